"""Host-side checks of the attention entry points that need no GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def binding():
    import __graft_entry__ as g
    g.build()
    from paper_2504_04704_b200 import binding as b
    return b


def test_workspace_sizes(binding):
    """Every smaller call fits the workspace of a larger one; bad shapes have none."""
    plan = binding.Plan(4, 8, 128, 16, 128, device=-1)
    size = lambda *a: int(plan.lib.lagkv_attend_workspace_bytes(plan.handle, *a))  # noqa: E731
    top = size(64, 64, 2000, 64)
    for T in (1, 2, 5, 16, 33, 64):
        for G in (1, 2, 7, 8):
            assert 0 < size(T, 8 * G, 0, 0) <= size(T, 8 * G, 100, 8) <= top
            assert size(T, 8 * G, 0, 0) % 256 == 0
    for bad in ((0, 8, 0, 0), (65, 8, 0, 0), (1, 12, 0, 0), (1, 4, 0, 0), (1, 8 * 65, 0, 0), (1, 8, -1, 0), (1, 8, 10, 0),
                (1, 8, 1 << 40, 4)):
        assert size(*bad) == 0
    assert plan.lib.lagkv_attend_workspace_bytes(None, 1, 8, 0, 0) == 0


def test_host_only_plan_refuses_attention(binding):
    plan = binding.Plan(1, 2, 128, 4, 64, device=-1)
    q = binding.lagkv_query(1, 2, 0.0, 0.0, 0.0, 0, 0, 0)
    p = [ctypes.c_void_p(256 * (i + 1)) for i in range(8)]
    assert plan.lib.lagkv_attend_tree(plan.handle, ctypes.byref(q), p[0], p[1], p[2], 64, p[3], None, None, p[4], None, p[5],
                                      1 << 30, None) == binding.LAGKV_EINVAL
    assert plan.lib.lagkv_tree_commit(plan.handle, p[0], p[1], 64, p[2], None, 4, p[3], p[4], p[5], 4096, None) == binding.LAGKV_EINVAL
    assert plan.lib.lagkv_attend_workspace_init(plan.handle, p[0], 4096, None) == binding.LAGKV_EINVAL


def test_strides_that_reach_behind_either_pool_are_refused(binding):
    """Both pools are checked against their own storage, and a stride of 0 counts as the dense one it stands for."""
    import torch
    H, rows, D = 2, 16, 64
    plan = binding.Plan(1, H, D, 4, 64, device=-1)
    size = H * rows * D
    store = torch.zeros(4 * size, dtype=torch.bfloat16)
    short = torch.zeros(3 * size, dtype=torch.bfloat16)
    table = torch.zeros((1, 4), dtype=torch.int32)
    view = lambda x, at=0: x.as_strided((1, H, rows, D), (size, rows * D, D, 1), at)  # noqa: E731
    dense = (size, rows * D, D, rows)

    def refused(K, V, strides, pages):
        with pytest.raises(TypeError) as e:                       # what a pool on the host meets behind this check is another
            plan._paged_pool(K, V, table, strides, pages)
        return "reach behind the pool" in str(e.value)

    assert not refused(view(store), view(store), dense, 4)
    assert refused(view(store), view(store), dense, 5)
    assert refused(view(store), view(short), dense, 4)            # V alone is too short
    assert refused(view(store), view(store, size), dense, 4)      # V begins behind K's first page
    assert not refused(view(store), view(short), dense, 3)
    for strides in ((0, 0, 0, rows), (0, rows * D, D, rows), (size, 0, D, rows), (size, rows * D, 0, rows)):
        assert not refused(view(store), view(store), strides, 4)
        assert refused(view(store), view(store), strides, 5)
