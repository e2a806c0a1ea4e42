"""Host-side checks of the operators on caches in 8 bits that need no GPU."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    import __graft_entry__ as g
    g.build()
    from paper_2504_04704_b200 import binding as b
    return b


def test_workspace_sizes(binding):
    """Every smaller call fits the workspace of a larger one; bad shapes have none."""
    for D in (64, 96, 128, 256):
        plan = binding.Plan(4, 8, D, 16, 128, device=-1)
        size = lambda *a: int(plan.lib.lagkv_attend_quant_workspace_bytes(plan.handle, *a))  # noqa: E731
        got = [size(T, 8 * G) for G in (1, 2, 7, 8) for T in (1, 2, 5, 16, 33, 64)]
        assert all(0 < n <= size(64, 64) and n % 256 == 0 for n in got)
        for bad in ((0, 8), (65, 8), (1, 12), (1, 4), (1, 8 * 65)):
            assert size(*bad) == 0
    assert plan.lib.lagkv_attend_quant_workspace_bytes(None, 1, 8) == 0


def cpu_cache(binding, B=1, H=2, S=64, D=128, R=32, dtype=torch.int8):
    codes = [torch.zeros((B, H, S, D), dtype=torch.uint8).view(dtype) for _ in "KV"]
    return binding.QuantCache(*codes, *(torch.zeros((B, H, -(-S // R))) for _ in "KV"), block_rows=R)


def test_host_only_plan_refuses(binding):
    plan = binding.Plan(1, 2, 128, 4, 64, device=-1)
    p = [ctypes.c_void_p(256 * (i + 1)) for i in range(8)]
    q = binding.lagkv_query(1, 2, 0.0, 0.0, 0.0, 0, 0, 0)
    c = binding.lagkv_quant_cache(256, 512, 1024, 2048, 0, 32, 2, 0, 0, 0)
    s = binding.lagkv_quant_source(1, 0, None, 0, 0, 0, 0, 0)
    r = ctypes.byref
    assert plan.lib.lagkv_quant_write(plan.handle, r(c), 64, r(s), p[5], p[6], None, p[3], p[4], 4096, None) == binding.LAGKV_EINVAL
    assert plan.lib.lagkv_quant_read(plan.handle, r(c), 64, None, p[3], None, 64, p[5], p[6], p[4], 4096, None) == binding.LAGKV_EINVAL
    assert plan.lib.lagkv_attend_quant(plan.handle, r(q), 0.0, r(c), p[5], 64, p[3], None, None, p[6], None, p[4], 1 << 30, None) == binding.LAGKV_EINVAL


def test_cache_object_refuses(binding):
    K = torch.zeros((1, 2, 64, 128), dtype=torch.int8)
    s = torch.zeros((1, 2, 2))
    binding.QuantCache(K, K.clone(), s, s.clone(), block_rows=32)
    for bad in (dict(K=K.to(torch.uint8)), dict(V=K.view(torch.float8_e4m3fn)), dict(V=K[:, :, :32]), dict(K_scale=s.double()),
                dict(V_scale=s[..., :1]), dict(K=K[0], V=K[0]), dict(V=torch.zeros((1, 2, 128, 64), dtype=torch.int8).transpose(2, 3)),
                dict(K=K[:, :1].expand(1, 2, 64, 128), V=K[:, :1].expand(1, 2, 64, 128)), dict(V=K.transpose(1, 2).contiguous().transpose(1, 2))):
        args = dict(K=K, V=K.clone(), K_scale=s, V_scale=s.clone())
        args.update(bad)
        with pytest.raises(TypeError):
            binding.QuantCache(**args)


def test_strides_are_kept_and_dense_ones_left_out(binding):
    x = torch.zeros((3, 2, 50, 64), dtype=torch.int8)
    assert binding._dense_strides(x, "x") == (0, 0, 0)
    y = torch.zeros((3, 50, 2, 80), dtype=torch.int8)[..., :64].transpose(1, 2)
    assert binding._dense_strides(y, "y") == (50 * 2 * 80, 80, 160)
    one = torch.zeros((3, 50, 1, 64), dtype=torch.int8).transpose(1, 2)[:, :, :1]   # a dimension of one: its stride says nothing
    assert binding._dense_strides(one, "one")[1] % 64 == 0
    with pytest.raises(TypeError):
        binding._dense_strides(x[..., ::2], "x")
    with pytest.raises(TypeError):
        binding._dense_strides(x[:, :1].expand(3, 2, 50, 64), "x")


def test_tensors_elsewhere_are_refused(binding):
    """Everything has to be on the plan's device: nothing of the CPU's reaches the library."""
    plan = binding.Plan(1, 2, 128, 4, 64, device=-1)
    cache = cpu_cache(binding)
    x = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    n, ws = torch.zeros(1, dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
    plan.device = 0
    with pytest.raises(TypeError):
        plan.quant_write(cache, x, x, n, ws)
    with pytest.raises(TypeError):
        plan.quant_read(cache, n, ws, K_out=x)
    with pytest.raises(TypeError):
        plan.attend_quant(x.transpose(1, 2).contiguous(), cache, n, ws)


def test_cache_object_keeps_its_tensors(binding):
    """What a call passes is what the attributes name: nothing can be assigned, and memory that was exchanged is refused."""
    plan = binding.Plan(1, 2, 128, 4, 64, device=-1)
    cache = cpu_cache(binding)
    was = bytes(cache.arg)
    for name in ("K", "V", "K_scale", "V_scale", "block_rows", "rows", "shape", "arg", "other"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name, 1))
    with pytest.raises(AttributeError):
        del cache.K_scale
    with pytest.raises(AttributeError):                            # sequences in another order, as a batch's slots change hands
        cache.K_scale = cache.K_scale[torch.zeros(1, dtype=torch.long)]
    assert bytes(cache.arg) == was and cache.arg.K == cache.K.data_ptr() and cache.arg.K_scale == cache.K_scale.data_ptr()
    cache.K.add_(1)
    cache.K_scale.fill_(2.0)
    assert plan._check_quant(cache, False) is cache.ref and plan._check_quant(cache, True) is cache.ref
    for name in ("K", "V", "K_scale", "V_scale"):
        cache = cpu_cache(binding)
        t = getattr(cache, name)
        t.resize_((1, 2, 4 * t.shape[2]) + t.shape[3:])            # a pool that grows
        for paged in (False, True):
            with pytest.raises(TypeError):
                plan._check_quant(cache, paged)
        cache = cpu_cache(binding)
        t = getattr(cache, name)
        t.data = t.clone()
        with pytest.raises(TypeError):
            plan._check_quant(cache, False)


def test_pools_with_strides_carry_them_in_the_layout(binding):
    """What a paged call passes for pools that are not contiguous; strides that reach behind the memory are refused."""
    plan = binding.Plan(2, 3, 64, 4, 64, device=-1)
    store = torch.zeros((5, 2, 3, 16, 80), dtype=torch.int8)
    K, V = store[:, 0, :, :, :64], store[:, 1, :, :, :64]
    scales = torch.zeros((2, 2, 3, 4))
    cache = binding.QuantCache(K, V, scales[0], scales[1], block_rows=16)
    ref = plan._check_quant(cache, True)
    arg = cache.paged
    assert ref is cache.paged_ref and (arg.stride_b, arg.stride_h, arg.stride_s) == (0, 0, 0) and arg.K == K.data_ptr() and arg.V == V.data_ptr()
    assert (cache.arg.stride_b, cache.arg.stride_h, cache.arg.stride_s) == K.stride()[:3]
    table = torch.zeros((2, 4), dtype=torch.int32)
    plan._paged = lambda pool, tab, strides: strides               # a table on the host goes no further
    assert plan._quant_pool(cache, table) == (K.stride()[:3] + (16,), 5)
    dense = torch.zeros((2, 5, 3, 16, 64), dtype=torch.int8)
    assert plan._quant_pool(binding.QuantCache(dense[0], dense[1], scales[0], scales[1], block_rows=16), table) == (None, 5)
