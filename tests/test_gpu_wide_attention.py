"""The kernel for wide trees at its special cases: every test says that its capacity takes that kernel."""
import random

import pytest
import torch

import serve_util as U

pytestmark = pytest.mark.gpu

BF16, FP16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
DEV = "cuda:0"
IDS = dict(ids=["bf16", "fp16", "fp8"])


@pytest.fixture(scope="module")
def binding():
    from paper_2504_04704_b200 import binding as b
    b.load_library()
    return b


def word_of(value, dtype):
    return U.bits(torch.tensor([value], device=DEV).to(dtype))[0]


def takes_wide(binding, call, ws, D, groups=1):
    """The call takes the wide kernel with `groups` groups of 128 query rows: the partials of that kernel, two per SM, are
    more than the others need, and a workspace without room for them is refused."""
    least = torch.cuda.get_device_properties(0).multi_processor_count * 2 * groups * 128 * (D + 2) * 4
    with pytest.raises(binding.LagKVError) as e:
        call(ws[:least])
    assert e.value.code == binding.LAGKV_EWORKSPACE


class Paged:
    """Sequences in pages at random places, behind a table whose capacity is far above the lengths."""

    def __init__(self, binding, B, H, G, D, T, dtype, page, lens, drafts=None, capacity=1 << 17, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.rng = random.Random(seed)
        self.dims, self.page, self.lens, self.dtype = (B, H, G, D, T), page, lens, dtype
        self.drafts = [min(T, n) for n in lens] if drafts is None else drafts
        nb = max(1, -(-max(lens) // page))
        self.K, self.V, self.ks, self.vs = U.make_cache((B, H, nb * page, D), dtype, g)
        self.Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(U.out_dtype(dtype))
        self.mask = U.random_tree(B, T, self.rng).to(DEV)
        self.pages = B * nb + 1
        perm = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
        self.table = torch.full((B, capacity // page), -1, dtype=torch.int32, device=DEV)
        for b, n in enumerate(lens):
            self.table[b, :-(-n // page)] = perm[b, :-(-n // page)]
        self.perm = perm
        self.seq, self.draft = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, self.drafts))
        self.plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
        self.ws = self.plan.new_attend_workspace(T, H * G)

    def pools(self):
        """K and V as pages; rows behind the last one are not finite."""
        K, V = self.K.clone(), self.V.clone()
        for b, n in enumerate(self.lens):
            for x in (K, V):
                U.bits(x)[b, :, n:] = word_of(float("nan"), self.dtype)
        return [U.to_pages(x, self.page, self.perm, self.pages, float("nan")) for x in (K, V)]

    def call(self, pools, ws=None):
        return self.plan.attend_tree_paged(self.Q, *pools, self.table, self.seq, self.ws if ws is None else ws, draft_len=self.draft,
                                           tree_mask=self.mask, k_scale=self.ks, v_scale=self.vs, want_lse=True)

    def reference(self, gone=()):
        """`gone`: (sequence, block) pairs whose rows are not there."""
        B, H, G, D, T = self.dims
        out = torch.zeros((B, T, H * G, D), dtype=torch.float64, device=DEV)
        lse = torch.full((B, T, H * G), -float("inf"), dtype=torch.float64, device=DEV)
        to, tl = torch.zeros_like(out), torch.zeros_like(lse)
        for b, n in enumerate(self.lens):
            seen = U.tree_seen(self.mask[b].tolist(), T, self.drafts[b], n)
            for x, j in gone:
                if x == b:
                    seen[:, j * self.page:(j + 1) * self.page] = False
            seen = seen.to(DEV).repeat_interleave(G, 0)
            for h in range(H):
                sl = slice(h * G, (h + 1) * G)
                q = self.Q[b, :, sl].reshape(T * G, D)
                o, l, eo, el = U.attention64(q, self.K[b, h, :n].float(), self.V[b, h, :n].float(), seen, D ** -0.5, self.ks, self.vs, self.dtype)
                out[b, :, sl], to[b, :, sl] = o.view(T, G, D), eo.view(T, G, D)
                lse[b, :, sl], tl[b, :, sl] = l.view(T, G), el.view(T, G)
        return out, lse, to, tl


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("T,G,page,D", [(12, 4, 16, 128), (33, 1, 32, 64), (40, 4, 64, 128), (40, 4, 16, 96), (20, 4, 128, 64), (64, 4, 256, 128)])
def test_missing_pages_under_drafted_rows(binding, dtype, T, G, page, D):
    """Drafts across pages of which the first, the last or all are not in the pool, one that is nothing but its draft
    among them: those rows are as not there, whatever shared memory held before."""
    lens = [page * 5 - min(T // 2, page) + T] * 3 + [page * 5 + 3 + T, T]
    c = Paged(binding, len(lens), 2, G, D, T, dtype, page, lens)
    pools = c.pools()
    blocks = [((n - T) // page, (n - 1) // page) for n in lens]
    gone = [(0, blocks[0][0]), (1, blocks[1][1])]
    gone += [(b, j) for b in (2, 4) for j in range(blocks[b][0], blocks[b][1] + 1)]
    # first a call whose tiles are nothing but NaN
    nan = [torch.full(p.shape, float("nan"), device=DEV).to(dtype) for p in pools]
    takes_wide(binding, lambda ws: c.call(nan, ws), c.ws, D, 2 if T * G > 128 else 1)
    c.call(nan)
    assert c.plan.read_status(c.ws)[0] == 0
    for i, (b, j) in enumerate(gone):
        c.table[b, j] = (-1, c.pages, -(1 << 31), (1 << 31) - 1)[i % 4]
    got = c.call(pools)
    assert c.plan.read_status(c.ws)[0] == binding.LAGKV_EINVAL
    U.assert_attention(got, c.reference(gone))
    assert not got["out"][4].any() and torch.isneginf(got["lse"][4]).all()


@pytest.mark.parametrize("T,G", [(12, 4), (40, 4)])
def test_tiny_queries_over_fp8(binding, T, G):
    """Queries whose factor and scale multiply to less than fp32 holds: all logits are nearly 0, hidden rows stay hidden."""
    c = Paged(binding, 3, 2, G, 128, T, FP8, 64, [T, 300, 129 + T])
    c.Q = (c.Q.float() * 2.0 ** -122).to(BF16)
    c.ks = 1e-7
    pools = c.pools()
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, 128, 2 if T * G > 128 else 1)
    got = c.call(pools)
    assert c.plan.read_status(c.ws)[0] == 0
    U.assert_attention(got, c.reference())


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_scales_that_vanish(binding, dtype):
    """A scale that is 0 in fp32: every row that is seen weighs the same."""
    T, G = 40, 4
    c = Paged(binding, 2, 2, G, 64, T, dtype, 64, [300, 129 + T])
    c.ks = 1e-60
    pools = c.pools()
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, 64, 2)
    got = c.call(pools)
    assert c.plan.read_status(c.ws)[0] == 0
    U.assert_attention(got, c.reference())
