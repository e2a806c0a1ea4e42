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


def same(a, b):
    return torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def dense_cache(c, S):
    """K and V of `c` as [B, H, S, D], rows behind the last one not finite."""
    B, H, G, D, T = c.dims
    out = []
    for x in (c.K, c.V):
        y = torch.empty((B, H, S, D), dtype=c.dtype, device=DEV)
        U.bits(y).fill_(int(word_of(float("nan"), c.dtype)))
        for b, n in enumerate(c.lens):
            U.bits(y)[b, :, :n] = U.bits(x)[b, :, :n]
        out.append(y)
    return out


def hide(c, odd):
    """Token t sees drafted row t at least; rows `odd` are seen by their own tokens alone."""
    T = c.dims[4]
    bit = sum(1 << j for j in odd)
    m = c.mask.cpu()
    for b in range(m.shape[0]):
        for t in range(T):
            word = ((int(m[b, t]) & ~bit) | ((1 << t) if t in odd else 0)) & ((1 << 64) - 1)
            m[b, t] = word - (1 << 64) if word >> 63 else word
    c.mask = m.to(DEV)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=["nan", "inf"])
@pytest.mark.parametrize("T,G,page,D", [(40, 2, 16, 128), (64, 4, 32, 64), (33, 4, 64, 96), (12, 4, 128, 64)])
def test_hidden_drafted_rows_may_hold_anything(binding, dtype, value, T, G, page, D):
    """Drafted rows that are not finite reach the tokens that see them and no others, in pages and without."""
    odd = [1, T // 2, T - 2]
    c = Paged(binding, 3, 2, G, D, T, dtype, page, [150 + T, T, 128 + T // 2])
    hide(c, odd)
    clean = [c.K.clone(), c.V.clone()]
    for b, n in enumerate(c.lens):
        for j in odd:
            for x, z in zip((c.K, c.V), clean):
                U.bits(x)[b, :, n - T + j] = word_of(value, dtype)
                U.bits(z)[b, :, n - T + j] = 0
    pools, dense = c.pools(), dense_cache(c, 32768)
    c.K, c.V = clean
    want = c.reference()
    keep = torch.tensor([t not in odd for t in range(T)], device=DEV)
    groups = 2 if T * G > 128 else 1
    contiguous = lambda ws: c.plan.attend_tree(c.Q, *dense, c.seq, ws, draft_len=c.draft, tree_mask=c.mask, k_scale=c.ks,  # noqa: E731
                                               v_scale=c.vs, want_lse=True)
    for call in (lambda ws: c.call(pools, ws), contiguous):
        takes_wide(binding, call, c.ws, D, groups)
        got = call(c.ws)
        assert c.plan.read_status(c.ws)[0] == 0
        U.assert_attention({k: v[:, keep] for k, v in got.items()}, tuple(x[:, keep] for x in want))
        assert torch.isnan(got["out"][:, odd].float()).all()


@pytest.mark.parametrize("T,G", [(12, 4), (40, 4)])
def test_one_infinite_value_of_a_seen_row(binding, T, G):
    """V of one drafted row is finite but for one channel: that channel alone is infinite for those who see it."""
    c = Paged(binding, 2, 2, G, 64, T, BF16, 64, [300, T])
    for b, n in enumerate(c.lens):
        c.K[b, :, n - T + 2] = 0
        c.V[b, :, n - T + 2, 5] = float("inf")
    pools = c.pools()
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, 64, 2 if T * G > 128 else 1)
    got = c.call(pools)["out"].float()
    sees = (c.mask >> 2 & 1).bool()
    assert torch.isinf(got[..., 5][sees]).all() and torch.isfinite(got[~sees]).all()
    got[..., 5] = 0
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("T,G,page,D", [(12, 4, 16, 128), (33, 4, 32, 96), (40, 4, 64, 64), (20, 4, 128, 128), (64, 4, 256, 64), (64, 2, 16, 64)])
def test_missing_pages_under_the_rows_that_all_see(binding, dtype, T, G, page, D):
    """Pages outside the pool, one of them before the draft's, one the first."""
    c = Paged(binding, 3, 2, G, D, T, dtype, page, [6 * page + T, 4 * page + T, 3 * page])
    pools = c.pools()
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, D, 2 if T * G > 128 else 1)
    nan = [torch.full(p.shape, float("nan"), device=DEV).to(dtype) for p in pools]
    c.call(nan)
    gone = [(0, 1), (0, 2), (1, 0)]
    for i, (b, j) in enumerate(gone):
        c.table[b, j] = (-1, c.pages, 1 << 30)[i]
    got = c.call(pools)
    assert c.plan.read_status(c.ws)[0] == binding.LAGKV_EINVAL
    U.assert_attention(got, c.reference(gone))


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("T,G,page,D", [(33, 1, 16, 128), (64, 2, 32, 96), (40, 4, 64, 128), (64, 7, 128, 64), (33, 4, 16, 64)])
def test_pages_and_lengths_around_every_tile(binding, dtype, T, G, page, D):
    """Empty slots, all draft, lengths next to the 128-row tiles, ragged drafts, tokens that see no drafted row; the
    contiguous cache of the same capacity gives the same bits."""
    lens = [0, T, T + 1, 127 + T, 128, 129, 255, 256, 257, 512 + T // 2, 700]
    lens = [max(n, T) if n else 0 for n in lens]
    drafts = [0 if n == 0 else T - (i % 3) * (T // 3) for i, n in enumerate(lens)]
    S = 16384
    c = Paged(binding, len(lens), 2, G, D, T, dtype, page, lens, drafts, capacity=S)
    c.mask[1, ::2] = 0
    pools, dense = c.pools(), dense_cache(c, S)
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, D, 2 if T * G > 128 else 1)
    got = c.call(pools)
    U.assert_attention(got, c.reference())
    assert not got["out"][0].any() and not got["out"][1, drafts[1]:].any()
    assert same(got, c.plan.attend_tree(c.Q, *dense, c.seq, c.ws, draft_len=c.draft, tree_mask=c.mask, k_scale=c.ks, v_scale=c.vs, want_lse=True))
    assert c.plan.read_status(c.ws)[0] == 0


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("T,G,page", [(12, 4, 16), (40, 4, 64)])
def test_captured_and_replayed(binding, dtype, T, G, page):
    """One captured call serves every later length and draft; two such graphs share a workspace in turn."""
    cases = [Paged(binding, 3, 2, G, 128, T, dtype, page, [900, 333, T], seed=s) for s in (1, 2)]
    graphs, outs = [], []
    ws = cases[0].ws
    for c in cases:
        pools = c.kept = [U.to_pages(x, page, c.perm, c.pages, float("nan")) for x in (c.K, c.V)]
        c.table[:, :c.perm.shape[1]] = c.perm
        takes_wide(binding, lambda w: c.call(pools, w), ws, 128, 2 if T * G > 128 else 1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(c.call(pools, ws))
        graphs.append(graph)
    for lens, drafts in (([900, 333, T], [T, T, T]), ([0, 129, T], [0, 1, T - 1]), ([128, 900, 200], [T, 0, 5])):
        for c in cases:
            c.lens, c.drafts = lens, drafts
            c.seq.copy_(torch.tensor(lens, dtype=torch.int32))
            c.draft.copy_(torch.tensor(drafts, dtype=torch.int32))
        for order in ((0, 1), (1, 0, 0)):
            for i in order:
                graphs[i].replay()
            torch.cuda.synchronize()
            for c, out in zip(cases, outs):
                U.assert_attention(out, c.reference())
    assert cases[0].plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("T,G,B,longest", [(12, 4, 4, 9000), (40, 4, 4, 9000), (33, 1, 600, 300)])
def test_shared_units_large_batches_and_repeats(binding, dtype, T, G, B, longest):
    """Sequences shared by many CTAs, more sequences than a CTA has threads; the same bits again, on two streams at once."""
    rng = random.Random(3)
    lens = [rng.randint(T, longest) for _ in range(B)]
    c = Paged(binding, B, 1, G, 64, T, dtype, 64, lens, capacity=1 << 16)
    pools = c.pools()
    takes_wide(binding, lambda ws: c.call(pools, ws), c.ws, 64, 2 if T * G > 128 else 1)
    got = c.call(pools)
    U.assert_attention(got, c.reference())
    streams, spaces = [torch.cuda.Stream(), torch.cuda.Stream()], [c.ws, c.plan.new_attend_workspace(T, G)]
    torch.cuda.synchronize()
    again = []
    for _ in range(5):
        for s, ws in zip(streams, spaces):
            with torch.cuda.stream(s):
                again.append(c.call(pools, ws))
    torch.cuda.synchronize()
    assert all(same(got, x) for x in again)
    assert all(c.plan.read_status(ws)[0] == 0 for ws in spaces)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], **IDS)
@pytest.mark.parametrize("T,G,D", [(12, 4, 96), (40, 4, 128)])
def test_other_arrangements(binding, dtype, T, G, D):
    """[B, S, H, D] caches with padded rows, pools with rows outside heads, queries cut out of a fused projection."""
    B, H, S, page, extra = 2, 3, 32768, 32, 16
    c = Paged(binding, B, H, G, D, T, dtype, page, [700, 131 + T])
    fused = torch.zeros((B, T, H * G + 4, D + 8), dtype=c.Q.dtype, device=DEV)
    fused[:, :, 2:2 + H * G, :D] = c.Q
    Q = fused[:, :, 2:2 + H * G, :D]
    kw = dict(draft_len=c.draft, tree_mask=c.mask, k_scale=c.ks, v_scale=c.vs, want_lse=True)
    want = c.reference()
    wide = []
    for x in dense_cache(c, S):
        y = torch.empty((B, S, H, D + extra), dtype=dtype, device=DEV)
        U.bits(y).fill_(int(word_of(float("nan"), dtype)))
        U.bits(y)[..., :D] = U.bits(x).permute(0, 2, 1, 3)
        wide.append(y.permute(0, 2, 1, 3)[..., :D])
    K, V = wide
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype, strides=(K.stride(0), K.stride(1), K.stride(2)))
    groups = 2 if T * G > 128 else 1
    takes_wide(binding, lambda ws: plan.attend_tree(Q, K, V, c.seq, ws, **kw), c.ws, D, groups)
    U.assert_attention(plan.attend_tree(Q, K, V, c.seq, c.ws, **kw), want)
    pools = []
    for x in c.pools():
        y = torch.empty((c.pages, page, H, D + extra), dtype=dtype, device=DEV)
        U.bits(y).fill_(int(word_of(float("nan"), dtype)))
        U.bits(y)[..., :D] = U.bits(x).permute(0, 2, 1, 3)
        pools.append(y)
    strides = (page * H * (D + extra), D + extra, H * (D + extra), page)
    call = lambda ws: c.plan.attend_tree_paged(Q, *pools, c.table, c.seq, ws, strides=strides, num_pages=c.pages, **kw)  # noqa: E731
    takes_wide(binding, call, c.ws, D, groups)
    U.assert_attention(call(c.ws), want)
    assert c.plan.read_status(c.ws)[0] == 0


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
def test_offsets_beyond_32_bits(binding, dtype):
    """Pages, heads and sequences more than 2^32 bytes apart."""
    D, H, B, G, T, page = 128, 2, 2, 4, 16, 64
    size = 1 if dtype == FP8 else 2
    far = ((1 << 32) + 8192) // size
    g = torch.Generator(device=DEV).manual_seed(3)
    store = [torch.empty(4 * far, dtype=torch.uint8 if dtype == FP8 else BF16, device=DEV).view(dtype) for _ in range(2)]
    Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(BF16)
    # contiguous: heads `far` apart, a capacity that none of the sequences fills
    S = 1 << 20
    K, V = (x.as_strided((B, H, S, D), (2 * far, far, D, 1)) for x in store)
    lens = [300, 141]
    small = [torch.randn((B, H, 300, D), generator=g, device=DEV).to(dtype) for _ in range(2)]
    for x, y in zip((K, V), small):
        U.bits(x)[:, :, :300] = U.bits(y)
    plan = binding.Plan(B, H, D, sink=0, lag=32, strides=(2 * far, far, D), dtype=dtype)
    ws = plan.new_attend_workspace(T, H * G)
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    takes_wide(binding, lambda w: plan.attend_tree(Q, K, V, seq, w), ws, D)
    U.assert_attention(plan.attend_tree(Q, K, V, seq, ws, want_lse=True), U.tree_reference(Q, *small, seq, [T, T], None))
    # pages `far` apart in one pool, one head
    pool = [x.as_strided((4, 1, page, D), (far, page * D, D, 1)) for x in store]
    fresh = [torch.randn((4, 1, page, D), generator=g, device=DEV).to(dtype) for _ in range(2)]
    for x, y in zip(pool, fresh):
        U.bits(x)[:] = U.bits(y)
    table = torch.full((B, 8192), -1, dtype=torch.int32, device=DEV)
    table[:, :2] = torch.tensor([[3, 0], [2, 1]], dtype=torch.int32)
    plan1 = binding.Plan(B, 1, D, sink=0, lag=32, dtype=dtype)
    q1 = Q[:, :, :G].contiguous()
    seq1 = torch.tensor([128, 77], dtype=torch.int32, device=DEV)
    call = lambda w, **kw: plan1.attend_tree_paged(q1, store[0], store[1], table, seq1, w, strides=(far, page * D, D, page), num_pages=4, **kw)  # noqa: E731
    takes_wide(binding, call, ws, D)
    dense = [U.bits(x)[table[:, :2].long()].view(B, 1, 128, D).view(dtype) for x in fresh]
    U.assert_attention(call(ws, want_lse=True), U.tree_reference(q1, *dense, seq1, [T, T], None))
    assert plan.read_status(ws)[0] == 0
