"""Block bounds and the attention over chosen blocks against float64 statements (tests/serve_util.py)."""
import random

import pytest
import torch

import serve_util as U

pytestmark = pytest.mark.gpu

BF16, FP16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
DEV = "cuda:0"


@pytest.fixture(scope="module")
def binding():
    from paper_2504_04704_b200 import binding as b
    b.load_library()
    return b


def bounds_reference(K, lens, rows, before=None, from_len=None):
    """float64 [B, H, blocks, 2, D]; blocks nobody writes keep `before`."""
    B, H, S, D = K.shape
    blocks = -(-S // rows)
    want = torch.zeros((B, H, blocks, 2, D), dtype=torch.float64, device=K.device) if before is None else before.double().clone()
    k = K.float().double()
    for b, n in enumerate(lens):
        first = 0 if from_len is None else from_len[b] // rows
        for j in range(first, -(-n // rows)):
            part = k[b, :, j * rows:min(n, (j + 1) * rows)]
            want[b, :, j, 0], want[b, :, j, 1] = part.amin(1), part.amax(1)
    return want


def choose(q, lo, hi, nb, keep, sink, recent):
    """Blocks for one token and KV head: q [G, D], lo / hi [blocks, D], all float64."""
    if nb <= keep:
        return list(range(nb))
    score = torch.stack([torch.maximum(g * lo[:nb], g * hi[:nb]).sum(-1) for g in q]).amax(0).tolist()
    forced = set(range(sink)) | set(range(nb - recent, nb))
    rest = sorted((j for j in range(nb) if j not in forced), key=lambda j: (-score[j], j))
    return sorted(list(forced) + rest[:keep - len(forced)])


def reference(c, rows, keep, sink, recent, scale=None):
    Q, K, V = c["Q"], c["K"], c["V"]
    B, T, Hq, D = Q.shape
    H = K.shape[1]
    G = Hq // H
    scale = D ** -0.5 if scale is None else scale
    bd = c["bounds"].float().double()
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, T, Hq), -float("inf"), dtype=torch.float64, device=DEV)
    to, tl = torch.zeros_like(out), torch.zeros_like(lse)
    idx = torch.full((B, T, H, keep), -1, dtype=torch.int32)
    for b, n in enumerate(c["seq"].tolist()):
        if n < T:
            continue
        for t in range(T):
            end = n - (T - 1 - t)
            for h in range(H):
                q = Q[b, t, h * G:(h + 1) * G]
                pick = choose(q.double(), bd[b, h, :, 0], bd[b, h, :, 1], -(-end // rows), keep, sink, recent)
                idx[b, t, h, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
                at = [r for j in pick for r in range(j * rows, min(end, (j + 1) * rows))]
                seen = torch.ones((G, len(at)), dtype=torch.bool, device=DEV)
                o, l, eo, el = U.attention64(q, K[b, h].float()[at], V[b, h].float()[at], seen, scale, c["ks"], c["vs"], K.dtype)
                sl = slice(h * G, (h + 1) * G)
                out[b, t, sl], lse[b, t, sl], to[b, t, sl], tl[b, t, sl] = o, l, eo, el
    return (out, lse, to, tl), idx


def case(binding, B, H, G, D, S, T, dtype, rows, seed, lens=None, keep=8):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    K, V, ks, vs = U.make_cache((B, H, S, D), dtype, g)
    c = dict(K=K, V=V, ks=ks, vs=vs, Q=torch.randn((B, T, H * G, D), generator=g, device=DEV).to(U.out_dtype(dtype)))
    lens = [rng.randint(T, S) for _ in range(B)] if lens is None else lens
    for x in (K, V):                                              # rows behind the last one must not matter
        word = U.bits(torch.tensor([float("nan")], device=DEV).to(dtype))[0]
        for b, n in enumerate(lens):
            U.bits(x)[b, :, n:] = word
    c["seq"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    c["plan"] = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    c["bounds"] = c["plan"].new_block_bounds(S, rows)
    c["ws"] = c["plan"].new_attend_workspace(T, H * G, blocks=c["bounds"].shape[2], keep=keep)
    c["plan"].block_bounds(K, c["seq"], c["bounds"], c["ws"], block_rows=rows)
    return c


def run(c, rows, keep, sink=1, recent=2, **kw):
    got = c["plan"].attend_blocks(c["Q"], c["K"], c["V"], c["seq"], c["bounds"], c["ws"], block_rows=rows, keep=keep, sink_blocks=sink,
                                  recent_blocks=recent, k_scale=c["ks"], v_scale=c["vs"], want_lse=True, want_idx=True, **kw)
    assert c["plan"].read_status(c["ws"])[0] == 0
    return got


def check(c, rows, keep, sink=1, recent=2, **kw):
    got = run(c, rows, keep, sink, recent, **kw)
    want, idx = reference(c, rows, keep, sink, recent)
    assert torch.equal(got["idx"].cpu(), idx)
    U.assert_attention(got, want)
    return got


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("rows", [16, 32, 64, 128])
def test_bounds_are_exact(binding, dtype, D, rows):
    lens = [0, 1, rows - 1, rows, rows + 1, 300, 517]
    B, H, S = len(lens), 2, 517
    g = torch.Generator(device=DEV).manual_seed(D)
    K = U.make_cache((B, H, S, D), dtype, g)[0]
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    ws = plan.new_workspace()
    bounds = plan.new_block_bounds(S, rows)
    U.bits(bounds).fill_(3)
    before = bounds.float()
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    plan.block_bounds(K, seq, bounds, ws, block_rows=rows)
    assert torch.equal(bounds.float().double(), bounds_reference(K, lens, rows, before))
    # only the blocks from `from_len` on are made again
    K2 = U.make_cache((B, H, S, D), dtype, g)[0]
    start = [min(n, x) for n, x in zip(lens, (0, 0, 5, rows, 1, 150, 517))]
    before = bounds.float()
    plan.block_bounds(K2, seq, bounds, ws, block_rows=rows, from_len=torch.tensor(start, dtype=torch.int32, device=DEV))
    assert torch.equal(bounds.float().double(), bounds_reference(K2, lens, rows, before, start))
    # the same cache in pages
    page, nb = 32, 17
    perm = torch.randperm(B * nb, generator=torch.Generator().manual_seed(1)).view(B, nb).to(torch.int32).to(DEV)
    pool = U.to_pages(K, page, perm, B * nb, float("nan"))
    paged = plan.new_block_bounds(nb * page, rows)
    plan.block_bounds_paged(pool, perm, seq, paged, ws, block_rows=rows)
    blocks = bounds.shape[2]
    assert torch.equal(paged.float().double()[:, :, :blocks], bounds_reference(K, lens, rows))
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("T,G,H", [(1, 4, 2), (3, 7, 1), (1, 1, 2), (2, 20, 1)])
def test_every_type_and_head_dim(binding, dtype, D, T, G, H):
    c = case(binding, 3, H, G, D, 700, T, dtype, 16, seed=D + T, lens=[700, 333, 90])
    check(c, 16, 8)


@pytest.mark.parametrize("rows", [16, 32, 64, 128])
@pytest.mark.parametrize("keep,sink,recent", [(1, 0, 0), (1, 0, 1), (3, 1, 2), (5, 0, 1), (7, 3, 0), (13, 2, 2)])
def test_choices_and_lengths(binding, rows, keep, sink, recent):
    """Lengths next to every border: empty, one row, fewer blocks than kept, one more."""
    lens = [0, 1, rows, rows + 1, keep * rows - 1, keep * rows, keep * rows + 1, 20 * rows - 3, 20 * rows]
    c = case(binding, len(lens), 2, 2, 64, 20 * rows, 1, BF16, rows, seed=keep, lens=[min(n, 20 * rows) for n in lens], keep=keep)
    got = check(c, rows, keep, sink, recent)
    assert not got["out"][0].any() and (got["idx"][0] == -1).all()


def test_many_blocks(binding):
    """Thousands of blocks to choose from, one sequence; twice the same bits."""
    c = case(binding, 1, 2, 4, 64, 60000, 2, FP16, 16, seed=3, lens=[59990], keep=40)
    a = check(c, 16, 40)
    b = run(c, 16, 40)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_equal_scores_go_to_the_lowest_block(binding):
    """A cache of few distinct blocks: many exact ties, at and around the border."""
    c = case(binding, 2, 1, 2, 64, 16 * 90, 1, BF16, 16, seed=4, lens=[16 * 90, 16 * 51 + 5], keep=33)
    base = c["K"][:, :, :48].clone()
    c["K"][:, :, :16 * 90] = base.repeat(1, 1, 30, 1)
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    for keep in (4, 17, 33):
        check(c, 16, keep)
    c["K"].zero_()                                                # every score is zero
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    assert run(c, 16, 6)["idx"][0, 0, 0].tolist() == [0, 1, 2, 3, 88, 89]


def test_scores_next_to_the_border(binding):
    """Blocks whose scores differ by less than fp32 sums resolve."""
    c = case(binding, 1, 1, 1, 128, 16 * 40, 1, BF16, 16, seed=5, lens=[640], keep=9)
    c["Q"].fill_(1.0)
    c["K"].fill_(1.0)
    for j in range(40):                                           # 64 + j * 2^-26 after cancellation of large terms
        c["K"][0, 0, j * 16:(j + 1) * 16, 0] = 4096.0
        c["K"][0, 0, j * 16:(j + 1) * 16, 1] = -4096.0
        c["K"][0, 0, j * 16:(j + 1) * 16, 2] = ((j * 7) % 40) * 2.0 ** -20
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    check(c, 16, 9)


@pytest.mark.parametrize("keep", [3, 700, 1990])
def test_thousands_of_scores_next_to_the_border(binding, keep):
    """More blocks that 32-bit sums cannot tell apart than are ranked one against another, ties among them."""
    n = 2000
    c = case(binding, 1, 1, 2, 64, 16 * n, 1, BF16, 16, seed=6, lens=[16 * n], keep=keep)
    c["Q"].fill_(1.0)
    c["K"].fill_(1.0)
    c["K"][..., 0], c["K"][..., 1] = 4096.0, -4096.0
    v = (torch.arange(n, device=DEV) * 7) % 1500                  # 64 + v * 2^-20 after cancellation, 500 values twice
    c["K"][0, 0, :, 2] = ((v % 200) * 2.0 ** -20).to(BF16).repeat_interleave(16)
    c["K"][0, 0, :, 3] = ((v // 200) * 200 * 2.0 ** -20).to(BF16).repeat_interleave(16)
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    check(c, 16, keep)


@pytest.mark.parametrize("q,k", [(0, 0), (-80, 0), (-100, 0), (0, -80), (-40, -60), (-126, 0)])
def test_scores_next_to_the_border_of_tiny_values(binding, q, k):
    """Blocks whose scores differ by less than the rounding of 32-bit sums, at queries and keys whose squares vanish."""
    n, D, keep = 64, 128, 9
    c = case(binding, 1, 1, 1, D, 16 * n, 1, BF16, 16, seed=11, lens=[16 * n], keep=keep)
    g = torch.Generator(device=DEV).manual_seed(12)
    base = (torch.randn(D - 1, generator=g, device=DEV) * torch.exp2(torch.rand(D - 1, generator=g, device=DEV) * 22 - 16)).to(BF16).float()
    for i in range(3):                                            # large terms that cancel
        base[i] = 0
        base[i] = -base.sum().to(BF16).float()
    rows = torch.zeros((n, D), device=DEV)
    for j in range(n):                                            # the same terms in another order, and one that decides
        rows[j, :D - 1] = base[torch.randperm(D - 1, generator=g, device=DEV)]
        rows[j, D - 1] = ((j * 37) % n) * 2.0 ** -26
    c["K"][0, 0] = (rows * 2.0 ** k).repeat_interleave(16, 0).to(BF16)
    c["Q"].fill_(2.0 ** q)
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    check(c, 16, keep)


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("page,rows", [(16, 64), (64, 16), (32, 32)])
def test_paged_equals_contiguous(binding, dtype, page, rows):
    B, H, G, D, S, T = 3, 2, 4, 128, 600, 2
    lens = [600, 0, 331]
    c = case(binding, B, H, G, D, S, T, dtype, rows, seed=page, lens=lens)
    nb = -(-S // page)
    perm = torch.randperm(B * nb + 1, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    pools = [U.to_pages(c[x], page, perm, B * nb + 1, float("nan")) for x in "KV"]
    for b, n in enumerate(lens):
        perm[b, -(-n // page):] = -1
    plan = c["plan"]
    bounds = plan.new_block_bounds(nb * page, rows)
    ws = plan.new_attend_workspace(T, H * G, blocks=bounds.shape[2], keep=5)
    plan.block_bounds_paged(pools[0], perm, c["seq"], bounds, ws, block_rows=rows)
    got = plan.attend_blocks_paged(c["Q"], *pools, perm, c["seq"], bounds, ws, block_rows=rows, keep=5, k_scale=c["ks"], v_scale=c["vs"],
                                   want_lse=True, want_idx=True)
    assert plan.read_status(ws)[0] == 0
    same = check(c, rows, 5)
    assert all(torch.equal(got[k], same[k]) for k in got)


def test_keeping_every_block_is_dense_attention(binding):
    c = case(binding, 2, 2, 4, 128, 500, 1, BF16, 32, seed=2, lens=[500, 77], keep=16)
    a = run(c, 32, 16)
    b = c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], want_lse=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_lengths_that_do_not_describe_the_cache(binding):
    c = case(binding, 4, 1, 2, 64, 200, 3, BF16, 16, seed=2, lens=[200, 150, 100, 90])
    c["seq"][1], c["seq"][2] = 201, 2                              # too long; shorter than its tokens
    want, idx = reference(dict(c, seq=torch.tensor([200, 0, 0, 90])), 16, 5, 1, 2)
    got = c["plan"].attend_blocks(c["Q"], c["K"], c["V"], c["seq"], c["bounds"], c["ws"], block_rows=16, keep=5, want_lse=True, want_idx=True)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    assert torch.equal(got["idx"].cpu(), idx)
    U.assert_attention(got, want)
    c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=16)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL


def test_captured_and_replayed_while_the_cache_grows(binding):
    """A decode loop: append a row, renew the last block's bounds, attend; one captured step, replayed."""
    B, H, G, D, S, rows, keep = 2, 2, 2, 64, 400, 16, 6
    c = case(binding, B, H, G, D, S, 1, BF16, rows, seed=9, lens=[150, 310])
    g = torch.Generator(device=DEV).manual_seed(1)
    new = torch.randn((60, 2, B, H, D), generator=g, device=DEV).to(BF16)
    step = torch.zeros(1, dtype=torch.long, device=DEV)
    plan, old = c["plan"], torch.empty_like(c["seq"])
    b = torch.arange(B, device=DEV)[:, None]
    h = torch.arange(H, device=DEV)[None]
    out, got = torch.empty_like(c["Q"]), {}

    def token():
        old.copy_(c["seq"])
        row = new[step].squeeze(0)
        c["K"][b, h, old.long()[:, None]] = row[0]
        c["V"][b, h, old.long()[:, None]] = row[1]
        c["seq"].add_(1)
        step.add_(1)
        plan.block_bounds(c["K"], c["seq"], c["bounds"], c["ws"], block_rows=rows, from_len=old)
        got.update(plan.attend_blocks(c["Q"], c["K"], c["V"], c["seq"], c["bounds"], c["ws"], block_rows=rows, keep=keep, want_lse=True,
                                      want_idx=True, out=out))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            token()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(40):
        graph.replay()
        if i % 13 == 0:
            full = torch.zeros_like(c["bounds"])
            plan.block_bounds(c["K"], c["seq"], full, c["ws"], block_rows=rows)
            assert torch.equal(full, c["bounds"])
            want, idx = reference(c, rows, keep, 1, 2)
            assert torch.equal(got["idx"].cpu(), idx)
            U.assert_attention(got, want)
    assert plan.read_status(c["ws"])[0] == 0


def test_refusals_touch_nothing(binding):
    import ctypes
    c = case(binding, 2, 2, 2, 64, 256, 1, BF16, 32, seed=1)
    plan, lib = c["plan"], c["plan"].lib
    E = binding.LAGKV_EINVAL
    ptr = lambda t, off=0: None if t is None else ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731
    kept = c["bounds"].clone()
    args = [plan.handle, ptr(c["K"]), 256, None, ptr(c["seq"]), 32, ptr(c["bounds"]), 8, ptr(c["ws"]), c["ws"].numel(), None]
    for i, bad in ((1, None), (1, ptr(c["K"], 2)), (2, 0), (4, None), (5, 24), (5, 256), (6, None), (6, ptr(c["bounds"], 8)), (7, 7)):
        assert lib.lagkv_block_bounds(*(args[:i] + [bad] + args[i + 1:])) == E, (i, bad)
    assert lib.lagkv_block_bounds(*(args[:9] + [100, None])) == binding.LAGKV_EWORKSPACE
    query = binding.lagkv_query(1, 4, 0.0, 1.0, 1.0, 0, 0, 0)
    out = torch.full_like(c["Q"], 7)

    def call(q=query, nbytes=None, bounds=c["bounds"], V=c["V"], **kw):
        ch = binding.lagkv_block_choice(**{**dict(block_rows=32, keep=4, sink_blocks=1, recent_blocks=1, blocks=8), **kw})
        return lib.lagkv_attend_blocks(plan.handle, ctypes.byref(q), ctypes.byref(ch), ptr(c["Q"]), ptr(c["K"]), ptr(V), 256, ptr(c["seq"]),
                                       ptr(bounds), ptr(out), None, None, ptr(c["ws"]), c["ws"].numel() if nbytes is None else nbytes, None)

    for kw in (dict(block_rows=48), dict(keep=0), dict(sink_blocks=-1), dict(recent_blocks=-1), dict(sink_blocks=3, recent_blocks=2),
               dict(blocks=0), dict(blocks=7), dict(bounds=None), dict(V=None), dict(q=binding.lagkv_query(1, 3, 0.0, 1.0, 1.0, 0, 0, 0))):
        assert call(**kw) == E, kw
    for kw in (dict(keep=4097), dict(blocks=24577)):
        assert call(**kw) == binding.LAGKV_EUNSUPPORTED, kw
    assert call(nbytes=8192) == binding.LAGKV_EWORKSPACE and call(blocks=24000) == binding.LAGKV_EWORKSPACE
    torch.cuda.synchronize()
    assert (out == 7).all() and torch.equal(kept, c["bounds"])
