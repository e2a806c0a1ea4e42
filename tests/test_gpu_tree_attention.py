"""Tree attention and the commit of accepted rows against float64 statements (tests/serve_util.py)."""
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


def case(binding, B, H, G, D, S, T, dtype, seed, lens=None, drafts=None, tree=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    K, V, ks, vs = U.make_cache((B, H, S, D), dtype, g)
    Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(U.out_dtype(dtype))
    lens = [rng.randint(T, S) for _ in range(B)] if lens is None else lens
    drafts = [min(T, n) for n in lens] if drafts is None else drafts
    c = dict(K=K, V=V, Q=Q, ks=ks, vs=vs, seq=torch.tensor(lens, dtype=torch.int32, device=DEV),
             draft=torch.tensor(drafts, dtype=torch.int32, device=DEV),
             mask=U.random_tree(B, T, rng).to(DEV) if tree else None)
    c["plan"] = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    c["ws"] = c["plan"].new_attend_workspace(T, H * G)
    return c


def poison(c, value=float("nan")):
    """Rows at and behind seq_len hold what must never be used."""
    K, V = U.bits(c["K"]), U.bits(c["V"])
    word = U.bits(torch.tensor([value], device=DEV).to(c["K"].dtype))[0]
    for b, n in enumerate(c["seq"].tolist()):
        K[b, :, n:] = word
        V[b, :, n:] = word


def run(c, **kw):
    got = c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"],
                                k_scale=c["ks"], v_scale=c["vs"], want_lse=True, **kw)
    assert c["plan"].read_status(c["ws"])[0] == 0
    return got


def reference(c, scale=None):
    return U.tree_reference(c["Q"], c["K"], c["V"], c["seq"], c["draft"], c["mask"], scale, c["ks"], c["vs"])


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("T,G,H", [(1, 4, 2), (1, 7, 4), (5, 1, 3), (13, 4, 2), (32, 4, 1), (64, 8, 1)])
def test_every_type_and_head_dim(binding, dtype, D, T, G, H):
    c = case(binding, 3, H, G, D, 333, T, dtype, seed=D + T, lens=[max(T, 100), 333, max(T, 257)])
    poison(c)
    U.assert_attention(run(c), reference(c))


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("T", [1, 4, 40])
def test_lengths_around_every_tile(binding, dtype, T):
    """Empty sequences, sequences that are all draft, and every length next to a multiple of 16 or 64."""
    lens = [0, T, T + 1, 15 + T, 16 + T, 17 + T, 63 + T, 64 + T, 65 + T, 128, 129, 200]
    c = case(binding, len(lens), 2, 3, 128, 200, T, dtype, seed=5, lens=lens)
    poison(c)
    got = run(c)
    U.assert_attention(got, reference(c))
    assert not got["out"][0].any() and (got["lse"][0] == float("-inf")).all()


def test_chain_without_lengths_and_masks(binding):
    """No draft_len: T everywhere; no mask: token t sees drafted rows 0 .. t."""
    c = case(binding, 4, 2, 4, 128, 300, 6, BF16, seed=9, tree=False)
    got = c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], want_lse=True)
    U.assert_attention(got, reference(c))
    assert "lse" not in c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"])


@pytest.mark.parametrize("T", [1, 9, 64])
def test_padded_batch_and_rows_that_see_nothing(binding, T):
    """Draft lengths from 0 on; tokens whose mask is empty in a cache without other rows."""
    B = 5
    drafts = [0, min(1, T), T // 2, T, T]
    lens = [50, 33, T // 2, T, 90 + T]              # sequences 2 and 3 are nothing but their draft
    c = case(binding, B, 2, 4, 128, 200, T, FP16, seed=T, lens=lens, drafts=drafts)
    c["mask"][3, ::2] = 0
    c["mask"][4] = -1
    poison(c, float("inf"))
    got = run(c)
    U.assert_attention(got, reference(c))
    assert not got["out"][0].any() and not got["out"][3, ::2].any()
    assert torch.isneginf(got["lse"][3, 0]).all()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,G", [(7, 2), (40, 4), (64, 4)])
def test_hidden_drafted_rows_may_hold_anything(binding, dtype, value, T, G):
    """Drafted rows that are not finite reach the tokens that see them and no others."""
    c = case(binding, 2, 2, G, 128, 150, T, dtype, seed=3, lens=[150, T])
    odd = [1, T - 2]
    bit = sum(1 << j for j in odd)
    # tokens 1 and T - 2 see their own row, nobody else sees either
    m = c["mask"].cpu()
    for t in range(T):
        word = ((int(m[0, t]) & ~bit) | ((1 << t) if t in odd else 0)) & ((1 << 64) - 1)
        m[:, t] = word - (1 << 64) if word >> 63 else word
    c["mask"] = m.to(DEV)
    word = U.bits(torch.tensor([value], device=DEV).to(dtype))[0]
    for b, n in enumerate(c["seq"].tolist()):
        for j in odd:
            U.bits(c["K"])[b, :, n - T + j] = word
            U.bits(c["V"])[b, :, n - T + j] = word
    clean = dict(c, K=c["K"].clone(), V=c["V"].clone())
    for b, n in enumerate(c["seq"].tolist()):
        for j in odd:
            U.bits(clean["K"])[b, :, n - T + j] = 0
            U.bits(clean["V"])[b, :, n - T + j] = 0
    got, want = run(c), reference(clean)
    keep = torch.tensor([t not in odd for t in range(T)], device=DEV)
    U.assert_attention({k: v[:, keep] for k, v in got.items()}, tuple(x[:, keep] for x in want))
    assert torch.isnan(got["out"][:, odd].float()).all()


@pytest.mark.parametrize("T,G", [(6, 4), (33, 4)])
def test_one_infinite_value_of_a_seen_row(binding, T, G):
    """V of one drafted row is finite but for one channel: that channel alone is infinite for those who see it."""
    c = case(binding, 1, 1, G, 64, 90, T, BF16, seed=8, lens=[80])
    c["K"][0, 0, 80 - T + 2] = 0
    c["V"][0, 0, 80 - T + 2, 5] = float("inf")
    got = run(c)["out"].float()
    sees = (c["mask"][0] >> 2 & 1).bool()
    assert torch.isinf(got[0, sees, :, 5]).all() and torch.isfinite(got[0, ~sees]).all()
    got[..., 5] = 0
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("page,T", [(16, 1), (16, 20), (64, 1), (128, 33)])
def test_paged_equals_contiguous(binding, dtype, page, T):
    B, H, G, D, S = 4, 2, 4, 128, 300
    lens = [0, max(T, 17), 299, 300]
    c = case(binding, B, H, G, D, S, T, dtype, seed=page, lens=lens)
    poison(c)
    nb = -(-S // page)
    perm = torch.randperm(B * nb + 2, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    pools = [U.to_pages(c[x], page, perm, B * nb + 2, float("nan")) for x in "KV"]
    for b, n in enumerate(lens):                     # entries behind the last row may be anything
        perm[b, -(-n // page):] = -1 if b % 2 else 1 << 30
    got = c["plan"].attend_tree_paged(c["Q"], *pools, perm, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"],
                                      k_scale=c["ks"], v_scale=c["vs"], want_lse=True)
    assert c["plan"].read_status(c["ws"])[0] == 0
    same = run(c)
    assert torch.equal(got["out"], same["out"]) and torch.equal(got["lse"], same["lse"])
    U.assert_attention(got, reference(c))


def test_paged_pool_with_padded_strides(binding):
    B, H, G, D, S, T, page = 2, 2, 4, 64, 100, 3, 32
    c = case(binding, B, H, G, D, S, T, BF16, seed=2, lens=[100, 64])
    perm = torch.tensor([[3, 0, 6, 2], [1, 5, 4, 7]], dtype=torch.int32, device=DEV)
    pools = []
    for x in "KV":
        dense = U.to_pages(c[x], page, perm, 8, 0.0)
        wide = torch.full((8, page, H, D + 8), float("nan"), dtype=BF16, device=DEV)    # rows outside heads, padded
        wide[..., :D] = dense.permute(0, 2, 1, 3)
        pools.append(wide)
    strides = (page * H * (D + 8), D + 8, H * (D + 8), page)
    got = c["plan"].attend_tree_paged(c["Q"], *pools, perm, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"],
                                      want_lse=True, strides=strides, num_pages=8)
    U.assert_attention(got, reference(c))


def test_a_page_outside_the_pool_is_not_read(binding):
    """Recorded, and its rows count as not there; other sequences are as without it."""
    B, H, G, D, S, T, page = 3, 1, 4, 128, 256, 2, 64
    c = case(binding, B, H, G, D, S, T, BF16, seed=4, lens=[256, 256, 200])
    perm = torch.randperm(12, generator=torch.Generator().manual_seed(2)).view(3, 4).to(torch.int32).to(DEV)
    pools = [U.to_pages(c[x], page, perm, 12, 0.0) for x in "KV"]
    table = perm.clone()
    table[0, 1], table[1, 2] = -7, 12
    got = c["plan"].attend_tree_paged(c["Q"], *pools, table, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    for b, gone in ((0, 1), (1, 2), (2, None)):
        K, V = (c[x][b:b + 1] for x in "KV")
        n = int(c["seq"][b])
        if gone is not None:
            keep = torch.tensor([r // page != gone for r in range(S)], device=DEV)
            K, V, n = K[:, :, keep], V[:, :, keep], n - page
        want = U.tree_reference(c["Q"][b:b + 1], K, V, [n], [T], c["mask"][b:b + 1])
        U.assert_attention({k: v[b:b + 1] for k, v in got.items()}, want)


def test_lengths_that_do_not_describe_the_cache(binding):
    c = case(binding, 5, 2, 4, 128, 128, 4, BF16, seed=6, lens=[100, 90, 80, 70, 128])
    c["seq"][1], c["draft"][2], c["seq"][3] = 129, 5, 3          # too long, too wide, draft above the length
    got = c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    assert not got["out"][1:4].any() and torch.isneginf(got["lse"][1:4]).all()
    good = [0, 4]
    want = U.tree_reference(c["Q"][good], c["K"][good], c["V"][good], c["seq"][good], c["draft"][good], c["mask"][good])
    U.assert_attention({k: v[good] for k, v in got.items()}, want)


def test_strided_cache_and_queries(binding):
    """[B, S, H, D] caches with padded rows, queries cut out of a fused projection."""
    B, H, G, D, S, T = 2, 3, 2, 96, 120, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    wide = torch.randn((2, B, S, H, D + 16), generator=g, device=DEV).to(BF16)
    K, V = (wide[i].permute(0, 2, 1, 3)[..., :D] for i in range(2))
    fused = torch.randn((B, T, H * G + 4, D + 8), generator=g, device=DEV).to(BF16)
    Q = fused[:, :, 2:2 + H * G, :D]
    plan = binding.Plan(B, H, D, sink=0, lag=32, strides=(K.stride(0), K.stride(1), K.stride(2)))
    ws = plan.new_attend_workspace(T, H * G)
    seq = torch.tensor([120, 77], dtype=torch.int32, device=DEV)
    got = plan.attend_tree(Q, K, V, seq, ws, want_lse=True, scale=0.3)
    U.assert_attention(got, U.tree_reference(Q, K, V, seq, [T, T], None, 0.3))


@pytest.mark.parametrize("T,G,B,S", [(1, 4, 1, 40000), (64, 4, 1, 9000), (24, 2, 3, 5000), (2, 7, 40, 700), (1, 1, 600, 90)])
def test_shared_units_and_large_batches(binding, T, G, B, S):
    """Long sequences shared by many CTAs, and more sequences than a CTA has threads; twice the same bits."""
    c = case(binding, B, 2, G, 128, S, T, BF16, seed=S)
    got = run(c)
    U.assert_attention(got, reference(c))
    again = run(c)
    assert torch.equal(got["out"], again["out"]) and torch.equal(got["lse"], again["lse"])


def test_one_workspace_serves_every_smaller_call(binding):
    """Shapes in turn on one workspace: each equals its run on a workspace of its own, bit for bit."""
    shapes = [(64, 4), (1, 4), (7, 2), (1, 1), (33, 4), (64, 4)]
    big = None
    for T, G in shapes:
        c = case(binding, 3, 2, G, 128, 3000, T, BF16, seed=T, lens=[3000, 1500, 64])
        own = run(c)
        if big is None:
            big = c["ws"]
        c["ws"] = big
        shared = run(c)
        assert torch.equal(own["out"], shared["out"]) and torch.equal(own["lse"], shared["lse"])


def test_captured_and_replayed_with_other_lengths(binding):
    """One captured call serves every later length and draft; another stream than the default."""
    c = case(binding, 3, 2, 4, 128, 2000, 8, BF16, seed=1, lens=[8, 8, 8])
    out = torch.empty_like(c["Q"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(c, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"],
                                        want_lse=True, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for lens, drafts in (([2000, 8, 0], [8, 3, 0]), ([17, 900, 1999], [1, 8, 0])):
        c["seq"].copy_(torch.tensor(lens, dtype=torch.int32))
        c["draft"].copy_(torch.tensor(drafts, dtype=torch.int32))
        graph.replay()
        U.assert_attention(got, reference(c))


def test_offsets_beyond_32_bits(binding):
    """Heads and sequences more than 2^32 bytes apart."""
    D, S, H, B = 128, 70, 2, 2
    far = (1 << 31) + 4096                                      # elements between heads
    store = [torch.empty(3 * far + S * D, dtype=BF16, device=DEV) for _ in range(2)]
    K, V = (x.as_strided((B, H, S, D), (2 * far, far, D, 1)) for x in store)
    g = torch.Generator(device=DEV).manual_seed(3)
    for x in (K, V):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
    plan = binding.Plan(B, H, D, sink=0, lag=32, strides=(2 * far, far, D))
    Q = torch.randn((B, 2, 4, D), generator=g, device=DEV).to(BF16)
    seq = torch.tensor([70, 41], dtype=torch.int32, device=DEV)
    ws = plan.new_attend_workspace(2, 4)
    U.assert_attention(plan.attend_tree(Q, K, V, seq, ws, want_lse=True), U.tree_reference(Q, K, V, seq, [2, 2], None))
    # the same rows as pages far apart in one pool
    pool = [x.as_strided((4, 1, 32, D), (far, 0, D, 1)) for x in store]
    table = torch.tensor([[3, 0], [2, 1]], dtype=torch.int32, device=DEV)
    for i, x in enumerate(pool):
        x.copy_(torch.randn((4, 1, 32, D), generator=g, device=DEV))
    plan1 = binding.Plan(B, 1, D, sink=0, lag=32)
    q1 = Q[:, :, :2].contiguous()
    seq1 = torch.tensor([64, 33], dtype=torch.int32, device=DEV)
    got = plan1.attend_tree_paged(q1, store[0], store[1], table, seq1, ws, want_lse=True, strides=(far, 32 * D, D, 32), num_pages=4)
    dense = [x[table.long()].reshape(B, 1, 64, D) for x in pool]
    U.assert_attention(got, U.tree_reference(q1, *dense, seq1, [2, 2], None))


def test_large_logits_and_scales(binding):
    """Logits of hundreds, tiny and large scales: the running maximum moves at every tile."""
    c = case(binding, 2, 2, 4, 128, 400, 3, FP16, seed=12, lens=[400, 399])
    ramp = torch.linspace(0, 6, 400, device=DEV)[None, None, :, None]
    c["K"] = (c["K"].float().clamp(-3, 3) + ramp * c["Q"].float().mean((1, 2))[:, None, None, :].sign()).to(FP16)
    for scale in (1e-4, 0.5, 3.0):
        U.assert_attention(run(c, scale=scale), reference(c, scale))


# ------------------------------------------------------------------------------------------- commit
def commit_reference(K, V, lens, drafts, paths):
    K, V, out = U.bits(K).clone(), U.bits(V).clone(), []
    for b, path in enumerate(paths):
        base = lens[b] - drafts[b]
        rows = [base + p for p in path]
        for X in (K, V):
            X[b, :, base:base + len(path)] = X[b][:, rows].clone()
        out.append(base + len(path))
    return K, V, out


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D,T,H", [(64, 1, 1), (96, 5, 3), (128, 64, 8), (256, 33, 2)])
def test_commit_moves_the_accepted_path(binding, dtype, D, T, H):
    rng = random.Random(T)
    B, S = 6, 150
    drafts = [T, T, max(1, T // 2), 0, T, T]
    lens = [S, T, 100, 40, T + 17, 99]
    paths = [sorted(rng.sample(range(d), rng.randint(0, d))) for d in drafts]
    paths[0] = list(range(T))                                    # all accepted: nothing moves
    paths[1] = list(range(T // 2, T))
    g = torch.Generator(device=DEV).manual_seed(D)
    K, V, _, _ = U.make_cache((B, H, S, D), dtype, g)
    wantK, wantV, want_len = commit_reference(K, V, lens, drafts, paths)
    acc = torch.full((B, T), -5, dtype=torch.int32)
    for b, p in enumerate(paths):
        acc[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    plan = binding.Plan(B, H, D, sink=0, lag=32, dtype=dtype)
    ws = plan.new_workspace()
    page, nb = 16, 10
    perm = torch.randperm(B * nb, generator=torch.Generator().manual_seed(2)).view(B, nb).to(torch.int32).to(DEV)
    pools = [U.to_pages(x, page, perm, B * nb, 0.0) for x in (K, V)]
    seq, draft = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, drafts))
    seq2 = seq.clone()
    plan.tree_commit(K, V, seq, acc.to(DEV), n, ws, draft_len=draft)
    assert torch.equal(U.bits(K), wantK) and torch.equal(U.bits(V), wantV) and seq.tolist() == want_len
    plan.tree_commit_paged(*pools, perm, seq2, acc.to(DEV), n, ws, draft_len=draft)
    for pool, want in zip(pools, (wantK, wantV)):
        assert torch.equal(U.bits(U.from_pages(pool, perm, page))[:, :, :S], want)
    assert seq2.tolist() == want_len and plan.read_status(ws)[0] == 0


def test_commit_refuses_paths_that_are_none(binding):
    """Not ascending, outside the draft, too long, lengths that do not fit: untouched and recorded, others done."""
    B, H, S, D, T = 7, 2, 64, 64, 4
    K, V, _, _ = U.make_cache((B, H, S, D), BF16, torch.Generator(device=DEV).manual_seed(1))
    k0, v0 = K.clone(), V.clone()
    acc = torch.tensor([[2, 1, 0, 0], [0, 4, 0, 0], [-1, 0, 0, 0], [1, 1, 0, 0], [0, 1, 2, 3], [0, 1, 2, 3], [1, 3, 0, 0]], dtype=torch.int32, device=DEV)
    n = torch.tensor([2, 2, 1, 2, 5, 1, 2], dtype=torch.int32, device=DEV)
    seq = torch.tensor([30, 30, 30, 30, 30, 65, 30], dtype=torch.int32, device=DEV)
    plan = binding.Plan(B, H, D, sink=0, lag=32)
    ws = plan.new_workspace()
    plan.tree_commit(K, V, seq, acc, n, ws)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    assert seq.tolist() == [30, 30, 30, 30, 30, 65, 28]
    assert torch.equal(K[:6], k0[:6]) and torch.equal(V[:6], v0[:6])
    assert torch.equal(K[6, :, 26:28], k0[6][:, [27, 29]]) and torch.equal(V[6, :, 26:28], v0[6][:, [27, 29]])
    table = torch.tensor([[0, 1, 2, 3]] * B, dtype=torch.int32, device=DEV)
    table[:, 1] = 77                                              # the draft's page is not in the pool
    pool = torch.zeros((8, H, 16, D), dtype=BF16, device=DEV)
    seq = torch.full((B,), 30, dtype=torch.int32, device=DEV)
    plan.tree_commit_paged(pool, pool.clone(), table, seq, acc, torch.ones_like(n), ws)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL and seq.tolist() == [30] * B


# ------------------------------------------------------------------------------------------- refusals
def test_refusals_touch_nothing(binding):
    """Everything the host can see is refused with its status, before any launch."""
    import ctypes
    B, H, G, D, S, T = 2, 2, 4, 128, 64, 3
    c = case(binding, B, H, G, D, S, T, BF16, seed=1)
    plan, lib = c["plan"], c["plan"].lib
    out, lse = torch.full_like(c["Q"], 7), torch.full((B, T, H * G), 7.0, device=DEV)
    ptr = lambda t, off=0: None if t is None else ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731

    def call(q=None, Q=c["Q"], K=c["K"], V=c["V"], S_cap=S, seq=c["seq"], draft=c["draft"], mask=c["mask"], o=out, l=lse, ws=c["ws"],
             nbytes=None, off=None):
        off = off or {}
        query = dict(T=T, H_q=H * G, scale=0.0, k_scale=1.0, v_scale=1.0, stride_b=0, stride_t=0, stride_h=0)
        query.update(q or {})
        query = binding.lagkv_query(**query)
        return lib.lagkv_attend_tree(plan.handle, ctypes.byref(query), ptr(Q, off.get("Q", 0)), ptr(K, off.get("K", 0)), ptr(V), S_cap,
                                     ptr(seq, off.get("seq", 0)), ptr(draft), ptr(mask, off.get("mask", 0)), ptr(o), ptr(l), ptr(ws, off.get("ws", 0)),
                                     c["ws"].numel() if nbytes is None else nbytes, None)

    E = binding.LAGKV_EINVAL
    for q in (dict(T=0), dict(T=65), dict(H_q=H * G + 1), dict(H_q=1), dict(H_q=H * 65), dict(scale=-1.0), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(k_scale=-1.0), dict(v_scale=float("inf")), dict(stride_h=4), dict(stride_b=-8)):
        assert call(q) == E, q
    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(seq=None), dict(o=None), dict(S_cap=0), dict(S_cap=1 << 31), dict(o=c["Q"]),
               dict(off={"Q": 2}), dict(off={"K": 8}), dict(off={"seq": 2}), dict(off={"mask": 4}), dict(off={"ws": 16})):
        assert call(**kw) == E, kw
    assert call(ws=None) == binding.LAGKV_EWORKSPACE and call(nbytes=1024) == binding.LAGKV_EWORKSPACE
    assert call(nbytes=c["ws"].numel() // 2) == binding.LAGKV_EWORKSPACE
    torch.cuda.synchronize()
    assert (out == 7).all() and (lse == 7).all()
    with pytest.raises(TypeError):
        plan.attend_tree(c["Q"].float(), c["K"], c["V"], c["seq"], c["ws"])
    with pytest.raises(TypeError):
        plan.attend_tree(c["Q"], c["K"][:, :, ::2], c["V"][:, :, ::2], c["seq"], c["ws"])
    with pytest.raises(TypeError):
        plan.attend_tree(c["Q"], c["K"], c["V"], c["seq"].cpu(), c["ws"])
    with pytest.raises(TypeError):
        plan.attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], tree_mask=c["mask"][:, :2])
    pool, table = torch.zeros((4, H, 16, D), dtype=BF16, device=DEV), torch.zeros((B, 2), dtype=torch.int32, device=DEV)
    lay = lambda **kw: binding.lagkv_paged_layout(**{**dict(block_table=table.data_ptr(), max_blocks=2, page_size=16), **kw})  # noqa: E731
    query = binding.lagkv_query(T, H * G, 0.0, 1.0, 1.0, 0, 0, 0)
    for kw, pages in ((dict(page_size=8), 4), (dict(page_size=24), 4), (dict(max_blocks=0), 4), (dict(block_table=None), 4), ({}, 0),
                      (dict(stride_s=4), 4)):
        layout = lay(**kw)
        assert lib.lagkv_attend_tree_paged(plan.handle, ctypes.byref(query), ptr(c["Q"]), ptr(pool), ptr(pool), ctypes.byref(layout), pages,
                                           ptr(c["seq"]), None, None, ptr(out), None, ptr(c["ws"]), c["ws"].numel(), None) == E, kw
    acc, n = torch.zeros((B, T), dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    args = [plan.handle, ptr(c["K"]), ptr(c["V"]), S, ptr(c["seq"]), None, T, ptr(acc), ptr(n), ptr(c["ws"]), c["ws"].numel(), None]
    for i, bad in ((1, None), (2, args[1]), (3, 0), (4, None), (6, 0), (6, 65), (7, None), (8, None)):
        assert lib.lagkv_tree_commit(*(args[:i] + [bad] + args[i + 1:])) == E, i
    assert lib.lagkv_tree_commit(*(args[:10] + [128, None])) == binding.LAGKV_EWORKSPACE


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("T,G,page", [(12, 4, 16), (40, 4, 64), (20, 4, 128)])
def test_missing_pages_under_wide_trees(binding, dtype, T, G, page):
    """A page outside the pool, among the rows that everybody sees, with more query rows than one narrow unit."""
    B, H, D, S = 2, 1, 128, 640
    c = case(binding, B, H, G, D, S, T, dtype, seed=4, lens=[640, 513])
    nb = S // page
    perm = torch.randperm(B * nb, generator=torch.Generator().manual_seed(2)).view(B, nb).to(torch.int32).to(DEV)
    pools = [U.to_pages(c[x], page, perm, B * nb, 0.0) for x in "KV"]
    gone = [1, (S // 2) // page]
    table = perm.clone()
    table[0, gone[0]], table[1, gone[1]] = -1, B * nb
    got = c["plan"].attend_tree_paged(c["Q"], *pools, table, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True,
                                      k_scale=c["ks"], v_scale=c["vs"])
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    for b in range(B):
        keep = torch.tensor([r // page != gone[b] for r in range(S)], device=DEV)
        K, V = (U.bits(c[x])[b:b + 1][:, :, keep].view(dtype) for x in "KV")
        want = U.tree_reference(c["Q"][b:b + 1], K, V, [int(c["seq"][b]) - page], [T], c["mask"][b:b + 1], None, c["ks"], c["vs"])
        U.assert_attention({k: v[b:b + 1] for k, v in got.items()}, want)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_wide_trees_over_many_lengths(binding, dtype, D):
    """Lengths around the 128-row tiles, empty slots, units of one and two groups of query rows, ragged drafts."""
    for T, G in ((33, 1), (32, 4), (33, 4), (64, 4), (64, 7)):
        lens = [0, T, T + 1, 127 + T, 128, 129, 255, 256, 257, 640, 700]
        lens = [max(n, T) if n else 0 for n in lens]
        drafts = [0 if n == 0 else T - (i % 3) for i, n in enumerate(lens)]
        c = case(binding, len(lens), 2, G, D, 700, T, dtype, seed=T, lens=lens, drafts=drafts)
        poison(c)
        U.assert_attention(run(c), reference(c))


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("T,G", [(16, 4), (40, 4)])
def test_wide_trees_in_a_batch_of_short_sequences(binding, dtype, T, G):
    """Several units per CTA, of one tile and of several, in every order."""
    lens = [(40, 130, 300, 41, 129, 128, 500)[(i * i + i // 3) % 7] for i in range(300)]
    c = case(binding, 300, 2, G, 64, 500, T, dtype, seed=T, lens=lens)
    poison(c)
    U.assert_attention(run(c), reference(c))


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
def test_commit_of_a_batch_with_empty_slots(binding, paged):
    """Without draft_len an empty slot has no tokens, as for the attention: no error, nothing moves.  One that claims an
    accepted row is refused."""
    B, H, S, D, T = 4, 2, 64, 64, 4
    K, V, _, _ = U.make_cache((B, H, S, D), BF16, torch.Generator(device=DEV).manual_seed(1))
    lens, paths = [0, 30, 0, T], [[], [1, 3], [], [2]]
    wantK, wantV, want_len = commit_reference(K, V, lens, [0, T, 0, T], paths)
    acc = torch.zeros((B, T), dtype=torch.int32)
    for b, p in enumerate(paths):
        acc[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    acc, seq = acc.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    plan = binding.Plan(B, H, D, sink=0, lag=32)
    ws = plan.new_workspace()
    table = torch.arange(B * 4, dtype=torch.int32, device=DEV).view(B, 4)
    pools = [U.to_pages(x, 16, table, B * 4, 0.0) for x in (K, V)]
    table[0], table[2] = -1, -1

    def commit():
        if paged:
            plan.tree_commit_paged(*pools, table, seq, acc, n, ws)
        else:
            plan.tree_commit(K, V, seq, acc, n, ws)

    commit()
    assert plan.read_status(ws)[0] == 0 and seq.tolist() == want_len
    for b in (1, 3) if paged else range(B):
        for x, pool, want in zip((K, V), pools, (wantK, wantV)):
            got = U.from_pages(pool, table[b:b + 1], 16)[0] if paged else x[b]
            assert torch.equal(U.bits(got), want[b])
    n[0] = 1
    commit()
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL and int(seq[0]) == 0


def test_scales_at_the_ends_of_fp32(binding):
    """scale * k_scale * log2(e) above fp32 is refused, also where scale * k_scale alone is not; below it all rows weigh the same."""
    c = case(binding, 2, 2, 4, 128, 300, 3, BF16, seed=1)
    poison(c)
    for kw in (dict(scale=3e38), dict(scale=1e30, k_scale=2.5e8), dict(scale=1e30, k_scale=1e30), dict(v_scale=1e39)):
        with pytest.raises(binding.LagKVError) as e:
            c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"], **kw)
        assert e.value.code == binding.LAGKV_EINVAL
    for scale in (1e-37, 1e-45, 1e-60):
        U.assert_attention(run(c, scale=scale), reference(c, scale))
