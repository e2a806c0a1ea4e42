"""Attention over caches in 8 bits with block scales against a float64 statement (tests/quant_util.py)."""
import math
import random

import pytest
import torch

import quant_util as QU
import serve_util as U

pytestmark = pytest.mark.gpu

BF16, FP16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
DEV = "cuda:0"
KINDS = [("int8", BF16), ("e4m3", BF16), ("int8", FP16), ("e4m3", FP16)]
KIND_IDS = ["int8-bf16", "e4m3-bf16", "int8-fp16", "e4m3-fp16"]


@pytest.fixture(scope="module")
def binding():
    from paper_2504_04704_b200 import binding as b
    b.load_library()
    return b


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# Which kernel serves a call goes by the query rows and the capacity of the cache: small caches take units of 8 or 16 query rows,
# with this much room units of 16 and 32 and, from some 40 query rows on, the kernel on tensor memory take over (int8: two units of 128 rows
# in one from 129 rows on).
ROOM = 40000


def case(binding, kind, B, H, G, D, S, T, R, seed, lens=None, drafts=None, tree=True, spread=3.0, room=0):
    form, dtype = kind
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    K, V, ks, vs = QU.random_cache(B, H, S, D, form, R, g, spread)
    if room:  # more room behind the rows
        blocks, some = -(-room // R), ks.shape[2]
        store = torch.full((2, B, H, room, D), 0x7f, dtype=torch.uint8, device=DEV)
        scales = torch.full((2, B, H, blocks), float("nan"), device=DEV)
        for i, (x, s) in enumerate(((K, ks), (V, vs))):
            store[i, :, :, :S] = x.view(torch.uint8)
            scales[i, :, :, :some] = s
        K, V, ks, vs = store[0].view(K.dtype), store[1].view(K.dtype), scales[0], scales[1]
    lens = [rng.randint(T, S) for _ in range(B)] if lens is None else lens
    drafts = [min(T, n) for n in lens] if drafts is None else drafts
    c = dict(form=form, S=S, R=R, cache=binding.QuantCache(K, V, ks, vs, block_rows=R), lens=lens, drafts=drafts,
             Q=torch.randn((B, T, H * G, D), generator=g, device=DEV).to(dtype), seq=i32(lens), draft=i32(drafts),
             mask=U.random_tree(B, T, rng).to(DEV) if tree else None)
    c["plan"] = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    c["ws"] = c["plan"].new_attend_quant_workspace(T, H * G)
    return c


def poison(c):
    """Rows at and behind seq_len, and the scales of blocks without a row, hold what must never be used."""
    cache = c["cache"]
    for b, n in enumerate(c["lens"]):
        for x in (cache.K, cache.V):
            x.view(torch.uint8)[b, :, n:] = 0x7f if c["form"] == "e4m3" else 0x80
        for s in (cache.K_scale, cache.V_scale):
            s[b, :, -(-n // c["R"]):] = float("nan")


def run(c, **kw):
    got = c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True, **kw)
    assert c["plan"].read_status(c["ws"])[0] == 0
    return got


def reference(c, **kw):
    cache, R, S = c["cache"], c["R"], c["S"]
    K, V = (QU.row_values(x[:, :, :S], s[:, :, :-(-S // R)], R) for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))
    return QU.attention_reference(c["Q"], K, V, c["lens"], c["drafts"], c["mask"], form=c["form"],
                                  V_scale=cache.V_scale.nan_to_num(nan=0.0), **kw)


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("T,G,H,R", [(1, 4, 2, 16), (1, 7, 4, 64), (5, 1, 3, 32), (3, 5, 2, 128), (6, 5, 2, 32), (13, 4, 2, 64), (32, 4, 1, 16), (64, 8, 1, 64)])
@pytest.mark.parametrize("room", [0, ROOM])
def test_every_type_and_head_dim(binding, kind, D, T, G, H, R, room):
    c = case(binding, kind, 3, H, G, D, 333, T, R, seed=D + T, lens=[max(T, 100), 333, max(T, 257)], room=room)
    poison(c)
    QU.assert_attention(run(c), reference(c))


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("T,room", [(1, 0), (4, 0), (9, 8000), (40, 0), (20, 8000), (60, ROOM)])
def test_lengths_around_every_tile(binding, kind, T, room):
    """Empty sequences, sequences that are all draft, and every length next to a multiple of 16, 32 or 64."""
    lens = [0, T, T + 1, 15 + T, 16 + T, 17 + T, 31 + T, 32 + T, 63 + T, 64 + T, 65 + T, 128, 129, 200]
    c = case(binding, kind, len(lens), 2, 3, 128, 200, T, 32, seed=5, lens=lens, room=room)
    poison(c)
    got = run(c)
    QU.assert_attention(got, reference(c))
    assert not got["out"][0].any() and (got["lse"][0] == float("-inf")).all()


@pytest.mark.parametrize("kind", KINDS[:2], ids=KIND_IDS[:2])
def test_chain_without_lengths_and_masks(binding, kind):
    c = case(binding, kind, 4, 2, 4, 128, 300, 6, 64, seed=9, tree=False)
    got = c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"], want_lse=True)
    QU.assert_attention(got, reference(c))
    assert "lse" not in c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"])


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("T,room", [(1, 0), (9, 0), (64, 0), (7, ROOM), (20, ROOM), (64, ROOM)])
def test_padded_batch_and_rows_that_see_nothing(binding, kind, T, room):
    """Draft lengths from 0 on; tokens whose mask is empty in a cache without other rows."""
    drafts = [0, min(1, T), T // 2, T, T]
    lens = [50, 33, T // 2, T, 90 + T]              # sequences 2 and 3 are nothing but their draft
    c = case(binding, kind, 5, 2, 4, 128, 200, T, 16, seed=T, lens=lens, drafts=drafts, room=room)
    c["mask"][3, ::2] = 0
    c["mask"][4] = -1
    poison(c)
    got = run(c)
    QU.assert_attention(got, reference(c))
    assert not got["out"][0].any() and not got["out"][3, ::2].any() and torch.isneginf(got["lse"][3, 0]).all()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("T,G,room", [(7, 1, 0), (7, 2, 0), (40, 4, 0), (7, 4, ROOM), (40, 4, ROOM), (64, 4, ROOM)])
def test_hidden_drafted_rows_may_hold_nan(binding, dtype, D, T, G, room):
    """e4m3 NaN in drafted rows reaches the tokens that see them and no others."""
    c = case(binding, ("e4m3", dtype), 2, 2, G, D, 150, T, 16, seed=3, lens=[150, T], room=room)
    odd = [1, T - 2]
    bit = sum(1 << j for j in odd)
    m = c["mask"].cpu()
    for t in range(T):
        word = ((int(m[0, t]) & ~bit) | ((1 << t) if t in odd else 0)) & ((1 << 64) - 1)
        m[:, t] = word - (1 << 64) if word >> 63 else word
    c["mask"] = m.to(DEV)
    for b, n in enumerate(c["lens"]):
        for x in (c["cache"].K, c["cache"].V):
            x.view(torch.uint8)[b, :, n - T + 1, 3::5] = 0x7f
            x.view(torch.uint8)[b, :, n - T + T - 2, 1::7] = 0xff
    got = run(c)
    clean = [t for t in range(T) if t not in odd]
    out, lse, t_out, t_lse = reference(c)
    QU.assert_attention({"out": got["out"][:, clean], "lse": got["lse"][:, clean]}, (out[:, clean], lse[:, clean], t_out[:, clean], t_lse[:, clean]))
    assert torch.isnan(got["out"][:, odd]).any(-1).all()


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("T,G,room", [(1, 4, 0), (6, 4, 0), (6, 4, ROOM), (32, 4, ROOM), (64, 4, ROOM)])
@pytest.mark.parametrize("way", ["up", "down", "mixed", "zeros"])
def test_scales_far_apart(binding, kind, T, G, room, way):
    """V scales that climb by 2^40 in the order of the rows, fall, or lie anywhere; blocks whose scales are 0."""
    c = case(binding, kind, 2, 2, G, 128, 640, T, 16, seed=T, lens=[640, 613], room=room)
    cache = c["cache"]
    e = torch.linspace(-20, 20, 640 // 16, device=DEV)
    if way == "zeros":
        cache.K_scale[:, :, 3::5] = 0
        cache.V_scale[:, :, ::3] = 0
        cache.V_scale[:, 1] = 0
    else:
        e = e if way == "up" else e.flip(0) if way == "down" else e[torch.randperm(len(e), generator=torch.Generator().manual_seed(1)).to(DEV)]
        cache.V_scale[:, :, :640 // 16].mul_(torch.exp2(e))
    got = run(c)
    QU.assert_attention(got, reference(c))
    if way == "zeros":
        assert not got["out"][:, :, G:].any()


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("T,G,room", [(1, 4, 0), (5, 7, 0), (4, 7, ROOM), (24, 4, ROOM), (33, 4, ROOM)])
@pytest.mark.parametrize("cap", [0.5, 30.0, 1e5])
def test_capped_logits(binding, kind, T, G, room, cap):
    """A cap far below the logits, near them, and far above (where it must not lose them)."""
    c = case(binding, kind, 2, 2, G, 128, 500, T, 64, seed=2, lens=[500, 333], room=room)
    poison(c)
    QU.assert_attention(run(c, cap=cap), reference(c, cap=cap))


@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("T,G,cap", [(5, 7, 30.0), (5, 7, 4.0), (64, 4, 10.0)])
def test_capped_logits_of_every_head_dim(binding, kind, D, T, G, cap):
    """Long ragged caches whose logits lie on both sides of the cap, within warps and among them."""
    c = case(binding, kind, 2, 1, G, D, 5000, T, 32, seed=3, lens=[5000, 3777], spread=2.0, room=2 * ROOM if T > 5 else 0)
    QU.assert_attention(run(c, cap=cap), reference(c, cap=cap))


@pytest.mark.parametrize("kind", KINDS[:2], ids=KIND_IDS[:2])
@pytest.mark.parametrize("T,G,room", [(1, 4, 0), (12, 4, 0), (5, 4, 2 * ROOM), (12, 4, 2 * ROOM), (40, 4, 2 * ROOM)])
def test_factors_and_large_logits(binding, kind, T, G, room):
    """scale, k_scale and v_scale; logits in the hundreds, whose largest comes late."""
    c = case(binding, kind, 2, 1, G, 128, 300, T, 32, seed=11, lens=[300, 299], room=room)
    c["cache"].K_scale[:, :, 8:10] *= 16
    got = run(c, scale=0.5, k_scale=2.0, v_scale=0.25)
    QU.assert_attention(got, reference(c, scale=1.0, v_scale=0.25))


@pytest.mark.parametrize("kind", KINDS[:2], ids=KIND_IDS[:2])
@pytest.mark.parametrize("T,room", [(3, 0), (15, 2 * ROOM)])
def test_queries_at_the_ends_of_their_type(binding, kind, T, room):
    """Rows of queries of very different size keep their own factor; zero rows attend evenly."""
    c = case(binding, kind, 1, 2, 4, 128, 200, T, 64, seed=12, lens=[200], room=room)
    c["Q"] *= torch.exp2(torch.linspace(-100, 3, 8 * T, device=DEV)).view(1, T, 8, 1).to(BF16)
    c["Q"][0, 0, 0] = 0
    QU.assert_attention(run(c), reference(c))


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("T,G,room", [(1, 7, 0), (4, 4, 0), (4, 4, ROOM), (7, 4, ROOM), (20, 4, ROOM), (40, 4, ROOM)])
@pytest.mark.parametrize("page,R", [(16, 16), (32, 16), (64, 64), (128, 32), (256, 128)])
def test_pages(binding, form, T, G, room, page, R):
    """Random pages; a table entry outside the pool counts as rows that nobody sees."""
    B, H, D, S = 3, 2, 128, 512
    room = room // page * page
    c = case(binding, (form, BF16), B, H, G, D, S, T, R, seed=page + T, lens=[S, 250 + T, T], room=room)
    nb = S // page
    pages = B * nb + 2
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    cache = c["cache"]
    pool = binding.QuantCache(*(QU.pool_of(x[:, :, :S].contiguous(), page, table, pages) for x in (cache.K, cache.V)), cache.K_scale, cache.V_scale, block_rows=R)
    if room:  # entries of blocks that no sequence reaches
        table = torch.cat([table, torch.full((B, room // page - nb), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    call = lambda tab: c["plan"].attend_quant_paged(c["Q"], pool, tab, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)  # noqa: E731
    got = call(table)
    assert c["plan"].read_status(c["ws"])[0] == 0
    QU.assert_attention(got, reference(c))
    flat = run(c)
    assert torch.equal(flat["out"], got["out"]) and torch.equal(flat["lse"], got["lse"])
    # the second page of sequence 0 is gone: as a cache in which those rows are hidden
    bad = table.clone()
    bad[0, 1], bad[2, nb - 1] = -1, pages                          # the last page of sequence 2 is behind its rows
    lost = call(bad)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    assert torch.equal(lost["out"][1:], got["out"][1:])
    K, V = (QU.row_values(x[:1, :, :S], s[:1, :, :S // R], R) for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))
    want = QU.attention_reference(c["Q"][:1], K, V, [S], [c["drafts"][0]], c["mask"][:1], form=form, V_scale=cache.V_scale[:1].nan_to_num(nan=0.0),
                                  gone=slice(page, 2 * page))
    QU.assert_attention({"out": lost["out"][:1], "lse": lost["lse"][:1]}, want)


def test_strides_of_queries_and_cache(binding):
    """Queries and caches as projections leave them: tokens first, padded rows."""
    B, H, G, D, S, T, R = 2, 4, 2, 96, 210, 3, 32
    c = case(binding, ("int8", BF16), B, H, G, D, S, T, R, seed=1, lens=[210, 100])
    want = reference(c)
    cache = c["cache"]
    K, V = (torch.zeros((B, S, H, D + 16), dtype=torch.int8, device=DEV)[..., :D].transpose(1, 2).copy_(x) for x in (cache.K, cache.V))
    c["cache"] = binding.QuantCache(K, V, cache.K_scale, cache.V_scale, block_rows=R)
    c["Q"] = torch.zeros((B, T, H * G, D + 8), dtype=BF16, device=DEV)[..., :D].copy_(c["Q"])
    QU.assert_attention(run(c), want)


def test_refusals(binding):
    """What does not fit is refused with nothing launched."""
    c = case(binding, ("int8", BF16), 2, 2, 4, 128, 128, 2, 32, seed=1, lens=[128, 100])
    plan, cache, ws = c["plan"], c["cache"], c["ws"]
    for cap in (-1.0, float("nan"), float("inf"), 1e-40):
        with pytest.raises(binding.LagKVError):
            plan.attend_quant(c["Q"], cache, c["seq"], ws, cap=cap)
    for kw in (dict(scale=-1.0), dict(k_scale=float("inf")), dict(v_scale=-2.0)):
        with pytest.raises(binding.LagKVError):
            plan.attend_quant(c["Q"], cache, c["seq"], ws, **kw)
    for rows in (8, 48, 256, 16):                                   # 16: too few blocks for the rows
        with pytest.raises(binding.LagKVError):
            plan.attend_quant(c["Q"], binding.QuantCache(cache.K, cache.V, cache.K_scale, cache.V_scale, block_rows=rows), c["seq"], ws)
    with pytest.raises(binding.LagKVError):
        plan.attend_quant(c["Q"], binding.QuantCache(cache.K, cache.K, cache.K_scale, cache.V_scale, block_rows=32), c["seq"], ws)
    with pytest.raises(binding.LagKVError) as e:
        plan.attend_quant(c["Q"], cache, c["seq"], ws[:4096])
    assert e.value.code == binding.LAGKV_EWORKSPACE
    with pytest.raises(TypeError):
        plan.attend_quant(c["Q"].half(), cache, c["seq"], ws)
    with pytest.raises(TypeError):
        plan.attend_quant(c["Q"], cache, c["seq"].long(), ws)
    fp8 = binding.Plan(2, 2, 128, sink=4, lag=64, dtype=FP8)
    with pytest.raises(binding.LagKVError) as e:
        fp8.attend_quant(c["Q"], cache, c["seq"], ws)
    assert e.value.code == binding.LAGKV_EUNSUPPORTED
    x = torch.zeros((2, 2, 5, 128), dtype=BF16, device=DEV)
    fw = plan.new_workspace()
    with pytest.raises(TypeError):
        plan.quant_write(cache, x, x[:, :, :3], c["seq"], fw)
    with pytest.raises(TypeError):
        plan.quant_write(cache, x, x, c["seq"], fw, take=torch.zeros((2, 3, 4), dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        plan.quant_read(cache, c["seq"], fw)
    with pytest.raises(binding.LagKVError):
        plan.quant_read(cache, c["seq"], fw, from_len=c["seq"], idx=torch.zeros((2, 2, 3), dtype=torch.int32, device=DEV))
    out = torch.zeros((2, 2, 128, 128), dtype=BF16, device=DEV)
    with pytest.raises(binding.LagKVError):
        plan.quant_read(cache, c["seq"], fw, K_out=out, V_out=out)
    assert plan.read_status(fw)[0] == 0 and plan.read_status(ws)[0] == 0


def test_bad_lengths_are_recorded(binding):
    """A sequence whose lengths do not describe the cache counts as without tokens; the others get theirs."""
    c = case(binding, ("e4m3", BF16), 5, 2, 4, 128, 128, 3, 32, seed=1, lens=[128, 100, 90, 80, 70])
    want = reference(c)
    c["seq"].copy_(i32([129, 100, -1, 80, 2]))
    c["draft"].copy_(i32([3, 4, 3, 3, 3]))
    got = c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    QU.assert_attention({k: v[3:4] for k, v in got.items()}, tuple(w[3:4] for w in want))
    for b in (0, 1, 2, 4):
        assert not got["out"][b].any() and torch.isneginf(got["lse"][b]).all()


@pytest.mark.parametrize("kind", KINDS[:2], ids=KIND_IDS[:2])
@pytest.mark.parametrize("T,G,room", [(1, 4, 0), (4, 8, ROOM), (16, 8, ROOM), (64, 4, ROOM)])
def test_graph_replay_and_repeats(binding, kind, T, G, room):
    """One captured call serves every length, and the same call gives the same bits; on another stream, too."""
    c = case(binding, kind, 3, 2, G, 128, 3000, T, 64, seed=4, lens=[3000, 1700, T], room=room)
    first = run(c)
    again = run(c)
    assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])
    out = torch.empty_like(c["Q"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], out=out)
    torch.cuda.current_stream().wait_stream(side)
    for lens in ([3000, 1700, T], [0, 64 + T, 2999], [T, T, T]):
        c["lens"], c["drafts"] = lens, [min(T, n) for n in lens]
        c["seq"].copy_(i32(lens))
        c["draft"].copy_(i32(c["drafts"]))
        graph.replay()
        QU.assert_attention({"out": out}, reference(c))


@pytest.mark.parametrize("T", [2, 40])
def test_two_calls_at_once_with_their_own_workspaces(binding, T):
    c = case(binding, ("int8", BF16), 2, 4, 4, 128, 4096, T, 64, seed=7, lens=[4096, 4000], room=20000)
    want = run(c)
    other = c["plan"].new_attend_quant_workspace(T, 16)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for st, ws in zip(streams, (c["ws"], other)):
            with torch.cuda.stream(st):
                got.append(c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], ws, draft_len=c["draft"], tree_mask=c["mask"], want_lse=True))
    torch.cuda.synchronize()
    for x in got:
        assert torch.equal(x["out"], want["out"]) and torch.equal(x["lse"], want["lse"])


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("T,G", [(1, 4), (2, 16), (16, 4)])
def test_a_long_cache(binding, form, T, G):
    """Offsets behind 2^32 bytes: only the last rows have large logits, the others weigh evenly."""
    D, S, R = 128, (1 << 25) + (1 << 24), 128
    plan = binding.Plan(1, 1, D, sink=4, lag=64)
    cache, ws = plan.new_quant_cache(S, form, block_rows=R), plan.new_attend_quant_workspace(T, G)
    n, tail = S - 5, 300
    g = torch.Generator(device=DEV).manual_seed(1)
    kt, vt, kst, vst = QU.random_cache(1, 1, tail + (n - tail) % R, D, form, R, g)
    lo = (n - tail) // R * R
    for x, s, xt, st in ((cache.K, cache.K_scale, kt, kst), (cache.V, cache.V_scale, vt, vst)):
        x.view(torch.uint8)[:, :, lo:n] = xt.view(torch.uint8)
        s[:, :, lo // R:lo // R + st.shape[2]] = st
    Q = torch.randn((1, T, G, D), generator=g, device=DEV).to(BF16) * 3
    got = plan.attend_quant(Q, cache, i32([n]), ws, want_lse=True)
    assert plan.read_status(ws)[0] == 0
    k, v = QU.row_values(kt, kst, R)[0, 0], QU.row_values(vt, vst, R)[0, 0]
    z = (Q[0].double().reshape(T * G, D) @ k.T) / math.sqrt(D)
    seen = U.tree_seen(None, T, T, len(k)).to(DEV).repeat_interleave(G, 0)
    z = torch.where(seen, z, -math.inf)
    p = torch.exp(z)
    total = p.sum(-1, keepdim=True) + lo                           # lo rows of zeros: logit 0, value 0
    out = (p @ v) / total
    # the rounding of probabilities and of the output; sums of positive fp32 terms, per thread and tile some S / 64 of them, then joined
    tol = (p @ v.abs()) / total * (2.0 ** -11 + 2.0 ** -17 + S * 2.0 ** -30) + out.abs() * 2.0 ** -8 + S * 2.0 ** -32 * float(v.abs().max()) / total
    assert ((got["out"][0].reshape(T * G, D).double() - out).abs() <= tol).all()
    assert ((got["lse"][0].reshape(-1).double() - torch.log(total[:, 0])).abs() <= S * 2.0 ** -30 + 2.0 ** -17).all()


def read_back(plan, cache, seq, ws, S, dtype):
    out = torch.zeros((2,) + cache.K.shape[:2] + (S, cache.K.shape[3]), dtype=dtype, device=DEV)
    plan.quant_read(cache, seq, ws, K_out=out[0], V_out=out[1])
    return out


@pytest.mark.parametrize("form,dtype", [("int8", BF16), ("e4m3", FP16)], ids=["int8", "e4m3"])
def test_a_sequence_from_prompt_to_compression(binding, form, dtype):
    """The compress pass picks rows of a raw cache, which go to 8 bits directly; decode steps write and attend; a draft is written, its
    accepted path kept by a list; then the window is read back, compressed in place and written again."""
    B, H, G, D, L, sink, R, S0 = 2, 2, 4, 128, 64, 16, 32, 16 + 6 * 64 + 20
    g = torch.Generator(device=DEV).manual_seed(5)
    raw = torch.randn((2, B, H, S0, D), generator=g, device=DEV).to(dtype)
    plan = binding.Plan(B, H, D, sink=sink, lag=L, keep_ratio=0.25, dtype=dtype)
    ws, aws = plan.new_workspace(4), plan.new_attend_quant_workspace(8, H * G)
    picked = plan.compress_prefill(raw[0], raw[1], ws, want_rows=True)
    n, cap = picked["L_R"], 400
    cache = plan.new_quant_cache(cap, form, block_rows=R)
    seq = i32([n] * B)
    plan.quant_write(cache, raw[0], raw[1], seq, ws, take=picked["idx"])
    whole = plan.new_quant_cache(cap, form, block_rows=R)
    plan.quant_write(whole, picked["K_out"], picked["V_out"], seq, ws, at_positions=True)
    for a, b in ((cache.K, whole.K), (cache.V, whole.V)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(cache.K_scale, whole.K_scale) and torch.equal(cache.V_scale, whole.V_scale)

    def check(Q, lens, drafts, mask):
        got = plan.attend_quant(Q, cache, seq, aws, draft_len=i32(drafts), tree_mask=mask, want_lse=True)
        K, V = (QU.row_values(x, s, R) for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))
        QU.assert_attention(got, QU.attention_reference(Q, K, V, lens, drafts, mask, form=form, V_scale=cache.V_scale))

    fresh = lambda t: torch.randn((2, B, H, t, D), generator=g, device=DEV).to(dtype)  # noqa: E731
    queries = lambda t: torch.randn((B, t, H * G, D), generator=g, device=DEV).to(dtype)  # noqa: E731
    for _ in range(5):                                             # decode steps
        new, old = fresh(1), seq.clone()
        seq += 1
        plan.quant_write(cache, new[0], new[1], seq, ws, from_len=old)
        n += 1
        check(queries(1), [n] * B, [1] * B, None)
    new, old = fresh(6), seq.clone()                               # a draft of six, of which tokens 0, 2, 5 and 1 are kept
    seq += 6
    plan.quant_write(cache, new[0], new[1], seq, ws, from_len=old)
    check(queries(6), [n + 6] * B, [6] * B, U.random_tree(B, 6, random.Random(1)).to(DEV))
    seq.copy_(old + i32([3, 1]))
    plan.quant_write(cache, new[0], new[1], seq, ws, from_len=old, take=i32([[0, 2, 5, 0], [1, 0, 0, 0]]))
    got = read_back(plan, cache, seq, ws, cap, dtype)
    path = torch.stack([new[0][0][:, [0, 2, 5]], new[1][0][:, [0, 2, 5]]]).double()
    kept = got[:, 0, :, n:n + 3].double()
    steps = torch.stack([t[0, :, n // R:-(-(n + 3) // R)].amax(-1) for t in (cache.K_scale, cache.V_scale)])[..., None, None].double()
    # int8: half a step, the scale; e4m3: half a step of 2^-3, and of its subnormals; then 16 bits
    bound = steps / 2 if form == "int8" else path.abs() * 2.0 ** -4 + steps * 2.0 ** -10
    assert ((kept - path).abs() <= bound + path.abs() * torch.finfo(dtype).eps).all()
    lens = seq.tolist()
    check(queries(2), lens, [1, 1], None)
    # the window grows to two lags, is read back, compressed in place and written behind the rows that stay
    static = i32([sink + 5 * plan.k] * B)
    more = fresh(2 * L)
    old = seq.clone()
    seq += 2 * L
    plan.quant_write(cache, more[0], more[1], seq, ws, from_len=old)
    full = read_back(plan, cache, seq, ws, cap, dtype)
    before, static0 = full.clone(), static.clone()
    lens0 = seq.tolist()
    plan.compress_append(full[0], full[1], seq, static, ws, max_new_chunks=4)
    assert (seq < i32(lens0)).all() and (static > static0).all()
    plan.quant_write(cache, full[0], full[1], seq, ws, from_len=static0, at_positions=True)
    assert plan.read_status(ws)[0] == 0
    again = read_back(plan, cache, seq, ws, cap, dtype)
    for b, m in enumerate(seq.tolist()):
        s = int(static0[b])
        # rows below the static part are what they were, but for those that share its last block with new rows
        assert torch.equal(again[:, b, :, :s // R * R], before[:, b, :, :s // R * R])
        far = (again[:, b, :, s:m].double() - full[:, b, :, s:m].double()).abs()
        scale = torch.stack([cache.K_scale[b], cache.V_scale[b]]).double().repeat_interleave(R, -1)[:, :, s:m, None]
        x = full[:, b, :, s:m].double().abs()
        bound = scale / 2 if form == "int8" else x * 2.0 ** -4 + scale * 2.0 ** -10
        assert (far <= bound + x * torch.finfo(dtype).eps).all()
    check(queries(3), seq.tolist(), [3, 3], None)


def test_forked_pages_with_their_scales(binding):
    """Pools of codes are forked by a plan of 8-bit format; scales follow the sequences."""
    B, H, G, D, page, R, S = 3, 2, 4, 128, 32, 32, 192
    g = torch.Generator(device=DEV).manual_seed(9)
    plan, pager = binding.Plan(B, H, D, sink=4, lag=64), binding.Plan(B, H, D, sink=4, lag=64, dtype=FP8)
    nb, pages = S // page, 20
    cache = plan.new_quant_cache(S, "int8", block_rows=R, num_pages=pages, page_size=page)
    table, refs = torch.full((B, nb), -1, dtype=torch.int32, device=DEV), torch.zeros(pages, dtype=torch.int32, device=DEV)
    ws, pws, aws = plan.new_workspace(), pager.new_pages_workspace(pages), plan.new_attend_quant_workspace(1, H * G)
    seq, static = i32([150, 0, 70]), i32([100, 0, 70])
    pager.pages_reserve(table, refs, seq, pws, page)
    x = torch.randn((2, B, H, 150, D), generator=g, device=DEV).to(BF16)
    plan.quant_write_paged(cache, table, x[0], x[1], seq, ws)
    pool = [t.view(FP8) for t in (cache.K, cache.V)]
    pager.pages_fork(pool[0], pool[1], table, refs, seq, static, i32([0]), i32([1]), pws)
    for s in (cache.K_scale, cache.V_scale):
        s[1] = s[0]
    # both go on on their own
    old = seq.clone()
    seq += i32([1, 2, 1])
    pager.pages_reserve(table, refs, seq, pws, page)
    y = torch.randn((2, B, H, 2, D), generator=g, device=DEV).to(BF16) * 3
    plan.quant_write_paged(cache, table, y[0], y[1], seq, ws, from_len=old)
    Q = torch.randn((B, 1, H * G, D), generator=g, device=DEV).to(BF16)
    got = plan.attend_quant_paged(Q, cache, table, seq, aws, want_lse=True)
    assert plan.read_status(ws)[0] == 0 and plan.read_status(aws)[0] == 0 and pager.read_status(pws)[0] == 0
    K, V = (QU.row_values(QU.dense_of(t, table, page), s, R) for t, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))
    QU.assert_attention(got, QU.attention_reference(Q, K, V, seq.tolist(), [1] * B, None, V_scale=cache.V_scale))
    assert (table[0, :3] == table[1, :3]).all() and table[0, 4] != table[1, 4]
    both = torch.cat([x[0, 0], y[0, 0, :, :1]], 1), torch.cat([x[0, 0], y[0, 1]], 1)
    for b, rows in enumerate(both):
        off = (K[b, :, :rows.shape[1]] - rows.double()).abs()
        assert (off <= cache.K_scale[b].double().repeat_interleave(R, -1)[:, :rows.shape[1], None] * 1.01).all()


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nb", [4, 512])
def test_many_short_units_of_many_query_rows(binding, form, D, nb):
    """Units of one or two tiles one behind the other in a CTA, whose query rows differ in size: each keeps its own factors."""
    B, H, G, T, page, R = 96, 6, 4, 40, 64, 64
    rng = random.Random(nb)
    lens = [rng.choice([40, 100, 128, 129, 200, 256]) for _ in range(B)]
    c = case(binding, (form, BF16), B, H, G, D, 256, T, R, seed=D + nb, lens=lens, spread=1.0)
    c["Q"] *= torch.exp2(-torch.randint(0, 12, (B, T, H * G, 1), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).float()).to(BF16)
    want = reference(c)
    cache, pages = c["cache"], B * 4
    used = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).view(B, 4).to(torch.int32).to(DEV)
    table = torch.full((B, nb), -1, dtype=torch.int32, device=DEV)
    table[:, :4] = used
    scales = torch.full((2, B, H, nb), float("nan"), device=DEV)
    scales[0, :, :, :4], scales[1, :, :, :4] = cache.K_scale, cache.V_scale
    paged = binding.QuantCache(QU.pool_of(cache.K, page, used, pages), QU.pool_of(cache.V, page, used, pages), scales[0], scales[1], block_rows=R)
    first = None
    for _ in range(5):
        got = c["plan"].attend_quant_paged(c["Q"], paged, table, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)
        assert c["plan"].read_status(c["ws"])[0] == 0
        first = first or got
        assert torch.equal(got["out"], first["out"]) and torch.equal(got["lse"], first["lse"])
    QU.assert_attention(first, want)
