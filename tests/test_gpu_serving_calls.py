"""Calls of the attention operators that overlap, repeat or share: streams, graphs, workspaces, views."""
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


def make(binding, B, H, G, D, S, T, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    K, V, ks, vs = U.make_cache((B, H, S, D), dtype, g)
    Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(U.out_dtype(dtype))
    seq = torch.tensor([S - 37 * i for i in range(B)], dtype=torch.int32, device=DEV)
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    ws = plan.new_attend_workspace(T, H * G, -(-S // 64), 8)
    bounds = plan.new_block_bounds(S, 64)
    plan.block_bounds(K, seq, bounds, ws)
    return dict(K=K, V=V, Q=Q, ks=ks, vs=vs, seq=seq, plan=plan, ws=ws, bounds=bounds)


def tree(c, ws=None, out=None):
    return c["plan"].attend_tree(c["Q"], c["K"], c["V"], c["seq"], c["ws"] if ws is None else ws, k_scale=c["ks"], v_scale=c["vs"],
                                 want_lse=True, out=out)


def blocks(c, ws=None, out=None):
    return c["plan"].attend_blocks(c["Q"], c["K"], c["V"], c["seq"], c["bounds"], c["ws"] if ws is None else ws, keep=8,
                                   k_scale=c["ks"], v_scale=c["vs"], want_lse=True, out=out)


def same(a, b):
    return torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


SHAPES = [(1, 1, 4, 128, 9000, 1), (3, 2, 4, 64, 700, 5), (2, 2, 4, 128, 1500, 20), (2, 1, 4, 96, 900, 40)]


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("B,H,G,D,S,T", SHAPES)
def test_the_same_call_gives_the_same_bits(binding, dtype, B, H, G, D, S, T):
    c = make(binding, B, H, G, D, S, T, dtype, 1)
    first = tree(c), blocks(c)
    U.assert_attention(first[0], U.tree_reference(c["Q"], c["K"], c["V"], c["seq"], torch.full_like(c["seq"], T), None, None, c["ks"], c["vs"]))
    for _ in range(5):
        assert same(tree(c), first[0]) and same(blocks(c), first[1])
    c["ws"][4096:].fill_(0xA5)                      # what a call leaves behind its status block is of no use to the next
    assert same(tree(c), first[0]) and same(blocks(c), first[1])
    assert c["plan"].read_status(c["ws"])[0] == 0


@pytest.mark.parametrize("B,H,G,D,S,T", SHAPES)
def test_two_streams_with_workspaces_of_their_own(binding, B, H, G, D, S, T):
    cases = [make(binding, B, H, G, D, S, T, BF16, seed) for seed in (2, 3)]
    want = [(tree(c), blocks(c)) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append((tree(c), blocks(c)))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(same(t, want[i][0]) and same(b, want[i][1]) for t, b in got[i])


@pytest.mark.parametrize("B,H,G,D,S,T", SHAPES)
def test_two_graphs_share_a_workspace_one_after_the_other(binding, B, H, G, D, S, T):
    a = make(binding, B, H, G, D, S, T, BF16, 4)
    b = make(binding, B, H, G, D, S // 2, max(1, T // 2), BF16, 5)
    want = tree(a), blocks(a), tree(b), blocks(b)
    outs = [{k: torch.zeros_like(v) for k, v in w.items()} for w in want]
    graphs = []
    for c, i in ((a, 0), (b, 2)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs[i], outs[i + 1] = tree(c, a["ws"]), blocks(c, a["ws"])
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for o in outs:
            o["out"].fill_(9)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))
    assert a["plan"].read_status(a["ws"])[0] == 0


def test_queries_as_views(binding):
    """A view with strides is read as it is; one that repeats elements, or a workspace elsewhere, is refused."""
    c = make(binding, 2, 2, 4, 128, 300, 3, BF16, 6)
    want = tree(c)
    wide = torch.zeros((2, 3, 8, 256), dtype=BF16, device=DEV)
    wide[..., :128] = c["Q"]
    assert same(tree({**c, "Q": wide[..., :128]}), want)
    for shape, view in (((2, 1, 8, 128), c["Q"][:, :1].expand(2, 3, 8, 128)), ((1,), c["Q"][:1, :1, :1].expand(2, 3, 8, 128)),
                        ((2,), c["Q"][:, :, :1].expand(2, 3, 8, 128))):
        with pytest.raises(TypeError):
            tree({**c, "Q": view})
        with pytest.raises(TypeError):
            blocks({**c, "Q": view})
    for ws in (c["ws"].cpu(), c["ws"][::2]):
        with pytest.raises(TypeError):
            tree(c, ws)
        with pytest.raises(TypeError):
            blocks(c, ws)
        with pytest.raises(TypeError):
            c["plan"].block_bounds(c["K"], c["seq"], c["bounds"], ws)
    pool, table = torch.zeros((4, 2, 16, 128), dtype=BF16, device=DEV), torch.zeros((2, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError):
        c["plan"].attend_tree_paged(c["Q"], pool, pool.clone(), table, c["seq"], c["ws"], strides=(2 * 16 * 128, 16 * 128, 128, 16), num_pages=5)
    assert c["plan"].read_status(c["ws"])[0] == 0


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_the_most_query_rows(binding, dtype, D):
    """64 tokens of 64 query heads per KV head, over a cache that is hardly longer; the blocks of 2 tokens of them."""
    c = make(binding, 2, 1, 64, D, 190, 64, dtype, 7)
    U.assert_attention(tree(c), U.tree_reference(c["Q"], c["K"], c["V"], c["seq"], torch.full_like(c["seq"], 64), None, None, c["ks"], c["vs"]))
    c = make(binding, 2, 1, 64, D, 190, 2, dtype, 8)                # all blocks kept: dense attention
    want = U.tree_reference(c["Q"], c["K"], c["V"], c["seq"], torch.full_like(c["seq"], 2), None, None, c["ks"], c["vs"])
    U.assert_attention(tree(c), want)
    U.assert_attention(blocks(c), want)
    assert c["plan"].read_status(c["ws"])[0] == 0


@pytest.mark.parametrize("dtype,D,T,G", [(BF16, 64, 5, 4), (FP16, 96, 4, 8), (BF16, 128, 17, 1), (FP8, 64, 8, 4)], ids=str)
def test_large_capacities(binding, dtype, D, T, G):
    """Half a million rows of capacity, most of them unused or all of them used, under 17 to 32 query rows."""
    c = make(binding, 2, 1, G, D, 1 << 18, T, dtype, 9)
    for lens in ([1 << 18, 37], [3000, T], [0, 100000]):
        c["seq"].copy_(torch.tensor(lens, dtype=torch.int32))
        draft = torch.tensor([min(T, n) for n in lens], dtype=torch.int32, device=DEV)
        want = U.tree_reference(c["Q"], c["K"], c["V"], c["seq"], draft, None, None, c["ks"], c["vs"])
        U.assert_attention(tree(c), want)
        page = 64
        table = torch.randperm(2 << 12, generator=torch.Generator().manual_seed(3)).view(2, -1).to(torch.int32).to(DEV)
        pools = [U.to_pages(x, page, table, 2 << 12, 0.0) for x in (c["K"], c["V"])]
        got = c["plan"].attend_tree_paged(c["Q"], *pools, table, c["seq"], c["ws"], k_scale=c["ks"], v_scale=c["vs"], want_lse=True)
        U.assert_attention(got, want)
    assert c["plan"].read_status(c["ws"])[0] == 0


def test_choices_of_one_workspace_in_turn(binding):
    """Calls back to back on one workspace, each with another choice in the same place: none sees the other's."""
    a = make(binding, 3, 2, 4, 64, 4000, 2, BF16, 10)
    b = {**a, "Q": -a["Q"], "seq": a["seq"] - 900}
    want = [blocks(c) for c in (a, b)]
    assert not same(*want)
    got = [(blocks(a), blocks(b)) for _ in range(50)]
    assert all(same(g[i], want[i]) for g in got for i in (0, 1))
    assert a["plan"].read_status(a["ws"])[0] == 0
