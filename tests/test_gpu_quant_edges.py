"""Caches in 8 bits with block scales: calls at the edges of what the header promises, every kernel family at odd layouts."""
import pytest
import torch

import quant_util as QU
import test_gpu_quant_attention as A
import test_gpu_quant_cache as W
from test_gpu_quant_attention import BF16, DEV, FP16, ROOM, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2504_04704_b200 import binding as b
    b.load_library()
    return b


def room_of(heads):
    """Capacity from which int8 calls of more than 128 query rows to a KV head take units of 256."""
    return (1600000 // heads // 256 + 1) * 256


@pytest.mark.parametrize("bad", [-1, -2, -3, -2 ** 31, 40, 2 ** 31 - 1])
def test_every_entry_outside_the_source_is_recorded(binding, bad):
    """Whatever number it is: recorded, and its row is 0."""
    D, R, T, n = 64, 32, 40, 50
    g, K, V, ks, vs = W.start_state(1, 2, 64, D, "int8", R, seed=1)
    x = torch.randn((2, 1, 2, T, D), generator=g, device=DEV).to(BF16)
    plan, cache = binding.Plan(1, 2, D, sink=4, lag=64), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    take = torch.randint(0, T - 1, (1, n), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    pick = take.clone()
    take[0, 7], pick[0, 7] = bad, T - 1
    clean = x.clone()
    clean[:, :, :, T - 1] = 0                                      # the statement's stand-in for a row that is not there
    want = W.expected(K, V, ks, vs, clean[0], clean[1], [3], [3 + n], R, "int8", lambda b, h, i: int(pick[0, i]))
    plan.quant_write(cache, x[0], x[1], i32([3 + n]), ws, from_len=i32([3]), take=take.to(DEV))
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    W.same(cache, want)
    assert not cache.K[0, :, 10].any()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("T,G,room", [(2, 1, 0), (7, 2, 0), (7, 4, 0), (2, 4, ROOM), (7, 4, ROOM), (40, 4, ROOM)])
@pytest.mark.parametrize("tree", [True, False])
def test_nan_in_rows_before_the_draft_reaches_every_token(binding, dtype, D, T, G, room, tree):
    """e4m3 NaN in a row that every token sees, beside the draft in one tile or not."""
    c = A.case(binding, ("e4m3", dtype), 3, 2, G, D, 180, T, 16, seed=3, lens=[150, T + 9, 128 + T], tree=tree, room=room)
    base = [n - T for n in c["lens"]]
    c["cache"].V.view(torch.uint8)[0, :, base[0] - 1, 3::5] = 0x7f
    c["cache"].V.view(torch.uint8)[1, 0, base[1] - 9, 1] = 0xff
    c["cache"].V.view(torch.uint8)[2, 1, base[2] - 20, D - 1] = 0x7f
    got = A.run(c)
    out, lse, t_out, t_lse = A.reference(c)
    odd = torch.isnan(out)
    assert odd.any(-1).any(-1).all(-1).all() and torch.equal(torch.isnan(got["out"]), odd)
    zero = lambda x: torch.where(odd, 0.0, x)  # noqa: E731
    QU.assert_attention(dict(got, out=zero(got["out"])), (zero(out), lse, zero(t_out), t_lse))


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_scales_of_other_writers_below_the_least_normal_number(binding, form):
    """Zeros behind older rows under a scale of 1e-40 keep that scale and are codes of 0; other rows make it grow."""
    D, R, H = 64, 32, 8
    g, K, V, ks, vs = W.start_state(1, H, 64, D, form, R, seed=5)
    tiny = torch.tensor([1e-40, 1.1e-40, 1.2e-40, 1.3e-40, 3e-40, 7e-40, 2e-39, 2.0 ** -127], dtype=torch.float32).to(DEV)
    ks[0, :, 0], vs[0, :, 0] = tiny, tiny.flip(0)
    assert (ks[0, :, 0] > 0).all()
    x = torch.zeros((2, 1, H, 9, D), dtype=BF16, device=DEV)
    plan, cache = binding.Plan(1, H, D, sink=4, lag=64), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    want = W.expected(K, V, ks, vs, x[0], x[1], [11], [20], R, form)
    plan.quant_write(cache, x[0], x[1], i32([20]), ws, from_len=i32([11]))
    W.same(cache, want)
    assert not cache.K[0, :, 11:20].float().any()
    x += torch.exp2(torch.arange(-133, -125, device=DEV).float()).to(BF16).view(1, 1, H, 1, 1)
    want = W.expected(want[0][0], want[1][0], want[0][1], want[1][1], x[0], x[1], [20], [29], R, form)
    plan.quant_write(cache, x[0], x[1], i32([29]), ws, from_len=i32([20]))
    W.same(cache, want)
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_nothing_finite_but_zeros(binding, form, dtype):
    """A block of infinities, NaN and zeros has a scale of 0, under which every code is 0; beside older rows theirs holds."""
    D, R = 128, 16
    g, K, V, ks, vs = W.start_state(1, 1, 64, D, form, R, seed=7)
    x = torch.zeros((1, 1, 40, D), dtype=dtype, device=DEV)
    x[0, 0, 0, 1], x[0, 0, 1, 2], x[0, 0, 20, 3], x[0, 0, 21, 4] = float("inf"), float("nan"), float("-inf"), float("nan")
    plan, cache = binding.Plan(1, 1, D, sink=4, lag=64, dtype=dtype), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    want = W.expected(K, V, ks, vs, x, x, [5], [45], R, form)
    was = float(ks[0, 0, 0])
    plan.quant_write(cache, x, x, i32([45]), ws, from_len=i32([5]))
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    W.same(cache, want)
    assert float(cache.K_scale[0, 0, 0]) == was and float(cache.K[0, 0, 5, 1]) == QU.TOP[form]
    assert float(cache.K_scale[0, 0, 1]) == 0 and not cache.K[0, 0, 16:45].float().any()
    out = torch.full((1, 1, 64, D), 3.0, dtype=dtype, device=DEV)
    plan.quant_read(cache, i32([45]), ws, from_len=i32([16]), K_out=out)
    assert not out[0, 0, 16:45].any()


@pytest.mark.parametrize("kind", A.KINDS, ids=A.KIND_IDS)
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("T,G,room", [(3, 2, 0), (2, 4, ROOM), (4, 4, ROOM), (7, 4, ROOM), (20, 4, ROOM), (64, 4, room_of(6))])
def test_strides_in_every_kernel(binding, kind, D, T, G, room):
    """Codes and queries as projections leave them, tokens first, rows padded: clusters, units of 8, 16, 32, 128 and 256."""
    B, H, S, R = 2, 3, 210, 32
    c = A.case(binding, kind, B, H, G, D, S, T, R, seed=1, lens=[210, 100], room=room)
    A.poison(c)
    want = A.reference(c)
    cache = c["cache"]
    K, V = (torch.full((B, x.shape[2], H, D + 16), 0x7f, dtype=torch.uint8, device=DEV).view(x.dtype)[..., :D].transpose(1, 2) for x in (cache.K, cache.V))
    for to, x in ((K, cache.K), (V, cache.V)):
        to.view(torch.uint8).copy_(x.view(torch.uint8))
    c["cache"] = binding.QuantCache(K, V, cache.K_scale, cache.V_scale, block_rows=R)
    Q = torch.full((B, T, H * G, D + 8), float("nan"), dtype=c["Q"].dtype, device=DEV)[..., :D].copy_(c["Q"])
    heads_first = torch.full((B, H * G, T, D + 24), float("nan"), dtype=c["Q"].dtype, device=DEV)[..., :D].transpose(1, 2).copy_(c["Q"])
    for q in (Q, heads_first):
        c["Q"] = q
        QU.assert_attention(A.run(c), want)


@pytest.mark.parametrize("form,dtype", [("int8", BF16), ("e4m3", FP16)], ids=["int8-bf16", "e4m3-fp16"])
@pytest.mark.parametrize("D", [64, 96, 256])
@pytest.mark.parametrize("T,G,room", [(1, 7, 0), (2, 4, ROOM), (4, 4, ROOM), (8, 4, 2 * ROOM), (20, 4, 2 * ROOM), (64, 4, room_of(4))])
@pytest.mark.parametrize("page,R", [(16, 16), (64, 32), (128, 128)])
def test_attention_on_pages_of_every_head_dim(binding, form, dtype, D, T, G, room, page, R):
    """The same bits as from the contiguous cache, which is held against the statement; an entry outside the pool is recorded."""
    B, H, S = 2, 2, 384
    room = room // page * page
    c = A.case(binding, (form, dtype), B, H, G, D, S, T, R, seed=page + T, lens=[S, 200 + T], room=room)
    nb = S // page
    pages = B * nb + 2
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    cache = c["cache"]
    pool = binding.QuantCache(*(QU.pool_of(x[:, :, :S].contiguous(), page, table, pages) for x in (cache.K, cache.V)), cache.K_scale, cache.V_scale, block_rows=R)
    if room:  # entries of blocks that no sequence reaches
        table = torch.cat([table, torch.full((B, room // page - nb), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    call = lambda tab: c["plan"].attend_quant_paged(c["Q"], pool, tab, c["seq"], c["ws"], draft_len=c["draft"], tree_mask=c["mask"], want_lse=True)  # noqa: E731
    got, flat = call(table), A.run(c)
    QU.assert_attention(flat, A.reference(c))
    assert torch.equal(flat["out"], got["out"]) and torch.equal(flat["lse"], got["lse"])
    bad = table.clone()
    bad[0, 1] = pages
    lost = call(bad)
    assert c["plan"].read_status(c["ws"])[0] == binding.LAGKV_EINVAL
    assert torch.equal(lost["out"][1], got["out"][1])
    K, V = (QU.row_values(x[:1, :, :S], s[:1, :, :S // R], R) for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)))
    want = QU.attention_reference(c["Q"][:1], K, V, [S], [c["drafts"][0]], None if c["mask"] is None else c["mask"][:1], form=form,
                                  V_scale=cache.V_scale[:1].nan_to_num(nan=0.0), gone=slice(page, 2 * page))
    QU.assert_attention({"out": lost["out"][:1], "lse": lost["lse"][:1]}, want)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("D", [64, 96, 256])
@pytest.mark.parametrize("page,R", [(16, 16), (64, 32), (128, 128)])
def test_writing_and_reading_pages_of_every_head_dim(binding, form, D, page, R):
    """Ragged spans through a random table, read back whole and row by row."""
    B, H, nb = 3, 2, 256 // page
    S = nb * page
    g, K, V, ks, vs = W.start_state(B, H, S, D, form, R, seed=page)
    x = (torch.randn((2, B, H, 120, D), generator=g, device=DEV) * 2).to(FP16)
    pages = B * nb + 3
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=FP16)
    cache = binding.QuantCache(QU.pool_of(K, page, table, pages), QU.pool_of(V, page, table, pages), ks, vs, block_rows=R)
    ws = plan.new_workspace()
    starts, ends = [0, 37, 200], [120, 130, S]
    want = W.expected(K, V, ks, vs, x[0], x[1], starts, ends, R, form)
    plan.quant_write_paged(cache, table, x[0], x[1], i32(ends), ws, from_len=i32(starts))
    W.same(cache, want, table, page)
    values = [(c.float() * s.float().repeat_interleave(R, -1)[..., :S, None]).to(FP16) for c, s in want]
    out = torch.full((2, B, H, S, D), 3.0, dtype=FP16, device=DEV)
    plan.quant_read_paged(cache, table, i32(ends), ws, from_len=i32(starts), K_out=out[0], V_out=out[1])
    idx = torch.stack([torch.randint(0, e, (H, 33), generator=torch.Generator().manual_seed(e)) for e in ends]).to(torch.int32)
    picks = plan.quant_read_paged(cache, table, i32(ends), ws, idx=idx.to(DEV))
    for t, p, value in zip(out, picks, values):
        for b in range(B):
            assert torch.equal(t[b, :, starts[b]:ends[b]].cpu(), value[b, :, starts[b]:ends[b]])
            assert (t[b, :, :starts[b]] == 3).all() and (t[b, :, ends[b]:] == 3).all()
        assert torch.equal(p.cpu(), value.gather(2, idx.long()[..., None].expand(B, H, 33, D)))
    assert plan.read_status(ws)[0] == 0


INT8 = [A.KINDS[0], A.KINDS[2]]


@pytest.mark.parametrize("kind", INT8, ids=["bf16", "fp16"])
@pytest.mark.parametrize("D,T,G", [(64, 64, 8), (96, 48, 4), (128, 64, 8), (64, 35, 5), (128, 64, 3)])
def test_units_of_256_query_rows(binding, kind, D, T, G):
    """int8 caches with much room under many query rows, full units and others."""
    A.test_every_type_and_head_dim(binding, kind, D, T, G, 1, 64, room_of(3))


@pytest.mark.parametrize("kind", INT8, ids=["bf16", "fp16"])
def test_units_of_256_query_rows_over_every_length(binding, kind):
    A.test_lengths_around_every_tile(binding, kind, 60, room_of(28))
    A.test_padded_batch_and_rows_that_see_nothing(binding, kind, 64, room_of(10))


@pytest.mark.parametrize("kind", INT8, ids=["bf16", "fp16"])
@pytest.mark.parametrize("way", ["up", "down", "mixed", "zeros"])
def test_units_of_256_query_rows_under_scales_far_apart(binding, kind, way):
    A.test_scales_far_apart(binding, kind, 64, 4, room_of(4), way)


@pytest.mark.parametrize("kind", A.KINDS, ids=A.KIND_IDS)
@pytest.mark.parametrize("cap", [0.5, 30.0, 1e5])
def test_caps_under_many_query_rows(binding, kind, cap):
    """In units of 128 and, int8, of 256."""
    A.test_capped_logits(binding, kind, 64, 4, ROOM, cap)
    if kind[0] == "int8":
        A.test_capped_logits(binding, kind, 33, 4, room_of(4), cap)


@pytest.mark.parametrize("kind", A.KINDS[:2], ids=A.KIND_IDS[:2])
def test_factors_and_ends_of_the_type_under_many_query_rows(binding, kind):
    """In units of 128 and, int8, of 256."""
    A.test_factors_and_large_logits(binding, kind, 32, 4, 2 * ROOM)
    A.test_queries_at_the_ends_of_their_type(binding, kind, 32, 2 * ROOM)
    if kind[0] == "int8":
        A.test_factors_and_large_logits(binding, kind, 40, 4, room_of(2))
        A.test_queries_at_the_ends_of_their_type(binding, kind, 60, room_of(2))


@pytest.mark.parametrize("page,R", [(16, 16), (64, 64), (256, 128)])
def test_units_of_256_query_rows_on_pages(binding, page, R):
    A.test_pages(binding, "int8", 40, 4, room_of(6), page, R)


@pytest.mark.parametrize("kind", A.KINDS[:1], ids=A.KIND_IDS[:1])
def test_units_of_256_query_rows_replayed(binding, kind):
    A.test_graph_replay_and_repeats(binding, kind, 64, 4, room_of(6))


@pytest.mark.parametrize("H,S", [(2, 300), (8, 4096), (2, 20000)])
def test_the_first_call_of_a_plan_may_be_captured(binding, H, S):
    """What a plan asks the runtime once, it may ask while a stream is captured: clusters of CTAs, and the form without."""
    c = A.case(binding, ("int8", BF16), 1, H, 4, 128, S, 1, 64, seed=6, lens=[S])
    out, side, graph = torch.empty_like(c["Q"]), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c["plan"].attend_quant(c["Q"], c["cache"], c["seq"], c["ws"], out=out)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        out.zero_()
        graph.replay()
        QU.assert_attention({"out": out}, A.reference(c))


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("D,page,R", [(64, 16, 16), (128, 64, 32), (96, 128, 128)])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_pools_with_strides(binding, form, D, page, R, tokens_first):
    """K and V of a page side by side, heads or tokens first, rows padded: written, read and attended to like contiguous pools."""
    B, H, G, S = 2, 3, 4, 256
    g, K, V, ks, vs = W.start_state(B, H, S, D, form, R, seed=page)
    nb = S // page
    pages = B * nb + 3
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    plan = binding.Plan(B, H, D, sink=4, lag=64)
    ws = plan.new_workspace()
    dense = binding.QuantCache(QU.pool_of(K, page, table, pages), QU.pool_of(V, page, table, pages), ks, vs, block_rows=R)
    if tokens_first:
        store = torch.full((pages, page, 2, H, D + 16), 0x55, dtype=torch.uint8, device=DEV)
        both = [store[:, :, i, :, :D].transpose(1, 2) for i in range(2)]
    else:
        store = torch.full((pages, 2, H, page, D + 16), 0x55, dtype=torch.uint8, device=DEV)
        both = [store[:, i, :, :, :D] for i in range(2)]
    for to, x in zip(both, (dense.K, dense.V)):
        to.copy_(x.view(torch.uint8))
    cache = binding.QuantCache(*(t.view(dense.K.dtype) for t in both), ks.clone(), vs.clone(), block_rows=R)
    x = (torch.randn((2, B, H, 90, D), generator=g, device=DEV) * 2).to(BF16)
    starts, ends = [0, 37], [90, 111]
    for c in (dense, cache):
        plan.quant_write_paged(c, table, x[0], x[1], i32(ends), ws, from_len=i32(starts))
    assert torch.equal(cache.K_scale, dense.K_scale) and torch.equal(cache.V_scale, dense.V_scale)
    for a, b in ((cache.K, dense.K), (cache.V, dense.V)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert (store[..., D:] == 0x55).all()
    out = torch.zeros((4, B, H, S, D), dtype=BF16, device=DEV)
    plan.quant_read_paged(dense, table, i32([S, S]), ws, K_out=out[0], V_out=out[1])
    plan.quant_read_paged(cache, table, i32([S, S]), ws, K_out=out[2], V_out=out[3])
    assert torch.equal(out[:2], out[2:]) and plan.read_status(ws)[0] == 0
    for T, room in ((1, 0), (2, ROOM), (20, ROOM), (64, room_of(B * H))):
        wide = torch.cat([table, torch.full((B, max(0, room // page - nb)), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
        blocks = -(-wide.shape[1] * page // R)
        scales = lambda c: [torch.nn.functional.pad(s, (0, blocks - s.shape[2])) for s in (c.K_scale, c.V_scale)]  # noqa: E731
        Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(BF16)
        aws = plan.new_attend_quant_workspace(T, H * G)
        got = [plan.attend_quant_paged(Q, binding.QuantCache(c.K, c.V, *scales(c), block_rows=R), wide, i32([S, 200]), aws, want_lse=True) for c in (dense, cache)]
        assert plan.read_status(aws)[0] == 0
        assert torch.equal(got[0]["out"], got[1]["out"]) and torch.equal(got[0]["lse"], got[1]["lse"])
        kv = [QU.row_values(QU.dense_of(c, table, page), s, R) for c, s in ((dense.K, dense.K_scale), (dense.V, dense.V_scale))]
        QU.assert_attention(got[1], QU.attention_reference(Q, *kv, [S, 200], [T, T], None, form=form, V_scale=dense.V_scale))
