"""Caches in 8 bits with block scales: writing and reading back against float64 statements (tests/quant_util.py)."""
import random

import pytest
import torch

import quant_util as QU

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
DEV = "cuda:0"


@pytest.fixture(scope="module")
def binding():
    from paper_2504_04704_b200 import binding as b
    b.load_library()
    return b


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def start_state(B, H, S, D, form, R, seed, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    K, V, ks, vs = QU.random_cache(B, H, S, D, form, R, g, spread)
    return g, K, V, ks, vs


def expected(K, V, ks, vs, Kn, Vn, starts, ends, R, form, source=lambda b, h, i: i):
    """Codes and scales (float64, CPU) after the write."""
    got = []
    for code, scale, new in ((K, ks, Kn), (V, vs, Vn)):
        c, s, x = code.double().cpu(), scale.double().cpu(), new.cpu()
        for b, (a, e) in enumerate(zip(starts, ends)):
            for h in range(c.shape[1]):
                rows = [source(b, h, i) for i in range(e - a)]
                QU.write64(c[b, h], s[b, h], x[b, h, rows], a, e, R, form)
        got.append((c, s))
    return got


def same(cache, want, table=None, page=0):
    for codes, scale, (c, s) in ((cache.K, cache.K_scale, want[0]), (cache.V, cache.V_scale, want[1])):
        codes = QU.dense_of(codes, table, page)[:, :, :c.shape[2]] if page else codes
        assert torch.equal(scale.double().cpu(), s), "scales"
        off = codes.double().cpu() != c
        off &= ~(torch.isnan(codes.double().cpu()) & torch.isnan(c))
        assert not off.any(), f"{int(off.sum())} codes differ, first at {off.nonzero()[0].tolist()}"


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("R", [16, 32, 64, 128])
def test_every_type_size_and_start(binding, form, dtype, D, R):
    """Starts and ends inside, at and around blocks; nothing, one row, several blocks; older rows whose scale grows."""
    spans = [(0, 0), (0, 1), (0, R), (0, 3 * R + 5), (5, 5), (3, 4), (R - 1, R), (R - 1, R + 1), (R, R + 1), (R + 7, 3 * R), (300, 391)]
    B, H, S, T = len(spans), 2, 400, max(3 * R + 5, 91)
    g, K, V, ks, vs = start_state(B, H, S, D, form, R, seed=D + R)
    new = torch.randn((2, B, H, T, D), generator=g, device=DEV) * torch.exp(2 * torch.randn((2, B, H, T, 1), generator=g, device=DEV))
    Kn, Vn = new[0].to(dtype), new[1].to(dtype)
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    cache = binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    spans = [(a, min(e, S)) for a, e in spans]
    want = expected(K, V, ks, vs, Kn, Vn, *zip(*spans), R, form)
    plan.quant_write(cache, Kn, Vn, i32([e for _, e in spans]), ws, from_len=i32([a for a, _ in spans]))
    assert plan.read_status(ws)[0] == 0
    same(cache, want)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [1, 2, 3, 9, 64, 65, 200])
def test_row_by_row_and_in_chunks(binding, form, T):
    """The same rows in chunks of T: what each call leaves is what the definition says of the last state."""
    B, H, S, D, R = 2, 3, 203, 128, 64
    g, K, V, ks, vs = start_state(B, H, S, D, form, R, seed=T)
    x = (torch.randn((2, B, H, S, D), generator=g, device=DEV) * torch.linspace(0.1, 3, S, device=DEV)[:, None]).to(BF16)
    plan, cache = binding.Plan(B, H, D, sink=4, lag=64), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    want = [(K.double().cpu(), ks.double().cpu()), (V.double().cpu(), vs.double().cpu())]
    for at in range(0, S, T):
        end = min(S, at + T)
        part = [t[:, :, at:end].contiguous() for t in x]
        want = expected(want[0][0], want[1][0], want[0][1], want[1][1], *part, [at] * B, [end] * B, R, form)
        plan.quant_write(cache, *part, i32([end] * B), ws, from_len=i32([at] * B))
        if at // T < 8 or end == S:
            same(cache, want)
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("top", [1.0, 127.0, 0.7109375, 448.0, 450.0, 1.9921875, 60000.0, 3.1e-5])
def test_every_value_below_a_largest_one(binding, form, dtype, top):
    """All 16-bit values up to a largest one share a block: quotients on and next to every border."""
    D, R = 256, 128
    bits = torch.arange(0, 32768, dtype=torch.int32).to(torch.int16).view(dtype)
    t = float(torch.tensor(top).to(dtype))
    x = torch.where(bits.abs().double() <= t, bits, torch.tensor(t, dtype=dtype))
    x[1::2] = -x[1::2]
    Kn = x.view(1, 1, R, D).to(DEV)
    plan = binding.Plan(1, 1, D, sink=4, lag=64, dtype=dtype)
    cache, ws = plan.new_quant_cache(R, form, block_rows=R), plan.new_workspace()
    want = expected(cache.K, cache.V, cache.K_scale, cache.V_scale, Kn, -Kn, [0], [R], R, form)
    plan.quant_write(cache, Kn, -Kn, i32([R]), ws)
    same(cache, want)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_zeros_tiny_and_huge_values(binding, form):
    """Blocks of zeros (scale 0), of bf16 subnormals (least scale), of the largest bf16 values; older zeros under a new scale."""
    R, D = 16, 64
    x = torch.zeros((1, 1, 6 * R, D), device=DEV)
    x[:, :, R:2 * R] = 2.0 ** -130
    x[:, :, 2 * R:3 * R] = torch.linspace(-1, 1, D, device=DEV) * 3.38e38
    x[:, :, 3 * R:4 * R] = torch.linspace(-1, 1, D, device=DEV) * 2.0 ** -119
    x[:, :, 4 * R + 3] = 5.0
    x = x.to(BF16)
    plan = binding.Plan(1, 1, D, sink=4, lag=64)
    cache, ws = plan.new_quant_cache(6 * R, form, block_rows=R), plan.new_workspace()
    want = expected(cache.K, cache.V, cache.K_scale, cache.V_scale, x, x, [0], [4 * R + 2], R, form)
    plan.quant_write(cache, x, x, i32([4 * R + 2]), ws)
    same(cache, want)
    want = expected(want[0][0], want[1][0], want[0][1], want[1][1], x[:, :, 4 * R + 2:], x[:, :, 4 * R + 2:], [4 * R + 2], [6 * R], R, form)
    plan.quant_write(cache, x, x, i32([6 * R]), ws, from_len=i32([4 * R + 2]), at_positions=True)
    same(cache, want)
    K16 = torch.full((1, 1, 6 * R, D), 9.0, dtype=BF16, device=DEV)
    plan.quant_read(cache, i32([6 * R]), ws, K_out=K16)
    assert torch.isfinite(K16).all() and not K16[:, :, :R].any()
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_values_that_are_not_finite_are_recorded(binding, form, dtype):
    """They leave the scale to the others: infinities become the largest code, NaN 0."""
    B, H, D, R = 1, 2, 128, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn((B, H, 100, D), generator=g, device=DEV).to(dtype)
    x[0, 0, 3, 5], x[0, 0, 70, 6], x[0, 1, 8, 127], x[0, 1, 9, 0] = float("inf"), float("-inf"), float("nan"), -float("nan")
    plan = binding.Plan(B, H, D, sink=4, lag=64, dtype=dtype)
    cache, ws = plan.new_quant_cache(100, form, block_rows=R), plan.new_workspace()
    want = expected(cache.K, cache.V, cache.K_scale, cache.V_scale, x, x, [0], [100], R, form)
    plan.quant_write(cache, x, x, i32([100]), ws)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    same(cache, want)
    top = QU.TOP[form]
    assert cache.K[0, 0, 3, 5].double() == top and cache.K[0, 0, 70, 6].double() == -top and cache.K[0, 1, 8, 127].double() == 0


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_strides_of_source_and_cache(binding, form):
    """Tokens-first rows, as projections leave them, into a tokens-first cache with padded rows; read into a tokens-first cache."""
    B, H, S, D, R, T = 3, 4, 150, 96, 32, 40
    g = torch.Generator(device=DEV).manual_seed(8)
    x = torch.randn((2, B, T, H, D + 8), generator=g, device=DEV).to(BF16)[..., :D].transpose(2, 3)
    store = torch.full((2, B, S, H, D + 16), 0x55, dtype=torch.uint8, device=DEV)
    K, V = (t[..., :D].transpose(1, 2).view(QU.DTYPE[form]) for t in store)
    blocks = -(-S // R)
    ks, vs = torch.full((2, B, H, blocks), 0.01, device=DEV).unbind(0)
    plan = binding.Plan(B, H, D, sink=4, lag=64, strides=(S * H * D, D, H * D))
    cache, ws = binding.QuantCache(K, V, ks, vs, block_rows=R), plan.new_workspace()
    starts, ends = [0, 17, 110], [40, 50, 150]
    want = expected(K, V, ks, vs, x[0], x[1], starts, ends, R, form)
    plan.quant_write(cache, x[0], x[1], i32(ends), ws, from_len=i32(starts))
    same(cache, want)
    assert (store[..., D:] == 0x55).all()
    out = torch.full((2, B, S, H, D), 7.0, dtype=BF16, device=DEV).transpose(2, 3)
    plan.quant_read(cache, i32(ends), ws, from_len=i32(starts), K_out=out[0], V_out=out[1])
    for t, (c, s) in zip(out, want):
        value = (c.float() * s.float().repeat_interleave(R, -1)[..., :S, None]).to(BF16)
        for b in range(B):
            assert torch.equal(t[b, :, starts[b]:ends[b]].cpu(), value[b, :, starts[b]:ends[b]])
            assert (t[b, :, :starts[b]] == 7).all() and (t[b, :, ends[b]:] == 7).all()
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("shared", [False, True])
def test_rows_by_a_list(binding, shared):
    """take: rows in any order, some twice, per KV head or for all; entries outside the source are recorded and give 0."""
    B, H, S, D, R, T, n = 2, 3, 256, 128, 64, 500, 130
    rng = random.Random(3)
    g, K, V, ks, vs = start_state(B, H, S, D, "int8", R, seed=1)
    x = torch.randn((2, B, H, T, D), generator=g, device=DEV).to(FP16)
    take = torch.tensor([[[rng.randrange(T) for _ in range(n)] for _ in range(1 if shared else H)] for _ in range(B)], dtype=torch.int32, device=DEV)
    plan, cache = binding.Plan(B, H, D, sink=4, lag=64, dtype=FP16), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    starts, ends = [70, 0], [200, 99]
    pick = take.cpu()
    row = lambda b, h, i: int(pick[b, 0 if shared else h, i])  # noqa: E731
    want = expected(K, V, ks, vs, x[0], x[1], starts, ends, R, "int8", row)
    plan.quant_write(cache, x[0], x[1], i32(ends), ws, from_len=i32(starts), take=take[:, 0].contiguous() if shared else take)
    assert plan.read_status(ws)[0] == 0
    same(cache, want)
    take[0, 0, 5], take[1, -1, 7] = T, -1
    clean = x.clone()
    clean[:, :, :, T - 1] = 0                                      # the reference's stand-in for a row that is not there
    pick = torch.where((take < 0) | (take >= T), T - 1, torch.where(take == T - 1, 0, take)).cpu()
    good = torch.where(take == T - 1, 0, take)
    state = [(t.double().cpu(), s.double().cpu()) for t, s in ((cache.K, ks), (cache.V, vs))]
    want = expected(state[0][0], state[1][0], state[0][1], state[1][1], clean[0], clean[1], starts, ends, R, "int8", row)
    plan.quant_write(cache, x[0], x[1], i32(ends), ws, from_len=i32(starts), take=good[:, 0].contiguous() if shared else good)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    same(cache, want)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("page,R", [(16, 16), (64, 16), (64, 64), (128, 32)])
def test_pages(binding, form, page, R):
    """Random pages, ragged spans, rows of other pages untouched; a page outside the pool is left out and recorded."""
    B, H, D, nb = 3, 2, 128, 256 // page
    S = nb * page
    g, K, V, ks, vs = start_state(B, H, S, D, form, R, seed=page)
    x = torch.randn((2, B, H, 120, D), generator=g, device=DEV).to(BF16) * 2
    pages = B * nb + 4
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[:B * nb].view(B, nb).to(torch.int32).to(DEV)
    plan = binding.Plan(B, H, D, sink=4, lag=64)
    cache = binding.QuantCache(QU.pool_of(K, page, table, pages), QU.pool_of(V, page, table, pages), ks, vs, block_rows=R)
    ws = plan.new_workspace()
    starts, ends = [0, 37, 200], [120, 130, S]
    want = expected(K, V, ks, vs, x[0], x[1], starts, ends, R, form)
    before = cache.K.view(torch.uint8).clone()
    plan.quant_write_paged(cache, table, x[0], x[1], i32(ends), ws, from_len=i32(starts))
    assert plan.read_status(ws)[0] == 0
    same(cache, want, table, page)
    loose = sorted(set(range(pages)) - set(table.flatten().tolist()))
    assert torch.equal(cache.K.view(torch.uint8)[loose], before[loose])
    out = torch.full((2, B, H, S, D), 3.0, dtype=BF16, device=DEV)
    plan.quant_read_paged(cache, table, i32(ends), ws, from_len=i32(starts), K_out=out[0], V_out=out[1])
    for t, (c, s) in zip(out, want):
        value = (c.float() * s.float().repeat_interleave(R, -1)[..., :S, None]).to(BF16)
        for b in range(B):
            assert torch.equal(t[b, :, starts[b]:ends[b]].cpu(), value[b, :, starts[b]:ends[b]])
            assert (t[b, :, :starts[b]] == 3).all() and (t[b, :, ends[b]:] == 3).all()
    # sequence 1 loses the page of row 37
    bad, hole = table.clone(), 37 // page
    bad[1, hole] = pages
    kept = cache.K.view(torch.uint8).clone()
    out.fill_(3.0)
    plan.quant_write_paged(cache, bad, x[0], x[1], i32([0, 38, 0]), ws, from_len=i32([0, 37, 0]))
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    assert torch.equal(cache.K.view(torch.uint8), kept) and torch.equal(cache.K_scale.double().cpu(), want[0][1])
    plan.quant_read_paged(cache, bad, i32([0, 130, 0]), ws, K_out=out[0])
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    assert (out[0, 1, :, hole * page:(hole + 1) * page] == 3).all() and not (out[0, 1, :, (hole + 1) * page:130] == 3).all()
    if page > R:
        with pytest.raises(binding.LagKVError):                    # a block has to lie in one page
            wide = binding.QuantCache(cache.K, cache.V, ks, vs, block_rows=128 if page < 128 else 256)
            plan.quant_write_paged(wide, table, x[0], x[1], i32(ends), ws, from_len=i32(starts))


def test_read_of_chosen_rows(binding):
    """Any order, repeats, entries behind the sequence; one of the outputs alone."""
    B, H, S, D, R, n = 2, 2, 300, 64, 32, 77
    g, K, V, ks, vs = start_state(B, H, S, D, "e4m3", R, seed=2, spread=6)
    plan, cache = binding.Plan(B, H, D, sink=4, lag=64, dtype=FP16), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    lens = [300, 150]
    idx = torch.stack([torch.randint(0, m, (H, n), generator=g, device=DEV) for m in lens]).to(torch.int32)
    Ko, Vo = plan.quant_read(cache, i32(lens), ws, idx=idx)
    for out, c, s in ((Ko, K, ks), (Vo, V, vs)):
        value = (c.float() * s.repeat_interleave(R, -1)[..., :S, None]).clamp(-65504, 65504).to(FP16)
        assert torch.equal(out, value.gather(2, idx.long()[..., None].expand(B, H, n, D)))
    assert plan.read_status(ws)[0] == 0
    idx[1, 0, 3], idx[0, 1, 4] = 150, -1
    mark = torch.full_like(Ko, 5.0)
    got = plan.quant_read(cache, i32(lens), ws, idx=idx, V_out=mark)
    assert got[0] is None and got[1] is mark and plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    assert (mark[1, 0, 3] == 5).all() and (mark[0, 1, 4] == 5).all() and torch.equal(mark[1, 1], Vo[1, 1])


def test_values_beyond_fp16_saturate(binding):
    """65504 in e4m3 is 256 * 256: read back it is the largest fp16 again, not infinity."""
    x = torch.full((1, 1, 16, 64), 65504.0, dtype=FP16, device=DEV)
    x[..., ::2] *= -1
    plan = binding.Plan(1, 1, 64, sink=4, lag=64, dtype=FP16)
    for form in ("int8", "e4m3"):
        cache, ws = plan.new_quant_cache(16, form, block_rows=16), plan.new_workspace()
        plan.quant_write(cache, x, x, i32([16]), ws)
        Ko, _ = plan.quant_read(cache, i32([16]), ws, idx=torch.zeros((1, 1, 1), dtype=torch.int32, device=DEV))
        assert torch.equal(Ko[0, 0, 0].abs(), x[0, 0, 0].abs()), form


def test_lengths_that_do_not_fit_are_recorded(binding):
    """Such a sequence is left alone; the others are written and read."""
    B, H, S, D, R, T = 6, 1, 100, 64, 16, 30
    g, K, V, ks, vs = start_state(B, H, S, D, "int8", R, seed=6)
    x = torch.randn((2, B, H, T, D), generator=g, device=DEV).to(BF16)
    plan, cache = binding.Plan(B, H, D, sink=4, lag=64), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    starts, ends = [-1, 20, 90, 0, 5, 40], [3, 19, 101, 31, 35, 40]
    ok = [4, 5]
    want = expected(K, V, ks, vs, x[0], x[1], [s if b in ok else 0 for b, s in enumerate(starts)], [e if b in ok else 0 for b, e in enumerate(ends)], R, "int8")
    plan.quant_write(cache, x[0], x[1], i32(ends), ws, from_len=i32(starts))
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    same(cache, want)
    plan.quant_write(cache, x[0], x[1], i32([31] + [0] * 5), ws, from_len=i32([25] + [0] * 5), at_positions=True)  # row 30 of 30
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    same(cache, want)
    out = torch.full((B, H, 50, D), 3.0, dtype=BF16, device=DEV)
    plan.quant_read(cache, i32([50, 51, 101, 10, -1, 40]), ws, from_len=i32([-1, 0, 0, 11, 0, 40]), K_out=out)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL and (out == 3).all()


def test_graph_replay_and_streams(binding):
    """A captured append of one row per sequence, replayed while the lengths advance on the device; another stream's call."""
    B, H, S, D, R = 4, 2, 64, 128, 16
    plan = binding.Plan(B, H, D, sink=4, lag=64)
    cache, ws = plan.new_quant_cache(S, "int8", block_rows=R), plan.new_workspace()
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = (torch.randn((2, S, B, H, 1, D), generator=g, device=DEV) * torch.linspace(0.2, 2, S, device=DEV).view(S, 1, 1, 1, 1)).to(BF16)
    K, V = torch.zeros_like(rows[0, 0]), torch.zeros_like(rows[0, 0])
    start, end = i32([0, 5, 15, 16]), i32([1, 6, 16, 17])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            plan.quant_write(cache, K, V, end, ws, from_len=start)
            start += 1
            end += 1
    torch.cuda.current_stream().wait_stream(side)
    cache.K_scale.zero_()
    cache.V_scale.zero_()
    start.copy_(i32([0, 5, 15, 16]))
    end.copy_(i32([1, 6, 16, 17]))
    for n in range(40):
        K.copy_(rows[0, n])
        V.copy_(rows[1, n])
        graph.replay()
    want = [(torch.zeros((B, H, S, D), dtype=torch.float64), torch.zeros((B, H, 4), dtype=torch.float64)) for _ in "KV"]
    for n in range(40):
        at = [a + n for a in (0, 5, 15, 16)]
        want = expected(want[0][0], want[1][0], want[0][1], want[1][1], rows[0, n], rows[1, n], at, [a + 1 for a in at], R, "int8")
    same(cache, want)
    assert plan.read_status(ws)[0] == 0


def test_rows_far_into_a_cache(binding):
    """Offsets behind 2^32 bytes in the codes, the source and the 16-bit output."""
    D, S, R = 256, (1 << 24) + 1000, 128
    plan = binding.Plan(1, 1, D, sink=4, lag=64)
    cache, ws = plan.new_quant_cache(S, "e4m3", block_rows=R), plan.new_workspace()
    x = torch.zeros((1, 1, S, D), dtype=BF16, device=DEV)
    a, e = S - 333, S
    x[:, :, a:e] = torch.randn((333, D), device=DEV).to(BF16)
    plan.quant_write(cache, x, x, i32([e]), ws, from_len=i32([a]), at_positions=True)
    want = (torch.zeros((333 + a % R, D), dtype=torch.float64), torch.zeros(5, dtype=torch.float64))
    QU.write64(*want, x[0, 0, a:e].cpu(), a % R, a % R + 333, R, "e4m3")
    assert torch.equal(cache.K[0, 0, a:].double().cpu(), want[0][a % R:])
    n = -(-e // R) - a // R
    assert torch.equal(cache.V_scale[0, 0, a // R:].double().cpu(), want[1][:n]) and not cache.V_scale[0, 0, :a // R].any()
    x.fill_(2.0)
    plan.quant_read(cache, i32([e]), ws, from_len=i32([a]), K_out=x)
    scale = cache.K_scale[0, 0].repeat_interleave(R)[a:e, None]
    assert torch.equal(x[0, 0, a:e], (cache.K[0, 0, a:e].float() * scale).to(BF16)) and (x[0, 0, a - 5:a] == 2).all()
    idx = torch.arange(e - 40, e, dtype=torch.int32, device=DEV).view(1, 1, 40)
    assert torch.equal(plan.quant_read(cache, i32([e]), ws, idx=idx)[0][0, 0], x[0, 0, e - 40:e])
    assert plan.read_status(ws)[0] == 0


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_older_rows_under_a_scale_of_zero_stay_zero(binding, form):
    """A scale of 0 makes every code stand for 0, codes of another writer too: they become codes of 0 when the scale grows."""
    B, H, S, D, R = 2, 2, 64, 64, 32
    g, K, V, ks, vs = start_state(B, H, S, D, form, R, seed=4)
    ks[:, 0], vs[:, 1] = 0.0, 0.0
    x = torch.randn((2, B, H, 20, D), generator=g, device=DEV).to(BF16)
    plan, cache = binding.Plan(B, H, D, sink=4, lag=64), binding.QuantCache(K, V, ks, vs, block_rows=R)
    ws = plan.new_workspace()
    want = expected(K, V, ks, vs, x[0], x[1], [10, 33], [30, 50], R, form)
    plan.quant_write(cache, x[0], x[1], i32([30, 50]), ws, from_len=i32([10, 33]))
    assert plan.read_status(ws)[0] == 0
    same(cache, want)
    assert not cache.K[0, 0, :10].float().any() and not cache.V[1, 1, 32:33].float().any()
