"""The pages of a paged cache (release, reserve, fork, compact) against a plain statement of each, and a
whole serving run of the cache's operators together."""
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


class State:
    """Tables and counts on the host, with the four operations written out."""

    def __init__(self, B, nb, pages, page):
        self.table = [[-1] * nb for _ in range(B)]
        self.refs = [0] * pages
        self.page, self.B, self.nb = page, B, nb
        self.seq, self.static = [0] * B, [0] * B

    def need(self, n):
        return -(-n // self.page)

    def free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def release(self, keep):
        for b, n in enumerate(keep):
            for j in range(self.need(n), self.nb):
                if self.table[b][j] >= 0:
                    self.refs[self.table[b][j]] -= 1
                    self.table[b][j] = -1

    def reserve(self, want):
        lack = [(b, j) for b, n in enumerate(want) for j in range(self.need(n)) if self.table[b][j] < 0]
        free = self.free()
        if len(free) < len(lack):
            return False
        for (b, j), p in zip(lack, free):
            self.table[b][j] = p
            self.refs[p] = 1
        return True

    def fork(self, src, dst):
        """The copies (from, to) to make, or None when they do not fit."""
        taken, todo, copies = set(), [], []
        old = [row[:] for row in self.table]
        for s, d in zip(src, dst):
            if not (0 <= s < self.B and 0 <= d < self.B) or d in taken or any(p >= 0 for p in old[d]):
                continue
            if any(not 0 <= p < len(self.refs) for p in old[s][:self.need(self.seq[s])]):
                continue
            taken.add(d)
            todo.append((s, d))
        free = self.free()
        seq, static = self.seq[:], self.static[:]
        for s, d in todo:
            for j in range(self.need(seq[s])):
                if j < min(seq[s], static[s]) // self.page:
                    copies.append((d, j, old[s][j], None))
                else:
                    if not free:
                        return None
                    copies.append((d, j, old[s][j], free.pop(0)))
        moves = []
        for d, j, p, q in copies:
            self.table[d][j] = p if q is None else q
            self.refs[self.table[d][j]] += 1
            if q is not None:
                moves.append((p, q))
        for s, d in todo:
            self.seq[d], self.static[d] = seq[s], static[s]
        return moves

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        name = dict(zip(movers, holes))
        for a, b in name.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[name.get(p, p) for p in row] for row in self.table]
        return live, list(name.items())

    def device(self):
        t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        return dict(table=t(self.table), refs=t(self.refs), seq=t(self.seq), static=t(self.static))

    def same(self, d):
        assert d["table"].tolist() == self.table
        assert d["refs"].tolist() == self.refs
        assert d["seq"].tolist() == self.seq and d["static"].tolist() == self.static


def filled(B, nb, pages, page, rng, lens):
    """Sequences of `lens` rows on pages drawn at random."""
    s = State(B, nb, pages, page)
    order = list(range(pages))
    rng.shuffle(order)
    for b, n in enumerate(lens):
        for j in range(s.need(n)):
            s.table[b][j] = order.pop()
            s.refs[s.table[b][j]] = 1
        s.seq[b], s.static[b] = n, rng.randint(0, n)
    return s


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("B,nb,page,spare", [(1, 1, 16, 0), (5, 9, 16, 7), (3, 40, 64, 0), (70, 33, 32, 100), (2, 3000, 16, 5), (1500, 3, 16, 9)])
def test_release_and_reserve(binding, B, nb, page, spare):
    rng = random.Random(nb)
    lens = [rng.choice((0, 1, page - 1, page, nb * page, rng.randint(0, nb * page))) for _ in range(B)]
    s = filled(B, nb, B * nb + spare, page, rng, lens)
    d = s.device()
    plan = binding.Plan(B, 2, 64, sink=0, lag=32)
    ws = plan.new_pages_workspace(B * nb + spare)
    for _ in range(3):
        keep = [rng.choice((0, n, n // 2, min(nb * page, n + 5), nb * page)) for n in lens]
        plan.pages_release(d["table"], d["refs"], ints(keep), ws, page)
        s.release(keep)
        s.same(d)
        want = [rng.randint(0, nb * page) for _ in range(B)]
        plan.pages_reserve(d["table"], d["refs"], ints(want), ws, page)
        assert s.reserve(want)
        s.same(d)
    plan.pages_release(d["table"], d["refs"], ints([0] * B), ws, page)
    assert not d["refs"].any() and (d["table"] == -1).all()
    assert plan.read_status(ws)[0] == 0


def test_reserve_without_enough_pages_changes_nothing(binding):
    s = filled(4, 6, 20, 16, random.Random(1), [96, 60, 0, 30])
    d = s.device()
    plan = binding.Plan(4, 2, 64, sink=0, lag=32)
    ws = plan.new_pages_workspace(20)
    plan.pages_reserve(d["table"], d["refs"], ints([96, 96, 96, 96]), ws, 16)
    assert plan.read_status(ws)[0] == binding.LAGKV_ECAPACITY
    s.same(d)
    plan.pages_reserve(d["table"], d["refs"], ints([96, 96, 96, 32]), ws, 16)       # exactly as many as there are
    assert s.reserve([96, 96, 96, 32]) and plan.read_status(ws)[0] == 0
    s.same(d)
    plan.pages_reserve(d["table"], d["refs"], ints([96, 97, -1, 32]), ws, 16)       # lengths outside the table
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    s.same(d)


def test_release_of_entries_that_are_none(binding):
    s = filled(3, 4, 16, 16, random.Random(1), [64, 64, 20])
    d = s.device()
    d["table"][0, 3], d["refs"][int(d["table"][1, 2])] = 99, 0
    t, r = d["table"].clone(), d["refs"].clone()
    plan = binding.Plan(3, 2, 64, sink=0, lag=32)
    ws = plan.new_pages_workspace(16)
    plan.pages_release(d["table"], d["refs"], ints([48, 32, -5]), ws, 16)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    # the entry outside the pool and the uncounted page stay, the counted one beside it goes, sequence 2 is left alone
    p = int(t[1, 3])
    t[1, 3] = -1
    r[p] = 0
    assert torch.equal(d["table"], t) and torch.equal(d["refs"], r)


def pools(s, H, D, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [U.make_cache((len(s.refs), H, s.page, D), dtype, g)[i] for i in range(2)]


@pytest.mark.parametrize("dtype", [BF16, FP16, FP8], ids=["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("B,H,D,page,nb", [(6, 1, 64, 16, 5), (9, 8, 128, 64, 7), (4, 3, 96, 32, 20), (12, 2, 256, 16, 3)])
def test_fork(binding, dtype, B, H, D, page, nb):
    rng = random.Random(B)
    held = B // 2
    lens = [rng.choice((1, page, nb * page, rng.randint(1, nb * page))) for _ in range(held)] + [0] * (B - held)
    s = filled(B, nb, B * nb, page, rng, lens)
    s.static[0] = s.seq[0]                       # an uncompressed sequence: all full pages shared
    if held > 1:
        s.static[1] = s.seq[1] + 40              # a sink longer than the sequence
    d = s.device()
    K, V = pools(s, H, D, dtype, B)
    wantK, wantV = U.bits(K).clone(), U.bits(V).clone()
    plan = binding.Plan(B, H, D, sink=0, lag=32, dtype=dtype)
    ws = plan.new_pages_workspace(B * nb)
    src = [rng.randrange(held) for _ in range(B - held)]
    src[0] = 0
    dst = list(range(held, B))
    rng.shuffle(dst)
    plan.pages_fork(K, V, d["table"], d["refs"], d["seq"], d["static"], ints(src), ints(dst), ws)
    for a, b in s.fork(src, dst):
        wantK[b], wantV[b] = wantK[a], wantV[a]
    s.same(d)
    assert torch.equal(U.bits(K), wantK) and torch.equal(U.bits(V), wantV)
    assert plan.read_status(ws)[0] == 0
    for b in range(B):                            # a fork reads as its source
        n = s.seq[b]
        if b >= held:
            a = src[dst.index(b)]
            for X in (K, V):
                rows = U.bits(U.from_pages(X, d["table"][[a, b]], page))
                assert torch.equal(rows[0, :, :n], rows[1, :, :n])


def test_fork_refuses_pairs_that_are_none(binding):
    """Indexes outside the batch, targets that hold pages or come twice, sources without their pages: the others are done."""
    B, nb, page, H, D = 8, 4, 16, 2, 64
    s = filled(B, nb, 40, page, random.Random(3), [60, 33, 16, 20, 0, 0, 0, 0])
    s.table[3][1] = -1                           # sequence 3 lacks a page its length needs
    d = s.device()
    K, V = pools(s, H, D, BF16, 1)
    wantK = K.clone()
    plan = binding.Plan(B, H, D, sink=0, lag=32)
    ws = plan.new_pages_workspace(40)
    src, dst = [0, 8, 1, 3, 1, 0, -1, 4], [4, 5, 2, 5, 4, 6, 7, 7]
    plan.pages_fork(K, V, d["table"], d["refs"], d["seq"], d["static"], ints(src), ints(dst), ws)
    for a, b in s.fork(src, dst):
        wantK[b] = wantK[a]
    s.same(d)
    assert torch.equal(K, wantK) and plan.read_status(ws)[0] == binding.LAGKV_EINVAL


def test_fork_without_enough_pages_changes_nothing(binding):
    B, nb, page, H, D = 4, 4, 16, 2, 64
    s = filled(B, nb, 11, page, random.Random(3), [60, 50, 0, 0])
    s.static = [0] * B
    d = s.device()
    K, V = pools(s, H, D, BF16, 1)
    k0, v0 = K.clone(), V.clone()
    plan = binding.Plan(B, H, D, sink=0, lag=32)
    ws = plan.new_pages_workspace(11)
    plan.pages_fork(K, V, d["table"], d["refs"], d["seq"], d["static"], ints([0, 1]), ints([2, 3]), ws)
    assert plan.read_status(ws)[0] == binding.LAGKV_ECAPACITY
    s.same(d)
    assert torch.equal(K, k0) and torch.equal(V, v0)


@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
@pytest.mark.parametrize("B,H,D,page,nb,spare", [(6, 2, 64, 16, 5, 3), (9, 8, 128, 64, 7, 0), (3, 1, 96, 16, 900, 11), (40, 1, 64, 16, 300, 1)])
def test_compact(binding, dtype, B, H, D, page, nb, spare):
    rng = random.Random(B)
    lens = [rng.choice((0, rng.randint(1, nb * page))) for _ in range(B)]
    s = filled(B, nb, B * nb + spare, page, rng, lens)
    if B > 8:                                     # a shared page moves once, for everybody
        s.table[B - 1] = [-1] * nb
        s.refs = [0] * len(s.refs)
        s.table[B - 1][:s.need(s.seq[0])] = s.table[0][:s.need(s.seq[0])]
        for row in s.table:
            for p in row:
                if p >= 0:
                    s.refs[p] += 1
    d = s.device()
    K, V = pools(s, H, D, dtype, B)
    wantK, wantV = U.bits(K).clone(), U.bits(V).clone()
    plan = binding.Plan(B, H, D, sink=0, lag=32, dtype=dtype)
    ws = plan.new_pages_workspace(len(s.refs))
    live = plan.pages_compact(K, V, d["table"], d["refs"], ws)
    want, moves = s.compact()
    for a, b in moves:
        wantK[b], wantV[b] = wantK[a], wantV[a]
    assert live.tolist() == [want]
    s.same(d)
    assert torch.equal(U.bits(K), wantK) and torch.equal(U.bits(V), wantV)
    live = plan.pages_compact(K, V, d["table"], d["refs"], ws)      # dense already: nothing moves
    assert live.tolist() == [want] and torch.equal(U.bits(K), wantK)
    s.same(d)
    assert plan.read_status(ws)[0] == 0


def test_pools_with_padded_strides(binding):
    B, H, D, page, nb = 4, 2, 64, 32, 3
    s = filled(B, nb, 14, page, random.Random(2), [90, 50, 0, 0])
    s.static = [40, 0, 0, 0]
    d = s.device()
    wide = [torch.randn((14, page, H, D + 8), device=DEV).to(BF16) for _ in range(2)]
    want = [x.clone() for x in wide]
    plan = binding.Plan(B, H, D, sink=0, lag=32)
    ws = plan.new_pages_workspace(14)
    strides = (page * H * (D + 8), D + 8, H * (D + 8), page)
    plan.pages_fork(*wide, d["table"], d["refs"], d["seq"], d["static"], ints([0, 0]), ints([3, 2]), ws, strides=strides)
    for a, b in s.fork([0, 0], [3, 2]):
        for x in want:
            x[b, :, :, :D] = x[a, :, :, :D]
    s.same(d)
    assert all(torch.equal(x, y) for x, y in zip(wide, want))
    plan.pages_release(d["table"], d["refs"], ints([0, 50, 20, 90]), ws, page)
    s.release([0, 50, 20, 90])
    live = plan.pages_compact(*wide, d["table"], d["refs"], ws, strides=strides)
    n, moves = s.compact()
    for a, b in moves:
        for x in want:
            x[b, :, :, :D] = x[a, :, :, :D]
    s.same(d)
    assert live.tolist() == [n] and all(torch.equal(x, y) for x, y in zip(wide, want))


def test_an_entry_that_names_a_free_page(binding):
    s = filled(2, 3, 8, 16, random.Random(2), [48, 20])
    d = s.device()
    d["table"][1, 2] = max(p for p in range(8) if s.refs[p] == 0)
    K, V = pools(s, 1, 64, BF16, 1)
    plan = binding.Plan(2, 1, 64, sink=0, lag=32)
    ws = plan.new_pages_workspace(8)
    live = plan.pages_compact(K, V, d["table"], d["refs"], ws)
    n, _ = s.compact()
    got = plan.read_status(ws)[0]
    assert live.tolist() == [n]
    assert d["table"][1, 2].item() < n or got == binding.LAGKV_EINVAL


@pytest.mark.parametrize("name", ["hole", "behind", "outside"])
def test_an_entry_that_names_an_uncounted_page_is_cleared(binding, name):
    """Page 1 is free and below the number of live pages, page 7 free and behind: after the move their numbers may be
    another sequence's page, so an entry that names one, or no page of the pool, is recorded and becomes -1."""
    s = State(3, 3, 8, 16)
    s.table = [[0, 2, 5], [3, -1, -1], [6, -1, -1]]
    s.refs = [1, 0, 1, 1, 0, 1, 1, 0]
    s.seq, s.static = [48, 16, 16], [0, 0, 0]
    d = s.device()
    d["table"][1, 2] = {"hole": 1, "behind": 7, "outside": 8}[name]
    K, V = pools(s, 1, 64, BF16, 1)
    wantK, wantV = (U.bits(x).clone() for x in (K, V))
    plan = binding.Plan(3, 1, 64, sink=0, lag=32)
    ws = plan.new_pages_workspace(8)
    live = plan.pages_compact(K, V, d["table"], d["refs"], ws)
    assert plan.read_status(ws)[0] == binding.LAGKV_EINVAL
    n, moves = s.compact()
    assert moves == [(5, 1), (6, 4)]
    for a, b in moves:
        wantK[b], wantV[b] = wantK[a], wantV[a]
    assert live.tolist() == [n]
    s.same(d)
    assert torch.equal(U.bits(K), wantK) and torch.equal(U.bits(V), wantV)
    plan.pages_compact(K, V, d["table"], d["refs"], ws)
    assert plan.read_status(ws)[0] == 0


def test_refusals_touch_nothing(binding):
    import ctypes
    s = filled(2, 3, 8, 16, random.Random(2), [48, 0])
    d = s.device()
    K, V = pools(s, 1, 64, BF16, 1)
    plan = binding.Plan(2, 1, 64, sink=0, lag=32)
    lib, ws, E = plan.lib, plan.new_pages_workspace(8), binding.LAGKV_EINVAL
    ptr = lambda t, off=0: ctypes.c_void_p(t.data_ptr() + off)  # noqa: E731
    keep = ints([0, 0])
    args = [plan.handle, ptr(d["table"]), 3, 16, 8, ptr(d["refs"]), ptr(keep), ptr(ws), ws.numel(), None]
    for fn in (lib.lagkv_pages_release, lib.lagkv_pages_reserve):
        for i, bad in ((1, None), (1, ptr(d["table"], 2)), (2, 0), (3, 8), (3, 24), (4, 0), (5, None), (6, None), (7, ptr(ws, 4))):
            assert fn(*(args[:i] + [bad] + args[i + 1:])) == E, (i, bad)
        assert fn(*(args[:8] + [512, None])) == binding.LAGKV_EWORKSPACE
    lay = binding.lagkv_paged_layout(d["table"].data_ptr(), 3, 16)
    src, dst = ints([0]), ints([1])
    args = [plan.handle, ptr(K), ptr(V), ctypes.byref(lay), 8, ptr(d["refs"]), ptr(d["seq"]), ptr(d["static"]), ptr(src), ptr(dst), 1, ptr(ws),
            ws.numel(), None]
    for i, bad in ((1, None), (2, args[1]), (1, ptr(K, 8)), (3, None), (4, 0), (5, None), (6, None), (7, None), (8, None), (9, None), (10, 3), (10, -1)):
        assert lib.lagkv_pages_fork(*(args[:i] + [bad] + args[i + 1:])) == E, (i, bad)
    live = ints([0])
    args = [plan.handle, ptr(K), ptr(V), ctypes.byref(lay), 8, ptr(d["refs"]), ptr(live), ptr(ws), ws.numel(), None]
    for i, bad in ((1, None), (2, None), (3, None), (5, None), (6, None)):
        assert lib.lagkv_pages_compact(*(args[:i] + [bad] + args[i + 1:])) == E, (i, bad)
    torch.cuda.synchronize()
    s.same(d)
    with pytest.raises(TypeError):
        plan.pages_fork(K, V, d["table"], d["refs"][:7], d["seq"], d["static"], src, dst, ws)


# ------------------------------------------------------------------------------------------- together
def test_a_serving_run(binding, oracle):
    """A prompt in pages, forked, drafted trees attended and committed, the cache compressed in place, pages freed and
    the pool made dense, then block-sparse decoding: every attention against float64 on rows kept on the host."""
    B, H, G, D, page, nb, pages = 3, 2, 4, 64, 16, 40, 100
    sink, lag, T = 4, 64, 8
    rng = random.Random(7)
    g = torch.Generator(device=DEV).manual_seed(7)
    plan = binding.Plan(B, H, D, sink=sink, lag=lag, keep_ratio=0.25)
    K, V = (torch.zeros((pages, H, page, D), dtype=BF16, device=DEV) for _ in range(2))
    table = torch.full((B, nb), -1, dtype=torch.int32, device=DEV)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    seq, static = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    pws, aws = plan.new_pages_workspace(pages), plan.new_attend_workspace(T, H * G, blocks=nb * page // 16, keep=6)
    cws = plan.new_workspace(8)
    rows = [[torch.zeros((H, 0, D), dtype=BF16, device=DEV) for _ in range(2)] for _ in range(B)]   # what each sequence holds

    def append(b, k, v):
        n = rows[b][0].shape[1]
        for i, (pool, x) in enumerate(((K, k), (V, v))):
            for r in range(x.shape[1]):
                pool[int(table[b, (n + r) // page]), :, (n + r) % page] = x[:, r]
            rows[b][i] = torch.cat((rows[b][i], x), 1)
        seq[b] += k.shape[1]

    def fresh(n):
        return [torch.randn((H, n, D), generator=g, device=DEV).to(BF16) for _ in range(2)]

    def dense():
        S = max(r[0].shape[1] for r in rows)
        out = [torch.zeros((B, H, S, D), dtype=BF16, device=DEV) for _ in range(2)]
        for b in range(B):
            for i in range(2):
                out[i][b, :, :rows[b][i].shape[1]] = rows[b][i]
        return out

    def consistent():
        count = torch.zeros(pages, dtype=torch.int64)
        for p in table.cpu().reshape(-1).tolist():
            if p >= 0:
                count[p] += 1
        assert torch.equal(count.to(torch.int32), refs.cpu())
        for b in range(B):
            n = rows[b][0].shape[1]
            assert int(seq[b]) == n
            for i, pool in enumerate((K, V)):
                assert torch.equal(U.from_pages(pool, table[b:b + 1], page)[0, :, :n], rows[b][i])

    plan.pages_reserve(table, refs, ints([300, 0, 0]), pws, page)
    append(0, *fresh(300))
    static[0] = sink
    plan.compress_append_paged(K, V, table, seq, static, cws, max_new_chunks=8)

    def compressed(b, before_static):
        ks, vs = (x.view(torch.int16)[None].cpu().numpy().view("uint16") for x in rows[b])
        k2, v2, s2, st2, _ = oracle.compress_append(ks, vs, [rows[b][0].shape[1]], [before_static], lag, plan.k)
        n = int(s2[0])
        for i, x in enumerate((k2, v2)):
            rows[b][i] = torch.from_numpy(x.view("int16"))[0, :, :n].contiguous().view(BF16).to(DEV)
        assert int(seq[b]) == n and int(static[b]) == int(st2[0])

    compressed(0, sink)
    plan.pages_release(table, refs, seq, pws, page)
    consistent()
    plan.pages_fork(K, V, table, refs, seq, static, ints([0, 0]), ints([2, 1]), pws)
    rows[1], rows[2] = [x.clone() for x in rows[0]], [x.clone() for x in rows[0]]
    consistent()
    assert int((refs > 1).sum()) == int(static[0]) // page
    for step in range(14):
        plan.pages_reserve(table, refs, seq + T, pws, page)
        masks = U.random_tree(B, T, rng).to(DEV)
        Q = torch.randn((B, T, H * G, D), generator=g, device=DEV).to(BF16)
        for b in range(B):
            append(b, *fresh(T))
        got = plan.attend_tree_paged(Q, K, V, table, seq, aws, tree_mask=masks, want_lse=True)
        U.assert_attention(got, U.tree_reference(Q, *dense(), seq, [T] * B, masks))
        paths = [sorted(rng.sample(range(T), rng.randint(1, T))) for _ in range(B)]
        acc = torch.zeros((B, T), dtype=torch.int32)
        for b, p in enumerate(paths):
            acc[b, :len(p)] = torch.tensor(p)
        plan.tree_commit_paged(K, V, table, seq, acc.to(DEV), ints([len(p) for p in paths]), aws)
        for b, p in enumerate(paths):
            base = rows[b][0].shape[1] - T
            rows[b] = [torch.cat((x[:, :base], x[:, [base + j for j in p]]), 1) for x in rows[b]]
        before = static.tolist()
        plan.compress_append_paged(K, V, table, seq, static, cws, max_new_chunks=8)
        for b in range(B):
            compressed(b, before[b])
        plan.pages_release(table, refs, seq, pws, page)
        if step == 8:
            live = plan.pages_compact(K, V, table, refs, pws)
            assert not refs[int(live):].any() and refs[:int(live)].all()
        consistent()
    bounds = plan.new_block_bounds(nb * page, 16)
    plan.block_bounds_paged(K, table, seq, bounds, aws, block_rows=16)
    Q = torch.randn((B, 1, H * G, D), generator=g, device=DEV).to(BF16)
    got = plan.attend_blocks_paged(Q, K, V, table, seq, bounds, aws, block_rows=16, keep=6, want_lse=True, want_idx=True)
    for b in range(B):
        n = int(seq[b])
        for h in range(H):
            at = [r for j in got["idx"][b, 0, h].tolist() if j >= 0 for r in range(16 * j, min(n, 16 * j + 16))]
            assert n - 1 in at and 0 in at
            q = Q[b, 0, h * G:(h + 1) * G]
            o, l, to, tl = U.attention64(q, rows[b][0][h, at].float(), rows[b][1][h, at].float(), torch.ones((G, len(at)), dtype=torch.bool, device=DEV),
                                         D ** -0.5, 1.0, 1.0, BF16)
            sl = slice(h * G, (h + 1) * G)
            assert ((got["out"][b, 0, sl].double() - o).abs() <= to).all()
            assert ((got["lse"][b, 0, sl].double() - l).abs() <= tl).all()
    for ws in (pws, aws, cws):
        assert plan.read_status(ws)[0] == 0
