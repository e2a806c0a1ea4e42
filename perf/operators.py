"""The serving operators that read, score and manage a KV cache, as cases that can be timed and compared.

Three operators, each with a plain form in elementary torch operations and the library's calls:

* ``tree``   attention of T drafted tokens per sequence over a contiguous or paged cache (T = 1 is a decode step);
* ``sparse`` attention over the blocks of rows that a per-channel min / max bound selects for each query, and
  ``bounds``, which builds those bounds from a cache;
* ``fork``, ``turnover``, ``compact``: the pages of a paged cache shared and copied, freed and handed out, renumbered.

Cache shapes are those of the compress pass's own workloads (8 or 4 KV heads, head_dim 128, 32768 or 131072 rows
before and 9728 or 19968 after compression) and generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}
ELEM = {"bf16": 2, "fp16": 2, "fp8": 1}


def listed():
    return [
        # one user, the token after a short compressed prompt: latency alone counts
        dict(name="tree_t1_b1_short", op="tree", dtype="bf16", B=1, H=8, G=4, D=128, S=1216, T=1, page=0, tree=False),
        # a decode step of a served batch in pages, seven query heads to a KV head, ragged lengths
        dict(name="tree_t1_b16_paged", op="tree", dtype="bf16", B=16, H=4, G=7, D=128, S=16384, T=1, page=64, tree=False),
        # speculative decoding over caches that the compress pass cut from 32768 to 9728 rows
        dict(name="tree_t32_b16", op="tree", dtype="bf16", B=16, H=8, G=4, D=128, S=9728, T=32, page=0, tree=True),
        # an odd tree over an fp8 cache in small pages
        dict(name="tree_t13_b8_fp8_paged", op="tree", dtype="fp8", B=8, H=8, G=4, D=128, S=19968, T=13, page=16, tree=True),
        # the widest tree over the longest cache
        dict(name="tree_t64_b2_128k", op="tree", dtype="fp16", B=2, H=8, G=4, D=128, S=131072, T=64, page=0, tree=True),
        # one user with a 32768-row cache: 16 of its 512 blocks
        dict(name="sparse_b1_32k", op="sparse", dtype="bf16", B=1, H=8, G=4, D=128, S=32768, T=1, page=0, rows=64, keep=16),
        # a batch with odd lengths, five tokens each, head_dim 64, blocks of 32 rows
        dict(name="sparse_t5_b6_odd", op="sparse", dtype="fp16", B=6, H=4, G=7, D=64, S=16411, T=5, page=0, rows=32, keep=24),
        # a batch of the longest caches, in pages
        dict(name="sparse_b8_128k_paged", op="sparse", dtype="bf16", B=8, H=8, G=4, D=128, S=131072, T=1, page=64, rows=64, keep=64),
        # the bounds of all 32 layers' caches after a prompt
        dict(name="bounds_32k", op="bounds", dtype="bf16", B=32, H=8, D=128, S=32768, page=0, rows=64),
        # one prompt forked into four continuations
        dict(name="fork_1_to_4", op="fork", dtype="bf16", B=8, H=8, D=128, S=1216, page=16, forks=4, recent=272),
        # a batch of prompts forked, each once, windows of three partitions of 1024 rows copied
        dict(name="fork_16", op="fork", dtype="bf16", B=32, H=8, D=128, S=9728, page=64, forks=16, recent=2500),
        # a pool left full of holes by freed sequences, made dense
        dict(name="compact_half", op="compact", dtype="bf16", B=16, H=8, D=128, S=8192, page=64, holes=2),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(("tree", "tree", "tree", "sparse", "sparse", "bounds", "fork", "compact", "turnover"))
    H, G, D = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8)), rng.choice((64, 96, 128, 128, 256))
    dtype, page = rng.choice(("bf16", "bf16", "fp16", "fp8")), rng.choice((0, 0, 16, 32, 64, 128))
    if op in ("tree", "sparse"):
        B, S = log(1, 32), log(70, 100000)
        while B * H * S * D > 1 << 28:
            B, S = max(1, B // 2), S * 3 // 4
        if op == "tree":
            T = rng.choice((1, 1, 2, log(3, 64), log(3, 64)))
            while B * H * G * T * S * D > 1 << 34:
                T, S = max(1, T // 2), max(70, S * 3 // 4)
            return dict(op=op, dtype=dtype, B=B, H=H, G=G, D=D, S=S, T=T, page=page, tree=T > 1 and rng.random() < 0.7)
        return dict(op=op, dtype=dtype, B=B, H=H, G=G, D=D, S=S, T=rng.choice((1, 1, 1, log(2, 8))), page=page,
                    rows=rng.choice((16, 32, 64, 128)), keep=log(3, 96))
    if op == "bounds":
        B, S = log(1, 64), log(1, 60000)
        while B * H * S * D > 1 << 29:
            B, S = max(1, B // 2), S * 3 // 4
        return dict(op=op, dtype=dtype, B=B, H=H, D=D, S=S, page=page, rows=rng.choice((16, 32, 64, 128)))
    page, dtype = rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "fp16"))
    B, S = log(3, 48), log(100, 12000)
    while B * H * S * D > 1 << 28:
        B, S = max(3, B // 2), S * 3 // 4
    if op == "fork":
        return dict(op=op, dtype=dtype, B=B, H=H, D=D, S=S, page=page, forks=rng.randint(1, max(1, B // 2)), recent=min(S, log(1, 3000)))
    if op == "compact":
        return dict(op=op, dtype=dtype, B=B, H=H, D=D, S=S, page=page, holes=rng.choice((2, 3, 4)))
    return dict(op="turnover", dtype=dtype, B=B, H=H, D=D, S=S, page=page, room=rng.randint(1, 64))


# ------------------------------------------------------------------------------------ the inputs
def lengths(case):
    """Rows of each sequence: the case's length, and ragged shorter ones down to half of it."""
    S, T = case["S"], case.get("T", 1)
    return [max(T, min(S, S - (S * ((b * 7) % 16)) // 32 - (b % 3 if b else 0))) for b in range(case["B"])]


def _draw_kv(shape, dim_h, g, dev, sigma, dtype):
    """Values with outlier channels of each head (what keys look like), or without (values): sigma 0."""
    x = torch.randn(shape, generator=g, device=dev, dtype=torch.float32)
    if sigma:
        per = [1] * len(shape)
        per[dim_h], per[-1] = shape[dim_h], shape[-1]
        x *= torch.exp(sigma * torch.randn(per, generator=g, device=dev, dtype=torch.float32))
    if dtype == torch.float8_e4m3fn:
        unit = float(x.abs().max()) / 400.0
        return (x / unit).to(dtype), unit
    return x.to(dtype), 1.0


def _tree_masks(B, T, rng):
    """64-bit masks of random trees: a token sees itself and its ancestors."""
    parent = np.array([[rng.integers(max(-1, i - 6), i) for i in range(T)] for _ in range(B)])
    masks = np.zeros((B, T), dtype=np.uint64)
    for i in range(T):
        up = np.where(parent[:, i] >= 0, masks[np.arange(B), np.maximum(parent[:, i], 0)], np.uint64(0))
        masks[:, i] = up | np.uint64(1 << i)
    return masks.view(np.int64)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    op, B, H, D, S, page = case["op"], case["B"], case["H"], case["D"], case["S"], case["page"]
    dtype = DTYPES[case["dtype"]]
    s = {"case": dict(case), "op": op}
    lens = lengths(case)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    if op in ("fork", "compact", "turnover"):
        return _prepare_pages(s, case, lens, g, rng, dev, dtype)
    if page:
        nb = -(-S // page)
        pages = B * nb + 3
        s["table"] = torch.from_numpy(rng.permutation(pages)[:B * nb].reshape(B, nb).astype(np.int32)).to(dev)
        shape = (pages, H, page, D)
    else:
        shape = (B, H, S, D)
    s["K"], s["k_scale"] = _draw_kv(shape, 1, g, dev, 1.0, dtype)
    if op != "bounds":
        s["V"], s["v_scale"] = _draw_kv(shape, 1, g, dev, 0.0, dtype)
        T, G = case["T"], case["G"]
        qdt = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
        s["Q"] = torch.randn((B, T, H * G, D), generator=g, device=dev, dtype=torch.float32).to(qdt)
    if op == "tree":
        s["draft_len"] = torch.full((B,), case["T"], dtype=torch.int32, device=dev)
        s["mask"] = torch.from_numpy(_tree_masks(B, case["T"], rng)).to(dev) if case["tree"] else None
    if op in ("sparse", "bounds"):
        nblk = -(-S // case["rows"]) if not page else -(-(nb * page) // case["rows"])
        s["bounds"] = torch.zeros((B, H, nblk, 2, D), dtype=dtype, device=dev)
        if op == "sparse":
            _plain_bounds(s)
    if own:
        from paper_2504_04704_b200 import binding
        s["plan"] = binding.Plan(B, H, D, sink=16, lag=128, dtype=dtype, device=torch.cuda.current_device())
        if op == "bounds":
            s["ws"] = s["plan"].new_workspace()
        else:
            s["ws"] = s["plan"].new_attend_workspace(case["T"], H * case["G"], blocks=s["bounds"].shape[2] if op == "sparse" else 0,
                                                     keep=case.get("keep", 0))
    return s


def _prepare_pages(s, case, lens, g, rng, dev, dtype):
    op, B, H, D, S, page = case["op"], case["B"], case["H"], case["D"], case["S"], case["page"]
    nb = -(-(S + case.get("room", 0)) // page)
    table = np.full((B, nb), -1, dtype=np.int32)
    if op == "fork":  # the first sequences hold rows, the last ones are empty and take the forks
        sources = max(1, B - case["forks"])
        lens = [n if b < sources else 0 for b, n in enumerate(lens)]
        src = [i % sources for i in range(case["forks"])]
        if case["forks"] < B // 2 or sources == 1:
            src = [0] * case["forks"]
        s["src"] = torch.tensor(src, dtype=torch.int32, device=dev)
        s["dst"] = torch.tensor([B - 1 - i for i in range(min(case["forks"], B - 1))][:len(src)], dtype=torch.int32, device=dev)
        s["src"] = s["src"][:s["dst"].numel()].contiguous()
    if op == "compact":  # every `holes`-th sequence has ended: its pages are free
        lens = [0 if b % case["holes"] == 1 else n for b, n in enumerate(lens)]
    pages = B * nb + 5
    perm = rng.permutation(pages).astype(np.int32)
    used, need = 0, np.array([-(-n // page) for n in lens])
    for b in range(B):
        table[b, :need[b]] = perm[used:used + need[b]]
        used += need[b]
    refs = np.zeros(pages, dtype=np.int32)
    refs[table[table >= 0]] = 1
    s["table"] = torch.from_numpy(table).to(dev)
    s["refs"] = torch.from_numpy(refs).to(dev)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["static_len"] = torch.clamp(s["seq_len"] - case.get("recent", 0), min=0)
    if op == "turnover":  # the compress pass has just shortened these sequences; then the next rows need room
        s["keep"] = (s["seq_len"].long() * 5 // 8).to(torch.int32)
        s["want"] = s["keep"] + case["room"]
    else:
        s["K"] = _draw_kv((pages, H, page, D), 1, g, dev, 1.0, dtype)[0]
        s["V"] = _draw_kv((pages, H, page, D), 1, g, dev, 0.0, dtype)[0]
    if own:
        from paper_2504_04704_b200 import binding
        s["plan"] = binding.Plan(B, H, D, sink=16, lag=128, dtype=dtype, device=torch.cuda.current_device())
        s["ws"] = s["plan"].new_pages_workspace(pages)
    return s


# ------------------------------------------------------------------------------------ one pass
def run(s):
    return {"tree": _tree, "sparse": _sparse, "bounds": _bounds, "fork": _fork, "compact": _compact,
            "turnover": _turnover}[s["op"]](s)


def _tree(s):
    if own:
        kw = dict(draft_len=s["draft_len"], tree_mask=s["mask"], k_scale=s["k_scale"], v_scale=s["v_scale"], want_lse=True)
        if s["case"]["page"]:
            return s["plan"].attend_tree_paged(s["Q"], s["K"], s["V"], s["table"], s["seq_len"], s["ws"], **kw)
        return s["plan"].attend_tree(s["Q"], s["K"], s["V"], s["seq_len"], s["ws"], **kw)
    return _plain_tree(s)


def _sparse(s):
    if own:
        kw = dict(block_rows=s["case"]["rows"], keep=s["case"]["keep"], sink_blocks=1, recent_blocks=2, k_scale=s["k_scale"],
                  v_scale=s["v_scale"], want_lse=True, want_idx=True)
        if s["case"]["page"]:
            return s["plan"].attend_blocks_paged(s["Q"], s["K"], s["V"], s["table"], s["seq_len"], s["bounds"], s["ws"], **kw)
        return s["plan"].attend_blocks(s["Q"], s["K"], s["V"], s["seq_len"], s["bounds"], s["ws"], **kw)
    return _plain_sparse(s)


def _bounds(s):
    if own:
        if s["case"]["page"]:
            s["plan"].block_bounds_paged(s["K"], s["table"], s["seq_len"], s["bounds"], s["ws"], block_rows=s["case"]["rows"])
        else:
            s["plan"].block_bounds(s["K"], s["seq_len"], s["bounds"], s["ws"], block_rows=s["case"]["rows"])
    else:
        _plain_bounds(s)
    return s["bounds"].float() if s["case"]["dtype"] == "fp8" else s["bounds"]


def _fork(s):
    # the tables are the program's own and change with the call: a copy, so that the pass can be made again
    t = {k: s[k].clone() for k in ("table", "refs", "seq_len", "static_len")}
    if own:
        s["plan"].pages_fork(s["K"], s["V"], t["table"], t["refs"], t["seq_len"], t["static_len"], s["src"], s["dst"], s["ws"])
    else:
        _plain_fork(s, t)
    return dict(t, K=s["K"], V=s["V"])


def _compact(s):
    t = {k: s[k].clone() for k in ("table", "refs")}
    if own:
        t["live"] = s["plan"].pages_compact(s["K"], s["V"], t["table"], t["refs"], s["ws"])
    else:
        t["live"] = _plain_compact(s, t)
    return dict(t, K=s["K"], V=s["V"])


def _turnover(s):
    t = {k: s[k].clone() for k in ("table", "refs")}
    if own:
        s["plan"].pages_release(t["table"], t["refs"], s["keep"], s["ws"], page_size=s["case"]["page"])
        s["plan"].pages_reserve(t["table"], t["refs"], s["want"], s["ws"], page_size=s["case"]["page"])
    else:
        _plain_release(t, s["keep"], s["case"]["page"])
        _plain_reserve(t, s["want"], s["case"]["page"])
    return t


# ------------------------------------------------------------------------------------ plain forms
def _dense(s, x):
    """The cache as [B, H, rows, D] (pages looked up in the table)."""
    if not s["case"]["page"]:
        return x
    bits = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    t = bits[s["table"].long()]
    B, nb, H, page, D = t.shape
    return t.permute(0, 2, 1, 3, 4).reshape(B, H, nb * page, D).view(x.dtype)


def _attention(q, k, v, seen, scale, v_scale):
    """Softmax attention in 32 bits: q [..., M, D], k / v [..., R, D], seen [..., M, R] (or one that broadcasts to it)."""
    logits = (q @ k.transpose(-1, -2)) * scale
    logits = torch.where(seen, logits, float("-inf"))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, 1.0, total) * v_scale
    return out, (top + torch.log(total)).squeeze(-1)


def _plain_tree(s):
    c, Q, n = s["case"], s["Q"], s["seq_len"].long()
    B, H, G, D, T = c["B"], c["H"], c["G"], c["D"], c["T"]
    K, V = _dense(s, s["K"]), _dense(s, s["V"])
    R = K.shape[2]
    q = Q.float().view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    at = torch.arange(R, device=Q.device)[None, None] - (n - s["draft_len"].long())[:, None, None]  # [B, 1, R], drafted rows from 0
    token = torch.arange(T, device=Q.device)[None, :, None]
    if s["mask"] is None:
        hit = at <= token
    else:
        hit = ((s["mask"][:, :, None] >> at.clamp(0, 63)) & 1) != 0
    seen = (at < 0) | ((at < s["draft_len"].long()[:, None, None]) & hit)
    seen = seen & (token < s["draft_len"].long()[:, None, None])
    seen = seen[:, None, :, None].expand(B, 1, T, G, R).reshape(B, 1, T * G, R)
    out, lse = _attention(q, K.float(), V.float(), seen, s["k_scale"] / math.sqrt(D), s["v_scale"])
    out = out.view(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(Q.dtype)
    return {"out": out, "lse": lse.view(B, H, T, G).permute(0, 2, 1, 3).reshape(B, T, H * G).contiguous()}


def _plain_bounds(s):
    c = s["case"]
    rows, bounds = c["rows"], s["bounds"]
    K = _dense(s, s["K"])
    B, H, R, D = K.shape
    blocks = bounds.shape[2]
    k = torch.nn.functional.pad(K.to(torch.float16 if c["dtype"] == "fp8" else K.dtype), (0, 0, 0, blocks * rows - R)).view(B, H, blocks, rows, D)
    valid = (torch.arange(blocks * rows, device=K.device)[None] < s["seq_len"].long()[:, None]).view(B, 1, blocks, rows, 1)
    low = torch.where(valid, k, float("inf")).amin(3)
    high = torch.where(valid, k, float("-inf")).amax(3)
    used = valid.any(3)
    bounds.copy_(torch.where(used[:, :, :, None], torch.stack((low, high), 3).float(), bounds.float()))


def _plain_sparse(s):
    c, Q, n = s["case"], s["Q"], s["seq_len"].long()
    B, H, G, D, T, rows, keep = c["B"], c["H"], c["G"], c["D"], c["T"], c["rows"], c["keep"]
    dev = Q.device
    blocks = s["bounds"].shape[2]
    q = Q.view(B, T, H, G, D).permute(0, 2, 1, 3, 4)                                         # [B, H, T, G, D]
    bound = s["bounds"].to(torch.float64)
    q64 = q.reshape(B, H, T * G, D).to(torch.float64)
    score = q64.clamp(min=0) @ bound[:, :, :, 1].transpose(-1, -2) + q64.clamp(max=0) @ bound[:, :, :, 0].transpose(-1, -2)
    score = score.view(B, H, T, G, blocks).amax(3)                                            # next to the border: 64 bits
    end = n[:, None] - (T - 1) + torch.arange(T, device=dev)[None]                            # rows that token t sees
    nblk = ((end + rows - 1) // rows)[:, None, :, None]
    j = torch.arange(blocks, device=dev)[None, None, None]
    score = torch.where((j < 1) | (j >= nblk - 2), float("inf"), score)
    score = torch.where(j < nblk, score, float("-inf"))
    best, order = torch.sort(score, dim=-1, descending=True, stable=True)
    kept = min(keep, blocks)
    order = torch.where(best[..., :kept] > float("-inf"), order[..., :kept], blocks)
    order = torch.sort(order, dim=-1).values                                                  # ascending, missing ones last
    at = (order[..., None] * rows + torch.arange(rows, device=dev)).reshape(B, H, T, kept * rows)
    seen = at < end[:, None, :, None]
    cap = (s["K"].shape[2] if not c["page"] else s["table"].shape[1] * c["page"]) - 1
    at = torch.where(seen, at, 0).clamp(max=cap)
    head = torch.arange(H, device=dev)[None, :, None, None]
    seq = torch.arange(B, device=dev)[:, None, None, None]
    if c["page"]:
        where = (s["table"].long()[seq, at // c["page"]], head, at % c["page"])
    else:
        where = (seq, head, at)
    k, v = (x.view(torch.uint8)[where].view(x.dtype).float() if c["dtype"] == "fp8" else x[where].float() for x in (s["K"], s["V"]))
    out, lse = _attention(q.float(), k, v, seen[:, :, :, None], s["k_scale"] / math.sqrt(D), s["v_scale"])
    idx = torch.full((B, T, H, keep), -1, dtype=torch.int32, device=dev)
    idx[..., :kept] = torch.where(order < blocks, order, -1).permute(0, 2, 1, 3).to(torch.int32)
    return {"out": out.permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(Q.dtype),
            "lse": lse.permute(0, 2, 1, 3).reshape(B, T, H * G).contiguous(), "idx": idx}


def _plain_fork(s, t):
    page, table, refs = s["case"]["page"], t["table"], t["refs"]
    src, dst = s["src"].long(), s["dst"].long()
    nb = table.shape[1]
    n, static = t["seq_len"][src].long(), t["static_len"][src].long()
    j = torch.arange(nb, device=table.device)[None]
    used = (n + page - 1) // page
    shared = j < torch.minimum(static // page, used)[:, None]
    copied = (j < used[:, None]) & ~shared
    free = torch.argsort((refs != 0).to(torch.uint8), stable=True)                            # free pages first, lowest first
    old = table[src].long()
    rank = (torch.cumsum(copied.reshape(-1).long(), 0) - 1).clamp(min=0).view_as(old)
    new = torch.where(copied, free[rank.clamp(max=free.numel() - 1)], old)
    refs.index_add_(0, old.clamp(min=0).reshape(-1), shared.reshape(-1).to(torch.int32))
    refs.index_add_(0, new.clamp(min=0).reshape(-1), copied.reshape(-1).to(torch.int32))
    table[dst] = torch.where(j < used[:, None], new, -1).to(torch.int32)
    t["seq_len"][dst], t["static_len"][dst] = t["seq_len"][src], t["static_len"][src]
    pick = copied.reshape(-1).nonzero().squeeze(1)
    a, b = old.reshape(-1)[pick], new.reshape(-1)[pick]
    s["K"][b], s["V"][b] = s["K"][a], s["V"][a]


def _plain_compact(s, t):
    table, refs = t["table"], t["refs"]
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.numel(), device=refs.device)
    hole = (~live) & (at < count)
    mover = live & (at >= count)
    to, frm = hole.nonzero().squeeze(1), mover.nonzero().squeeze(1)
    name = at.clone()
    name[frm] = to
    s["K"][to], s["V"][to] = s["K"][frm], s["V"][frm]
    refs[to] = refs[frm]
    refs[frm] = 0
    table.copy_(torch.where(table >= 0, name[table.clamp(min=0).long()].to(torch.int32), table))
    return count.to(torch.int32).reshape(1)


def _plain_release(t, keep, page):
    table, refs = t["table"], t["refs"]
    j = torch.arange(table.shape[1], device=table.device)[None]
    drop = (j >= ((keep.long() + page - 1) // page)[:, None]) & (table >= 0)
    refs.index_add_(0, table.clamp(min=0).long().reshape(-1), -drop.reshape(-1).to(torch.int32))
    table.copy_(torch.where(drop, -1, table))


def _plain_reserve(t, want, page):
    table, refs = t["table"], t["refs"]
    j = torch.arange(table.shape[1], device=table.device)[None]
    lack = (j < ((want.long() + page - 1) // page)[:, None]) & (table < 0)
    free = torch.argsort((refs != 0).to(torch.uint8), stable=True)
    rank = (torch.cumsum(lack.reshape(-1).long(), 0) - 1).clamp(0, free.numel() - 1).view_as(lack)
    new = free[rank]
    refs.index_add_(0, torch.where(lack, new, 0).reshape(-1), lack.reshape(-1).to(torch.int32))
    table.copy_(torch.where(lack, new.to(torch.int32), table))


# ------------------------------------------------------------------------------------ what a pass has to do
def work(case):
    op, B, H, D = case["op"], case["B"], case["H"], case["D"]
    eb, lens = ELEM[case["dtype"]], lengths(case)
    row = D * eb
    if op == "tree":
        T, Hq = case["T"], H * case["G"]
        return {"bytes": sum(lens) * H * 2 * row + 2 * B * T * Hq * D * 2 + 4 * B * T * Hq, "flops": 4 * T * Hq * D * sum(lens)}
    if op == "sparse":
        T, Hq, rows, keep = case["T"], H * case["G"], case["rows"], case["keep"]
        blocks = sum(-(-n // rows) for n in lens)
        read = sum(min(n - T + 1 + t, keep * rows) for n in lens for t in range(T))
        return {"bytes": blocks * H * 2 * row + read * H * 2 * row + 2 * B * T * Hq * D * 2 + 4 * B * T * (Hq + H * keep),
                "flops": 4 * Hq * D * (read + T * blocks)}
    if op == "bounds":
        return {"bytes": sum(lens) * H * row + sum(-(-n // case["rows"]) for n in lens) * H * 2 * row, "flops": 2 * sum(lens) * H * D}
    page, nb = case["page"], -(-(case["S"] + case.get("room", 0)) // case["page"])
    tables = 2 * 4 * (B * nb + B * nb + 5)
    if op == "fork":
        sources = max(1, B - case["forks"])
        src = [i % sources for i in range(case["forks"])]
        if case["forks"] < B // 2 or sources == 1:
            src = [0] * case["forks"]
        src = src[:B - 1]
        copied = sum(-(-lens[b] // page) - max(0, lens[b] - case["recent"]) // page for b in src)
        return {"bytes": copied * page * H * 4 * row + tables, "flops": 0}
    if op == "compact":
        lens = [0 if b % case["holes"] == 1 else n for b, n in enumerate(lens)]
        live = sum(-(-n // page) for n in lens)
        moved = live - live * live // (B * nb + 5)                # pages lie in random order
        return {"bytes": moved * page * H * 4 * row + tables, "flops": 0}
    return {"bytes": 2 * tables, "flops": 0}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def _row64(s, x, b, h, rows):
    """Rows `rows` of one head of one sequence, in 64 bits."""
    c = s["case"]
    if c["page"]:
        p = s["table"][b, torch.div(rows, c["page"], rounding_mode="floor")].long()
        x, i = x[:, h], (p, rows % c["page"])
    else:
        x, i = x[b, h], (rows,)
    return (x.view(torch.uint8)[i].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[i]).double()


def exact(case, seed):
    s = prepare(case, seed)
    op, B, H, D = case["op"], case["B"], case["H"], case["D"]
    if op in ("tree", "sparse"):
        T, G = case["T"], case["G"]
        out = torch.zeros((B, T, H, G, D), dtype=torch.float64, device=s["Q"].device)
        lse = torch.full((B, T, H, G), -math.inf, dtype=torch.float64, device=out.device)
        unit = 1.0 / math.sqrt(D) * s["k_scale"]
        for b, n in enumerate(lengths(case)):
            for h in range(H):
                q = s["Q"][b, :, h * G:(h + 1) * G].double()
                if op == "tree":
                    rows = torch.arange(n, device=out.device)
                    k, v = (_row64(s, s[x], b, h, rows) for x in "KV")
                    z = torch.einsum("tgd,rd->tgr", q, k) * unit
                    if s["mask"] is None:
                        hid = torch.ones((T, T), dtype=torch.bool, device=out.device).triu(1)
                    else:
                        bits = s["mask"][b].cpu().numpy().view(np.uint64)
                        hid = torch.tensor([[not (int(m) >> i) & 1 for i in range(T)] for m in bits], device=out.device)
                    z[:, :, n - T:].masked_fill_(hid[:, None], -math.inf)
                    lse[b, :, h] = torch.logsumexp(z, -1)
                    out[b, :, h] = torch.einsum("tgr,rd->tgd", torch.softmax(z, -1), v) * s["v_scale"]
                    continue
                R, keep = case["rows"], case["keep"]
                lo, hi = s["bounds"][b, h, :, 0].double(), s["bounds"][b, h, :, 1].double()
                for t in range(T):
                    end = n - (T - 1 - t)
                    m = -(-end // R)
                    worth = torch.stack([torch.maximum(q[t, g] * lo[:m], q[t, g] * hi[:m]).sum(-1) for g in range(G)]).amax(0).cpu().numpy()
                    worth[:1] = math.inf
                    worth[max(0, m - 2):] = math.inf
                    pick = np.sort(np.argsort(-worth, kind="stable")[:keep])
                    rows = (torch.from_numpy(pick).to(out.device)[:, None] * R + torch.arange(R, device=out.device)).reshape(-1)
                    rows = rows[rows < end]
                    k, v = (_row64(s, s[x], b, h, rows) for x in "KV")
                    z = (q[t] @ k.T) * unit
                    lse[b, t, h] = torch.logsumexp(z, -1)
                    out[b, t, h] = torch.softmax(z, -1) @ v * s["v_scale"]
        return {"out": out.reshape(B, T, H * G, D), "lse": lse.reshape(B, T, H * G), "idx": None}
    if op == "bounds":
        R = case["rows"]
        want = s["bounds"].double()
        for b, n in enumerate(lengths(case)):
            whole = n // R
            for h in range(H):
                k = _row64(s, s["K"], b, h, torch.arange(n, device=want.device))
                full = k[:whole * R].view(whole, R, D)
                if whole:
                    want[b, h, :whole, 0], want[b, h, :whole, 1] = full.min(1).values, full.max(1).values
                if n % R:
                    want[b, h, whole, 0], want[b, h, whole, 1] = k[whole * R:].min(0).values, k[whole * R:].max(0).values
        return want
    if op == "turnover":
        return None  # whole numbers alone
    table, refs = s["table"].cpu().numpy(), s["refs"].cpu().numpy()
    pairs = []
    if op == "fork":
        free = iter(np.flatnonzero(refs == 0).tolist())
        n, static = s["seq_len"].tolist(), s["static_len"].tolist()
        for b in s["src"].tolist():
            pairs += [(int(table[b, j]), next(free)) for j in range(static[b] // case["page"], -(-n[b] // case["page"]))]
    else:
        count = int((refs > 0).sum())
        pairs = list(zip((count + np.flatnonzero(refs[count:] > 0)).tolist(), np.flatnonzero(refs[:count] == 0).tolist()))
    a, b = (torch.tensor([p[i] for p in pairs], dtype=torch.long, device=s["K"].device) for i in (0, 1))
    got = {}
    for x in "KV":
        y = s[x].double()
        y[b] = y[a]
        got[x] = y
    return got
