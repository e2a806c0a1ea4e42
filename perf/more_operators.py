"""A KV cache held in 8 bits with a scale for each block of rows and head, as cases that can be timed and compared.

Three operators, each with a plain form in elementary torch operations and the library's calls:

* ``attend`` attention of T drafted tokens per sequence over such a cache (T = 1 is a decode step), contiguous or paged;
* ``store``  rows of K and V quantised as they are written, and the blocks they lie in read back in 16 bits;
* ``read``   a cache, or chosen rows of it, read back in 16 bits.

Codes are int8 (the scale is the largest magnitude of the block over 127) or e4m3 (the least power of two that brings
it to 448 or below).  Cache shapes are those of the compress pass's own workloads (8 or 4 KV heads, head_dim 128, 32768
rows before and 9728 after compression) and generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FORMATS = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -126


def listed():
    return [
        # one user, the token after a short compressed prompt: latency alone counts
        dict(name="attend_t1_b1_short", op="attend", dtype="bf16", form="int8", B=1, H=8, G=4, D=128, S=1216, T=1, page=0, rows=64, tree=False, cap=0.0),
        # a decode step of a served batch in pages, seven query heads to a KV head, ragged lengths
        dict(name="attend_t1_b16_paged", op="attend", dtype="bf16", form="e4m3", B=16, H=4, G=7, D=128, S=16384, T=1, page=64, rows=64, tree=False, cap=0.0),
        # a decode step of a large batch of long, uncompressed caches
        dict(name="attend_t1_b32_32k", op="attend", dtype="bf16", form="int8", B=32, H=8, G=4, D=128, S=32768, T=1, page=0, rows=128, tree=False, cap=0.0),
        # a small tree for a model that caps its logits, head_dim 64, odd lengths
        dict(name="attend_t5_b6_odd", op="attend", dtype="fp16", form="int8", B=6, H=4, G=7, D=64, S=16411, T=5, page=0, rows=32, tree=True, cap=30.0),
        # speculative decoding over caches that the compress pass cut from 32768 to 9728 rows
        dict(name="attend_t32_b16", op="attend", dtype="bf16", form="e4m3", B=16, H=8, G=4, D=128, S=9728, T=32, page=0, rows=64, tree=True, cap=0.0),
        # the widest tree over the longest cache
        dict(name="attend_t64_b2_128k", op="attend", dtype="fp16", form="int8", B=2, H=8, G=4, D=128, S=131072, T=64, page=0, rows=64, tree=True, cap=0.0),
        # the new row of each sequence of a batch, into blocks that hold rows already
        dict(name="store_step_b32", op="store", dtype="bf16", form="int8", B=32, H=8, D=128, S=4096, T=1, page=64, rows=64, take=False),
        # a chunk of a prompt behind ragged prefixes, small pages
        dict(name="store_chunk_b8", op="store", dtype="fp16", form="e4m3", B=8, H=8, D=128, S=9728, T=1024, page=16, rows=16, take=False),
        # the rows that the compress pass keeps of 32 layers' prompts, quantised straight from the raw caches
        dict(name="store_prompt_kept", op="store", dtype="bf16", form="int8", B=32, H=8, D=128, S=9728, T=9728, page=0, rows=64, take=True),
        # odd sizes: head_dim 96, five sequences, three heads
        dict(name="store_odd", op="store", dtype="bf16", form="e4m3", B=5, H=3, D=96, S=7001, T=2503, page=0, rows=32, take=False),
        # whole caches read back before the compress pass runs on them again
        dict(name="read_b32", op="read", dtype="bf16", form="e4m3", B=32, H=8, D=128, S=9728, page=0, rows=64, picks=0),
        # chosen rows of paged caches
        dict(name="read_picks_paged", op="read", dtype="fp16", form="int8", B=4, H=8, D=128, S=16384, page=32, rows=32, picks=1216),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(("attend", "attend", "attend", "store", "store", "read"))
    H, G, D = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8)), rng.choice((64, 96, 128, 128, 256))
    c = dict(op=op, dtype=rng.choice(("bf16", "fp16")), form=rng.choice(("int8", "e4m3")), B=log(1, 32), H=H, D=D)
    c["page"] = rng.choice((0, 0, 16, 32, 64, 128))
    c["rows"] = rng.choice([r for r in (16, 32, 64, 128) if r <= (c["page"] or 128)])
    if op == "attend":
        S, T = log(70, 100000), rng.choice((1, 1, 2, log(3, 64), log(3, 64)))
        while c["B"] * H * S * D > 1 << 28:
            c["B"], S = max(1, c["B"] // 2), S * 3 // 4
        while c["B"] * H * G * T * S * D > 1 << 34:
            T, S = max(1, T // 2), max(70, S * 3 // 4)
        return dict(c, G=G, S=S, T=T, tree=T > 1 and rng.random() < 0.7, cap=rng.choice((0.0, 0.0, 20.0, 50.0)))
    S = log(70, 20000)
    while c["B"] * H * S * D > 1 << 27:
        c["B"], S = max(1, c["B"] // 2), S * 3 // 4
    if op == "store":
        take = rng.random() < 0.3
        return dict(c, S=S, T=rng.choice((1, log(1, S), log(1, S))), take=take)
    return dict(c, S=S, picks=rng.choice((0, log(1, S))))


# ------------------------------------------------------------------------------------ the inputs
def lengths(case):
    """Rows of each sequence: the case's length, and ragged shorter ones down to half of it."""
    S, T = case["S"], case.get("T", 1)
    if case.get("take"):
        return [S] * case["B"]
    return [max(T, min(S, S - (S * ((b * 7) % 16)) // 32 - (b % 3 if b else 0))) for b in range(case["B"])]


def _draw_kv(shape, g, dev, sigma, dtype):
    """Values [B, H, rows, D] with outlier channels of each head (what keys look like), or without (values): sigma 0."""
    x = torch.randn(shape, generator=g, device=dev, dtype=torch.float32)
    if sigma:
        x *= torch.exp(sigma * torch.randn((1, shape[1], 1, shape[3]), generator=g, device=dev, dtype=torch.float32))
    return x.to(dtype)


def _tree_masks(B, T, rng):
    """64-bit masks of random trees: a token sees itself and its ancestors."""
    parent = np.array([[rng.integers(max(-1, i - 6), i) for i in range(T)] for _ in range(B)])
    masks = np.zeros((B, T), dtype=np.uint64)
    for i in range(T):
        up = np.where(parent[:, i] >= 0, masks[np.arange(B), np.maximum(parent[:, i], 0)], np.uint64(0))
        masks[:, i] = up | np.uint64(1 << i)
    return masks.view(np.int64)


def _kept_rows(B, H, n, rng):
    """[B, H, n] ascending source rows: a sink of 16, a quarter of each stretch of 1024 after it, then everything."""
    heads = np.empty((8, n), dtype=np.int32)
    for i in range(8):
        rows, at = [np.arange(min(16, n))], 16
        while sum(len(r) for r in rows) + 256 < n - 1024:
            rows.append(at + np.sort(rng.permutation(1024)[:256]))
            at += 1024
        left = n - sum(len(r) for r in rows)
        heads[i] = np.concatenate(rows + [at + np.arange(left)])[:n]
    return heads[np.arange(B * H) % 8].reshape(B, H, n), int(heads.max()) + 1


def _bytes(x):
    """Codes as plain bytes, which can be indexed whatever their format."""
    return x.view(torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    op, B, H, D, S, page, R, form = (case[k] for k in ("op", "B", "H", "D", "S", "page", "rows", "form"))
    dtype = DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    lens = lengths(case)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    cap = -(-S // page) * page if page else S
    s["capacity"] = cap
    if page:
        nb = cap // page
        pages = B * nb + 3
        s["table"] = torch.from_numpy(rng.permutation(pages)[:B * nb].reshape(B, nb).astype(np.int32)).to(dev)
    for x, sigma in (("K", 1.0), ("V", 0.0)):  # what the cache holds: every block quantised as a whole
        dense = torch.empty((B, H, cap, D), dtype=FORMATS[form], device=dev)
        scale = torch.empty((B, H, -(-cap // R)), dtype=torch.float32, device=dev)
        for b in range(B):
            v = _draw_kv((1, H, cap, D), g, dev, sigma, dtype)[0].float()
            v = torch.nn.functional.pad(v, (0, 0, 0, -cap % R)).view(H, -1, R, D)
            f = _fit(v.abs().amax((2, 3)), form)
            scale[b] = f
            dense[b] = _encode(v, f[:, :, None, None], form).view(H, -1, D)[:, :cap]
        if page:
            pool = torch.zeros((pages, H, page, D), dtype=torch.uint8, device=dev)
            pool[s["table"].reshape(-1).long()] = _bytes(dense).view(B, H, nb, page, D).permute(0, 2, 1, 3, 4).reshape(B * nb, H, page, D)
            dense = pool.view(FORMATS[form])
        s[x], s[x + "_scale"] = dense, scale
    if op == "attend":
        T, G = case["T"], case["G"]
        s["Q"] = torch.randn((B, T, H * G, D), generator=g, device=dev, dtype=torch.float32).to(dtype)
        s["draft_len"] = torch.full((B,), T, dtype=torch.int32, device=dev)
        s["mask"] = torch.from_numpy(_tree_masks(B, T, rng)).to(dev) if case["tree"] else None
    else:
        s["K16"] = torch.zeros((B, H, cap, D), dtype=dtype, device=dev)
        s["V16"] = torch.zeros((B, H, cap, D), dtype=dtype, device=dev)
    if op == "store":
        T = case["T"]
        s["from_len"] = torch.tensor([n - T for n in lens], dtype=torch.int32, device=dev)
        s["back"] = s["from_len"] // R * R       # the blocks that change, read back whole
        s["take"], rows = None, T
        if case["take"]:
            take, rows = _kept_rows(B, H, T, rng)
            s["take"] = torch.from_numpy(take).to(dev)
        s["K_new"] = torch.cat([_draw_kv((1, H, rows, D), g, dev, 1.0, dtype) for _ in range(B)])
        s["V_new"] = torch.cat([_draw_kv((1, H, rows, D), g, dev, 0.0, dtype) for _ in range(B)])
    if op == "read" and case["picks"]:
        low = min(lens)
        s["idx"] = torch.sort(torch.randint(0, low, (B, H, case["picks"]), generator=g, device=dev), -1).values.to(torch.int32)
    if own:
        from paper_2504_04704_b200 import binding
        s["plan"] = binding.Plan(B, H, D, sink=16, lag=128, dtype=dtype, device=torch.cuda.current_device())
        s["cache"] = binding.QuantCache(s["K"], s["V"], s["K_scale"], s["V_scale"], block_rows=R)
        s["ws"] = s["plan"].new_attend_quant_workspace(case["T"], H * case["G"]) if op == "attend" else s["plan"].new_workspace()
    return s


# ------------------------------------------------------------------------------------ one pass
def run(s):
    return {"attend": _attend, "store": _store, "read": _read}[s["case"]["op"]](s)


def _attend(s):
    if own:
        c = s["case"]
        kw = dict(draft_len=s["draft_len"], tree_mask=s["mask"], cap=c["cap"], want_lse=True)
        if c["page"]:
            return s["plan"].attend_quant_paged(s["Q"], s["cache"], s["table"], s["seq_len"], s["ws"], **kw)
        return s["plan"].attend_quant(s["Q"], s["cache"], s["seq_len"], s["ws"], **kw)
    return _plain_attend(s)


def _store(s):
    if own:
        kw = dict(from_len=s["from_len"], take=s["take"])
        back = dict(from_len=s["back"], K_out=s["K16"], V_out=s["V16"])
        if s["case"]["page"]:
            s["plan"].quant_write_paged(s["cache"], s["table"], s["K_new"], s["V_new"], s["seq_len"], s["ws"], **kw)
            s["plan"].quant_read_paged(s["cache"], s["table"], s["seq_len"], s["ws"], **back)
        else:
            s["plan"].quant_write(s["cache"], s["K_new"], s["V_new"], s["seq_len"], s["ws"], **kw)
            s["plan"].quant_read(s["cache"], s["seq_len"], s["ws"], **back)
    else:
        for x in "KV":
            _plain_write(s, x)
            _plain_read(s, x, s["back"])
    return {"K": s["K16"], "V": s["V16"], "K_scale": s["K_scale"], "V_scale": s["V_scale"]}


def _read(s):
    picks = s["case"]["picks"]
    if own:
        kw = dict(idx=s["idx"]) if picks else dict(K_out=s["K16"], V_out=s["V16"])
        if s["case"]["page"]:
            K, V = s["plan"].quant_read_paged(s["cache"], s["table"], s["seq_len"], s["ws"], **kw)
        else:
            K, V = s["plan"].quant_read(s["cache"], s["seq_len"], s["ws"], **kw)
        return {"K": K, "V": V}
    if picks:
        return {x: _plain_picks(s, x) for x in "KV"}
    for x in "KV":
        _plain_read(s, x, torch.zeros_like(s["seq_len"]))
    return {"K": s["K16"], "V": s["V16"]}


# ------------------------------------------------------------------------------------ plain forms
def _fit(top, form):
    """The scale that the largest magnitude of a block asks for."""
    if form == "int8":
        f = (top.double() / TOP[form]).float()                # correctly rounded
    else:
        m, e = torch.frexp(top.float())                      # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
        f = torch.ldexp(torch.ones_like(m), e - 9 + (m > 0.875).to(e.dtype))
    return torch.where(top > 0, f.clamp(min=TINY), torch.zeros_like(f))


def _encode(x, scale, form):
    """Codes of x (32 bits; quotients next to the border between two codes are worked out in 64)."""
    safe = torch.where(scale > 0, scale, 1.0)
    if form == "int8":
        return torch.round(x.double() / safe.double()).clamp(-127, 127).to(torch.int8)
    return (x / safe).to(torch.float8_e4m3fn)


def _dense(s, x):
    """The codes as [B, H, rows, D] (pages looked up in the table)."""
    if not s["case"]["page"]:
        return s[x]
    t = _bytes(s[x])[s["table"].long()]
    B, nb, H, page, D = t.shape
    return t.permute(0, 2, 1, 3, 4).reshape(B, H, nb * page, D).view(s[x].dtype)


def _row_scale(s, x):
    """[B, H, rows, 1]: the scale of each row."""
    return s[x + "_scale"].repeat_interleave(s["case"]["rows"], 2)[:, :, :s["capacity"], None]


def _plain_write(s, x):
    c, n, n0 = s["case"], s["seq_len"].long(), s["from_len"].long()
    B, H, D, R, cap, form = c["B"], c["H"], c["D"], c["rows"], s["capacity"], c["form"]
    src = s[x + "_new"]
    r = torch.arange(cap, device=src.device)[None]
    new = (r >= n0[:, None]) & (r < n[:, None])                                              # [B, cap]
    i = (r - n0[:, None]).clamp(0, c["T"] - 1)[:, None].expand(B, H, cap)
    if s["take"] is not None:
        i = s["take"].long().gather(2, i)
    rows = src.gather(2, i[..., None].expand(B, H, cap, D)).float()
    blocks = lambda t: torch.nn.functional.pad(t, (0, 0, 0, -cap % R)).view(B, -1, t.shape[2] // R + (t.shape[2] % R > 0), R, t.shape[3])  # noqa: E731
    rows = blocks(torch.where(new[:, None, :, None], rows, 0.0))
    fresh = blocks(new[:, None, :, None].float()) > 0                                        # [B, 1, blocks, R, 1]
    touched = fresh.any(3).squeeze(-1)                                                       # [B, 1, blocks]
    start = torch.arange(rows.shape[2], device=src.device)[None, None] * R
    older = (start < n0[:, None, None]) & touched                                            # blocks that hold rows already
    was = s[x + "_scale"]
    fit = _fit(rows.abs().amax((3, 4)), form)
    now = torch.where(touched, torch.where(older, torch.maximum(fit, was), fit), was)
    before = torch.nn.functional.pad(_dense(s, x).float(), (0, 0, 0, -cap % R)).view(rows.shape)
    again = before.double() * torch.where(older, was, 0.0).double()[..., None, None]
    code = _encode(torch.where(fresh, rows.double(), again), now.double()[..., None, None], form).float()
    keep = ~touched[..., None, None] | (~fresh & (~older[..., None, None] | (now <= was)[..., None, None] | (blocks(r[:, None, :, None].expand(B, 1, cap, 1).float()) >= n0.view(B, 1, 1, 1, 1))))
    code = torch.where(keep, before, code).view(B, H, -1, D)[:, :, :cap].to(FORMATS[form])
    if c["page"]:
        nb = cap // c["page"]
        _bytes(s[x])[s["table"].reshape(-1).long()] = _bytes(code.contiguous()).view(B, H, nb, c["page"], D).permute(0, 2, 1, 3, 4).reshape(B * nb, H, c["page"], D)
    else:
        s[x].copy_(code)
    was.copy_(now)


def _plain_read(s, x, first):
    r = torch.arange(s["capacity"], device=first.device)[None]
    there = (r >= first.long()[:, None]) & (r < s["seq_len"].long()[:, None])
    value = (_dense(s, x).float() * _row_scale(s, x)).to(s[x + "16"].dtype)
    s[x + "16"].copy_(torch.where(there[:, None, :, None], value, s[x + "16"]))


def _plain_picks(s, x):
    i = s["idx"].long()
    at = i[..., None].expand(*i.shape, s["case"]["D"])
    code = _bytes(_dense(s, x)).gather(2, at).view(s[x].dtype).float()
    return (code * s[x + "_scale"].gather(2, torch.div(i, s["case"]["rows"], rounding_mode="floor"))[..., None]).to(s[x + "16"].dtype)


def _plain_attend(s):
    c, Q, n = s["case"], s["Q"], s["seq_len"].long()
    B, H, G, D, T = c["B"], c["H"], c["G"], c["D"], c["T"]
    K, V = (_dense(s, x).float() * _row_scale(s, x) for x in "KV")
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
    logits = (q @ K.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    if c["cap"]:
        logits = c["cap"] * torch.tanh(logits / c["cap"])
    logits = torch.where(seen, logits, float("-inf"))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ V) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)
    out = out.view(B, H, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(Q.dtype)
    return {"out": out, "lse": lse.view(B, H, T, G).permute(0, 2, 1, 3).reshape(B, T, H * G).contiguous()}


# ------------------------------------------------------------------------------------ what a pass has to do
def work(case):
    op, B, H, D, R = case["op"], case["B"], case["H"], case["D"], case["rows"]
    lens = lengths(case)
    blocks = lambda lo, hi: -(-hi // R) - lo // R  # noqa: E731
    if op == "attend":
        T, Hq = case["T"], H * case["G"]
        return {"bytes": sum(n * D + 4 * blocks(0, n) for n in lens) * H * 2 + 2 * B * T * Hq * D * 2 + 4 * B * T * Hq + 8 * B * T,
                "flops": 4 * T * Hq * D * sum(lens)}
    if op == "store":
        T = case["T"]
        new = B * H * T * D * 2                                     # elements of K and V that are written
        back = sum(n - (n - T) // R * R for n in lens) * H * D * 2  # and read back: their blocks' older rows too
        scales = sum(blocks(n - T, n) for n in lens) * H * 2 * 4
        return {"bytes": 2 * new + new + (4 * B * H * T if case["take"] else 0) + back + 2 * back + 2 * scales, "flops": 4 * new}
    if case["picks"]:
        e = B * H * case["picks"] * D * 2
        return {"bytes": 3 * e + 12 * B * H * case["picks"], "flops": e}
    return {"bytes": sum(3 * n * D + 4 * blocks(0, n) for n in lens) * H * 2, "flops": sum(lens) * H * D * 2}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def _codes64(s, x, b, h):
    """Codes of one head of one sequence, [rows, D], in 64 bits."""
    if not s["case"]["page"]:
        return s[x][b, h].double()
    return torch.cat([s[x][int(p), h].double() for p in s["table"][b].tolist()])


def _nearest64(y, form):
    """The code values nearest to y, ties to the even one."""
    if form == "int8":
        return torch.round(y).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # e4m3: 3 fraction bits, exponents from -6 on
    return (torch.round(y / step) * step).clamp(-448, 448)


def _scale64(top, form):
    if top == 0:
        return 0.0
    if form == "int8":
        return max(float(np.float32(top / 127.0)), TINY)
    m, e = math.frexp(top / 448.0)
    return max(2.0 ** (e - 1 if m == 0.5 else e), TINY)


def exact(case, seed):
    s = prepare(case, seed)
    op, B, H, D, R, form = (case[k] for k in ("op", "B", "H", "D", "rows", "form"))
    lens, dev = lengths(case), s["seq_len"].device
    if op == "attend":
        T, G, cap = case["T"], case["G"], case["cap"]
        out = torch.zeros((B, T, H, G, D), dtype=torch.float64, device=dev)
        lse = torch.full((B, T, H, G), -math.inf, dtype=torch.float64, device=dev)
        for b, n in enumerate(lens):
            hid = torch.ones((T, T), dtype=torch.bool, device=dev).triu(1)
            if s["mask"] is not None:
                bits = s["mask"][b].cpu().numpy().view(np.uint64)
                hid = torch.tensor([[not (int(m) >> i) & 1 for i in range(T)] for m in bits], device=dev)
            at = torch.div(torch.arange(n, device=dev), R, rounding_mode="floor")
            for h in range(H):
                k, v = (_codes64(s, x, b, h)[:n] * s[x + "_scale"][b, h].double()[at][:, None] for x in "KV")
                z = torch.einsum("tgd,rd->tgr", s["Q"][b, :, h * G:(h + 1) * G].double(), k) / math.sqrt(D)
                if cap:
                    z = cap * torch.tanh(z / cap)
                z[:, :, n - T:].masked_fill_(hid[:, None], -math.inf)
                lse[b, :, h] = torch.logsumexp(z, -1)
                out[b, :, h] = torch.einsum("tgr,rd->tgd", torch.softmax(z, -1), v)
        return {"out": out.reshape(B, T, H * G, D), "lse": lse.reshape(B, T, H * G)}
    if op == "read" and case["picks"]:
        got = {}
        for x in "KV":
            got[x] = torch.zeros((B, H, case["picks"], D), dtype=torch.float64, device=dev)
            for b in range(B):
                for h in range(H):
                    i = s["idx"][b, h].long()
                    got[x][b, h] = _codes64(s, x, b, h)[i] * s[x + "_scale"][b, h].double()[torch.div(i, R, rounding_mode="floor")][:, None]
        return got
    got = {}
    if op == "store" and sum(-(-n // R) - (n - case["T"]) // R for n in lens) * H > 60000:
        return None  # block by block: minutes
    for x in "KV":
        value, scales = s[x + "16"].double(), s[x + "_scale"].double()
        for b, n in enumerate(lens):
            for h in range(H):
                code = _codes64(s, x, b, h)
                if op == "read":
                    value[b, h, :n] = code[:n] * scales[b, h].repeat_interleave(R)[:n, None]
                    continue
                first = n - case["T"]
                tops = scales[b, h].tolist()
                new = s[x + "_new"][b, h].double()
                if s["take"] is not None:
                    new = new[s["take"][b, h].long()]
                high = torch.zeros(len(tops), dtype=torch.float64, device=dev)
                high.index_reduce_(0, torch.div(torch.arange(first, n, device=dev), R, rounding_mode="floor"), new.abs().amax(1), "amax")
                high = high.tolist()
                for j in range(first // R, -(-n // R)):
                    lo, hi, old = j * R, min(n, (j + 1) * R), tops[j]
                    f = _scale64(high[j], form)
                    if lo < first:
                        f = max(f, old)
                        if f > old:
                            code[lo:first] = _nearest64(code[lo:first] * old / f, form)
                    scales[b, h, j] = f
                    a = max(lo, first)
                    code[a:hi] = _nearest64(new[a - first:hi - first] / f, form) if f else 0.0
                    value[b, h, lo:hi] = code[lo:hi] * f
        got[x] = value
        if op == "store":
            got[x + "_scale"] = scales
    return got
