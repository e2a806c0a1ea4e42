"""Plain float64 statements of the operators on caches in 8 bits with block scales, and the error each is allowed.

Writing is exact: codes and scales are compared for equality.  Reading back rounds the fp32 product once: compared with
torch's fp32 product rounded to 16 bits, for equality.

Attention.  A probability times its V scale is rounded once to fp16 (half a step: 2^-11 relative), an output once to its
own type; logits are fp32 sums of D products times fp32 factors, off by at most (D + 6) * 2^-23 * scale * sum |q k|
(one step per addition or product, tensor cores may truncate), a capped one by 2^-22 of itself more, which moves a probability by that
factor.  The largest probability counts 2^8 and the largest V scale seen less than 2^ve <= 2 * scale, so that products that fall among
fp16's subnormals are off by 2^-25 of 2^8 / 2^ve: n * 2^-32 of the largest scale times the largest code in all.  Sums of n
positive fp32 terms are off by n * 2^-24 relative, 2^x by 2^-22.
"""
import math

import torch

import serve_util as U

TOP = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def fit(top, form):
    """The scale that a largest magnitude (a Python float) asks for."""
    if top == 0:
        return 0.0
    if form == "int8":
        return max(float(torch.tensor(top / 127.0, dtype=torch.float64).float()), 2.0 ** -126)
    m, e = math.frexp(top / 448.0)
    return max(2.0 ** (e - 1 if m == 0.5 else e), 2.0 ** -126)


def nearest(y, form):
    """Code values nearest to y (float64), ties to the even one."""
    if form == "int8":
        return torch.round(y).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def write64(code, scale, X, start, end, R, form):
    """One (sequence, head): code [S, D] and scale [blocks] (float64, changed in place); X [end - start, D]: its new rows."""
    for j in range(start // R, -(-end // R) if end > start else 0):
        lo, hi = j * R, min(end, (j + 1) * R)
        a = max(lo, start)
        x = X[a - start:hi - start].double()
        fin = torch.where(torch.isfinite(x), x, 0.0)
        s = fit(float(fin.abs().max()), form)
        if lo < start:
            was = float(scale[j])
            s = max(s, was)
            if s > was:
                code[lo:start] = nearest(code[lo:start] * was / s, form)
        scale[j] = s
        x = torch.where(torch.isnan(x), 0.0, x).clamp(-TOP[form] * s, TOP[form] * s)
        code[a:hi] = nearest(x / s, form) if s else 0.0


def values(codes):
    """Codes as float64."""
    return codes.double()


def row_values(codes, scale, R):
    """[..., S, D] codes and [..., blocks] scales -> float64 values."""
    S = codes.shape[-2]
    return codes.double() * scale.double().repeat_interleave(R, -1)[..., :S, None]


def random_cache(B, H, S, D, form, R, g, spread=0.0, device="cuda"):
    """Codes and scales as a writer leaves them; block scales vary by 2^(+-spread)."""
    blocks = -(-S // R)
    x = torch.randn((2, B, H, S, D), generator=g, device=device) * TOP[form] / 4
    x[0] *= torch.exp(0.5 * torch.randn((1, H, 1, D), generator=g, device=device))
    codes = (x.round().clamp(-127, 127) if form == "int8" else x.clamp(-448, 448)).to(DTYPE[form])
    e = (torch.rand((2, B, H, blocks), generator=g, device=device) * 2 - 1) * spread
    scale = torch.exp2(torch.round(e)) * 4 / TOP[form]
    if form == "int8":
        scale = scale * (1 + torch.rand(scale.shape, generator=g, device=device))
    return codes[0], codes[1], scale[0].contiguous(), scale[1].contiguous()


def attention64(q, k, v, seen, scale, cap, v_reach, out_dtype):
    """q [M, D], k / v [n, D] (values), seen [M, n] -> out, lse and the error each may have (float64)."""
    D, n = q.shape[-1], k.shape[0]
    q, some_see = q.double(), seen.any(0)[:, None]
    k, v = torch.where(some_see, k.double(), 0.0), torch.where(some_see, v.double(), 0.0)
    z = (q @ k.T) * scale
    spread = (torch.where(seen, q.abs() @ k.abs().T, 0.0).amax(-1, keepdim=True) if n else torch.zeros((q.shape[0], 1), dtype=torch.float64, device=q.device)) * scale
    delta = (D + 6) * 2.0 ** -23 * spread + n * 2.0 ** -24 + 2.0 ** -21
    if cap:
        z = cap * torch.tanh(z / cap)
        delta = delta + 2.0 ** -22 * torch.clamp(spread, max=cap)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True) if n else torch.full((q.shape[0], 1), -math.inf, dtype=torch.float64, device=q.device)
    top0 = torch.where(torch.isinf(top), 0.0, top)
    p = torch.where(seen, torch.exp(z - top0), 0.0)
    total = p.sum(-1, keepdim=True)
    some = total > 0
    safe = torch.where(some, total, 1.0)
    odd = seen.double() @ torch.isnan(v).double() > 0                # NaN reaches those who see it, and not through 0 * NaN
    v = v.nan_to_num(nan=0.0)
    out = torch.where(odd, math.nan, torch.where(some, (p @ v) / safe, 0.0))
    lse = torch.where(some, top0 + torch.log(safe), -math.inf).squeeze(-1)
    weight = (p @ v.abs()) / safe
    tol = weight * (2.0 ** -11 + 2 * delta) * 1.01 + n * 2.0 ** -32 * v_reach + out.abs() * (torch.finfo(out_dtype).eps / 2) * 1.02
    return out, lse, tol + torch.finfo(out_dtype).tiny, 2 * delta.squeeze(-1) + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)


def assert_attention(got, want):
    """serve_util.assert_attention(); results that lie beyond the output's type round to infinity."""
    out, lse, t_out, t_lse = want
    most = torch.finfo(got["out"].dtype).max
    most = most * (1 + torch.finfo(got["out"].dtype).eps / 4)           # half a step further still rounds to the largest value
    beyond = torch.isinf(got["out"]) & (torch.sign(got["out"].double()) == torch.sign(out)) & (out.abs() + t_out >= most)
    U.assert_attention(dict(got, out=torch.where(beyond, 0.0, got["out"])), (torch.where(beyond, 0.0, out), lse, torch.where(beyond, 0.0, t_out), t_lse))


def attention_reference(Q, K, V, seq_len, draft_len, mask, scale=None, cap=0.0, v_scale=1.0, form="int8", V_scale=None, gone=None):
    """K, V [B, H, S, D] float64 values -> out, lse, and their tolerances [B, T, H_q, ...]; nobody sees rows `gone` (a slice)."""
    B, T, Hq, D = Q.shape
    H = K.shape[1]
    G = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=Q.device)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=Q.device)
    t_out, t_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, d = int(seq_len[b]), int(draft_len[b])
        seen = U.tree_seen(None if mask is None else mask[b].tolist(), T, d, n).to(Q.device).repeat_interleave(G, 0)
        if gone is not None:
            seen[:, gone] = False
        for h in range(H):
            q = Q[b, :, h * G:(h + 1) * G].reshape(T * G, D)
            reach = (float(V_scale[b, h].max()) * TOP[form] if V_scale is not None else float(V[b, h, :n].abs().max()) if n else 0.0) * v_scale
            o, l, to, tl = attention64(q, K[b, h, :n], V[b, h, :n] * v_scale, seen, scale, cap, reach, Q.dtype)
            out[b, :, h * G:(h + 1) * G] = o.view(T, G, D)
            lse[b, :, h * G:(h + 1) * G] = l.view(T, G)
            t_out[b, :, h * G:(h + 1) * G] = to.view(T, G, D)
            t_lse[b, :, h * G:(h + 1) * G] = tl.view(T, G)
    return out, lse, t_out, t_lse


def pool_of(dense, page, perm, pages, fill=0x7f):
    """Dense codes [B, H, S, D] -> pool [pages, H, page, D] behind table perm [B, nb]; other rows hold the byte `fill`."""
    B, H, S, D = dense.shape
    nb = perm.shape[1]
    pad = torch.full((B, H, nb * page, D), fill, dtype=torch.uint8, device=dense.device)
    pad[:, :, :S] = dense.view(torch.uint8)
    pool = torch.full((pages, H, page, D), fill, dtype=torch.uint8, device=dense.device)
    pool[perm.reshape(-1).long()] = pad.view(B, H, nb, page, D).permute(0, 2, 1, 3, 4).reshape(B * nb, H, page, D)
    return pool.view(dense.dtype)


def dense_of(pool, table, page):
    B, nb = table.shape
    x = pool.view(torch.uint8)[table.clamp(min=0).long()]
    return x.permute(0, 2, 1, 3, 4).reshape(B, pool.shape[1], nb * page, pool.shape[3]).contiguous().view(pool.dtype)
