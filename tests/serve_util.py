"""Plain float64 statements of the serving operators, and the error each is allowed.

Tolerances.  Each probability is rounded once to the 16-bit type of the matrix products (half a step:
2^-8 for bf16, 2^-11 for fp16 and fp8 caches), each output once to its own type; logits are fp32 sums of
D products, off by at most (D + 4) * 2^-23 * scale * sum |q k| (one step per addition, tensor cores may
truncate), which moves a probability by that factor.  fp16 probabilities are held up to 2^8, so one that
falls among the subnormals is off by 2^-25 of a largest one of 2^8.  Sums of n positive fp32 terms are off
by n * 2^-24 relative, 2^x by 2^-22.
"""
import math

import torch

U_P = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -11}


def out_dtype(dtype):
    return torch.float16 if dtype == torch.float16 else torch.bfloat16


def attention64(q, k, v, seen, scale, k_scale, v_scale, dtype):
    """q [M, D], k / v [R, D], seen [M, R] -> out, lse and the error each may have (float64)."""
    q, D, n = q.double(), q.shape[-1], k.shape[0]
    k = torch.where(seen.any(0)[:, None], k.double(), 0.0)           # rows nobody sees may hold anything
    z = (q @ k.T) * (scale * k_scale)
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True) if n else torch.full((q.shape[0], 1), -math.inf, dtype=torch.float64, device=q.device)
    top0 = torch.where(torch.isinf(top), 0.0, top)
    p = torch.where(seen, torch.exp(z - top0), 0.0)
    total = p.sum(-1, keepdim=True)
    some = total > 0
    safe = torch.where(some, total, 1.0)
    vs = torch.where(seen.any(0)[:, None], v.double(), 0.0)
    out = torch.where(some, (p @ vs) / safe * v_scale, 0.0)
    lse = torch.where(some, top0 + torch.log(safe), -math.inf).squeeze(-1)
    spread = (torch.where(seen, (q.abs() @ k.abs().T), 0.0).amax(-1, keepdim=True) if n else torch.zeros_like(total)) * scale * k_scale
    delta = (D + 4) * 2.0 ** -23 * spread + n * 2.0 ** -24 + 2.0 ** -21
    weight = (p @ vs.abs()) / safe * v_scale
    big = vs.abs().amax() * v_scale if n else 0.0
    u = U_P[dtype]
    tol = weight * (u + 2 * delta) * 1.01 + n * 2.0 ** -33 * big + out.abs() * (torch.finfo(out_dtype(dtype)).eps / 2) * 1.02
    tol = tol + torch.finfo(out_dtype(dtype)).tiny
    return out, lse, tol, (2 * delta.squeeze(-1) + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0))


def tree_seen(mask_row, T, draft, n):
    """seen [T, n] of one sequence: mask_row int64 [T] or None (a chain)."""
    base = n - draft
    seen = torch.zeros((T, n), dtype=torch.bool)
    for t in range(draft):
        seen[t, :base] = True
        for j in range(draft):
            seen[t, base + j] = (j <= t) if mask_row is None else bool((int(mask_row[t]) >> j) & 1)
    return seen


def tree_reference(Q, K, V, seq_len, draft_len, mask, scale=None, k_scale=1.0, v_scale=1.0):
    """Dense K, V [B, H, S, D]; returns out, lse, tol_out, tol_lse as [B, T, H_q, ...] float64 on Q's device."""
    B, T, Hq, D = Q.shape
    H = K.shape[1]
    G = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=Q.device)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=Q.device)
    t_out, t_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, d = int(seq_len[b]), int(draft_len[b])
        seen = tree_seen(None if mask is None else mask[b].tolist(), T, d, n).to(Q.device).repeat_interleave(G, 0)
        for h in range(H):
            q = Q[b, :, h * G:(h + 1) * G].reshape(T * G, D)
            o, l, to, tl = attention64(q, K[b, h, :n].float(), V[b, h, :n].float(), seen, scale, k_scale, v_scale, K.dtype)
            out[b, :, h * G:(h + 1) * G] = o.view(T, G, D)
            lse[b, :, h * G:(h + 1) * G] = l.view(T, G)
            t_out[b, :, h * G:(h + 1) * G] = to.view(T, G, D)
            t_lse[b, :, h * G:(h + 1) * G] = tl.view(T, G)
    return out, lse, t_out, t_lse


def assert_attention(got, want):
    out, lse, t_out, t_lse = want
    far = (got["out"].double() - out).abs()
    bad = ~(far <= t_out)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {far[bad].max().item():.3g} (allowed {t_out[bad].min().item():.3g})"
    if "lse" in got and got["lse"] is not None:
        g = got["lse"].double()
        assert torch.equal(torch.isinf(g), torch.isinf(lse))
        fin = torch.isfinite(lse)
        assert ((g - lse).abs()[fin] <= t_lse[fin]).all(), f"lse off by {(g - lse).abs()[fin].max().item():.3g}"


def make_cache(shape, dtype, g, device="cuda"):
    """K with outlier channels and V, in the storage format; fp8 with the scales its values stand for."""
    k = torch.randn(shape, generator=g, device=device) * torch.exp(0.8 * torch.randn((1, shape[1], 1, shape[3]), generator=g, device=device))
    v = torch.randn(shape, generator=g, device=device)
    if dtype == torch.float8_e4m3fn:
        ks, vs = float(k.abs().max()) / 400, float(v.abs().max()) / 400
        return (k / ks).to(dtype), (v / vs).to(dtype), ks, vs
    return k.to(dtype), v.to(dtype), 1.0, 1.0


def bits(t):
    """The storage of a 16- or 8-bit tensor as integers (indexing and comparing fp8 tensors)."""
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.view(torch.int16)


def to_pages(X, page, perm, num_pages, fill):
    """Dense [B, H, S, D] -> pool [num_pages, H, page, D] with table perm [B, nb]; other rows hold `fill`."""
    B, H, S, D = X.shape
    nb = perm.shape[1]
    pad = torch.full((B, H, nb * page, D), fill, dtype=torch.float32, device=X.device).to(X.dtype)
    bits(pad)[:, :, :S] = bits(X)
    pool = torch.full((num_pages, H, page, D), fill, dtype=torch.float32, device=X.device).to(X.dtype)
    bits(pool)[perm.reshape(-1).long()] = bits(pad).view(B, H, nb, page, D).permute(0, 2, 1, 3, 4).reshape(B * nb, H, page, D)
    return pool


def from_pages(pool, table, page):
    B, nb = table.shape
    x = bits(pool)[table.clamp(min=0).long()]
    return x.permute(0, 2, 1, 3, 4).reshape(B, pool.shape[1], nb * page, pool.shape[3]).view(pool.dtype)


def random_tree(B, T, rng):
    """int64 masks [B, T]: each token sees itself and the ancestors that a random tree gives it."""
    rows = []
    for _ in range(B):
        m = []
        for i in range(T):
            p = rng.randint(max(-1, i - 5), i - 1)
            m.append((m[p] if p >= 0 else 0) | (1 << i))
        rows.append([x - (1 << 64) if x >> 63 else x for x in m])
    return torch.tensor(rows, dtype=torch.int64)
