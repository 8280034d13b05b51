"""Plain 64-bit forms of the language-model block's operators, with bounds on what 16-bit products may be off by.

Rounding steps: u = eps/2 of the storage type (bfloat16 2^-8, binary16 2^-11, binary32 2^-24).  A probability or score gradient that
enters a product is rounded once (u), a result once more (u).  Scores are binary32 sums of at most 128 exact products: off by
at most 128 * 2^-24 sum |q||k|, which the tests keep below 1e-4 in p (E32).
"""
import math

import torch

U = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}
E32 = 1e-4
F8 = torch.float64


def seen_matrix(Nq, Nk, B, causal, window=0, kv_len=None, q_start=None, prefix=None, doc=None):
    """(B, Nq, Nk) truth values from the definition, pair by pair"""
    out = torch.zeros(B, Nq, Nk, dtype=torch.bool)
    j = torch.arange(Nk)
    for b in range(B):
        n = min(Nk, int(kv_len[b])) if kv_len is not None else Nk
        for i in range(Nq):
            p = i + (int(q_start[b]) if q_start is not None else Nk - Nq)
            if p < 0 or p >= n:
                continue
            s = j < n
            if causal:
                s &= (j <= p) | ((j < int(prefix[b])) if prefix is not None else False)
            if window:
                s &= j > p - window
                if not causal:
                    s &= j < p + window
            if doc is not None:
                s &= doc[b] == doc[b, p]
            out[b, i] = s
    return out


def intervals(seen):
    """lo, hi (B, Nq) int32 of a truth matrix whose rows are intervals"""
    n = seen.sum(-1)
    first = seen.to(torch.int8).argmax(-1)
    lo = torch.where(n > 0, first, 0)
    return lo.int(), (lo + n).int()


def scores(q, k, scale, cap, slopes, start, seen):
    """(B, Hq, Nq, Nk) scores and the cap's slope; q (B, Nq, Hq, D), k (B, Nk, Hk, D) in 64 bits; start: place of query 0"""
    B, Nq, Hq, D = q.shape
    Nk = k.shape[1]
    k = k.repeat_interleave(Hq // k.shape[2], 2)
    s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1).contiguous()) * scale
    slope = torch.ones_like(s)
    if cap:
        t = torch.tanh(s / cap)
        s, slope = cap * t, 1 - t * t
    if slopes is not None:
        p = start.to(q.device).to(F8)[:, None] + torch.arange(Nq, device=q.device, dtype=F8)
        far = (p[:, :, None] - torch.arange(Nk, device=q.device, dtype=F8)).abs()
        s = s - slopes.to(F8)[None, :, None, None] * far[:, None]
    return s.masked_fill(~seen[:, None], -math.inf), slope


def clean(x, keep):
    """rows that nobody sees, whatever they hold, as zeros; keep (B, N)"""
    return torch.where(keep[..., None, None], x, torch.zeros((), dtype=x.dtype, device=x.device)).to(F8)


def attention(q, k, v, scale, cap, slopes, start, seen):
    """o (B, Nq, Hq, D), lse (B, Hq, Nq) and the bound of o in storage type dt, all in 64 bits"""
    dt = q.dtype
    u = U[dt]
    group = q.shape[2] // k.shape[2]
    rows, keys = seen.any(-1), seen.any(1)
    q, k, v = clean(q, rows), clean(k, keys), clean(v, keys)
    s, _ = scores(q, k, scale, cap, slopes, start, seen)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0)[..., None])
    V = v.repeat_interleave(group, 2).transpose(1, 2).contiguous()
    o, mag = torch.matmul(p, V), torch.matmul(p, V.abs())
    bound = (u + E32) * mag + u * o.abs() * (1 + u) + 2.0**-25 * torch.matmul(seen[:, None].to(F8).expand_as(p).contiguous(), V.abs()) + 2.0**-24
    return o.transpose(1, 2), lse, bound.transpose(1, 2)


def attention_bwd(q, k, v, o, lse, do, scale, cap, slopes, start, seen):
    """(dq, dk, dv) and their bounds, in 64 bits; q, k, v as the products take them (de-quantized to dt)"""
    dt = q.dtype
    u = U[dt]
    B, Nq, Hq, D = q.shape
    Nk, Hk = k.shape[1], k.shape[2]
    group = Hq // Hk
    rows, keys = seen.any(-1), seen.any(1)
    q, o, do = clean(q, rows), clean(o, rows), clean(do, rows)
    k, v = clean(k, keys), clean(v, keys)
    s, slope = scores(q, k, scale, cap, slopes, start, seen)
    p = torch.exp(s - torch.where(torch.isfinite(lse), lse, 0).to(F8)[..., None])
    p = torch.where(seen[:, None], p, 0)
    Q, O, G = (t.transpose(1, 2).contiguous() for t in (q, o, do))
    K, V = (t.repeat_interleave(group, 2).transpose(1, 2).contiguous() for t in (k, v))
    T = lambda t: t.transpose(-1, -2).contiguous()  # noqa: E731
    dp, delta = torch.matmul(G, T(V)), (G * O).sum(-1, keepdim=True)
    ds = p * (dp - delta) * slope
    dp_off = D * 2.0**-24 * (torch.matmul(G.abs(), T(V.abs())) + (G * O).abs().sum(-1, keepdim=True))
    small = 2.0**-37 * (G.norm(dim=-1).amax() * V.norm(dim=-1).amax() + delta.abs().amax())   # binary16: half of the least subnormal, undone
    ds_off = ds.abs() * (u + E32) + p * dp_off + seen[:, None] * small
    join = lambda t: t.reshape(B, Hk, group, Nk, D).sum(2).transpose(1, 2)  # noqa: E731
    dq, dk, dv = torch.matmul(ds, K) * scale, torch.matmul(T(ds), Q) * scale, torch.matmul(T(p), G)
    eq = torch.matmul(ds_off, K.abs()) * scale
    ek = torch.matmul(T(ds_off), Q.abs()) * scale
    ev = torch.matmul(T(p * (u + E32) + seen[:, None] * 2.0**-33), G.abs())
    out = (dq.transpose(1, 2), join(dk), join(dv))
    off = (eq.transpose(1, 2), join(ek), join(ev))
    least = 2.0**-24 if dt == torch.float16 else 2.0**-133    # a result below the type's normal values
    return out, tuple(e + u * (x.abs() + e) + least for x, e in zip(out, off))


def angles(pos, freq, sections):
    """(T, 1, rot/2) cosines and sines in 64 bits"""
    axis = torch.cat([torch.full((n,), a, dtype=torch.long) for a, n in enumerate(sections)]).to(pos.device)
    a = pos.to(F8)[axis].t() * freq.to(F8)
    return a.cos()[:, None], a.sin()[:, None]


def turn(z, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out = z.clone()
    out[..., first] = z[..., first] * cos - z[..., second] * sin
    out[..., second] = z[..., second] * cos + z[..., first] * sin
    return out


def dequantize(q, alpha, beta, dt=None):
    """(..., heads, D) codes; dt None: 64 bits, else rounded as the library does"""
    if dt is None:
        return (q.to(F8) + 128) * (alpha.to(F8) / 255)[:, None] + beta.to(F8)[:, None]
    # 255 as a tensor: a division by a plain number would multiply by its rounded reciprocal
    return ((q.float() + 128) * (alpha / torch.full_like(alpha, 255))[:, None] + beta[:, None]).to(dt)
