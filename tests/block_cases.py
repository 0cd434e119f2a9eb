"""Attention, rotary positions and layer norm from their definitions in 64 bits, with bounds on what 32-bit sums and the documented roundings may differ by.

Bounds are worst cases, not fits (tests/layer_cases.py has the units).  A sum of n products in 32 bits is off by at most n * STEP * (sum of the absolute
values); a score's exponential is off, relatively, by the score's error and by STEP for each unit of the exponent; weights and score gradients
are rounded once to the type as operands (U relative, and what float16 loses below its normal numbers, TINY of the largest), results once more.
Exponentials below 2^-126, the smallest normal number of 32 bits, may be zero, and so may a product or a sum: FLUSH for a weight, times what it is
multiplied with, and for a result.
"""
import math

import torch

from tests.layer_cases import D, STEP, TINY, U

FLUSH = 2.0 ** -125


def spans(rows, offsets):
    """(first, end) of each sequence"""
    if offsets is None:
        return [(0, rows)]
    o = offsets.tolist()
    return [tuple(p) for p in o] if offsets.dim() == 2 else list(zip(o, o[1:]))


def attention(q, k, v, dy=None, offsets=None, k_offsets=None, scale=None, cap=0.0, slopes=None, causal=False, prefix=None):
    """{name: (value, bound)} of y, lse, and with dy of dq, dk, dv"""
    t, dim, group = q.dtype, q.shape[2], q.shape[1] // k.shape[1]
    u, tiny = U[t], TINY[t] if t == torch.float16 else 0.0
    scale = dim ** -0.5 if scale is None else scale
    q, k, v = q.to(D), k.to(D), v.to(D)
    dy = None if dy is None else dy.to(D)
    zero = lambda x: (torch.zeros_like(x), torch.zeros_like(x))
    out = {"y": zero(q), "lse": (torch.full_like(q[..., 0], -math.inf), torch.zeros_like(q[..., 0]))}
    if dy is not None:
        out.update(dq=zero(q), dk=zero(k), dv=zero(v))
    if k_offsets is None and offsets is not None:
        k_offsets = offsets
    for s, ((a, b), (c, e)) in enumerate(zip(spans(q.shape[0], offsets), spans(k.shape[0], k_offsets))):
        n, m = b - a, e - c
        if n <= 0 or m <= 0:
            continue
        place = torch.arange(m - n, m, device=q.device)[:, None]
        key = torch.arange(m, device=q.device)[None]
        seen = torch.ones(n, m, dtype=torch.bool, device=q.device)
        if causal:
            seen = key <= place
            if prefix is not None:
                seen = seen | (key < int(prefix[s]))
        far = (place - key).abs().to(D)
        for h in range(q.shape[1]):
            g = h // group
            Q, K, V = q[a:b, h], k[c:e, g], v[c:e, g]
            r = scale * Q @ K.t()
            e_r = (dim + 4) * STEP * abs(scale) * (Q.abs() @ K.abs().t())
            x, bent, e_bent = r, torch.ones_like(r), torch.zeros_like(r)
            e_a = e_r
            if cap:
                th = torch.tanh(r / cap)
                x, bent = cap * th, 1.0 - th * th
                e_a = e_r + cap * 2.0 ** -20
                e_bent = 0.77 / cap * e_r + 2.0 ** -19
            if slopes is not None:
                x = x - slopes[h].to(D) * far
                e_a = e_a + 4 * STEP * slopes[h].to(D).abs() * far
            e_a = e_a + 4 * STEP * (x.abs() + 1)
            x = x.masked_fill(~seen, -math.inf)
            some = seen.any(1, keepdim=True)
            lse = torch.logsumexp(x, 1, keepdim=True)
            p = torch.where(some, torch.exp(x - lse), torch.zeros_like(x))
            top = torch.where(seen, e_a, torch.zeros_like(e_a)).amax(1, keepdim=True)
            spread = torch.where(seen, (x - lse).abs(), torch.zeros_like(x)).amax(1, keepdim=True)
            e_w = top + STEP * (spread + 16)                       # of a weight, relative
            y = p @ V
            e_y = (p * (2 * e_w + u + (m + 16) * STEP)) @ V.abs() + (tiny + FLUSH) * (seen.to(D) @ V.abs()) + FLUSH
            y_off = e_y + u * (y.abs() + e_y) + TINY[t]
            lse_off = e_w + STEP * (lse.abs() + m + 16)
            out["y"][0][a:b, h], out["y"][1][a:b, h] = y, y_off
            out["lse"][0][a:b, h], out["lse"][1][a:b, h] = lse[:, 0], torch.where(some, lse_off, torch.zeros_like(lse_off))[:, 0]
            if dy is None:
                continue
            E = dy[a:b, h]
            dp, delta = E @ V.t(), (E * y).sum(1, keepdim=True)
            e_dp = (dim + 4) * STEP * (E.abs() @ V.abs().t())
            e_delta = (E.abs() * y_off).sum(1, keepdim=True) + (dim + 4) * STEP * (E.abs() * (y.abs() + y_off)).sum(1, keepdim=True)
            e_p = e_a + torch.where(some, lse_off, torch.zeros_like(lse_off)) + STEP * (torch.where(seen, (x - lse).abs(), torch.zeros_like(x)) + 16)
            w = p * (dp - delta)
            e_ds = p * e_p * (dp - delta).abs() + p * (e_dp + e_delta) * (1 + e_p) + 4 * STEP * w.abs() + FLUSH * seen * (1 + (dp - delta).abs())
            ds = w * bent
            e_ds = e_ds * bent + (w.abs() + e_ds) * e_bent
            ds_off = e_ds + u * (ds.abs() + e_ds)
            row_off, key_off = (ds_off + tiny * ds.abs().amax(i, keepdim=True) for i in (1, 0))
            v_, e_ = scale * ds @ K, FLUSH + abs(scale) * (row_off + (m + 4) * STEP * (ds.abs() + row_off)) @ K.abs()
            out["dq"][0][a:b, h], out["dq"][1][a:b, h] = v_, e_ + u * (v_.abs() + e_) + TINY[t]
            N = n * group + 64
            out["dk"][0][c:e, g] += scale * ds.t() @ Q
            out["dk"][1][c:e, g] += FLUSH + abs(scale) * (key_off + N * STEP * (ds.abs() + key_off)).t() @ Q.abs()
            out["dv"][0][c:e, g] += p.t() @ E
            out["dv"][1][c:e, g] += (p * (e_p + u + N * STEP) + (tiny + FLUSH) * seen).t() @ E.abs() + FLUSH
    for name in ("dk", "dv"):
        if name in out:
            v_, e_ = out[name]
            out[name] = v_, e_ + u * (v_.abs() + e_) + TINY[t]
    return out


def within(name, got, ref):
    """Equal where the value is infinite, else inside the bound."""
    value, bound = ref
    got = got.to(D)
    bad = torch.where(torch.isinf(value), got != value, ~((got - value).abs() <= bound))
    assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[0].tolist(), float(((got - value).abs() / bound).nan_to_num(0.0).max()))


def rotary(x, positions, frequencies, interleaved, scale, back=False):
    """(value, bound)"""
    t, half = x.dtype, frequencies.numel()
    x = x.to(D)
    angle = (positions.to(D)[:, None] * frequencies)[:, None]
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale * (-1.0 if back else 1.0)
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    else:
        a, b = x[..., :half], x[..., half:2 * half]
    value, off = x.clone(), torch.zeros_like(x)
    # a turn in 64 bits: 2^-52 of the angle; cut to 32 bits: 2^-25 of a turn, 2^-22 of a radian; sines to two units, their scale, products and sum rounded
    e = (a.abs() + b.abs()) * abs(scale) * (2.0 ** -52 * angle.abs() + 2.0 ** -20)
    for part, v in ((0, a * c - b * s), (1, a * s + b * c)):
        at = (slice(None), slice(None), slice(part, 2 * half, 2) if interleaved else slice(part * half, (part + 1) * half))
        value[at], off[at] = v, e + U[t] * (v.abs() + e) + TINY[t]
    return value, off


def norm(x, weight, bias, eps, dy=None):
    """{name: (value, bound)} of y, mean, rstd, and with dy of dx, dweight, dbias"""
    t, (rows, n) = x.dtype, x.shape
    x = x.to(D)
    w = torch.ones(n, dtype=D, device=x.device) if weight is None else weight.to(D)
    mean = x.mean(1, keepdim=True)
    e_mean = (n + 2) * STEP * x.abs().mean(1, keepdim=True)
    d = x - mean
    e_d = e_mean + STEP * (d.abs() + mean.abs())
    var = (d * d).mean(1, keepdim=True)
    e_var = (2 * d.abs() * e_d + e_d * e_d).mean(1, keepdim=True) + (n + 4) * STEP * ((d.abs() + e_d) ** 2).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    low = torch.clamp(var - e_var, min=0.0) + eps
    e_rstd = 1.0 / torch.sqrt(low) - rstd + 6 * STEP * rstd
    h = d * rstd
    e_h = e_d * (rstd + e_rstd) + d.abs() * e_rstd + 2 * STEP * h.abs()
    y = h * w + (0.0 if bias is None else bias.to(D))
    e_y = e_h * w.abs() + 4 * STEP * ((h * w).abs() + y.abs())
    rounded = lambda v, e: (v, e + U[t] * (v.abs() + e) + TINY[t])
    out = {"y": rounded(y, e_y), "mean": (mean[:, 0], e_mean[:, 0]), "rstd": (rstd[:, 0], e_rstd[:, 0])}
    if dy is None:
        return out
    dy = dy.to(D)
    g = dy * w
    e_g = STEP * g.abs()
    m1, m2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    e_m1 = (e_g + (n + 2) * STEP * g.abs()).mean(1, keepdim=True)
    e_m2 = (e_g * h.abs() + g.abs() * e_h + (n + 4) * STEP * g.abs() * (h.abs() + e_h)).mean(1, keepdim=True)
    v = g - m1 - h * m2
    e = e_g + e_m1 + e_h * m2.abs() + (h.abs() + e_h) * e_m2 + 4 * STEP * (g.abs() + m1.abs() + (h * m2).abs())
    out["dx"] = rounded(rstd * v, rstd * e + (e_rstd + 2 * STEP * rstd) * (v.abs() + e))
    out["dweight"] = rounded((dy * h).sum(0), (dy.abs() * e_h + (rows + 4) * STEP * dy.abs() * (h.abs() + e_h)).sum(0))
    out["dbias"] = rounded(dy.sum(0), (rows + 4) * STEP * dy.abs().sum(0))
    return out
