"""The layer operators from their definition in 64 bits, with bounds on what a 32-bit sum and one rounding may differ by.

Bounds are worst cases, not fits.  A sum of n products in 32 bits is off by at most n * 2^-23 * (sum of the absolute values) whatever
its order (2^-24 a step for rounding to nearest, twice that for an accumulator that cuts); a result is rounded once to its type,
at most U relative, and below its smallest normal number at most TINY.  Activations are smooth with slopes up to 1.13, and computed
in 32 bits with a few units in the last place: 2^-20 of |z| + 1 is allowed.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -23}     # half a unit, or a whole one in 32 bits
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}
STEP = 2.0 ** -23
ACT_ERR = 2.0 ** -20
D = torch.float64


def act(z, kind):
    """(value, slope); kinds are numbered as in the library."""
    if kind == 0:
        return z, torch.ones_like(z)
    if kind == 1:
        return torch.clamp(z, min=0.0), (z > 0).to(z.dtype)
    if kind == 2:
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == 3:
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return z * (1 + t) / 2, (1 + t) / 2 + z / 2 * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return z * s, s + z * s * (1 - s)


def forward(x, w, bias, residual, kind):
    """(y, bound of y, z, bound of z) for matrices of one type"""
    t, n = x.dtype, x.shape[1]
    x, w = x.to(D), w.to(D)
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.to(D), size + bias.to(D).abs()
    off = (n + 2) * STEP * size
    y = act(z, kind)[0]
    y_off = 1.13 * off + (ACT_ERR * (z.abs() + 1) if kind else 0.0)
    if residual is not None:
        y = y + residual.to(D)
        y_off = y_off + STEP * (y.abs() + residual.to(D).abs())
    return y, y_off + U[t] * (y.abs() + y_off) + TINY[t], z, off + U[t] * (z.abs() + off) + TINY[t]


def backward(dy, z, x, w, kind):
    """{name: (value, bound)} of dx, dw, dbias"""
    t, rows, n_out = dy.dtype, dy.shape[0], dy.shape[1]
    dy, x, w = dy.to(D), x.to(D), w.to(D)
    slope = act(z.to(D), kind)[1] if kind else torch.ones_like(dy)
    dz = dy * slope
    exact_off = (ACT_ERR * 2 + 2 * STEP) * dy.abs() if kind else torch.zeros_like(dy)
    off = exact_off + (U[t] * (dz.abs() + exact_off) + TINY[t] if kind else 0.0)
    out = {}
    for name, a, ao, b, n in (("dx", dz, off, w, n_out), ("dw", dz.t(), off.t(), x, rows)):
        v = a @ b
        e = (ao + (n + 1) * STEP * (a.abs() + ao)) @ b.abs()
        out[name] = (v, e + U[t] * (v.abs() + e) + TINY[t])
    v, e = dz.sum(0), exact_off.sum(0) + (rows + 1) * STEP * (dz.abs() + exact_off).sum(0)
    out["dbias"] = (v, e + U[t] * (v.abs() + e) + TINY[t])
    return out


def vocab(x, w, target, dloss):
    """{name: (value, bound)} of loss, lse, dx, dw"""
    t, (rows, n), words = x.dtype, x.shape, w.shape[0]
    x, w = x.to(D), w.to(D)
    l = x @ w.t()
    off = ((n + 1) * STEP * (x.abs() @ w.abs().t())).amax(1, keepdim=True)
    lse = torch.logsumexp(l, 1, keepdim=True)
    spread = l.amax(1, keepdim=True) - l.amin(1, keepdim=True)
    # a 32-bit exponential is off by 2^-23 of its exponent and two units, sums of `words` of them by a unit a step of the longest chain
    exp_off = STEP * (spread + 4)
    lse_off = off + exp_off + STEP * (lse.abs() + l.abs().amax(1, keepdim=True) + 64 + words / 64)
    here = target >= 0
    hot = torch.zeros_like(l)
    hot[torch.nonzero(here)[:, 0], target[here]] = 1.0
    loss = torch.where(here, lse[:, 0] - (l * hot).sum(1), torch.zeros((), dtype=D, device=x.device))
    loss_off = torch.where(here, (lse_off + off)[:, 0] + STEP * loss.abs(), torch.zeros((), dtype=D, device=x.device))
    out = {"loss": (loss, loss_off), "lse": (lse[:, 0], lse_off[:, 0])}
    if dloss is None:
        return out
    p, c = torch.exp(l - lse), torch.where(here, dloss.to(D), torch.zeros((), dtype=D, device=x.device))[:, None]
    g = (p - hot) * c
    top = c.abs().max()
    e = p * (off + lse_off + exp_off + STEP * (l - lse).abs()) * c.abs() + 4 * STEP * (p + hot) * c.abs()
    e = e + U[t] * (g.abs() + e) + TINY[t] * top / 2.0 ** 13
    for name, a, ao, b, k in (("dx", g, e, w, words), ("dw", g.t(), e.t(), x, rows)):
        v = a @ b
        s = (ao + (k + 16) * STEP * (a.abs() + ao)) @ b.abs()
        out[name] = (v, s + U[t] * (v.abs() + s) + TINY[t])
    return out


def normal(g, dtype, *size, scale=1.0):
    return (torch.randn(*size, device="cuda", generator=g) * scale).to(dtype)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def within(name, got, ref, bound):
    bad = ~((got.to(D) - ref).abs() <= bound)
    assert not bool(bad.any()), (name, int(bad.sum()), float(((got.to(D) - ref).abs() / bound).nan_to_num(1e9).max()))
