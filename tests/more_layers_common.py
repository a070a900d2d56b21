"""Layer norm, rotation at positions of several axes, gradient clipping and 8-bit
states: their definitions in 64 bits, with bounds on how far a kernel's results may
be off, derived from where it rounds as in layers_common.  A sum over n terms is
made of chains of at most chain(n) additions (64 or more lanes, then a tree), each
within E32 of the sum of magnitudes."""
import math

import torch

from .layers_common import E32, TINY, U, name_of


def chain(n):
    return min(n, n // 64 + 96)


# ---------------------------------------------------------------- layer norm
def layer_norm_ref(x, w, b, eps, dy=None, dres=None):
    """dict of (value, bound) for y and, given dy, dx, dw and db."""
    rows, W = x.shape
    dt = name_of(x.dtype)
    u, tiny, s = U[dt], TINY[dt], chain(W) * E32
    X = x.double()
    Wt = torch.ones(W, dtype=torch.float64, device=x.device) if w is None else w.double()
    B = torch.zeros_like(Wt) if b is None else b.double()
    d = X - X.mean(1, keepdim=True)
    r = 1 / torch.sqrt(d.square().mean(1, keepdim=True) + eps)
    n = d * r
    y = n * Wt + B
    # the first mean m is off by `off`, in units of the spread; x - m and its mean's
    # correction by a rounding of |x - m| each and a sum's error; the variance, mean
    # (x - m)^2 - c^2, by a sum's error relative to var + c^2
    off = (s + 2 * E32) * X.abs().mean(1, keepdim=True) * r
    en = 2 * E32 * (n.abs() + off) + s * (n.abs().mean(1, keepdim=True) + off) + \
        ((2 * s + 4 * E32) * (1 + off * off) + 16 * E32) * n.abs()
    out = dict(y=(y, u * y.abs() + en * Wt.abs() + 4 * E32 * ((n * Wt).abs() + B.abs()) + tiny))
    if dy is None:
        return out
    G = dy.double()
    g = G * Wt
    s1, s2 = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    D = torch.zeros_like(X) if dres is None else dres.double()
    dx = r * (g - s1 - n * s2) + D
    m1, m2 = g.abs().mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    # g, its mean, the mean of g n (whose n is off by en) and n times it
    es2 = (3 * s + 8 * E32) * (m2 + m1 * (1 + off)) + (g.abs() * en).mean(1, keepdim=True)
    er = (2 * s + 4 * E32) * (1 + off * off) + 16 * E32  # of r
    e = er * (g.abs() + m1 + n.abs() * m2) + s * m1 + n.abs() * es2 + en * m2
    out["dx"] = (dx, u * dx.abs() + r * e + 2 * E32 * D.abs() + tiny)
    t = chain(rows) * E32
    dw, db = (G * n).sum(0), G.sum(0)
    out["dw"] = (dw, u * dw.abs() + (G.abs() * (en + (t + 2 * E32) * n.abs())).sum(0) + tiny)
    out["db"] = (db, u * db.abs() + t * G.abs().sum(0) + tiny)
    return out


# ---------------------------------------------------------------- rotation
def axes_ref(x, w, table, pos, pair_axis, eps, interleaved, dy=None):
    """dict of (value, bound) for y and, given dy, dx and (with eps) dw."""
    T, H, D = x.shape
    dt = name_of(x.dtype)
    u, tiny = U[dt], TINY[dt]
    half = table.shape[2]
    a = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    b = a + (1 if interleaved else half)
    pairs = torch.arange(half, device=x.device)
    at = pos.long()[:, torch.tensor(list(pair_axis), device=x.device, dtype=torch.long)]
    c, s = table.double()[at, 0, pairs][:, None], table.double()[at, 1, pairs][:, None]

    def turn(n, sign):
        y = n.clone()
        y[..., a], y[..., b] = n[..., a] * c - sign * n[..., b] * s, sign * n[..., a] * s + n[..., b] * c
        return y

    def reach(n):
        y = n.abs().clone()
        y[..., a], y[..., b] = (n[..., a].abs() * c.abs() + n[..., b].abs() * s.abs(),
                                n[..., a].abs() * s.abs() + n[..., b].abs() * c.abs())
        return y
    X = x.double()
    if eps is None:
        out = dict(y=(turn(X, 1.0), u * turn(X, 1.0).abs() + 4 * E32 * reach(X) + tiny))
        if dy is not None:
            G = dy.double()
            out["dx"] = (turn(G, -1.0), u * turn(G, -1.0).abs() + 4 * E32 * reach(G) + tiny)
        return out
    W = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
    r = 1 / torch.sqrt((X * X).mean(2, keepdim=True) + eps)
    e = (D + 16) * E32
    n = X * r * W
    y = turn(n, 1.0)
    out = dict(y=(y, u * y.abs() + e * reach(n) + tiny))
    if dy is not None:
        G, rG = turn(dy.double(), -1.0), reach(dy.double())
        mean, rmean = (G * W * X).mean(2, keepdim=True), (rG * W.abs() * X.abs()).mean(2, keepdim=True)
        dx = r * (G * W - X * r * r * mean)
        out["dx"] = (dx, u * dx.abs() + 2 * e * r * (rG * W.abs() + X.abs() * r * r * rmean) + tiny)
        dw = (G * X * r).sum((0, 1))
        out["dw"] = (dw, u * dw.abs() + (2 * e + T * H * E32) * (rG * (X * r).abs()).sum((0, 1)) + tiny)
    return out


# ---------------------------------------------------------------- clipping
def clip_ref(grads, max_norm, eps=1e-6, out_dtypes=None):
    """((norm, bound), [(out, bound)])."""
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    c = 1.0 if math.isinf(max_norm) or norm + eps == 0.0 else min(1.0, max_norm / (norm + eps))
    outs = []
    for i, g in enumerate(grads):
        dt = name_of(g.dtype if out_dtypes is None else out_dtypes[i])
        o = g.double() * c
        # c is rounded to 32 bits, and the product
        outs.append((o, (U[dt] + 2 * E32) * o.abs() + TINY[dt] + 1e-300))
    return (norm, norm * 2 * E32 + 1e-300), outs


# ---------------------------------------------------------------- 8-bit states
BLOCK = 64


def allowed(B, S, kv_len, kv_mask, device):
    on = torch.ones(B, S, dtype=torch.bool, device=device)
    if kv_len is not None:
        on &= torch.arange(S, device=device) < kv_len[:, None]
    return on if kv_mask is None else on & kv_mask.bool()


def power_of_two(e):
    """2^e in 64 bits, by its bits (exp2 and ldexp round on some devices)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantize_ref(x, on):
    """(values as float64, scales as float32): steps of 2^-9 below 2^-6, of an
    eighth of the power of two above, ties to the even multiple."""
    B, S, H, D = x.shape
    X = torch.where(on[:, :, None, None], x.double(), torch.zeros((), dtype=torch.float64, device=x.device))
    finite = torch.isfinite(X)
    x8, scales = torch.zeros_like(X), []
    for t in range(0, S, BLOCK):
        most = torch.where(finite, X, 0.0)[:, t:t + BLOCK].abs().amax((1, 3))
        m, e = torch.frexp(most / 448.0)  # m in [1/2, 1)
        e = torch.where(m == 0.5, e - 1, e).clamp_min(-126)
        scale = torch.where(most > 0, power_of_two(e), 1.0)
        v = X[:, t:t + BLOCK] / scale[:, None, :, None]
        near = torch.where(finite[:, t:t + BLOCK], v, 0.0).abs().clamp_min(2.0 ** -6)
        step = power_of_two(torch.frexp(near)[1] - 4)
        v = torch.round(v / step) * step
        x8[:, t:t + BLOCK] = torch.where(finite[:, t:t + BLOCK], v, math.nan)
        scales.append(scale.float())
    return x8, torch.stack(scales, 1) if scales else x.new_zeros(B, 0, H, dtype=torch.float32)


def widened(x8, scale):
    """The values that 8-bit states stand for, in 64 bits."""
    return x8.float().double() * scale.double().repeat_interleave(BLOCK, 1)[:, :x8.shape[1], :, None]
