"""The layer operators' definitions in 64 bits, with a bound on how far a
kernel's results may be off, derived from where it rounds: inputs are exact, u
is half a unit in the last place of the data type (f16 2^-11, bf16 2^-8, f32
2^-24), 32-bit sums of n terms are within n 2^-24 of the sum of their
magnitudes, and 2^-20 covers the elementary functions."""
import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}  # half the smallest step
E32, EF = 2.0 ** -24, 2.0 ** -20


def name_of(dtype):
    return {v: k for k, v in DT.items()}[dtype]


def worst(got, ref, bound):
    """Largest error as a share of its bound (inf where a value is not finite)."""
    err = (got.double() - ref).abs()
    if err.numel() == 0:
        return 0.0
    if not bool(torch.isfinite(err).all()):
        return math.inf
    return float((err / bound).max())


def check(got, ref, bound, what):
    w = worst(got, ref, bound)
    assert w <= 1.0, f"{what}: {w:.3g} of its bound"


def attention_ref(q, k, v, q_len=None, kv_len=None, kv_mask=None, scale=None, do=None):
    """dict of (value, bound) for o, lse and, given do, dq, dk, dv."""
    (B, Sq, Hq, D), (Sk, Hkv) = q.shape, k.shape[1:3]
    dt = name_of(q.dtype)
    u, tiny = U[dt], TINY[dt]
    scale = D ** -0.5 if scale is None else scale
    f64 = dict(dtype=torch.float64, device=q.device)
    z = lambda *s: torch.zeros(*s, **f64)  # noqa: E731
    o, eo = z(B, Sq, Hq, D), z(B, Sq, Hq, D)
    lse, el = torch.full((B, Hq, Sq), -math.inf, **f64), z(B, Hq, Sq)
    dq, edq = z(B, Sq, Hq, D), z(B, Sq, Hq, D)
    dk, edk, dv, edv = (z(B, Sk, Hkv, D) for _ in range(4))
    for b in range(B):
        nq = Sq if q_len is None else max(0, min(int(q_len[b]), Sq))
        nk = Sk if kv_len is None else max(0, min(int(kv_len[b]), Sk))
        keys = torch.arange(nk, device=q.device)
        if kv_mask is not None:
            keys = keys[kv_mask[b, :nk].bool()]
        if nq == 0 or len(keys) == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            Q, K, V = q[b, :nq, h].double(), k[b, keys, g].double(), v[b, keys, g].double()
            A = scale * (Q @ K.t())
            L = torch.logsumexp(A, 1)
            P = torch.exp(A - L[:, None])
            # relative error of an unrounded p: its score's, and the log-sum's
            e = 2 * (D + 8) * E32 * scale * float((Q.abs() @ K.abs().t()).max()) + \
                4 * E32 * float(A.abs().max()) + len(keys) * E32 + EF
            O = P @ V
            o[b, :nq, h] = O
            lse[b, h, :nq] = L
            el[b, h, :nq] = 2 * e + 4 * E32 * L.abs()
            eO = (u + 2 * e) * (P @ V.abs()) + tiny * V.abs().sum(0) * 2
            eo[b, :nq, h] = u * O.abs() + eO + tiny
            if do is None:
                continue
            G = do[b, :nq, h].double()
            dP = G @ V.t()
            delta = (G * O).sum(1, keepdim=True)
            dS = P * (dP - delta)
            # delta takes o as it was rounded
            edelta = (G.abs() * (eO + u * O.abs() + tiny)).sum(1, keepdim=True) + \
                (D + 8) * E32 * (G * O).abs().sum(1, keepdim=True)
            eS = (u + 2 * e) * dS.abs() + P * (edelta + (D + 8) * E32 * (G.abs() @ V.abs().t())) + tiny
            dq[b, :nq, h] = scale * (dS @ K)
            edq[b, :nq, h] = u * dq[b, :nq, h].abs() + tiny + \
                scale * ((eS + len(keys) * E32 * dS.abs()) @ K.abs())
            n = nq * (Hq // Hkv)
            dk[b, keys, g] += scale * (dS.t() @ Q)
            edk[b, keys, g] += scale * ((eS + n * E32 * dS.abs()).t() @ Q.abs())
            dv[b, keys, g] += P.t() @ G
            edv[b, keys, g] += ((u + 2 * e + n * E32) * P + tiny).t() @ G.abs()
    out = dict(o=(o, eo + 1e-300), lse=(lse, el + 1e-300))
    if do is not None:
        out.update(dq=(dq, edq + 1e-300), dk=(dk, edk + u * dk.abs() + tiny),
                   dv=(dv, edv + u * dv.abs() + tiny))
    return out


def attention_value(q, k, v, do, scale):
    """sum(do . o) in 64 bits of 64-bit inputs, no masks."""
    B, Sq, Hq, D = q.shape
    Hkv = k.shape[2]
    t = 0.0
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            P = torch.softmax(scale * (q[b, :, h] @ k[b, :, g].t()), 1)
            t = t + (do[b, :, h] * (P @ v[b, :, g])).sum()
    return t


def norm_ref(x, w, table, pos, eps, interleaved, dy=None):
    """dict of (value, bound) for y and, given dy, dx and dw."""
    T, H, D = x.shape
    dt = name_of(x.dtype)
    u, tiny = U[dt], TINY[dt]
    half = 0 if table is None else table.shape[2]
    X = x.double()
    W = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
    r = 1 / torch.sqrt((X * X).mean(2, keepdim=True) + eps)
    a = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    b = a + (1 if interleaved else half)
    c = s = None
    if half:
        c, s = (table[pos.long(), i].double()[:, None] for i in (0, 1))

    def turn(n, sign):
        y = n.clone()
        if half:
            y[..., a], y[..., b] = n[..., a] * c - sign * n[..., b] * s, sign * n[..., a] * s + n[..., b] * c
        return y

    def reach(n):  # the magnitudes that meet in a rotated component
        y = n.abs().clone()
        if half:
            y[..., a], y[..., b] = (n[..., a].abs() * c.abs() + n[..., b].abs() * s.abs(),
                                    n[..., a].abs() * s.abs() + n[..., b].abs() * c.abs())
        return y
    e = (D + 16) * E32
    n = X * r * W
    y = turn(n, 1.0)
    out = dict(y=(y, u * y.abs() + e * reach(n) + tiny))
    if dy is not None:
        G = turn(dy.double(), -1.0)
        rG = reach(dy.double())
        mean, rmean = (G * W * X).mean(2, keepdim=True), (rG * W.abs() * X.abs()).mean(2, keepdim=True)
        dx = r * (G * W - X * r * r * mean)
        out["dx"] = (dx, u * dx.abs() + 2 * e * r * (rG * W.abs() + X.abs() * r * r * rmean) + tiny)
        dw = (G * X * r).sum((0, 1))
        out["dw"] = (dw, u * dw.abs() + (2 * e + T * H * E32) * (rG * (X * r).abs()).sum((0, 1)) + tiny)
    return out


def act(z, name):
    if name == "relu":
        return torch.relu(z)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z * math.sqrt(0.5)) + \
            z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        t = torch.sigmoid(z)
        return t * (1 + z * (1 - t))
    return torch.ones_like(z)


def linear_ref(x, w, bias=None, residual=None, activation="none", dy=None):
    """dict of (value, bound) for y, z and, given dy, dx, dw, db."""
    (M, K), N = x.shape, w.shape[1]
    dt = name_of(x.dtype)
    u, tiny = U[dt], TINY[dt]
    X, W = x.double(), w.double()
    b = torch.zeros(N, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    z = X @ W + b
    ez = (K + 8) * E32 * (X.abs() @ W.abs() + b.abs())
    y = act(z, activation)
    R = torch.zeros_like(y) if residual is None else residual.double()
    ey = 1.13 * ez + EF * (z.abs() + 1) + 4 * E32 * (y.abs() + R.abs())  # |act'| <= 1.13
    out = dict(z=(z, u * z.abs() + ez + tiny), y=(y + R, u * (y + R).abs() + ey + tiny))
    if dy is not None:
        G = dy.double()
        dz = G * slope(z, activation)
        # act' is taken at the rounded z: |act''| <= 0.8; relu's only jumps at 0
        off = u * z.abs() + ez + tiny
        es = {"none": torch.zeros_like(z), "relu": (z.abs() <= ez + tiny).double()}.get(
            activation, 0.8 * off + EF * (1 + z.abs()))
        ed = G.abs() * es
        er = ed + u * (dz.abs() + ed) + tiny  # dz as the products take it
        dx, dw, db = dz @ W.t(), X.t() @ dz, dz.sum(0)
        out["dx"] = (dx, u * dx.abs() + (er + (N + 8) * E32 * dz.abs()) @ W.abs().t() + tiny)
        out["dw"] = (dw, u * dw.abs() + X.abs().t() @ (er + (M + 8) * E32 * dz.abs()) + tiny)
        out["db"] = (db, u * db.abs() + (ed + (M + 8) * E32 * dz.abs()).sum(0) + tiny)
    return out
