"""Timed cases of the layer operators: a block by which pose hypotheses read an
image encoder's states, through the binding's entry points.

The operators are the products, norms and attention of a decoder block whose
queries are hypotheses (or tokens) and whose keys and values are an encoder's
states of another length: layers.cross_attention, layers.norm_rotate and
layers.linear with their backward passes.  Sizes come from the framework's
workloads where they have one (1 to 1024 hypotheses, the 16- and 32-pixel
patches of 640 x 480 and 800 x 800 images: 300, 1200, 2500) and are generic
otherwise (head widths 64 and 128, layer widths that are powers of two).

A case's kind: "attention" a forward pass, "attention_train" forward and
backward, and likewise "norm", "norm_train", "linear", "linear_train".  With
`own` false, run() evaluates the operators in elementary torch operations in 32
bits; with `own` true it calls the framework.  exact() evaluates the
definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
DEV = "cuda"


def listed():
    return [
        # one hypothesis reading a 640 x 480 image's 32-pixel patches: the
        # smallest call, all latency
        dict(name="attn_one", kind="attention", dtype="f16", B=1, Sq=1, Sk=300, Hq=8, Hkv=8, D=64,
             ragged=False),
        # one token for each of 64 images of up to 800 x 800 (16-pixel patches),
        # padded to the longest, some patches masked, shared heads
        dict(name="attn_token_ragged", kind="attention", dtype="bf16", B=64, Sq=1, Sk=2500, Hq=16,
             Hkv=4, D=128, ragged=True),
        # one token over a long set of encoder states
        dict(name="attn_token_long", kind="attention", dtype="f16", B=1, Sq=1, Sk=131109, Hq=32,
             Hkv=8, D=128, ragged=False),
        # 1024 hypotheses each for two 640 x 480 images (16-pixel patches)
        dict(name="attn_hypotheses", kind="attention", dtype="bf16", B=2, Sq=1024, Sk=1200, Hq=16,
             Hkv=16, D=64, ragged=True),
        # the largest forward pass: a long target over long states, shared heads
        dict(name="attn_prompt", kind="attention", dtype="f16", B=2, Sq=4096, Sk=8191, Hq=32, Hkv=8,
             D=128, ragged=False),
        # a training step over padded batches of odd lengths, shared heads
        dict(name="attn_train", kind="attention_train", dtype="bf16", B=2, Sq=2011, Sk=2500, Hq=16,
             Hkv=4, D=128, ragged=True),
        # the next token's queries of 64 sequences (the states' keys are there already)
        dict(name="norm_token", kind="norm", dtype="bf16", Tq=64, Tk=0, Hq=16, Hkv=4, D=128, R=128,
             interleaved=False),
        # queries and keys of a long batch in one pass
        dict(name="norm_prompt", kind="norm", dtype="bf16", Tq=8192, Tk=16382, Hq=32, Hkv=8, D=128,
             R=128, interleaved=False),
        # a training step with a part of each head rotated, pairs side by side
        dict(name="norm_train", kind="norm_train", dtype="f16", Tq=4022, Tk=5000, Hq=16, Hkv=16, D=64,
             R=32, interleaved=True),
        # four tokens through a wide layer: the weights' bytes
        dict(name="linear_token", kind="linear", dtype="bf16", M=4, K=4096, N=16384, act="silu",
             bias=True, residual=False),
        # a long batch through a wide layer, everything in the epilogue
        dict(name="linear_prompt", kind="linear", dtype="f16", M=4096, K=2048, N=8192, act="gelu",
             bias=True, residual=True),
        # a training step through a square layer, an odd number of rows
        dict(name="linear_train", kind="linear_train", dtype="bf16", M=4095, K=4096, N=4096,
             act="gelu", bias=True, residual=True),
    ]


def _span(rng, lo, hi):
    """A whole number of [lo, hi], uniform in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _draw_once(rng):
    kind = rng.choice(["attention", "attention", "attention_train", "norm", "norm_train", "linear",
                       "linear", "linear_train"])
    train = kind.endswith("_train")
    case = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]))
    if kind.startswith("attention"):
        Hkv = rng.choice([1, 2, 4, 8, 16])
        case.update(B=_span(rng, 1, 8 if train else 64),
                    Sq=1 if not train and rng.random() < 0.4 else _span(rng, 2, 4096),
                    Sk=_span(rng, 1, 8191), Hq=Hkv * rng.choice([1, 1, 2, 4, 8]), Hkv=Hkv,
                    D=rng.choice([32, 64, 64, 80, 96, 128, 128]), ragged=rng.random() < 0.5)
        if case["Sq"] == 1 and rng.random() < 0.3:
            case.update(B=1, Sk=_span(rng, 8192, 131109))
    elif kind.startswith("norm"):
        D = rng.choice([32, 64, 64, 80, 96, 128, 128])
        Hkv = rng.choice([1, 2, 4, 8, 16])
        case.update(dtype=rng.choice(["f32", "f16", "bf16"]), Tq=_span(rng, 1, 16384),
                    Tk=rng.choice([0, _span(rng, 1, 16384)]), Hq=Hkv * rng.choice([1, 2, 4]), Hkv=Hkv,
                    D=D, R=rng.choice([D, D // 2]), interleaved=rng.random() < 0.5)
    else:
        case.update(M=_span(rng, 33, 8192) if train or rng.random() < 0.6 else _span(rng, 1, 32),
                    K=_span(rng, 24, 8192), N=_span(rng, 3, 16384),
                    act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.7,
                    residual=rng.random() < 0.5)
        if rng.random() < 0.7:  # widths are mostly multiples of 8
            case.update(K=8 * max(1, case["K"] // 8), N=8 * max(1, case["N"] // 8))
    return case


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        case = _draw_once(rng)
        w, train = work(case), case["kind"].endswith("_train")
        if case["kind"].startswith("attention"):
            # the plain form's 32-bit scores stay below the largest listed case's
            scores = (4 if train else 1) * case["B"] * case["Hq"] * case["Sq"] * case["Sk"]
            if scores > 2 * 32 * 4096 * 8191:
                continue
        if all(w[k] <= max(m[k] for m in most) for k in w):
            return case


# ---------------------------------------------------------------- inputs
def _lengths(n, most, gen):
    """n lengths spread evenly over [most / 4, most], in an order from gen."""
    lens = [most - (i * (most - most // 4)) // max(n - 1, 1) for i in range(n)]
    return [lens[i] for i in torch.randperm(n, generator=gen).tolist()]


def _valid_share(case):
    """Mean share of the keys, and of the queries, that a ragged case holds."""
    if not case["ragged"]:
        return 1.0, 1.0

    def share(most):
        n = case["B"]
        lens = [most - (i * (most - most // 4)) // max(n - 1, 1) for i in range(n)]
        return sum(lens) / (n * most)
    return share(case["Sk"]), share(case["Sq"]) if case["Sq"] > 1 else 1.0


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dgen = torch.Generator(DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=dgen, device=DEV, dtype=torch.float32) * std).to(dtype)

    s = dict(case)
    kind = case["kind"]
    if kind.startswith("attention"):
        B, Sq, Sk, Hq, Hkv, D = (case[k] for k in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
        s["q"] = normal(B, Sq, Hq, D)
        # keys and values side by side, as one projection of the states leaves them
        kv = normal(B, Sk, 2, Hkv, D)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["q_len"] = s["kv_len"] = s["mask"] = None
        if case["ragged"]:
            s["kv_len"] = torch.tensor(_lengths(B, Sk, gen), dtype=torch.int32, device=DEV)
            if Sq > 1:
                s["q_len"] = torch.tensor(_lengths(B, Sq, gen), dtype=torch.int32, device=DEV)
            s["mask"] = torch.rand(B, Sk, generator=dgen, device=DEV) > 0.05
        if kind == "attention_train":
            s["do"] = normal(B, Sq, Hq, D)
    elif kind.startswith("norm"):
        Tq, Tk, Hq, Hkv, D, R = (case[k] for k in ("Tq", "Tk", "Hq", "Hkv", "D", "R"))
        s["q"], s["k"] = normal(Tq, Hq, D), normal(Tk, Hkv, D) if Tk else None
        s["wq"] = (1.0 + normal(D, std=0.1, dtype=torch.float32)).to(dt)
        s["wk"] = (1.0 + normal(D, std=0.1, dtype=torch.float32)).to(dt) if Tk else None
        n_pos = 4096
        freq = 10000.0 ** (-torch.arange(R // 2, dtype=torch.float64, device=DEV) / (R // 2))
        angle = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * freq
        s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float()
        start = int(torch.randint(0, n_pos, (1,), generator=gen))
        s["pos_q"] = ((torch.arange(Tq, device=DEV) + start) % n_pos).int()
        s["pos_k"] = (torch.arange(Tk, device=DEV) % n_pos).int() if Tk else None
        if kind == "norm_train":
            s["dq"], s["dk"] = normal(Tq, Hq, D), normal(Tk, Hkv, D) if Tk else None
    else:
        M, K, N = (case[k] for k in ("M", "K", "N"))
        s["x"], s["w"] = normal(M, K), normal(K, N, std=K ** -0.5)
        s["b"] = normal(N, std=0.5) if case["bias"] else None
        s["res"] = normal(M, N) if case["residual"] else None
        if kind == "linear_train":
            s["dy"] = normal(M, N)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2210_10108_amd import layers
    kind = s["kind"]
    if kind == "attention":
        return layers.cross_attention(s["q"], s["k"], s["v"], q_len=s["q_len"], kv_len=s["kv_len"],
                                      kv_mask=s["mask"])
    if kind == "attention_train":
        masks = dict(q_len=s["q_len"], kv_len=s["kv_len"], kv_mask=s["mask"])
        o, lse = layers.cross_attention(s["q"], s["k"], s["v"], return_lse=True, **masks)
        return (o, *layers.cross_attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, **masks))
    if kind == "norm":
        q, k = layers.norm_rotate(s["q"], s["k"], s["wq"], s["wk"], s["table"], s["pos_q"], s["pos_k"],
                                  eps=EPS, interleaved=s["interleaved"])
        return [q] if k is None else [q, k]
    if kind == "norm_train":
        rest = (s["q"], s["k"], s["wq"], s["wk"], s["table"], s["pos_q"], s["pos_k"])
        kw = dict(eps=EPS, interleaved=s["interleaved"])
        out = layers.norm_rotate(*rest, **kw)
        out += layers.norm_rotate_backward(s["dq"], s["dk"], *rest, **kw)
        return [t for t in out if t is not None]
    if kind == "linear":
        return layers.linear(s["x"], s["w"], s["b"], s["res"], activation=s["act"])
    y, z = layers.linear(s["x"], s["w"], s["b"], s["res"], activation=s["act"], return_preact=True)
    grads = layers.linear_backward(s["dy"], s["x"], s["w"], z, activation=s["act"],
                                   bias=s["b"] is not None)
    return [y] + [t for t in grads if t is not None]


def _rows(x, Hkv):
    """[B, S, H, D] as 32-bit [B, Hkv, (H / Hkv) S, D]: the rows that share a kv head."""
    B, S, H, D = x.shape
    return x.float().reshape(B, S, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)


def _unrows(x, S, dtype):
    B, Hkv, GS, D = x.shape
    return x.reshape(B, Hkv, GS // S, S, D).permute(0, 3, 1, 2, 4).reshape(B, S, -1, D).to(dtype)


def _plain_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    (B, Sq, Hq, D), (Sk, Hkv) = q.shape, k.shape[1:3]
    dt, scale = q.dtype, D ** -0.5
    valid = torch.ones(B, Sk, dtype=torch.bool, device=q.device)
    if s["kv_len"] is not None:
        valid = torch.arange(Sk, device=q.device) < s["kv_len"][:, None]
    if s["mask"] is not None:
        valid = valid & s["mask"]
    row = torch.ones(B, Sq, dtype=torch.bool, device=q.device)
    if s["q_len"] is not None:
        row = torch.arange(Sq, device=q.device) < s["q_len"][:, None]
    row = row[:, None, None, :, None].expand(B, 1, Hq // Hkv, Sq, 1).reshape(B, 1, -1, 1)
    zero = q.new_zeros((), dtype=torch.float32)
    qr, kr, vr = _rows(q, Hkv), _rows(k, Hkv), _rows(v, Hkv)
    kr, vr = (torch.where(valid[:, None, :, None], x, zero) for x in (kr, vr))
    a = torch.matmul(qr, kr.transpose(2, 3).contiguous()).mul_(scale)
    a.masked_fill_(~(valid[:, None, None, :] & row), -math.inf)
    m = a.amax(3, keepdim=True)
    p = a.sub_(torch.where(m == -math.inf, zero, m)).exp_()
    total = p.sum(3, keepdim=True)
    p.div_(torch.where(total == 0, zero + 1, total))
    o = torch.matmul(p, vr)
    out = _unrows(o, Sq, dt)
    if "do" not in s:
        return out
    do = torch.where(row, _rows(s["do"], Hkv), zero)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, vr.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(3, keepdim=True)) * scale
    dq = torch.matmul(ds, kr)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), qr)
    return out, _unrows(dq, Sq, dt), _unrows(dk, Sk, dt), _unrows(dv, Sk, dt)


def _rotate(x, table, pos, interleaved, sign):
    """Pairs of the first R components turned by sign * angle(position)."""
    half = table.shape[2]
    c, s = table[pos.long(), 0][:, None], sign * table[pos.long(), 1][:, None]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * c - b * s, a * s + b * c
    return y


def _plain_norm(s):
    out, grads, wgrads = [], [], []
    for x, w, pos, dy in ((s["q"], s["wq"], s["pos_q"], s.get("dq")),
                          (s["k"], s["wk"], s["pos_k"], s.get("dk"))):
        if x is None:
            continue
        xf, wf = x.float(), w.float()
        r = torch.rsqrt((xf * xf).mean(2, keepdim=True) + EPS)
        out.append(_rotate(xf * r * wf, s["table"], pos, s["interleaved"], 1.0).to(x.dtype))
        if dy is not None:
            g = _rotate(dy.float(), s["table"], pos, s["interleaved"], -1.0)
            wgrads.append((g * xf * r).sum((0, 1)).to(x.dtype))
            gw = g * wf
            grads.append((r * (gw - xf * r * r * (gw * xf).mean(2, keepdim=True))).to(x.dtype))
    return out + grads + wgrads


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + \
            z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return t * (1.0 + z * (1.0 - t))
    return torch.ones_like(z)


def _plain_linear(s):
    dt = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = torch.matmul(x, w)
    if s["b"] is not None:
        z += s["b"].float()
    y = _act(z, s["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    if "dy" not in s:
        return y.to(dt)
    dz = s["dy"].float() * _act_grad(z, s["act"])
    grads = [torch.matmul(dz, w.t()), torch.matmul(x.t(), dz)]
    if s["b"] is not None:
        grads.append(dz.sum(0))
    return [y.to(dt)] + [g.to(dt) for g in grads]


def _run_plain(s):
    kind = s["kind"]
    if kind.startswith("attention"):
        return _plain_attention(s)
    return _plain_norm(s) if kind.startswith("norm") else _plain_linear(s)


# ---------------------------------------------------------------- what a pass needs
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    kind, train = case["kind"], case["kind"].endswith("_train")
    if kind.startswith("attention"):
        B, Sq, Sk, Hq, Hkv, D = (case[k] for k in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
        fk, fq = _valid_share(case)
        rows, keys = B * Sq * Hq * D, B * Sk * Hkv * D
        pairs = fk * fq * B * Hq * Sq * Sk * D
        if train:  # q, do, k, v read; o, dq, dk, dv written
            return {"bytes": e * (rows * (2 * fq + 2) + keys * (2 * fk + 2)), "flops": 14 * pairs}
        return {"bytes": e * (rows * (fq + 1) + 2 * fk * keys), "flops": 4 * pairs}
    if kind.startswith("norm"):
        n = (case["Tq"] * case["Hq"] + case["Tk"] * case["Hkv"]) * case["D"]
        angles = 4 * case["R"] * min(4096, max(case["Tq"], case["Tk"]))
        # x (and dy) read; y (and dx) written
        return {"bytes": (4 if train else 2) * e * n + angles, "flops": (20 if train else 8) * n}
    M, K, N = case["M"], case["K"], case["N"]
    if train:  # x, w, residual, dy read; y, dx, dw written
        more = M * N * (2 + case["residual"]) + 2 * N * case["bias"]
        return {"bytes": e * (2 * M * K + 2 * K * N + more), "flops": 6 * M * K * N}
    more = M * N * (1 + case["residual"]) + N * case["bias"]
    return {"bytes": e * (M * K + K * N + more), "flops": 2 * M * K * N}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions in 64 bits, entry by entry, over the allowed keys alone."""
    s = prepare(case, seed)
    if case["kind"].startswith("attention"):
        return _exact_attention(s)
    if case["kind"].startswith("norm"):
        return _exact_norm(s)
    return _exact_linear(s)


def _exact_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    (B, Sq, Hq, D), (Sk, Hkv) = q.shape, k.shape[1:3]
    scale = 1.0 / math.sqrt(D)
    f64 = dict(dtype=torch.float64, device=q.device)
    o = torch.zeros(B, Sq, Hq, D, **f64)
    train = "do" in s
    if train:
        dq, dk, dv = torch.zeros_like(o), torch.zeros(B, Sk, Hkv, D, **f64), torch.zeros(B, Sk, Hkv, D, **f64)
    for b in range(B):
        nq = Sq if s["q_len"] is None else int(s["q_len"][b])
        nk = Sk if s["kv_len"] is None else int(s["kv_len"][b])
        keys = torch.arange(nk, device=q.device)
        if s["mask"] is not None:
            keys = keys[s["mask"][b, :nk]]
        if nq == 0 or len(keys) == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            Q, K, V = q[b, :nq, h].double(), k[b, keys, g].double(), v[b, keys, g].double()
            P = torch.softmax((Q @ K.t()) * scale, dim=1)
            o[b, :nq, h] = P @ V
            if train:
                G = s["do"][b, :nq, h].double()
                dP = G @ V.t()
                dS = P * (dP - (P * dP).sum(1, keepdim=True))
                dq[b, :nq, h] = scale * (dS @ K)
                dk[b, keys, g] += scale * (dS.t() @ Q)
                dv[b, keys, g] += P.t() @ G
    return (o, dq, dk, dv) if train else o


def _exact_norm(s):
    """The rotation as a product of complex numbers; the gradients by
    differentiating sum(dy . y) in 64 bits."""
    out, grads, wgrads = [], [], []
    for x, w, pos, dy in ((s["q"], s["wq"], s["pos_q"], s.get("dq")),
                          (s["k"], s["wk"], s["pos_k"], s.get("dk"))):
        if x is None:
            continue
        half = s["table"].shape[2]
        t = s["table"].double()[pos.long()]
        turn = torch.complex(t[:, 0], t[:, 1])[:, None]
        with torch.enable_grad():
            X, W = x.double().requires_grad_(), w.double().requires_grad_()
            n = X / torch.sqrt(X.square().sum(2, keepdim=True) / X.shape[2] + EPS) * W
            if s["interleaved"]:
                z = torch.complex(n[..., 0:2 * half:2], n[..., 1:2 * half:2]) * turn
                head = torch.stack([z.real, z.imag], 3).flatten(2)
            else:
                z = torch.complex(n[..., :half], n[..., half:2 * half]) * turn
                head = torch.cat([z.real, z.imag], 2)
            y = torch.cat([head, n[..., 2 * half:]], 2)
            out.append(y.detach())
            if dy is not None:
                gx, gw = torch.autograd.grad((dy.double() * y).sum(), (X, W))
                grads.append(gx)
                wgrads.append(gw)
    return out + grads + wgrads


def _exact_linear(s):
    x, w = s["x"].double(), s["w"].double()
    z = x @ w + (0.0 if s["b"] is None else s["b"].double())
    phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    gate = torch.sigmoid(z)
    y, slope = {
        "none": lambda: (z, torch.ones_like(z)),
        "relu": lambda: (torch.relu(z), torch.heaviside(z, torch.zeros_like(z))),
        "gelu": lambda: (z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)),
        "silu": lambda: (z * gate, gate + z * gate * (1 - gate)),
    }[s["act"]]()
    if s["res"] is not None:
        y = y + s["res"].double()
    if "dy" not in s:
        return y
    dz = s["dy"].double() * slope
    return [y, dz @ w.t(), x.t() @ dz] + ([] if s["b"] is None else [dz.sum(0)])
