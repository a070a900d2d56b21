"""Timed cases of the layer operators of a block that reads image patches, as it
is trained and as it is served, through the binding's entry points.

Training: layers.layer_norm (tokens of any width), layers.rotate_axes (heads
turned by a patch's time, row and column) with their backward passes, and
layers.clip_gradients before the optimiser's step.  Serving:
layers.quantize_states keeps an encoder's keys and values in 8 bits with a scale
for each block of 64 rows and head, layers.cross_attention_q8 reads them.  Sizes
come from the framework's workloads where they have one (1 to 1024 hypotheses,
the 16- and 32-pixel patches of 640 x 480 and 800 x 800 images: 300, 1200, 2500;
the proposal block of width 256 with its 16 parameters) and are generic otherwise
(head widths 64 and 128, layer widths that are powers of two).

A case's kind: "layer", "layer_train", "axes", "axes_train", "clip", "quant",
"q8"; _train is forward and backward.  With `own` false, run() evaluates the
operators in elementary torch operations in 32 bits (the sum of squares over all
gradients in 64); with `own` true it calls the framework.  exact() evaluates the
definitions in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-5
BLOCK = 64    # rows of the states that share a scale
POSITIONS = 4096
DEV = "cuda"


def listed():
    return [
        # 64 hypotheses at the proposal block's width: the smallest call, all latency
        dict(name="layer_token", kind="layer", dtype="bf16", rows=64, W=256, bias=True, residual=False),
        # a training step over a long batch of an odd number of tokens, the gradient
        # that goes past the norm added in the same pass
        dict(name="layer_train", kind="layer_train", dtype="bf16", rows=16381, W=2048, bias=True,
             residual=True),
        # the next token of 64 sequences, axes taken in turn over the pairs
        dict(name="axes_token", kind="axes", dtype="bf16", Tq=64, Tk=64, Hq=16, Hkv=4, D=128, R=128,
             axes=3, turns=True, norm=False, interleaved=False),
        # queries and keys of a long batch of video patches: pairs for time, rows and columns
        dict(name="axes_prompt", kind="axes", dtype="bf16", Tq=16382, Tk=16382, Hq=16, Hkv=8, D=128,
             R=128, axes=3, turns=False, norm=False, interleaved=False),
        # a training step: 1024 hypotheses a view against 2500 patches (800 x 800, 16 pixels),
        # normed heads, rows and columns
        dict(name="axes_train", kind="axes_train", dtype="f16", Tq=4096, Tk=10000, Hq=8, Hkv=4, D=64,
             R=64, axes=2, turns=False, norm=True, interleaved=False),
        # the proposal block's 16 gradients, for float32 masters: many small tensors
        dict(name="clip_block", kind="clip", dtype="bf16", out="f32", count=16, most=262144, mix=-1,
             active=True),
        # the gradients of a large network: 150 tensors from a few elements to 32 million
        dict(name="clip_network", kind="clip", dtype="bf16", out="bf16", count=150, most=1 << 25, mix=3,
             active=True),
        # keys and values of one 640 x 480 image's 32-pixel patches
        dict(name="quant_image", kind="quant", dtype="bf16", B=1, Sk=300, Hkv=2, D=64, ragged=False),
        # 64 views of up to 800 x 800 (16-pixel patches), padded, some patches masked
        dict(name="quant_views", kind="quant", dtype="f16", B=64, Sk=2500, Hkv=8, D=128, ragged=True),
        # one token for each of 64 views, padded to the longest, some patches masked, shared heads
        dict(name="q8_token_ragged", kind="q8", dtype="bf16", B=64, Sq=1, Sk=2500, Hq=16, Hkv=4, D=128,
             ragged=True),
        # one token over a long set of views' states
        dict(name="q8_token_long", kind="q8", dtype="f16", B=1, Sq=1, Sk=131109, Hq=32, Hkv=8, D=128,
             ragged=False),
        # 1024 hypotheses over the states of four 640 x 480 views (16-pixel patches), four batches
        dict(name="q8_hypotheses", kind="q8", dtype="bf16", B=4, Sq=1024, Sk=4800, Hq=16, Hkv=4, D=128,
             ragged=True),
    ]


def _span(rng, lo, hi):
    """A whole number of [lo, hi], uniform in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _draw_once(rng):
    kind = rng.choice(["layer", "layer_train", "layer_train", "axes", "axes_train", "clip", "clip",
                       "quant", "q8", "q8", "q8"])
    case = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]))
    if kind.startswith("layer"):
        W = _span(rng, 24, 16384)
        if rng.random() < 0.7:  # widths are mostly multiples of 8
            W = 8 * max(1, W // 8)
        case.update(dtype=rng.choice(["f32", "f16", "bf16"]), rows=_span(rng, 1, 32768), W=W,
                    bias=rng.random() < 0.7, residual=kind == "layer_train" and rng.random() < 0.5)
    elif kind.startswith("axes"):
        D = rng.choice([32, 64, 64, 80, 96, 128, 128])
        Hkv = rng.choice([1, 2, 4, 8, 16])
        case.update(dtype=rng.choice(["f32", "f16", "bf16"]), Tq=_span(rng, 1, 16384),
                    Tk=rng.choice([0, _span(rng, 1, 16384)]), Hq=Hkv * rng.choice([1, 2, 4]), Hkv=Hkv,
                    D=D, R=rng.choice([D, D, D // 2]), axes=rng.choice([2, 2, 3, 3, 4]),
                    turns=rng.random() < 0.3, norm=rng.random() < 0.5, interleaved=rng.random() < 0.3)
    elif kind == "clip":
        case["dtype"] = rng.choice(["f32", "f16", "bf16"])
        case.update(out=rng.choice([case["dtype"], "f32"]), count=_span(rng, 1, 150),
                    most=_span(rng, 64, 1 << 25), mix=rng.randrange(1 << 20), active=rng.random() < 0.7)
    else:
        Hkv = rng.choice([1, 2, 4, 8, 16])
        case.update(B=_span(rng, 1, 64), Sk=_span(rng, 1, 8191), Hkv=Hkv,
                    D=rng.choice([32, 64, 64, 80, 96, 128, 128]), ragged=rng.random() < 0.5)
        if kind == "q8":
            case.update(Sq=1 if rng.random() < 0.5 else _span(rng, 2, 2048),
                        Hq=Hkv * rng.choice([1, 1, 2, 4, 8]))
            if case["Sq"] == 1 and rng.random() < 0.3:
                case.update(B=1, Sk=_span(rng, 8192, 131109))
    return case


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        case = _draw_once(rng)
        w = work(case)
        # the plain form's 32-bit scores and copies of the states stay below the largest listed case's
        if case["kind"] == "q8" and (case["B"] * case["Hq"] * case["Sq"] * case["Sk"] > 4 * 16 * 1024 * 4800 or
                                     case["B"] * case["Hkv"] * case["Sk"] > 2 * 8 * 131109):
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
    return share(case["Sk"]), share(case["Sq"]) if case.get("Sq", 1) > 1 else 1.0


def _sizes(case):
    """The gradients' numbers of elements: the proposal block's (mix = -1), or
    weights and biases whose sizes are spread over their logarithm, some odd."""
    if case["mix"] < 0:
        w = 256
        return [16 * w, w, w, w * w, 48 * w, 64, 64, w * w, w, w, 4 * w * w, 4 * w, 4 * w * w, w, 8 * w, 8]
    rng = random.Random(case["mix"])
    sizes = []
    for i in range(case["count"]):
        n = _span(rng, 1, case["most"]) if i else case["most"]
        sizes.append(n if rng.random() < 0.2 else 8 * max(1, n // 8))
    return sizes


def _pair_axis(case):
    """The axis of every pair: in turn, or in runs of multiples of 8 where there are enough."""
    pairs, axes = case["R"] // 2, case["axes"]
    if case["turns"]:
        return bytes(j % axes for j in range(pairs))
    unit = 8 if pairs >= 8 * axes else 1
    first = pairs - (axes - 1) * (pairs // axes // unit * unit)
    return bytes(0 if j < first else 1 + (j - first) // (pairs // axes // unit * unit) for j in range(pairs))


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dgen = torch.Generator(DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=dgen, device=DEV, dtype=torch.float32) * std).to(dtype)

    s = dict(case)
    kind = case["kind"]
    if kind.startswith("layer"):
        rows, W = case["rows"], case["W"]
        # tokens whose mean is not 0, some features larger than the rest, as a residual stream has them
        size = 1.0 + 3.0 * (torch.rand(W, generator=dgen, device=DEV) < 0.02)
        s["x"] = (normal(rows, W, dtype=torch.float32) * size + 0.3).to(dt)
        s["w"] = (1.0 + normal(W, std=0.1, dtype=torch.float32)).to(dt)
        s["b"] = normal(W, std=0.1) if case["bias"] else None
        if kind == "layer_train":
            s["dy"], s["dres"] = normal(rows, W), normal(rows, W) if case["residual"] else None
    elif kind.startswith("axes"):
        Tq, Tk, Hq, Hkv, D, R, axes = (case[k] for k in ("Tq", "Tk", "Hq", "Hkv", "D", "R", "axes"))
        s["q"], s["k"] = normal(Tq, Hq, D), normal(Tk, Hkv, D) if Tk else None
        s["wq"] = (1.0 + normal(D, std=0.1, dtype=torch.float32)).to(dt) if case["norm"] else None
        s["wk"] = (1.0 + normal(D, std=0.1, dtype=torch.float32)).to(dt) if case["norm"] and Tk else None
        s["pair_axis"] = _pair_axis(case)
        freq = 10000.0 ** (-torch.arange(R // 2, dtype=torch.float64, device=DEV) / (R // 2))
        angle = torch.arange(POSITIONS, dtype=torch.float64, device=DEV)[:, None] * freq
        s["table"] = torch.stack([angle.cos(), angle.sin()], 1).float()
        start = int(torch.randint(0, POSITIONS, (1,), generator=gen))

        def walk(n):  # patches in order: a column fastest, then rows, then frames
            t = torch.arange(n, device=DEV) + start
            steps = [t // 2500, t // 50 % 50, t % 50, t % 7]
            return torch.stack([steps[a % 4] % POSITIONS for a in range(axes)], 1).int()
        s["pos_q"], s["pos_k"] = walk(Tq), walk(Tk) if Tk else None
        if kind == "axes_train":
            s["dq"], s["dk"] = normal(Tq, Hq, D), normal(Tk, Hkv, D) if Tk else None
    elif kind == "clip":
        sizes, odt = _sizes(case), DTYPES[case["out"]]
        start = [0]
        for n in sizes:  # every tensor starts on a whole chunk of its buffer
            start.append(start[-1] + (n + 63) // 64 * 64)
        flat = normal(start[-1], std=8.0 / math.sqrt(sum(sizes)))
        s["flat_out"] = torch.zeros(start[-1], dtype=odt, device=DEV)
        s["grads"] = [flat[a:a + n] for a, n in zip(start, sizes)]
        s["outs"] = [s["flat_out"][a:a + n] for a, n in zip(start, sizes)]
        s["max_norm"] = 1.0 if case["active"] else 100.0
    else:
        B, Sk, Hkv, D = (case[k] for k in ("B", "Sk", "Hkv", "D"))
        # keys and values side by side, as one projection of the states leaves them; heads and
        # stretches of rows of different sizes
        size = torch.exp(0.5 * normal(B, -(-Sk // 200), 2, Hkv, 1, dtype=torch.float32))
        kv = (normal(B, Sk, 2, Hkv, D, dtype=torch.float32) * size.repeat_interleave(200, 1)[:, :Sk]).to(dt)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["q_len"] = s["kv_len"] = s["mask"] = None
        if case["ragged"]:
            s["kv_len"] = torch.tensor(_lengths(B, Sk, gen), dtype=torch.int32, device=DEV)
            s["mask"] = torch.rand(B, Sk, generator=dgen, device=DEV) > 0.05
        if kind == "q8":
            Sq, Hq = case["Sq"], case["Hq"]
            s["q"] = normal(B, Sq, Hq, D)
            if case["ragged"] and Sq > 1:
                s["q_len"] = torch.tensor(_lengths(B, Sq, gen), dtype=torch.int32, device=DEV)
            s["k8"], s["v8"], s["ks"], s["vs"] = _plain_quant(s)
            del s["k"], s["v"]
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2210_10108_amd import layers
    kind = s["kind"]
    if kind == "layer":
        return layers.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
    if kind == "layer_train":
        y = layers.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
        grads = layers.layer_norm_backward(s["dy"], s["x"], s["w"], eps=EPS, bias=s["b"] is not None,
                                           residual_grad=s["dres"])
        return [y] + [t for t in grads if t is not None]
    if kind.startswith("axes"):
        rest = (s["q"], s["k"], s["table"], s["pos_q"], s["pos_k"], s["pair_axis"])
        kw = dict(q_weight=s["wq"], k_weight=s["wk"], eps=EPS if s["norm"] else None,
                  interleaved=s["interleaved"])
        out = layers.rotate_axes(*rest, **kw)
        if kind == "axes_train":
            out += layers.rotate_axes_backward(s["dq"], s["dk"], *rest, **kw)
        return [t for t in out if t is not None]
    if kind == "clip":
        norm = layers.clip_gradients(s["grads"], s["max_norm"], out=s["outs"])
        return [norm, s["flat_out"]]
    if kind == "quant":
        return list(layers.quantize_states(s["k"], s["v"], kv_len=s["kv_len"], kv_mask=s["mask"]))
    return layers.cross_attention_q8(s["q"], s["k8"], s["v8"], s["ks"], s["vs"], q_len=s["q_len"],
                                     kv_len=s["kv_len"], kv_mask=s["mask"])


def _plain_layer(s):
    dt = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    d = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    n = d * r
    y = n * w
    if s["b"] is not None:
        y = y + s["b"].float()
    if "dy" not in s:
        return y.to(dt)
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    if s["dres"] is not None:
        dx = dx + s["dres"].float()
    out = [y.to(dt), dx.to(dt), (dy * n).sum(0).to(dt)]
    return out + ([] if s["b"] is None else [dy.sum(0).to(dt)])


def _turn(x, c, s, interleaved):
    """Pairs of the first components of x turned by the angles of cosines c, sines s."""
    half = c.shape[-1]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * c - b * s, a * s + b * c
    return y


def _plain_axes(s):
    out, grads, wgrads = [], [], []
    table, inter = s["table"], s["interleaved"]
    pairs = torch.arange(table.shape[2], device=table.device)
    axis = torch.tensor(list(s["pair_axis"]), device=table.device)

    def side(x, w, pos, dy):
        at = pos.long()[:, axis]
        c, sn = table[at, 0, pairs][:, None], table[at, 1, pairs][:, None]
        xf = x.float()
        r = torch.rsqrt((xf * xf).mean(2, keepdim=True) + EPS) if s["norm"] else torch.ones_like(xf[..., :1])
        wf = torch.ones_like(xf[0, 0]) if w is None else w.float()
        out.append(_turn(xf * r * wf, c, sn, inter).to(x.dtype))
        if dy is None:
            return
        g = _turn(dy.float(), c, -sn, inter)
        if not s["norm"]:
            grads.append(g.to(x.dtype))
            return
        wgrads.append((g * xf * r).sum((0, 1)).to(x.dtype))
        gw = g * wf
        grads.append((r * (gw - xf * r * r * (gw * xf).mean(2, keepdim=True))).to(x.dtype))
    side(s["q"], s["wq"], s["pos_q"], s.get("dq"))
    if s["k"] is not None:
        side(s["k"], s["wk"], s["pos_k"], s.get("dk"))
    return out + grads + wgrads


def _plain_clip(s):
    total = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / (total + 1e-6)).clamp(max=1.0).float()
    [o.copy_(g.float() * c) for g, o in zip(s["grads"], s["outs"])]
    return [total.float(), s["flat_out"]]


def _allowed(s, B, Sk):
    dev = DEV
    on = torch.ones(B, Sk, dtype=torch.bool, device=dev)
    if s["kv_len"] is not None:
        on = torch.arange(Sk, device=dev) < s["kv_len"][:, None]
    return on if s["mask"] is None else on & s["mask"]


def _plain_quant(s):
    """e4m3 values and float32 scales: the least power of two with which a block's
    largest value is at most 448."""
    B, Sk, Hkv, D = s["k"].shape
    on = _allowed(s, B, Sk)[:, :, None, None]
    blocks = -(-Sk // BLOCK)

    def one(x):
        x = torch.where(on, x.float(), torch.zeros((), device=x.device))
        pad = torch.zeros(B, blocks * BLOCK - Sk, Hkv, D, device=x.device)
        x = torch.cat([x, pad], 1).view(B, blocks, BLOCK, Hkv, D)
        most = x.abs().amax((2, 4))
        m, e = torch.frexp(most / 448.0)  # m in [1/2, 1)
        scale = ((torch.where(m == 0.5, e - 1, e) + 127) << 23).view(torch.float32)  # by its bits: exact
        scale = torch.where(most == 0, torch.ones_like(scale), scale)
        x = (x / scale[:, :, None, :, None]).to(torch.float8_e4m3fn)
        return x.view(B, blocks * BLOCK, Hkv, D)[:, :Sk].contiguous(), scale
    (k8, ks), (v8, vs) = one(s["k"]), one(s["v"])
    return [k8, v8, ks, vs]


def _rows(x, Hkv):
    """[B, S, H, D] as 32-bit [B, Hkv, (H / Hkv) S, D]: the rows that share a kv head."""
    B, S, H, D = x.shape
    return x.float().reshape(B, S, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)


def _plain_q8(s):
    q, k8, v8 = s["q"], s["k8"], s["v8"]
    (B, Sq, Hq, D), (Sk, Hkv) = q.shape, k8.shape[1:3]
    valid = _allowed(s, B, Sk)
    row = torch.ones(B, Sq, dtype=torch.bool, device=q.device)
    if s["q_len"] is not None:
        row = torch.arange(Sq, device=q.device) < s["q_len"][:, None]
    row = row[:, None, None, :, None].expand(B, 1, Hq // Hkv, Sq, 1).reshape(B, 1, -1, 1)
    zero = q.new_zeros((), dtype=torch.float32)

    def states(x8, scale):
        x = x8.float() * scale.repeat_interleave(BLOCK, 1)[:, :Sk, :, None]
        return torch.where(valid[:, None, :, None], x.permute(0, 2, 1, 3), zero).contiguous()
    kr, vr = states(k8, s["ks"]), states(v8, s["vs"])
    a = torch.matmul(_rows(q, Hkv), kr.transpose(2, 3).contiguous()).mul_(D ** -0.5)
    a.masked_fill_(~(valid[:, None, None, :] & row), -math.inf)
    m = a.amax(3, keepdim=True)
    p = a.sub_(torch.where(m == -math.inf, zero, m)).exp_()
    total = p.sum(3, keepdim=True)
    p.div_(torch.where(total == 0, zero + 1, total))
    o = torch.matmul(p, vr)
    return o.reshape(B, Hkv, Hq // Hkv, Sq, D).permute(0, 3, 1, 2, 4).reshape(B, Sq, Hq, D).to(q.dtype)


def _run_plain(s):
    kind = s["kind"]
    if kind.startswith("layer"):
        return _plain_layer(s)
    if kind.startswith("axes"):
        return _plain_axes(s)
    return {"clip": _plain_clip, "quant": _plain_quant, "q8": _plain_q8}[kind](s)


# ---------------------------------------------------------------- what a pass needs
def work(case):
    e, kind = BYTES[case["dtype"]], case["kind"]
    if kind.startswith("layer"):
        n, W = case["rows"] * case["W"], case["W"]
        if kind == "layer":  # x in, y out
            return {"bytes": e * (2 * n + W * (1 + case["bias"])), "flops": 8 * n}
        # x, dy (and the residual's gradient) in; y, dx out
        return {"bytes": e * (n * (4 + case["residual"]) + W * (2 + 2 * case["bias"])), "flops": 24 * n}
    if kind.startswith("axes"):
        train = kind == "axes_train"
        n = (case["Tq"] * case["Hq"] + case["Tk"] * case["Hkv"]) * case["D"]
        angles = 4 * case["R"] * min(POSITIONS, max(case["Tq"], case["Tk"]))
        places = 4 * case["axes"] * (case["Tq"] + case["Tk"])
        # x (and dy; x again only where it is normed) read; y (and dx) written
        return {"bytes": (4 if train else 2) * e * n + angles + places, "flops": (20 if train else 8) * n}
    if kind == "clip":
        n = sum(_sizes(case))
        return {"bytes": n * (e + BYTES[case["out"]]), "flops": 3 * n}
    B, Sk, Hkv, D = (case[k] for k in ("B", "Sk", "Hkv", "D"))
    fk, fq = _valid_share(case)
    scales = 8 * B * -(-Sk // BLOCK) * Hkv
    if kind == "quant":  # 16-bit keys and values in, 8-bit ones out
        return {"bytes": 2 * B * Sk * Hkv * D * (fk * e + 1) + scales, "flops": 4 * B * Sk * Hkv * D}
    Sq, Hq = case["Sq"], case["Hq"]
    rows = B * Sq * Hq * D
    return {"bytes": e * rows * (fq + 1) + 2 * fk * B * Sk * Hkv * D + fk * scales,
            "flops": 4 * fk * fq * B * Hq * Sq * Sk * D}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The definitions in 64 bits, entry by entry, over the allowed keys alone."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("layer"):
        return _exact_layer(s)
    if kind.startswith("axes"):
        return _exact_axes(s)
    return {"clip": _exact_clip, "quant": _exact_quant, "q8": _exact_q8}[kind](s)


def _exact_layer(s):
    """The gradients by differentiating sum(dy . y + dres . x), a stretch of rows at a time."""
    ys, dxs = [], []
    dw = db = 0.0
    step = max(1, (1 << 25) // s["W"])
    for i in range(0, s["rows"], step):
        x = s["x"][i:i + step].double().requires_grad_()
        w = s["w"].double().requires_grad_()
        b = (torch.zeros_like(w) if s["b"] is None else s["b"].double()).detach().requires_grad_()
        with torch.enable_grad():
            mean = x.sum(1, keepdim=True) / x.shape[1]
            var = (x - mean).square().sum(1, keepdim=True) / x.shape[1]
            y = (x - mean) / torch.sqrt(var + EPS) * w + b
            if "dy" in s:
                value = (y * s["dy"][i:i + step].double()).sum()
                if s["dres"] is not None:
                    value = value + (x * s["dres"][i:i + step].double()).sum()
                gx, gw, gb = torch.autograd.grad(value, (x, w, b))
                dxs.append(gx)
                dw, db = dw + gw, db + gb
        ys.append(y.detach())
    y = torch.cat(ys)
    if "dy" not in s:
        return y
    return [y, torch.cat(dxs), dw] + ([] if s["b"] is None else [db])


def _exact_axes(s):
    """The rotation as a product of complex numbers, pair by pair at its axis's
    position; the gradients by differentiating sum(dy . y)."""
    out, grads, wgrads = [], [], []
    half = s["table"].shape[2]
    for x, w, pos, dy in ((s["q"], s["wq"], s["pos_q"], s.get("dq")),
                          (s["k"], s["wk"], s["pos_k"], s.get("dk"))):
        if x is None:
            continue
        T = s["table"].double()
        turn = torch.stack([torch.complex(T[pos[:, a].long(), 0, j], T[pos[:, a].long(), 1, j])
                            for j, a in enumerate(s["pair_axis"])], 1)[:, None]
        with torch.enable_grad():
            X = x.double().requires_grad_()
            W = torch.ones(x.shape[2], dtype=torch.float64, device=x.device) if w is None else w.double()
            W = W.detach().requires_grad_()
            n = X
            if s["norm"]:
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
                value = (dy.double() * y).sum()
                if s["norm"]:
                    gx, gw = torch.autograd.grad(value, (X, W))
                    wgrads.append(gw)
                else:
                    gx, = torch.autograd.grad(value, (X,))
                grads.append(gx)
    return out + grads + wgrads


def _exact_clip(s):
    norms = torch.stack([torch.linalg.vector_norm(g.double()) for g in s["grads"]])
    total = torch.linalg.vector_norm(norms)
    c = min(1.0, s["max_norm"] / (float(total) + 1e-6))
    flat = torch.zeros_like(s["flat_out"], dtype=torch.float64)
    base = s["flat_out"].data_ptr()
    for g, o in zip(s["grads"], s["outs"]):
        at = (o.data_ptr() - base) // o.element_size()
        flat[at:at + len(g)] = g.double() * c
    return [total, flat]


def _power_of_two(e):
    """2^e in 64 bits, by its bits (exp2 and ldexp round on some devices)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quant(s):
    """Scales by powers of two until the largest value fits; values to the nearest
    of e4m3's numbers (steps of 2^-9 below 2^-6, of an eighth of the power of two
    above), ties to the even one."""
    B, Sk, Hkv, D = s["k"].shape
    on = _allowed(s, B, Sk)
    values, scales = [], []
    for x in (s["k"], s["v"]):
        x8 = torch.zeros(B, Sk, Hkv, D, dtype=torch.float64, device=x.device)
        blocks = []
        for t in range(0, Sk, BLOCK):
            part = x[:, t:t + BLOCK].double() * on[:, t:t + BLOCK, None, None]
            most = part.abs().amax((1, 3))
            # most = m 2^e with m in [1/2, 1), and 448 = 7/8 2^9
            m, e = torch.frexp(most)
            power = torch.where(most > 0, torch.where(m <= 0.875, e - 9, e - 8), 0)
            blocks.append(_power_of_two(power))
            part = part / blocks[-1][:, None, :, None]
            step = _power_of_two(torch.frexp(part.abs().clamp_min(2.0 ** -6))[1] - 4)
            x8[:, t:t + BLOCK] = torch.round(part / step) * step
        values.append(x8)
        scales.append(torch.stack(blocks, 1))
    return [*values, *scales]


def _exact_q8(s):
    q = s["q"]
    (B, Sq, Hq, D), (Sk, Hkv) = q.shape, s["k8"].shape[1:3]
    on = _allowed(s, B, Sk)
    o = torch.zeros(B, Sq, Hq, D, dtype=torch.float64, device=q.device)
    for b in range(B):
        nq = Sq if s["q_len"] is None else int(s["q_len"][b])
        keys = torch.nonzero(on[b])[:, 0]
        if nq == 0 or len(keys) == 0:
            continue
        for g in range(Hkv):
            K = s["k8"][b, :, g].float().double()[keys] * s["ks"][b, keys // BLOCK, g, None].double()
            V = s["v8"][b, :, g].float().double()[keys] * s["vs"][b, keys // BLOCK, g, None].double()
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                P = torch.softmax((q[b, :nq, h].double() @ K.t()) / math.sqrt(D), dim=1)
                o[b, :nq, h] = P @ V
    return o
