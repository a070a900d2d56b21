"""The layer operators against their definitions in 64 bits, within the bounds
of layers_common, at the sizes, masks, strides and alignments where they can
go wrong."""
import math
import sys

import pytest
import torch

from . import layers_common as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


def say(*a):
    sys.stderr.write("[gpu] " + " ".join(str(x) for x in a) + "\n")
    sys.stderr.flush()


def normal(gen, *shape, dt="f16", std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(R.DT[dt])


def gen_of(seed):
    return torch.Generator("cuda").manual_seed(seed)


def check_attention(L, q, k, v, do, what, **masks):
    say("attention", what, tuple(q.shape), tuple(k.shape), q.dtype)
    ref = R.attention_ref(q, k, v, do=do, **masks)
    o, lse = L.cross_attention(q, k, v, return_lse=True, **masks)
    R.check(o, *ref["o"], what + " o")
    empty = torch.isinf(ref["lse"][0])
    assert torch.equal(empty, torch.isinf(lse) & (lse < 0)), what + " empty rows"
    assert bool((o.transpose(1, 2)[empty] == 0).all())
    R.check(lse[~empty], ref["lse"][0][~empty], ref["lse"][1][~empty], what + " lse")
    grads = L.cross_attention_backward(do, q, k, v, o, lse, **masks)
    for n, g in zip(("dq", "dk", "dv"), grads):
        R.check(g, *ref[n], f"{what} {n}")
    return o, lse, grads


# ---------------------------------------------------------------- attention
SHAPES = [  # B, Sq, Sk, Hq, Hkv, D
    (1, 1, 1, 1, 1, 64), (1, 1, 300, 8, 8, 64), (2, 1, 65, 8, 2, 128), (3, 2, 63, 4, 4, 32),
    (1, 7, 64, 4, 1, 96), (2, 33, 129, 6, 2, 80), (1, 128, 1, 2, 2, 128), (2, 130, 77, 4, 2, 64),
    (1, 5, 1000, 8, 1, 128), (1, 300, 513, 3, 3, 128), (4, 1, 700, 32, 8, 128), (1, 64, 2000, 2, 1, 64)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(L, shape, dt):
    B, Sq, Sk, Hq, Hkv, D = shape
    g = gen_of(1)
    q, do = normal(g, B, Sq, Hq, D, dt=dt), normal(g, B, Sq, Hq, D, dt=dt)
    k, v = normal(g, B, Sk, Hkv, D, dt=dt), normal(g, B, Sk, Hkv, D, dt=dt)
    check_attention(L, q, k, v, do, "plain")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(9, 300, 333, 16, 8, 128), (17, 257, 200, 16, 16, 64), (2, 3000, 130, 8, 8, 64),
                                   (1, 2000, 515, 16, 1, 128)], ids=str)
def test_attention_filling_the_chip(L, shape, dt):
    # more workgroups than compute units, and masks on top
    B, Sq, Sk, Hq, Hkv, D = shape
    g = gen_of(21)
    q, do = normal(g, B, Sq, Hq, D, dt=dt), normal(g, B, Sq, Hq, D, dt=dt)
    k, v = normal(g, B, Sk, Hkv, D, dt=dt), normal(g, B, Sk, Hkv, D, dt=dt)
    check_attention(L, q, k, v, do, "many")
    kv_len = torch.randint(0, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    q_len = torch.randint(0, Sq + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.rand(B, Sk, generator=g, device="cuda") > 0.3
    check_attention(L, q, k, v, do, "many, masked", q_len=q_len, kv_len=kv_len, kv_mask=mask)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [1, 7, 33, 100, 127])
def test_attention_odd_head_widths(L, D, dt):
    g = gen_of(2)
    q, do = normal(g, 2, 37, 4, D, dt=dt), normal(g, 2, 37, 4, D, dt=dt)
    k, v = normal(g, 2, 91, 2, D, dt=dt), normal(g, 2, 91, 2, D, dt=dt)
    check_attention(L, q, k, v, do, f"D={D}")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 45])
@pytest.mark.parametrize("D", [64, 100])
def test_attention_masks_and_what_lies_behind_them(L, dt, Sq, D):
    # lengths of 0, 1, a tile's end, all; lengths beyond the tensors and below 0
    # (clamped); a mask with holes, one that leaves nothing, one that leaves the
    # last key; NaN and infinities wherever nothing may be read
    B, Sk, Hq, Hkv = 8, 200, 4, 2
    g = gen_of(3)
    q, do = normal(g, B, Sq, Hq, D, dt=dt), normal(g, B, Sq, Hq, D, dt=dt)
    k, v = normal(g, B, Sk, Hkv, D, dt=dt), normal(g, B, Sk, Hkv, D, dt=dt)
    kv_len = torch.tensor([0, 1, 64, 200, 999, -5, 130, 130], dtype=torch.int32, device="cuda")
    q_len = torch.tensor([Sq, Sq, 0, Sq, max(Sq - 3, 1), Sq, 1, 99], dtype=torch.int32, device="cuda")
    mask = torch.rand(B, Sk, generator=g, device="cuda") > 0.4
    mask[1] = True
    mask[3] = False
    mask[7] = False
    mask[7, 129] = True
    seen = mask & (torch.arange(Sk, device="cuda") < kv_len[:, None])
    for junk in (float("nan"), float("inf"), float("-inf"), torch.finfo(R.DT[dt]).min):
        k2, v2 = k.clone(), v.clone()
        k2[~seen] = junk
        v2[~seen] = junk
        q2, do2 = q.clone(), do.clone()
        unread = torch.arange(Sq, device="cuda") >= q_len[:, None]
        q2[unread] = junk
        do2[unread] = junk
        for form in (mask, mask.to(torch.uint8) * 255):
            o, lse, grads = check_attention(L, q2, k2, v2, do2, f"masks junk={junk}", q_len=q_len,
                                            kv_len=kv_len, kv_mask=form)
        dq, dk, dv = grads
        assert bool((dk[~seen] == 0).all()) and bool((dv[~seen] == 0).all())
        assert bool((dq[unread] == 0).all())
    # a row without a key: whatever its gradient holds, nothing comes of it
    do3 = do2.clone()
    do3[[0, 3, 5]] = float("nan")
    grads = L.cross_attention_backward(do3, q2, k2, v2, o, lse, q_len=q_len, kv_len=kv_len, kv_mask=mask)
    for a, b in zip(grads, (dq, dk, dv)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_attention_zero_lengths(L, dt):
    g = gen_of(4)
    for B, Sq, Sk in ((2, 5, 0), (2, 0, 5), (0, 5, 5), (1, 0, 0)):
        q, do = normal(g, B, Sq, 4, 64, dt=dt), normal(g, B, Sq, 4, 64, dt=dt)
        k, v = normal(g, B, Sk, 2, 64, dt=dt), normal(g, B, Sk, 2, 64, dt=dt)
        o, lse = L.cross_attention(q, k, v, return_lse=True)
        grads = L.cross_attention_backward(do, q, k, v, o, lse)
        assert o.shape == q.shape and bool((o == 0).all()) and bool((lse == -math.inf).all())
        assert all(bool((t == 0).all()) for t in grads)


def _placed(t, kind):
    """The values of t [B, S, H, D] under another layout."""
    B, S, H, D = t.shape
    if kind == "heads first":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if kind == "batch inside":
        return t.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3)
    if kind == "part of a wider row":
        w = torch.full((B, S, 3, H, D + 8), float("nan"), dtype=t.dtype, device=t.device)
        w[:, :, 1, :, :D] = t
        return w[:, :, 1, :, :D]
    w = torch.full((B * S * H * (D + 3) + 1,), float("nan"), dtype=t.dtype, device=t.device)
    w = w[1:].view(B, S, H, D + 3)  # rows on odd addresses
    w[..., :D] = t
    return w[..., :D]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 70])
@pytest.mark.parametrize("kind", ["heads first", "batch inside", "part of a wider row", "unaligned"])
def test_attention_layouts(L, kind, Sq, dt):
    g = gen_of(5)
    q, do = normal(g, 3, Sq, 4, 64, dt=dt), normal(g, 3, Sq, 4, 64, dt=dt)
    k, v = normal(g, 3, 150, 2, 64, dt=dt), normal(g, 3, 150, 2, 64, dt=dt)
    want_o, want_lse, want = check_attention(L, q, k, v, do, "contiguous")
    ref = R.attention_ref(q, k, v, do=do)
    ins = [_placed(t, kind) for t in (q, k, v, do)]
    out = _placed(torch.zeros_like(q), kind)
    o, lse = L.cross_attention(*ins[:3], o=out, return_lse=True)
    assert o is out
    outs = [_placed(torch.zeros_like(t), kind) for t in (q, k, v)]
    got = L.cross_attention_backward(ins[3], *ins[:3], o, lse, dq=outs[0], dk=outs[1], dv=outs[2])
    if kind == "unaligned":  # other kernels
        for n, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *got)):
            R.check(t, *ref[n], n)
    else:  # the same kernels, bit for bit
        for a, b in zip((o, lse, *got), (want_o, want_lse, *want)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_attention_stride_of_a_single_row(L, dt):
    # whatever the stride of a dimension of one row says, no other row is there
    g = gen_of(22)
    for Sq, Sk in ((1, 200), (40, 1), (1, 1)):
        q, do, k, v = (normal(g, 3, n, h, 64, dt=dt) for n, h in ((Sq, 4), (Sq, 4), (Sk, 2), (Sk, 2)))
        for step in (0, 3, 1 << 33):
            ins = [t.as_strided(t.shape, (t.stride(0), step if t.shape[1] == 1 else t.stride(1), 64, 1))
                   for t in (q, k, v, do)]
            check_attention(L, *ins, f"stride {step}")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_linear_stride_of_a_single_row(L, dt):
    g = gen_of(23)
    for M, K, N in ((1, 64, 128), (40, 1, 64), (1, 2048, 1024), (1, 1, 8)):
        x, w, res, dy = (normal(g, *s, dt=dt) for s in ((M, K), (K, N), (M, N), (M, N)))
        for step in (0, 3, 1 << 33):
            one = [t.as_strided(t.shape, (step if t.shape[0] == 1 else t.stride(0), 1)) for t in (x, w, res, dy)]
            check_linear(L, one[0], one[1], None, one[2], "gelu", one[3], f"stride {step}")


def test_attention_broadcast_states(L):
    # one image's states for every batch entry: each entry's gradient is its own
    g = gen_of(6)
    q, do = normal(g, 5, 9, 4, 64), normal(g, 5, 9, 4, 64)
    k, v = normal(g, 1, 120, 2, 64).expand(5, -1, -1, -1), normal(g, 1, 120, 2, 64).expand(5, -1, -1, -1)
    check_attention(L, q, k, v, do, "broadcast")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_attention_scores_of_every_size(L, dt):
    # large scores (one key takes everything), equal scores, tiny ones, and a
    # maximum that keeps rising over the tiles
    g = gen_of(7)
    B, Sq, Sk, H, D = 1, 40, 400, 2, 64
    q, do = normal(g, B, Sq, H, D, dt=dt), normal(g, B, Sq, H, D, dt=dt)
    v = normal(g, B, Sk, H, D, dt=dt)
    rise = torch.linspace(0, 8, Sk, device="cuda")[None, :, None, None]
    for name, k, scale in (("large", normal(g, B, Sk, H, D, dt=dt, std=30.0), 1.0),
                           ("equal", torch.ones(B, Sk, H, D, dtype=R.DT[dt], device="cuda"), 1.0),
                           ("tiny", normal(g, B, Sk, H, D, dt=dt, std=1e-3), 1e-3),
                           ("rising", (q.float().mean(1, keepdim=True) * rise * 4).to(R.DT[dt]), 1.0)):
        check_attention(L, q, k, v, do, name, scale=scale)


def test_attention_offsets_beyond_32_bits(L):
    # rows 2^31 bytes and more apart: the last key lies past 2^32 bytes
    g = gen_of(8)
    Sk, step = 3, (1 << 30) + 64
    big = torch.zeros((Sk - 1) * step + 128, dtype=torch.float16, device="cuda")
    k = big.as_strided((1, Sk, 1, 64), (big.numel(), step, 64, 1))
    v = big[64:].as_strided((1, Sk, 1, 64), (big.numel(), step, 64, 1))
    k.copy_(normal(g, 1, Sk, 1, 64))
    v.copy_(normal(g, 1, Sk, 1, 64))
    for Sq in (1, 40):
        q, do = normal(g, 1, Sq, 1, 64), normal(g, 1, Sq, 1, 64)
        check_attention(L, q, k, v, do, "far rows")
    del k, v, big
    torch.cuda.empty_cache()


def test_attention_long_states_for_one_token(L):
    g = gen_of(9)
    q, do = normal(g, 1, 1, 8, 128), normal(g, 1, 1, 8, 128)
    k, v = normal(g, 1, 40003, 2, 128), normal(g, 1, 40003, 2, 128)
    check_attention(L, q, k, v, do, "long")


def test_attention_gradient_against_differences(L):
    g = gen_of(10)
    q, do = normal(g, 1, 6, 4, 32), normal(g, 1, 6, 4, 32)
    k, v = normal(g, 1, 11, 2, 32), normal(g, 1, 11, 2, 32)
    o, lse = L.cross_attention(q, k, v, return_lse=True)
    grads = L.cross_attention_backward(do, q, k, v, o, lse)
    ref = R.attention_ref(q, k, v, do=do)
    args = [t.double() for t in (q, k, v)]
    for i, (n, gr) in enumerate(zip(("dq", "dk", "dv"), grads)):
        for seed in range(4):
            way = torch.randn(args[i].shape, generator=gen_of(20 + seed), device="cuda", dtype=torch.float64)
            h = 1e-5
            hi, lo = ([a + (s * h * way if j == i else 0) for j, a in enumerate(args)] for s in (1, -1))
            diff = (R.attention_value(*hi, do.double(), 32 ** -0.5) -
                    R.attention_value(*lo, do.double(), 32 ** -0.5)) / (2 * h)
            bound = float((ref[n][1] * way.abs()).sum()) + 1e-6 * float((ref[n][0] * way).abs().sum())
            assert abs(float((gr.double() * way).sum() - diff)) <= bound, n


# ---------------------------------------------------------------- norm and rotation
def _table(n_pos, R_, seed=0):
    a = torch.rand(n_pos, R_ // 2, generator=gen_of(seed), device="cuda", dtype=torch.float64) * 6.3
    return torch.stack([a.cos(), a.sin()], 1).float()


def check_norm(L, q, k, wq, wk, table, pq, pk, eps, inter, dq, dk, what):
    say("norm", what, tuple(q.shape), q.dtype)
    out = L.norm_rotate(q, k, wq, wk, table, pq, pk, eps=eps, interleaved=inter)
    grads = L.norm_rotate_backward(dq, dk, q, k, wq, wk, table, pq, pk, eps=eps, interleaved=inter)
    for i, (x, w, pos, dy, n) in enumerate(((q, wq, pq, dq, "q"), (k, wk, pk, dk, "k"))):
        if x is None:
            assert out[i] is None and grads[i] is None and grads[2 + i] is None
            continue
        ref = R.norm_ref(x, w, table, pos, eps, inter, dy)
        R.check(out[i], *ref["y"], f"{what} {n}")
        R.check(grads[i], *ref["dx"], f"{what} d{n}")
        if w is None:
            assert grads[2 + i] is None
        else:
            R.check(grads[2 + i], *ref["dw"], f"{what} d{n}_weight")
    return out, grads


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("case", [(1, 0, 1, 1, 64, 64), (64, 0, 16, 4, 128, 128), (3, 5, 2, 1, 32, 16),
                                  (37, 21, 6, 3, 80, 80), (11, 13, 3, 3, 80, 32), (5, 9, 4, 2, 256, 128),
                                  (129, 300, 8, 2, 128, 64), (6, 2, 3, 1, 96, 0), (7, 3, 5, 2, 33, 10),
                                  (4, 4, 2, 2, 1, 0), (9, 2, 2, 1, 100, 100), (2, 2, 1, 1, 250, 6)], ids=str)
def test_norm_rotate(L, case, inter, dt):
    Tq, Tk, Hq, Hk, D, Rd = case
    g = gen_of(11)
    q, dq = normal(g, Tq, Hq, D, dt=dt), normal(g, Tq, Hq, D, dt=dt)
    k, dk = (normal(g, Tk, Hk, D, dt=dt), normal(g, Tk, Hk, D, dt=dt)) if Tk else (None, None)
    wq, wk = normal(g, D, dt=dt), normal(g, D, dt=dt) if Tk else None
    table = _table(50, Rd) if Rd else None
    pq, pk = (torch.randint(0, 50, (n,), generator=g, device="cuda", dtype=torch.int32) if Rd and n else None
              for n in (Tq, Tk))
    check_norm(L, q, k, wq, wk, table, pq, pk, 1e-5, inter, dq, dk, str(case))
    check_norm(L, q, k, None, None, table, pq, pk, 1e-5, inter, dq, dk, f"{case} no weights")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_norm_rotate_strides_and_in_place(L, dt):
    # heads inside a packed projection, rows on odd addresses, outputs in place
    g = gen_of(12)
    T, H, D = 19, 4, 64
    packed = normal(g, T, 3, H, D, dt=dt)
    q, k = packed[:, 0], packed[:, 1]
    w = normal(g, D, dt=dt)
    table, pos = _table(30, 64), torch.randint(0, 30, (T,), generator=g, device="cuda", dtype=torch.int32)
    dq, dk = normal(g, T, H, D, dt=dt), normal(g, T, H, D, dt=dt)
    (wantq, wantk), wantg = check_norm(L, q, k, w, w, table, pos, pos, 1e-6, False, dq, dk, "packed")
    odd = torch.empty(T * H * (D + 1) + 1, dtype=q.dtype, device="cuda")[1:].view(T, H, D + 1)[..., :D]
    odd.copy_(q)
    check_norm(L, odd, k, w, w, table, pos, pos, 1e-6, False, dq, dk, "odd rows")
    ref_odd = R.norm_ref(odd, w, table, pos, 1e-6, False)
    L.norm_rotate(q, k, w, w, table, pos, pos, eps=1e-6, q_out=q, k_out=k)
    assert torch.equal(q, wantq) and torch.equal(k, wantk)
    assert bool(torch.isfinite(packed[:, 2].float()).all())
    L.norm_rotate(odd, None, w, None, table, pos, None, eps=1e-6, q_out=odd)
    R.check(odd, *ref_odd["y"], "odd rows in place")
    x = normal(g, T, H, D, dt=dt)
    want = L.norm_rotate_backward(dq, None, x, None, w, None, table, pos, None)
    got = L.norm_rotate_backward(dq, None, x, None, w, None, table, pos, None, dq=dq)
    assert got[0] is dq and torch.equal(dq, want[0]) and torch.equal(got[2], want[2])


def test_norm_rotate_rows_of_every_size(L):
    # zero rows, rows far from 1, a position that the table does not have, one row with NaN
    g = gen_of(13)
    q = normal(g, 6, 2, 64, dt="f32")
    q[0] = 0
    q[1] *= 1e-12
    q[2] *= 1e12
    dq = normal(g, 6, 2, 64, dt="f32")
    w = normal(g, 64, dt="f32")
    table, pos = _table(8, 32), torch.tensor([0, 1, 2, 3, 4, 5], dtype=torch.int32, device="cuda")
    check_norm(L, q, None, w, None, table, pos, None, 1e-6, False, dq, None, "sizes")
    good, _ = L.norm_rotate(q, None, w, None, table, pos, None)
    pos2 = pos.clone()
    pos2[3], pos2[4] = 8, -1
    q2 = q.clone()
    q2[5, 0, 7] = float("nan")
    y, _ = L.norm_rotate(q2, None, w, None, table, pos2, None)
    assert torch.equal(y[:3], good[:3]) and torch.equal(y[5, 1], good[5, 1])
    assert bool(y[3:5, :, :32].isnan().all()) and torch.equal(y[3:5, :, 32:], good[3:5, :, 32:])
    assert bool(y[5, 0].isnan().all())


def test_norm_rotate_gradient_against_differences(L):
    g = gen_of(14)
    q, w, dq = normal(g, 5, 3, 16, dt="f32"), normal(g, 16, dt="f32"), normal(g, 5, 3, 16, dt="f32")
    table, pos = _table(9, 16), torch.randint(0, 9, (5,), generator=g, device="cuda", dtype=torch.int32)
    for inter in (False, True):
        gx, _, gw, _ = L.norm_rotate_backward(dq, None, q, None, w, None, table, pos, None, interleaved=inter)
        ref = R.norm_ref(q, w, table, pos, 1e-6, inter, dq)

        def value(x, v):
            n = x / torch.sqrt((x * x).mean(2, keepdim=True) + 1e-6) * v
            c, s = (table[pos.long(), i].double()[:, None] for i in (0, 1))
            a = torch.arange(8, device="cuda") * (2 if inter else 1)
            b = a + (1 if inter else 8)
            y = torch.empty_like(n)
            y[..., a], y[..., b] = n[..., a] * c - n[..., b] * s, n[..., a] * s + n[..., b] * c
            return (dq.double() * y).sum()
        for n, at, grad in (("dx", 0, gx), ("dw", 1, gw)):
            base = [q.double(), w.double()]
            way = torch.randn(base[at].shape, generator=gen_of(30), device="cuda", dtype=torch.float64)
            hi, lo = ([t + (s * 1e-5 * way if j == at else 0) for j, t in enumerate(base)] for s in (1, -1))
            diff = (value(*hi) - value(*lo)) / 2e-5
            bound = float((ref[n][1] * way.abs()).sum()) + 1e-6 * float((ref[n][0] * way).abs().sum())
            assert abs(float((grad.double() * way).sum() - diff)) <= bound, (n, inter)


# ---------------------------------------------------------------- linear
def check_linear(L, x, w, b, res, act, dy, what):
    say("linear", what, tuple(x.shape), tuple(w.shape), act, x.dtype)
    ref = R.linear_ref(x, w, b, res, act, dy)
    y, z = L.linear(x, w, b, res, activation=act, return_preact=True)
    R.check(y, *ref["y"], what + " y")
    R.check(z, *ref["z"], what + " z")
    assert torch.equal(L.linear(x, w, b, res, activation=act), y)
    dx, dw, db = L.linear_backward(dy, x, w, z if act != "none" else None, activation=act, bias=b is not None)
    R.check(dx, *ref["dx"], what + " dx")
    R.check(dw, *ref["dw"], what + " dw")
    if b is not None:
        R.check(db, *ref["db"], what + " db")
    else:
        assert db is None


LINEAR = [(1, 64, 64), (4, 256, 512), (32, 128, 264), (33, 72, 40), (1, 1, 1), (3, 5, 7), (17, 40, 3),
          (65, 129, 63), (130, 64, 192), (200, 513, 1), (1, 1000, 9), (5, 8, 2000), (300, 264, 520),
          (513, 256, 256), (260, 1032, 136), (31, 2048, 1000), (2, 17, 300)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("case", LINEAR, ids=str)
def test_linear(L, case, dt):
    M, K, N = case
    g = gen_of(15)
    x, w = normal(g, M, K, dt=dt), normal(g, K, N, dt=dt, std=K ** -0.5)
    b, res, dy = normal(g, N, dt=dt), normal(g, M, N, dt=dt), normal(g, M, N, dt=dt)
    for act in ("none", "relu", "gelu", "silu"):
        check_linear(L, x, w, b, res, act, dy, str(case))
    check_linear(L, x, w, None, None, "none", dy, f"{case} product alone")
    check_linear(L, x, w, None, res, "silu", dy, f"{case} no bias")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("case", [(222, 5690, 101), (45, 7085, 4), (57, 26, 4382), (29, 835, 62), (2000, 9, 31),
                                  (66, 129, 127)], ids=str)
def test_linear_odd_and_deep(L, case, dt):
    # sizes that are not of whole chunks, one axis long: in one of the three products
    # few tiles share a long contracted axis, in parts of which the last may be empty
    M, K, N = case
    g = gen_of(25)
    x, w = normal(g, M, K, dt=dt), normal(g, K, N, dt=dt, std=K ** -0.5)
    b, res, dy = normal(g, N, dt=dt), normal(g, M, N, dt=dt), normal(g, M, N, dt=dt)
    check_linear(L, x, w, b, res, "silu", dy, str(case))
    check_linear(L, x, w, None, None, "none", dy, f"{case} product alone")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("case", [(3500, 136, 3600), (3584, 64, 3840), (3400, 3500, 72), (77, 3480, 3610),
                                  (3333, 129, 3601), (5, 2100, 1001), (20, 1023, 2050), (700, 1000, 301)], ids=str)
def test_linear_large(L, case, dt):
    # sizes at which the largest tiles run, in each of the three products, inside
    # and at ragged edges; and sizes whose operands are copied to whole chunks first
    M, K, N = case
    g = gen_of(19)
    x, w = normal(g, M, K, dt=dt), normal(g, K, N, dt=dt, std=K ** -0.5)
    b, res, dy = normal(g, N, dt=dt), normal(g, M, N, dt=dt), normal(g, M, N, dt=dt)
    check_linear(L, x, w, b, res, "gelu", dy, str(case))
    check_linear(L, x, w, None, None, "none", dy, f"{case} product alone")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("M", [3, 40, 300])
def test_linear_strides(L, M, dt):
    # rows of wider tensors, aligned and not; one residual row for all; y over its residual
    g = gen_of(16)
    K, N = 72, 136
    for pad, off in ((8, 8), (3, 1)):
        def wide(*shape, std=1.0):
            t = torch.full((shape[0], shape[1] + pad + off), float("nan"), dtype=R.DT[dt], device="cuda")
            t[:, off:off + shape[1]] = normal(g, *shape, dt=dt, std=std)
            return t[:, off:off + shape[1]]
        x, w, dy, res = wide(M, K), wide(K, N, std=0.1), wide(M, N), wide(M, N)
        b = normal(g, N + 1, dt=dt)[1:]
        check_linear(L, x, w, b.clone(), res, "gelu", dy, f"pad {pad}")
        check_linear(L, x, w, b, normal(g, 1, N, dt=dt).expand(M, N), "relu", dy, "one residual row")
        want = L.linear(x, w, b, res, activation="silu")
        got = L.linear(x, w, b, res, activation="silu", y=res)
        assert got is res and torch.equal(res, want)
        dx, dw = torch.zeros_like(x.contiguous()), wide(K, N)
        ref = R.linear_ref(x, w, None, None, "none", dy)
        L.linear_backward(dy, x, w, bias=False, dx=dx, dw=dw)
        R.check(dx, *ref["dx"], "dx")
        R.check(dw, *ref["dw"], "dw")


def test_linear_without_rows(L):
    w = normal(gen_of(17), 24, 40)
    x, dy = w.new_empty(0, 24), w.new_empty(0, 40)
    y, z = L.linear(x, w, activation="gelu", return_preact=True)
    assert y.shape == (0, 40)
    dx, dw, db = L.linear_backward(dy, x, w, z, activation="gelu")
    assert dx.shape == (0, 24) and bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_linear_activation_far_out(L, act):
    # arguments from -60000 to 60000, zeros, infinities and NaN through the epilogue alone
    v = torch.tensor([0.0, -0.0, 1e-4, -1e-4, 1, -1, 3, -3, 5.5, -5.5, 12, -12, 90, -90, 6e4, -6e4],
                     device="cuda").half()
    x, w = v[:, None].contiguous(), torch.ones(1, 8, dtype=torch.float16, device="cuda")
    dy = torch.ones(16, 8, dtype=torch.float16, device="cuda")
    check_linear(L, x, w, None, None, act, dy, "far out")
    x[0], x[1], x[2] = float("inf"), float("-inf"), float("nan")
    y = L.linear(x, w, activation=act)[:, 0]
    assert y[0] == math.inf and bool(y[2].isnan())
    assert bool(torch.isfinite(y[3:]).all())


def test_linear_gradient_against_differences(L):
    g = gen_of(18)
    x, w, b = normal(g, 9, 12), normal(g, 12, 10, std=0.4), normal(g, 10)
    dy = normal(g, 9, 10)
    for act in ("none", "gelu", "silu"):
        _, z = L.linear(x, w, b, activation=act, return_preact=True)
        grads = L.linear_backward(dy, x, w, z, activation=act)
        ref = R.linear_ref(x, w, b, None, act, dy)
        base = [t.double() for t in (x, w, b)]
        for i, n in enumerate(("dx", "dw", "db")):
            way = torch.randn(base[i].shape, generator=gen_of(40 + i), device="cuda", dtype=torch.float64)
            hi, lo = ([t + (s * 1e-5 * way if j == i else 0) for j, t in enumerate(base)] for s in (1, -1))
            diff = ((dy.double() * R.act(hi[0] @ hi[1] + hi[2], act)).sum() -
                    (dy.double() * R.act(lo[0] @ lo[1] + lo[2], act)).sum()) / 2e-5
            bound = float((ref[n][1] * way.abs()).sum()) + 1e-6 * float((ref[n][0] * way).abs().sum())
            assert abs(float((grads[i].double() * way).sum() - diff)) <= bound, (n, act)


# ---------------------------------------------------------------- every operator
def _calls(L, g):
    q, k, v, do = (normal(g, 2, n, h, 64) for n, h in ((50, 4), (700, 2), (700, 2), (50, 4)))
    q1 = q[:, :1]
    lens = torch.tensor([700, 333], dtype=torch.int32, device="cuda")
    h, w = normal(g, 40, 4, 64), normal(g, 64)
    table, pos = _table(64, 64), torch.arange(40, dtype=torch.int32, device="cuda")
    x, wt, b, res, dy = normal(g, 100, 128), normal(g, 128, 256, std=0.1), normal(g, 256), \
        normal(g, 100, 256), normal(g, 100, 256)

    def run(**kw):
        o, lse = L.cross_attention(q, k, v, kv_len=lens, return_lse=True, **kw)
        out = [o, lse, *L.cross_attention_backward(do, q, k, v, o, lse, kv_len=lens, **kw)]
        out.append(L.cross_attention(q1, k, v, kv_len=lens, **kw))
        out.append(L.norm_rotate(h, None, w, None, table, pos, None, **kw)[0])
        out += [t for t in L.norm_rotate_backward(h, None, h, None, w, None, table, pos, None, **kw)
                if t is not None]
        y, z = L.linear(x, wt, b, res, activation="gelu", return_preact=True, **kw)
        out += [y, z, *L.linear_backward(dy, x, wt, z, activation="gelu", **kw)]
        out.append(L.linear(x[:3], wt, b, activation="silu", **kw))
        return out
    return run, (q, k, v, do, h, x, wt, dy)


def test_the_same_bits_on_every_call(L):
    run, _ = _calls(L, gen_of(50))
    first = run()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


def test_on_another_stream(L):
    run, ins = _calls(L, gen_of(51))
    want = run()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    busy = torch.zeros(1 << 27, device="cuda")
    for _ in range(3):
        for _ in range(4):
            busy.add_(1.0)  # the current stream is behind; the other does not wait for it
        got = run(stream=other)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.cuda.stream(other):
        got = run()
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_into_a_graph(L):
    run, ins = _calls(L, gen_of(52))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in range(4):
        g = gen_of(60 + seed)
        for t in ins:
            t.copy_(normal(g, *t.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), seed


def test_binding_refusals(L):
    g = gen_of(70)
    q, k = normal(g, 2, 5, 4, 64), normal(g, 2, 9, 2, 64)
    bad = [
        (TypeError, lambda: L.cross_attention(q, k.bfloat16(), k)),
        (TypeError, lambda: L.cross_attention(q, k.cpu(), k)),
        (TypeError, lambda: L.cross_attention(q.double(), k, k)),
        (ValueError, lambda: L.cross_attention(q, k, k[:, :4])),
        (ValueError, lambda: L.cross_attention(q[0], k, k)),
        (ValueError, lambda: L.cross_attention(q.transpose(2, 3).contiguous().transpose(2, 3), k, k)),
        (ValueError, lambda: L.cross_attention(q, k, k, kv_len=torch.ones(3, dtype=torch.int32, device="cuda"))),
        (TypeError, lambda: L.cross_attention(q, k, k, kv_len=torch.ones(2, device="cuda"))),
        (TypeError, lambda: L.cross_attention(q, k, k, kv_mask=torch.ones(2, 9, device="cuda"))),
        (ValueError, lambda: L.cross_attention(q, k, k, kv_mask=torch.ones(2, 8, device="cuda", dtype=torch.bool))),
        (ValueError, lambda: L.cross_attention(q, k, k, o=q[:, :3])),
        (ValueError, lambda: L.linear(q[0, 0], k[0, 0], activation="tanh")),
        (ValueError, lambda: L.linear(q[0, 0], k[0, 0])),
        (ValueError, lambda: L.linear(q, k)),
        (ValueError, lambda: L.norm_rotate(q, None, None, None, None, None, None)),
        (ValueError, lambda: L.norm_rotate(q[0], k[0, :, :, :32], None, None, None, None, None)),
        (ValueError, lambda: L.norm_rotate(q[0], None, None, None, torch.ones(3, 32, device="cuda"), None, None)),
    ]
    for kind, fn in bad:
        with pytest.raises(kind):
            fn()
    from paper_2210_10108_amd import pnerf
    for fn in (lambda: L.cross_attention(q.float(), k.float(), k.float()), lambda: L.linear(q[0, 0].float(), q[0, 0].float().t().contiguous()),
               lambda: L.cross_attention(normal(g, 1, 2, 1, 129), normal(g, 1, 2, 1, 129), normal(g, 1, 2, 1, 129))):
        with pytest.raises(pnerf.PnerfError) as e:
            fn()
        assert e.value.status == pnerf.ERR_NOT_SUPPORTED
    for fn in (lambda: L.cross_attention(normal(g, 1, 2, 3, 64), normal(g, 1, 2, 2, 64), normal(g, 1, 2, 2, 64)),
               lambda: L.cross_attention(q, k, k, scale=-1.0), lambda: L.cross_attention(q, k, k, o=q[:1].expand(2, -1, -1, -1)),
               lambda: L.norm_rotate(q[0], None, None, None, torch.ones(3, 2, 16, device="cuda"), None, None)):
        with pytest.raises(pnerf.PnerfError) as e:
            fn()
        assert e.value.status == pnerf.ERR_INVALID_ARG


# ---------------------------------------------------------------- more heads than workgroups
@pytest.mark.parametrize("case", [(1025, 1025, 24, 8, 128), (1030, 1030, 28, 4, 128), (513, 513, 12, 4, 256),
                                  (4100, 4099, 6, 2, 64), (1, 20000, 1, 1, 64), (20000, 1, 1, 3, 32)], ids=str)
def test_norm_rotate_uneven_shares_of_the_workgroups(L, case):
    # the gradient's workgroups are divided between queries and keys: shares that do not come out even
    Tq, Tk, Hq, Hk, D = case
    g = gen_of(80)
    q, k, dq, dk = (normal(g, T, H, D, dt="bf16") for T, H in ((Tq, Hq), (Tk, Hk), (Tq, Hq), (Tk, Hk)))
    wq, wk = normal(g, D, dt="bf16"), normal(g, D, dt="bf16")
    table = _table(64, D)
    pq, pk = (torch.randint(0, 64, (n,), generator=g, device="cuda", dtype=torch.int32) for n in (Tq, Tk))
    check_norm(L, q, k, wq, wk, table, pq, pk, 1e-6, False, dq, dk, str(case))
    odd = torch.empty(Tq * Hq * D + 1, dtype=q.dtype, device="cuda")[1:].view(Tq, Hq, D)
    odd.copy_(q)
    check_norm(L, odd, k, wq, wk, table, pq, pk, 1e-6, False, dq, dk, f"{case}, odd addresses")


# ---------------------------------------------------------------- GELU's tail
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_gelu_tail_is_relatively_exact(L, dt):
    # far below zero GELU is small and the data type holds it as exactly as any number: the
    # bound is relative.  2^-19 for the form and its steps, and 2^-23 z^2 for the exponent,
    # three of whose roundings (2^-24 each) weigh z^2 / 2 there.
    z = -torch.linspace(0.01, 5.5 if dt == "f16" else 12.5, 4000, device="cuda").to(R.DT[dt]).unique()
    x, w = z[:, None].contiguous(), torch.ones(1, 8, dtype=z.dtype, device="cuda")
    y, kept = L.linear(x, w, activation="gelu", return_preact=True)
    assert torch.equal(kept[:, 0], z)
    Z = z.double()
    phi = 0.5 * torch.special.erfc(-Z * math.sqrt(0.5))
    density = torch.exp(-0.5 * Z * Z) / math.sqrt(2 * math.pi)
    e = 2.0 ** -19 + 2.0 ** -23 * Z * Z
    R.check(y[:, 0], Z * phi, (R.U[dt] + e) * (Z * phi).abs() + R.TINY[dt], "gelu")
    dy = torch.zeros_like(y)
    dy[:, 0] = 1.0
    dx, _, _ = L.linear_backward(dy, x, w, kept, activation="gelu", bias=False)
    slope = phi + Z * density
    # dz is rounded, and its product with 1 once more
    R.check(dx[:, 0], slope, 2 * R.U[dt] * slope.abs() + e * (phi + (Z * density).abs()) + 2 * R.TINY[dt], "gelu'")


# ---------------------------------------------------------------- one very long row
@pytest.mark.parametrize("K,N", [(8, 1 << 26), (1 << 26, 8)])
def test_linear_gradient_of_one_very_long_row(L, K, N):
    # the rows that a tile has beyond the only one are zeros, however long a row is: an
    # infinity meets no other row's zero
    say("linear, one long row", K, N)
    x, dy = torch.ones(1, K, dtype=torch.float16, device="cuda"), torch.ones(1, N, dtype=torch.float16, device="cuda")
    w = torch.ones(1, N, dtype=torch.float16, device="cuda").expand(K, N)
    long = x if K > N else dy
    long[0, 12345], long[0, -1] = math.inf, 3.0
    dw = torch.empty(K, N, dtype=torch.float16, device="cuda")
    dx = torch.empty(1, K, dtype=torch.float16, device="cuda")
    L.linear_backward(dy, x, w, bias=False, dw=dw, dx=dx)
    want = long[0]
    for row in (dw.t() if K > N else dw):
        assert torch.equal(row, want)
    del dw, dx
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- small rows without eps
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 33])
def test_norm_rotate_small_rows_without_eps(L, D, dt):
    # with eps = 0 a row's size does not matter; here its mean square is a subnormal
    # number of 32 bits, exact to 2^-23 still
    g = gen_of(90)
    q, dq, w = normal(g, 9, 3, D, dt="f32"), normal(g, 9, 3, D, dt=dt), normal(g, D, dt=dt)
    q = (q * 8e-20).to(R.DT[dt])
    check_norm(L, q, None, w, None, None, None, None, 0.0, False, dq, None, f"small rows {D}")
