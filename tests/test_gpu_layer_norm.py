"""Layer norm against its definition in 64 bits, at the widths, row counts, strides
and values where it can go wrong."""
import math
import sys

import pytest
import torch

from . import layers_common as R
from . import more_layers_common as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


def say(*a):
    sys.stderr.write("[gpu] " + " ".join(str(x) for x in a) + "\n")
    sys.stderr.flush()


def normal(gen, *shape, dt="f16", std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(R.DT[dt])


def gen_of(seed):
    return torch.Generator("cuda").manual_seed(seed)


def check(L, x, w, b, dy, dres, eps, what):
    say("layer norm", what, tuple(x.shape), x.dtype)
    ref = M.layer_norm_ref(x, w, b, eps, dy, dres)
    y = L.layer_norm(x, w, b, eps=eps)
    R.check(y, *ref["y"], what + " y")
    dx, dw, db = L.layer_norm_backward(dy, x, w, eps=eps, bias=b is not None, residual_grad=dres)
    R.check(dx, *ref["dx"], what + " dx")
    assert (dw is None) == (w is None) and (db is None) == (b is None)
    if w is not None:
        R.check(dw, *ref["dw"], what + " dw")
    if b is not None:
        R.check(db, *ref["db"], what + " db")
    return y, dx, dw, db


SHAPES = [(1, 1), (1, 8), (5, 7), (3, 64), (64, 256), (33, 72), (130, 136), (7, 512), (9, 520), (257, 768),
          (5, 1000), (3, 1001), (19, 1024), (6, 2040), (4, 2048), (31, 4096), (5, 4104), (3, 8192), (2, 8200),
          (3, 12288), (2, 16384), (2, 16392), (1, 20007), (2, 65536), (1300, 256), (4500, 64), (9000, 24),
          (2100, 1032), (70000, 8), (1, 1 << 20)]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_layer_norm(L, shape, dt):
    g = gen_of(1)
    x, dy, dres = (normal(g, *shape, dt=dt, mean=m) for m in (0.5, 0.0, 0.0))
    w, b = normal(g, shape[1], dt=dt, std=0.3, mean=1.0), normal(g, shape[1], dt=dt)
    check(L, x, w, b, dy, dres, 1e-5, str(shape))
    check(L, x, None, None, dy, None, 1e-5, f"{shape} bare")
    check(L, x, w, None, dy, None, 1e-6, f"{shape} no bias")
    check(L, x, None, b, dy, dres, 1e-6, f"{shape} no weight")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("W", [64, 72, 1024, 1025, 4096])
def test_layer_norm_strides_and_in_place(L, W, dt):
    g = gen_of(2)
    rows = 37
    w, b = normal(g, W, dt=dt), normal(g, W, dt=dt)

    def wide(pad, off):
        t = torch.full((rows * (W + pad) + off,), float("nan"), dtype=R.DT[dt], device="cuda")
        t = t[off:].view(rows, W + pad)[:, :W]
        t.copy_(normal(g, rows, W, dt=dt))
        return t
    for pad, off in ((8, 8), (3, 1), (0, 1)):
        x, dy, dres = wide(pad, off), wide(pad, off), wide(pad, off)
        y, dx, dw, db = check(L, x, w, b, dy, dres, 1e-5, f"pad {pad} off {off}")
        out = wide(pad, off)
        assert L.layer_norm(x, w, b, y=out) is out and torch.equal(out, y)
        # dx over dy, over the residual's gradient, over x; y over x
        for target in (dy, dres, x):
            keep = target.clone()
            got = L.layer_norm_backward(dy, x, w, residual_grad=dres, dx=target)
            assert got[0] is target and all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
            target.copy_(keep)
        L.layer_norm(x, w, b, y=x)
        assert torch.equal(x, y)
    # one row for all: a stride of 0
    one = normal(g, 1, W, dt=dt).expand(rows, -1)
    check(L, one, w, b, one, one, 1e-5, "broadcast")
    # weights on odd addresses
    w2, b2 = normal(g, W + 1, dt=dt)[1:], normal(g, W + 1, dt=dt)[1:]
    x, dy = wide(0, 0), wide(0, 0)
    check(L, x, w2, b2, dy, None, 1e-5, "weights off 16 bytes")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("W", [96, 1024, 3000, 8192, 20000])
def test_layer_norm_rows_of_every_size(L, W, dt):
    # a mean far beside the spread, tiny and huge rows, a row of equal elements
    g = gen_of(3)
    x = normal(g, 7, W, dt="f32")
    x[1] += 1000.0
    x[2] = x[2] * 0.01 + 30000.0
    x[3] *= 1e-12
    x[4] *= 1e12
    x[5] = 3.0
    x[6, 0] += 5000.0  # one element far from all
    x, dy = x.to(R.DT[dt]), normal(g, 7, W, dt=dt)
    w, b = normal(g, W, dt=dt), normal(g, W, dt=dt)
    y, dx, _, _ = check(L, x, w, b, dy, None, 1e-5, "sizes")
    good = y.clone()
    x[0, 5], x[3, W - 1] = float("nan"), float("inf")
    y = L.layer_norm(x, w, b)
    assert bool(y[0].isnan().all()) and bool(y[3].isnan().all())
    for i in (1, 2, 4, 5, 6):
        assert torch.equal(y[i], good[i])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("W", [64, 33, 1024])
def test_layer_norm_small_rows_without_eps(L, W, dt):
    # the variance is a subnormal number of 32 bits; the squares that make it are exact to
    # half of 2^-149 each, so to 2^-20 of a variance of some 2^-129
    g = gen_of(4)
    x = (normal(g, 9, W, dt="f32") * 4e-20).to(R.DT[dt])
    dy, w = normal(g, 9, W, dt=dt), normal(g, W, dt=dt)
    ref = M.layer_norm_ref(x, w, None, 0.0)
    y = L.layer_norm(x, w, eps=0.0)
    value, bound = ref["y"]
    R.check(y, value, bound + 2.0 ** -19 * value.abs(), "small rows")


@pytest.mark.parametrize("W", [64, 100, 5000])
def test_layer_norm_without_rows(L, W):
    x = torch.empty(0, W, dtype=torch.float16, device="cuda")
    w = torch.ones(W, dtype=torch.float16, device="cuda")
    assert L.layer_norm(x, w, w).shape == (0, W)
    dx, dw, db = L.layer_norm_backward(x, x, w)
    assert dx.shape == (0, W) and bool((dw == 0).all()) and bool((db == 0).all())


def test_layer_norm_gradient_against_differences(L):
    g = gen_of(5)
    x, w, b, dy, dres = (normal(g, *s, dt="f32") for s in ((6, 40), (40,), (40,), (6, 40), (6, 40)))
    grads = L.layer_norm_backward(dy, x, w, eps=1e-5, residual_grad=dres)
    ref = M.layer_norm_ref(x, w, b, 1e-5, dy, dres)
    base = [t.double() for t in (x, w, b)]

    def value(x, w, b):
        n = torch.nn.functional.layer_norm(x, (40,), w, b, 1e-5)
        return (n * dy.double()).sum() + (x * dres.double()).sum()
    for i, n in enumerate(("dx", "dw", "db")):
        way = torch.randn(base[i].shape, generator=gen_of(6), device="cuda", dtype=torch.float64)
        hi, lo = ([t + (s * 1e-5 * way if j == i else 0) for j, t in enumerate(base)] for s in (1, -1))
        diff = (value(*hi) - value(*lo)) / 2e-5
        bound = float((ref[n][1] * way.abs()).sum()) + 1e-6 * float((ref[n][0] * way).abs().sum())
        assert abs(float((grads[i].double() * way).sum() - diff)) <= bound, n


def test_layer_norm_offsets_beyond_32_bits(L):
    # rows 2^32 bytes apart
    g = gen_of(7)
    step = (1 << 31) + 64
    big = torch.zeros(step + 512, dtype=torch.float16, device="cuda")
    x = big.as_strided((2, 256), (step, 1))
    x.copy_(normal(g, 2, 256))
    dy, w = normal(g, 2, 256), normal(g, 256)
    check(L, x, w, w, dy, None, 1e-5, "far rows")
    want = L.layer_norm(x, w, w)
    L.layer_norm(x, w, w, y=x)
    assert torch.equal(x, want)
    del x, big
    torch.cuda.empty_cache()


def test_layer_norm_refusals(L):
    from paper_2210_10108_amd import pnerf
    x = torch.zeros(4, 8, dtype=torch.float16, device="cuda")
    w = torch.ones(8, dtype=torch.float16, device="cuda")
    for kind, fn in [(TypeError, lambda: L.layer_norm(x.double(), w)), (TypeError, lambda: L.layer_norm(x, w.float())),
                     (ValueError, lambda: L.layer_norm(x, w[:4])), (ValueError, lambda: L.layer_norm(x[0], w)),
                     (ValueError, lambda: L.layer_norm(x, w.expand(8, 8)[:, 0])),
                     (ValueError, lambda: L.layer_norm(x.t(), None)),
                     (ValueError, lambda: L.layer_norm_backward(x[:2], x, w)),
                     (TypeError, lambda: L.layer_norm(x.cpu(), w))]:
        with pytest.raises(kind):
            fn()
    for fn in (lambda: L.layer_norm(x, w, eps=-1.0), lambda: L.layer_norm(x, w, eps=math.nan),
               lambda: L.layer_norm(x, w, y=x[:1].expand(4, -1))):
        with pytest.raises(pnerf.PnerfError) as e:
            fn()
        assert e.value.status == pnerf.ERR_INVALID_ARG
