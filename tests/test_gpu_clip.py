"""Gradient clipping against its definition in 64 bits."""
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


def gen_of(seed):
    return torch.Generator("cuda").manual_seed(seed)


def normal(gen, *shape, dt="f32", std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(R.DT[dt])


def check(L, grads, max_norm, what, outs=None, **kw):
    say("clip", what, len(grads))
    (norm, en), refs = M.clip_ref(grads, max_norm, out_dtypes=None if outs is None else [o.dtype for o in outs], **kw)
    before = [g.clone() for g in grads] if outs is not None else None
    got = L.clip_gradients(grads, max_norm, out=outs, **kw)
    assert got.shape == () and got.dtype == torch.float32
    assert abs(float(got) - norm) <= en, (what, float(got), norm)
    for i, (t, ref) in enumerate(zip(grads if outs is None else outs, refs)):
        R.check(t, *ref, f"{what} {i}")
    if before is not None:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))
    return got


SIZES = [[1], [0, 5, 0], [8], [8192], [8193, 8191, 16384], [7, 1, 100, 3, 8192 * 3 + 5], [300000, 17, 64, 1000003],
         [5] * 95, [9] * 96, [11] * 97, [33] * 200, [1 << 22, 3]]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_clip_gradients(L, sizes, dt):
    g = gen_of(1)
    for clips in (0.5, 1e9):
        grads = [normal(g, n, dt=dt, std=0.3) for n in sizes]
        kept = [t.clone() for t in grads]
        check(L, grads, clips, "in place")
        if clips == 1e9:
            assert all(torch.equal(a, b) for a, b in zip(grads, kept))
        for out in {dt, "f32"}:
            outs = [torch.full((n,), float("nan"), dtype=R.DT[out], device="cuda") for n in sizes]
            check(L, kept, clips, f"to {out}", outs)


def test_clip_gradients_of_several_types_and_shapes(L):
    g = gen_of(2)
    shapes = [(3, 5), (), (64, 129), (2, 3, 4, 5), (1000,), (1,), (0, 7), (257, 33)]
    grads = [normal(g, *s, dt=("f32", "f16", "bf16")[i % 3]) for i, s in enumerate(shapes)]
    outs = [torch.empty_like(t, dtype=torch.float32 if i % 2 else t.dtype) for i, t in enumerate(grads)]
    check(L, grads, 3.0, "mixed", outs)
    # some in place, some not
    mixed = [t if i % 2 else torch.empty_like(t) for i, t in enumerate(grads)]
    ref = M.clip_ref(grads, 3.0)[1]
    L.clip_gradients(grads, 3.0, out=mixed)
    for t, r in zip(mixed, ref):
        R.check(t, *r, "some in place")
    check(L, [normal(g, 40)], 0.1, "eps", eps=0.5)
    zeros = [torch.zeros(100, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.float16)]
    assert float(check(L, zeros, 1.0, "zeros")) == 0.0
    assert float(check(L, zeros, 1.0, "zeros, no eps", eps=0.0)) == 0.0


@pytest.mark.parametrize("off", [1, 3, 4, 8])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_clip_gradients_on_any_address(L, off, dt):
    # slices of one buffer, on addresses that are not of whole chunks; their neighbours stay
    g = gen_of(3)
    flat = normal(g, 70000, dt=dt)
    kept = flat.clone()
    spans = [(off, off + 20001), (30000 + off, 30000 + off + 7), (40000 + off, 40000 + off + 9 * 1111)]
    grads = [flat[a:b] for a, b in spans]
    outs = [torch.empty(b - a + 8, device="cuda")[8 - off % 8 or 0:][:b - a] for a, b in spans]
    check(L, grads, 1.0, f"off {off} to f32", outs)
    odd = [torch.empty(b - a + 1, dtype=flat.dtype, device="cuda")[1:] for a, b in spans]
    check(L, grads, 1.0, f"off {off} to odd addresses", odd)
    check(L, grads, 1.0, f"off {off} in place")
    mine = torch.zeros(70000, dtype=torch.bool, device="cuda")
    for a, b in spans:
        mine[a:b] = True
    assert torch.equal(flat[~mine], kept[~mine]) and not torch.equal(flat[mine], kept[mine])


def test_clip_gradients_of_every_size(L):
    # squares that float32 does not hold, above and below; one large among small
    g = gen_of(4)
    check(L, [normal(g, 1000, std=1e25), normal(g, 1000, std=1e-25)], 1.0, "large")
    check(L, [normal(g, 1000, std=1e-25)], 1e-26, "small", eps=0.0)
    check(L, [torch.full((1000,), 1e-30, device="cuda")], 1e-31, "smallest", eps=0.0)
    check(L, [normal(g, 100, dt="bf16", std=1e30)], 7.0, "bf16")
    one = normal(g, 1 << 20, std=1e-4)
    one[12345] = 1e4
    check(L, [one], 1.0, "one large")
    # the norm itself passes float32's range, the results do not
    big = [torch.full((9,), 3e38, device="cuda")]
    norm = L.clip_gradients(big, 1.0)
    assert float(norm) == math.inf
    assert float((big[0] - 1 / 3).abs().max()) <= 4 * R.E32


def test_clip_gradients_without_a_bound_and_not_finite(L):
    g = gen_of(5)
    a, b = normal(g, 5000), normal(g, 77, dt="bf16")
    kept = a.clone()
    check(L, [a, b], math.inf, "no bound")
    assert torch.equal(a, kept)
    for junk in (math.inf, -math.inf, math.nan):
        x, y = a.clone(), b.clone()
        x[77] = junk
        norm = float(L.clip_gradients([x, y], math.inf))
        assert (math.isnan(norm) if math.isnan(junk) else norm == math.inf)
        assert torch.equal(y, b) and torch.equal(x[:77], a[:77])
        L.clip_gradients([x, y], 1.0)
        if math.isnan(junk):
            assert bool(x.isnan().all()) and bool(y.isnan().all())
        else:
            assert bool(x[77].isnan()) and bool((x[:77] == 0).all()) and bool((y == 0).all())


def test_clip_gradients_beyond_32_bits(L):
    # more than 2^32 elements in one gradient
    n = (1 << 32) + 8197
    t = torch.full((n,), 2.0 ** -16, dtype=torch.float16, device="cuda")
    t[-1] = 3.0
    norm = L.clip_gradients([t], 0.75)
    want = math.sqrt((n - 1) * 2.0 ** -32 + 9.0)
    assert abs(float(norm) - want) <= 2 * R.E32 * want
    c = 0.75 / (want + 1e-6)
    assert abs(float(t[-1]) - 3.0 * c) <= (R.U["f16"] + 2 * R.E32) * 3.0 * c
    assert bool((t[:-1] == t[0]).all()) and abs(float(t[0]) - 2.0 ** -16 * c) <= R.TINY["f16"]
    del t
    torch.cuda.empty_cache()


def test_clip_gradients_refusals(L):
    from paper_2210_10108_amd import pnerf
    a = torch.zeros(64, device="cuda")
    h = torch.zeros(64, device="cuda", dtype=torch.float16)
    for kind, fn in [(ValueError, lambda: L.clip_gradients([], 1.0)),
                     (ValueError, lambda: L.clip_gradients([a], 1.0, out=[])),
                     (ValueError, lambda: L.clip_gradients([a.view(8, 8).t()], 1.0)),
                     (ValueError, lambda: L.clip_gradients([a], 1.0, out=[a[:32]])),
                     (TypeError, lambda: L.clip_gradients([a], 1.0, out=[h])),
                     (TypeError, lambda: L.clip_gradients([a, h.double()], 1.0)),
                     (TypeError, lambda: L.clip_gradients([a, h.cpu()], 1.0)),
                     (TypeError, lambda: L.clip_gradients([a.cpu()], 1.0)),
                     (TypeError, lambda: L.clip_gradients([a, h.long()], 1.0))]:
        with pytest.raises(kind):
            fn()
    for fn in (lambda: L.clip_gradients([a], 0.0), lambda: L.clip_gradients([a], -1.0),
               lambda: L.clip_gradients([a], math.nan), lambda: L.clip_gradients([a], 1.0, eps=-1.0),
               lambda: L.clip_gradients([a, a], 1.0), lambda: L.clip_gradients([a[:40], a[30:]], 1.0),
               lambda: L.clip_gradients([a[:8], a[8:16]], 1.0, out=[a[8:16], a[16:24]]),
               lambda: L.clip_gradients([a[:8]], 1.0, out=[a[4:12]])):
        with pytest.raises(pnerf.PnerfError) as e:
            fn()
        assert e.value.status == pnerf.ERR_INVALID_ARG
    # the same gradient twice, read only
    x = torch.ones(9, device="cuda")
    o = [torch.empty(9, device="cuda") for _ in range(2)]
    assert abs(float(L.clip_gradients([x, x], 100.0, out=o)) - math.sqrt(18)) < 1e-6
    assert torch.equal(o[0], x) and torch.equal(o[1], x)
