"""Layer norm of rows at the end of the numbers' range, and of equal elements, against
the definition in 64 bits."""
import math

import pytest
import torch

from . import layers_common as R
from . import more_layers_common as M
from .test_gpu_layers import gen_of, normal, say

pytestmark = pytest.mark.gpu
WIDTHS = [8, 33, 64, 200, 512, 1000, 1001, 2048, 3000, 8192, 12288, 20000]


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("W", WIDTHS)
def test_rows_whose_squares_pass_the_range(L, W, dt):
    # r is 0 where the squared differences' sum is no 32-bit number: y = b, dx = dres, and
    # the weights' gradients are those of the other rows
    g = gen_of(1)
    x = normal(g, 9, W, dt="f32")
    one = torch.randn(9, W, generator=g, device="cuda")
    far = torch.tensor([0, 1, 1, 0, 1, 1, 1, 0, 1], dtype=torch.bool, device="cuda")
    x[1] = 1e25 * one[1]
    x[2] = 1e28 * (1 + 0.1 * one[2])
    x[4] = -1e34 * (1 + 0.1 * one[4])
    x[5] = torch.where(torch.arange(W, device="cuda") % 2 == 0, 3e38, -3e38)
    x[6] = 3e38
    x[6, W // 2] = 2.9e38
    x[8] = 3.3e38 * torch.sign(one[8])
    x[8, 0], x[8, 1], x[8, 2] = 0.0, 3.3e38, -3.3e38
    x = x.to(R.DT[dt])
    dy, dres = normal(g, 9, W, dt=dt), normal(g, 9, W, dt=dt)
    w, b = normal(g, W, dt=dt), normal(g, W, dt=dt)
    say("large rows", W, dt)
    ref = M.layer_norm_ref(torch.where(far[:, None], torch.zeros_like(x), x), w, b, 1e-5, dy, dres)
    y = L.layer_norm(x, w, b)
    dx, dw, db = L.layer_norm_backward(dy, x, w, residual_grad=dres)
    assert torch.equal(y[far], b.expand(int(far.sum()), -1)) and torch.equal(dx[far], dres[far])
    R.check(y[~far], ref["y"][0][~far], ref["y"][1][~far], "y")
    R.check(dx[~far], ref["dx"][0][~far], ref["dx"][1][~far], "dx")
    R.check(dw, *ref["dw"], "dw")
    R.check(db, *ref["db"], "db")
    assert bool((L.layer_norm(x)[far] == 0).all())
    # an infinity or NaN still takes its whole row, whatever the others are
    for at, junk in ((0, math.inf), (W // 2, -math.inf), (W - 1, math.nan), (0, math.nan)):
        bad = x.clone()
        bad[:, at] = junk
        assert bool(L.layer_norm(bad, w, b).isnan().all()), (at, junk)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("W", [1, 7] + WIDTHS)
def test_rows_of_equal_elements(L, W, dt):
    # no difference at all: n is 0 exactly and r = 1 / sqrt(eps), at any size
    sizes = [0.0, 1.0, -3.3e-5, 7e3, 1.2345e4] + ([] if dt == "f16" else [
        1.1e6, -2.3e9, 5.7e12, 1.9e15, 1.2e18, 3e20, -8.1e24, 2.7e27, 1.3e30, 3.1e38, -3.3e38])
    x = torch.tensor(sizes, device="cuda").to(R.DT[dt])[:, None].expand(-1, W).contiguous()
    g = gen_of(2)
    dy, w, b = normal(g, len(sizes), W, dt=dt), normal(g, W, dt=dt), normal(g, W, dt=dt)
    ref = M.layer_norm_ref(torch.zeros_like(x), w, b, 1e-3, dy)
    assert torch.equal(L.layer_norm(x, w, b, eps=1e-3), b.expand(len(sizes), -1))
    dx, dw, db = L.layer_norm_backward(dy, x, w, eps=1e-3)
    R.check(dx, *ref["dx"], "dx")
    assert bool((dw == 0).all())
    R.check(db, *ref["db"], "db")


@pytest.mark.parametrize("shape", [(300001, 24), (70001, 250), (40001, 1000), (9001, 2048), (9001, 2999), (5001, 8192),
                                   (4301, 12288), (700, 20001)], ids=str)
def test_such_rows_among_many(L, shape):
    # rows of equal elements and rows past the range beside ordinary ones, in every step of
    # the kernels' walks; then rows without numbers, which take no other row with them
    g = gen_of(3)
    rows, W = shape
    x, dy, dres = (normal(g, rows, W, dt="bf16") for _ in range(3))
    w, b = normal(g, W, dt="bf16"), normal(g, W, dt="bf16")
    i = torch.arange(rows, device="cuda")
    far, equal = i % 7 == 3, i % 11 == 5
    equal &= ~far
    x[far] *= 1e30
    x[equal] = x[equal][:, :1] * 1e9
    say("rows among many", shape)
    ref = M.layer_norm_ref(torch.where((far | equal)[:, None], torch.zeros_like(x), x), w, b, 1e-5, dy, dres)
    y = L.layer_norm(x, w, b)
    dx, dw, db = L.layer_norm_backward(dy, x, w, residual_grad=dres)
    assert bool((y[far | equal] == b).all()) and torch.equal(dx[far], dres[far])
    R.check(y[~far], ref["y"][0][~far], ref["y"][1][~far], "y")
    R.check(dx[~far], ref["dx"][0][~far], ref["dx"][1][~far], "dx")
    R.check(dw, *ref["dw"], "dw")
    R.check(db, *ref["db"], "db")
    none = i % 5 == 1
    x[none, (i[none] * 31) % W] = math.nan
    x[i % 35 == 11, W - 1] = math.inf
    z = L.layer_norm(x, w, b)
    dz = L.layer_norm_backward(dy, x, w, residual_grad=dres)[0]
    assert bool(z[none].isnan().all()) and bool(dz[none].isnan().all())
    assert torch.equal(z[~none], y[~none]) and torch.equal(dz[~none], dx[~none])
