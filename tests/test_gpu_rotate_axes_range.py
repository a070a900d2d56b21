"""The rotation at positions of several axes: components that are no finite numbers
past the rotated part of a head, in every form of the kernels; the forms in which the
pairs' axes are given."""
import math

import numpy as np
import pytest
import torch

from .test_gpu_layers import gen_of, normal, say
from .test_gpu_rotate_axes import layout, table_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


def odd_rows(x):
    """The same numbers on odd addresses: the element-wise kernel."""
    T, H, D = x.shape
    t = torch.empty(T * H * (D + 1) + 1, dtype=x.dtype, device="cuda")[1:].view(T, H, D + 1)[..., :D]
    return t.copy_(x)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("kind", ["runs", "turns"])
@pytest.mark.parametrize("D,rotated", [(64, 32), (128, 64), (32, 16), (96, 48), (256, 16)])
def test_no_norm_leaves_the_rest_of_a_head_as_it_is(L, D, rotated, kind, inter, dt):
    g = gen_of(1)
    T, H = 23, 3
    x = normal(g, T, H, D, dt=dt)
    table, axis = table_of(40, rotated // 2), layout(kind, rotated // 2, 2)
    pos = torch.randint(0, 40, (T, 2), generator=g, device="cuda", dtype=torch.int32)
    bad = x.clone()
    junk = (math.inf, -math.inf, math.nan)
    for i in range(40):
        r, h, d = i % T, i % H, rotated + (i * 7) % (D - rotated)
        bad[r, h, d] = junk[i % 3]
    say("rotation, no numbers", D, rotated, kind, inter, dt)
    for q, clean in ((bad, x), (odd_rows(bad), odd_rows(x))):
        for fn in (lambda t: L.rotate_axes(t, None, table, pos, None, axis, interleaved=inter)[0],
                   lambda t: L.rotate_axes_backward(t, None, t, None, table, pos, None, axis, interleaved=inter)[0]):
            y, want = fn(q), fn(clean)
            assert torch.equal(y[..., :rotated], want[..., :rotated])
            rest = q[..., rotated:]
            assert bool(((y[..., rotated:] == rest) | (y[..., rotated:].isnan() & rest.isnan())).all())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("kind", ["runs", "turns"])
@pytest.mark.parametrize("D,rotated", [(64, 32), (128, 64), (256, 16)])
def test_norm_of_heads_that_hold_no_numbers(L, D, rotated, kind, inter, dt):
    # forward: an infinity has r = 0 for its head, so that the other components are 0;
    # gradient: one that reaches a component past the rotated part is in that component's
    # weight gradient and in its own head's dx alone
    g = gen_of(2)
    T, H = 19, 3
    x, dy, w = normal(g, T, H, D, dt=dt), normal(g, T, H, D, dt=dt), normal(g, D, dt=dt)
    table, axis = table_of(40, rotated // 2), layout(kind, rotated // 2, 2)
    pos = torch.randint(0, 40, (T, 2), generator=g, device="cuda", dtype=torch.int32)
    at = rotated + 5
    for make in (lambda t: t, odd_rows):
        kw = dict(q_weight=w, eps=1e-6, interleaved=inter)
        args = (table, pos, None, axis)
        want = L.rotate_axes(make(x), None, *args, **kw)[0]
        wdx, _, wdw, _ = L.rotate_axes_backward(make(dy), None, make(x), None, *args, **kw)
        bad = x.clone()
        bad[4, 1, at] = math.inf
        y = L.rotate_axes(make(bad), None, *args, **kw)[0]
        others = torch.ones(D, dtype=torch.bool, device="cuda")
        others[at] = False
        assert bool(y[4, 1, at].isnan()) and bool((y[4, 1, others] == 0).all())
        bad = dy.clone()
        bad[4, 1, at] = math.inf
        dx, _, dw, _ = L.rotate_axes_backward(make(bad), None, make(x), None, *args, **kw)
        assert not bool(torch.isfinite(dw[at])) and torch.equal(dw[others], wdw[others])
        heads = torch.ones(T, H, dtype=torch.bool, device="cuda")
        heads[4, 1] = False
        assert torch.equal(dx[heads], wdx[heads]) and torch.equal(want, L.rotate_axes(make(x), None, *args, **kw)[0])


def test_axes_of_pairs_as_bytes_or_numbers(L):
    g = gen_of(3)
    q, table = normal(g, 5, 2, 32), table_of(9, 16)
    pos = torch.randint(0, 9, (5, 3), generator=g, device="cuda", dtype=torch.int32)
    axis = [j % 3 for j in range(16)]
    want = L.rotate_axes(q, None, table, pos, None, bytes(axis))[0]
    for form in (axis, tuple(axis), bytearray(axis), iter(axis), np.array(axis), np.array(axis, dtype=np.int8),
                 torch.tensor(axis), torch.tensor(axis, dtype=torch.uint8)):
        assert torch.equal(L.rotate_axes(q, None, table, pos, None, form)[0], want)
    # a number is not the axes of that many pairs
    for bad in (16, np.int64(16), torch.tensor(16)):
        with pytest.raises(TypeError):
            L.rotate_axes(q, None, table, pos, None, bad)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rotated", [(64, 0), (64, 32), (128, 64), (256, 16)])
def test_norm_rotate_of_heads_that_hold_no_numbers(L, D, rotated, inter, dt):
    # the same of the operator with one position a row
    g = gen_of(4)
    T, H = 19, 3
    x, dy, w = normal(g, T, H, D, dt=dt), normal(g, T, H, D, dt=dt), normal(g, D, dt=dt)
    table = table_of(40, rotated // 2) if rotated else None
    pos = torch.randint(0, 40, (T,), generator=g, device="cuda", dtype=torch.int32) if rotated else None
    at = rotated + 5
    others = torch.ones(D, dtype=torch.bool, device="cuda")
    others[at] = False
    heads = torch.ones(T, H, dtype=torch.bool, device="cuda")
    heads[4, 1] = False
    for make in (lambda t: t, odd_rows):
        wdx, _, wdw, _ = L.norm_rotate_backward(make(dy), None, make(x), None, w, None, table, pos, None, interleaved=inter)
        bad = x.clone()
        bad[4, 1, at] = math.inf
        y = L.norm_rotate(make(bad), None, w, None, table, pos, None, interleaved=inter)[0]
        assert bool(y[4, 1, at].isnan()) and bool((y[4, 1, others] == 0).all())
        bad = dy.clone()
        bad[4, 1, at] = math.inf
        dx, _, dw, _ = L.norm_rotate_backward(make(bad), None, make(x), None, w, None, table, pos, None, interleaved=inter)
        assert not bool(torch.isfinite(dw[at])) and torch.equal(dw[others], wdw[others]) and torch.equal(dx[heads], wdx[heads])
