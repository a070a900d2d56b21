"""Layer norm and the rotation with several axes where their workgroups, of which no
more are launched than a fixed number, walk over several rows or groups of heads
each: the loads of the next step, the places in LDS that two steps use in turn, the
sums that are carried from row to row."""
import pytest
import torch

from . import layers_common as R
from . import more_layers_common as M
from .test_gpu_layer_norm import check as check_layer_norm
from .test_gpu_layers import gen_of, normal
from .test_gpu_rotate_axes import check as check_axes
from .test_gpu_rotate_axes import layout, table_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


# forward: 4096 workgroups of 64, 8, 4 rows and of one; gradient: 1024, 768 or 512 (256 past 8192)
@pytest.mark.parametrize("dt,shape", [
    ("f16", (600000, 8)), ("bf16", (600001, 31)), ("f16", (300000, 64)), ("bf16", (70000, 256)), ("f32", (70001, 250)),
    ("f16", (40000, 513)), ("bf16", (40000, 1024)), ("f32", (20000, 1000)), ("bf16", (9000, 2048)), ("f16", (9001, 1999)),
    ("f32", (9000, 2048)), ("bf16", (8300, 4096)), ("f16", (8300, 4095)), ("f32", (4200, 4096)), ("bf16", (8300, 8192)),
    ("f16", (4200, 8191)), ("bf16", (4500, 12288)), ("f32", (700, 12289)), ("f16", (4500, 16384)), ("bf16", (4500, 16392)),
    ("f16", (700, 16391)), ("f32", (700, 16392)), ("bf16", (530, 40001))], ids=str)
def test_layer_norm_of_many_rows(L, shape, dt):
    g = gen_of(1)
    x, dy, dres = (normal(g, *shape, dt=dt) for _ in range(3))
    w, b = normal(g, shape[1], dt=dt), normal(g, shape[1], dt=dt)
    check_layer_norm(L, x, w, b, dy, dres, 1e-5, "many rows")


@pytest.mark.parametrize("shape", [(9001, 1001), (40000, 77), (530, 16385)], ids=str)
def test_layer_norm_of_many_rows_apart(L, shape):
    # rows of odd widths and strides on odd addresses, in place
    g = gen_of(2)
    rows, W = shape

    def wide():
        t = torch.empty(rows * (W + 2) + 1, dtype=torch.bfloat16, device="cuda")[1:].view(rows, W + 2)[:, :W]
        return t.copy_(normal(g, rows, W, dt="bf16"))
    x, dy, dres = wide(), wide(), wide()
    w, b = normal(g, W, dt="bf16"), normal(g, W, dt="bf16")
    y, dx, _, _ = check_layer_norm(L, x, w, b, dy, dres, 1e-5, "many rows apart")
    L.layer_norm_backward(dy, x, w, residual_grad=dres, dx=dres)
    assert torch.equal(dres, dx)
    L.layer_norm(x, w, b, y=x)
    assert torch.equal(x, y)


# three steps and more of the forward (2048 workgroups with axes in turn, 4096 with runs) and the
# gradient (1024), 256 / lanes heads each; head counts that do not divide those
@pytest.mark.parametrize("eps", [None, 1e-6])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("kind", ["runs", "turns"])
@pytest.mark.parametrize("dt,Tq,Tk,Hq,Hk,D,rotated", [
    ("f16", 100000, 70000, 5, 1, 64, 64), ("bf16", 150001, 0, 3, 1, 64, 32), ("f16", 60000, 90001, 3, 2, 128, 128),
    ("f32", 400000, 0, 1, 1, 64, 64), ("bf16", 30000, 30000, 7, 1, 96, 96), ("f16", 9001, 9001, 7, 3, 256, 128),
    ("bf16", 300000, 0, 3, 1, 32, 32)], ids=str)
def test_rotation_of_many_heads(L, dt, Tq, Tk, Hq, Hk, D, rotated, kind, inter, eps):
    g = gen_of(3)
    q, dq = normal(g, Tq, Hq, D, dt=dt), normal(g, Tq, Hq, D, dt=dt)
    k, dk = (normal(g, Tk, Hk, D, dt=dt), normal(g, Tk, Hk, D, dt=dt)) if Tk else (None, None)
    table, axis = table_of(300, rotated // 2), layout(kind, rotated // 2, 3)
    pq, pk = (torch.randint(0, 300, (n, 3), generator=g, device="cuda", dtype=torch.int32) if n else None for n in (Tq, Tk))
    wq, wk = (normal(g, D, dt=dt), normal(g, D, dt=dt) if Tk else None) if eps else (None, None)
    check_axes(L, q, k, wq, wk, table, pq, pk, axis, eps, inter, dq, dk, f"many heads {kind}")


@pytest.mark.parametrize("eps", [None, 1e-6])
def test_rotation_of_many_heads_element_by_element(L, eps):
    # 4096 workgroups of 4 heads forward, 1024 in the gradient
    g = gen_of(4)
    T, H, D = 25001, 3, 50
    q, dq = normal(g, T, H, D), normal(g, T, H, D)
    table, axis = table_of(99, 11), layout("any", 11, 3)
    pos = torch.randint(0, 99, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    w = normal(g, D) if eps else None
    check_axes(L, q, None, w, None, table, pos, None, axis, eps, True, dq, None, "many heads, any width")
    # a head of the last step is as it is by itself
    y = L.rotate_axes(q, None, table, pos, None, axis, q_weight=w, eps=eps)[0]
    one = L.rotate_axes(q[-1:], None, table, pos[-1:].contiguous(), None, axis, q_weight=w, eps=eps)[0]
    assert torch.equal(y[-1:], one)
    R.check(y, *M.axes_ref(q, w, table, pos, axis, eps, False)["y"], "pairs half a head apart")
