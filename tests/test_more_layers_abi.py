"""The C ABI of layer norm, rotation with several axes, gradient clipping and 8-bit
states without a device: struct layouts, refusals on the host, workspaces and that
calls take them; and the kernels' registers, from the compiler."""
import ctypes as C
import math
import os
import random
import subprocess

import pytest
import torch

from paper_2210_10108_amd import build, layers, pnerf

from . import test_kernel_resources as kr
from .test_layers_abi import CAPACITY, HEADER, INVALID, PTR, UNSUPPORTED, _takes, attention, needs_hipcc, no_device, norm


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pnerf.LIB_PATH):
        build.build()
    return layers.lib()


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"pnerf_layer_norm_params": layers.LayerNormParams, "pnerf_rotate_axes_params": layers.RotateAxesParams,
               "pnerf_gradient": layers.Gradient, "pnerf_states_params": layers.StatesParams,
               "pnerf_attention_q8_params": layers.AttentionQ8Params}
    lines = []
    for c, py in structs.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f[0]} %zu\\n", offsetof({c}, {f[0]}));' for f in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) {%s\n'
                   'printf("block %%d\\n", PNERF_STATE_BLOCK);\nreturn 0; }' % (HEADER, "\n".join(lines)))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", str(src), "-o", str(exe)], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for c, py in structs.items():
        assert int(got[c]) == C.sizeof(py)
        for f in py._fields_:
            assert int(got[f"{c}.{f[0]}"]) == getattr(py, f[0]).offset, (c, f[0])
    assert int(got["block"]) == layers.STATE_BLOCK


# ---------------------------------------------------------------- refusals
def _set(p, kw):
    for k, v in kw.items():
        if isinstance(v, (tuple, bytes)):
            getattr(p, k)[:len(v)] = list(v)
        else:
            setattr(p, k, v)
    return p


def layer_norm(**kw):
    p = layers.LayerNormParams()
    p.dtype, p.rows, p.width, p.eps = 2, 6, 64, 1e-5
    p.x_stride = p.y_stride = p.dy_stride = p.dres_stride = p.dx_stride = 64
    return _set(p, kw)


def axes(base=None, **kw):
    p = layers.RotateAxesParams()
    p.base = norm(**(base or {}))
    p.norm, p.axes = 1, 3
    return _set(p, kw)


def states(**kw):
    p = layers.StatesParams()
    p.dtype, p.batch, p.kv_rows, p.kv_heads, p.head_dim = 1, 2, 100, 2, 64
    for n in ("k", "v", "k8", "v8"):
        getattr(p, n + "_stride")[:] = (100 * 128, 128, 64)
    for n in ("k_scale", "v_scale"):
        getattr(p, n + "_stride")[:] = (4, 2)
    return _set(p, kw)


def q8(attn=None, **kw):
    p = layers.AttentionQ8Params()
    p.attention = attention(**(attn or {}))
    p.k_scale_stride[:] = p.v_scale_stride[:] = (2, 2)
    return _set(p, kw)


def call(lib, p, **kw):
    r = C.byref(p)
    if isinstance(p, layers.LayerNormParams):
        t = dict(x=PTR, weight=PTR, bias=PTR, y=PTR, **kw) if not kw else {**dict(x=PTR, weight=PTR, bias=PTR, y=PTR), **kw}
        return lib.pnerf_layer_norm(r, t["x"], t["weight"], t["bias"], t["y"], None)
    if isinstance(p, layers.RotateAxesParams):
        t = {**dict(q=PTR, k=PTR, q_out=PTR, k_out=PTR), **kw}
        return lib.pnerf_rotate_axes(r, t["q"], t["k"], t["q_out"], t["k_out"], None)
    if isinstance(p, layers.StatesParams):
        t = {**dict.fromkeys(("k", "v", "k8", "v8", "k_scale", "v_scale"), PTR), **kw}
        return lib.pnerf_quantize_states(r, t["k"], t["v"], t["k8"], t["v8"], t["k_scale"], t["v_scale"], None)
    t = {**dict.fromkeys(("q", "k8", "v8", "k_scale", "v_scale", "o"), PTR), "lse": None, **kw}
    return lib.pnerf_cross_attention_q8(r, t["q"], t["k8"], t["v8"], t["k_scale"], t["v_scale"], t["o"], t["lse"], None, 0, None)


CASES = [
    (layer_norm, dict(dtype=3), INVALID, "dtype"), (layer_norm, dict(rows=-1), INVALID, "rows"),
    (layer_norm, dict(width=0), INVALID, "width"), (layer_norm, dict(width=(1 << 20) + 1), UNSUPPORTED, "width"),
    (layer_norm, dict(rows=1 << 30, width=1 << 20, x_stride=1 << 20), CAPACITY, "2^40"), (layer_norm, dict(eps=-1.0), INVALID, "eps"),
    (layer_norm, dict(eps=math.nan), INVALID, "eps"), (layer_norm, dict(eps=math.inf), INVALID, "eps"),
    (layer_norm, dict(x_stride=-1), INVALID, "x has stride"), (layer_norm, dict(y_stride=63), INVALID, "y overlaps"),
    (axes, dict(base=dict(dtype=-1)), INVALID, "dtype"), (axes, dict(base=dict(head_dim=257)), UNSUPPORTED, "head_dim"),
    (axes, dict(norm=2), INVALID, "norm="), (axes, dict(axes=0), INVALID, "axes="), (axes, dict(axes=5), INVALID, "axes="),
    (axes, dict(pair_axis=bytes(5) + b"\3"), INVALID, "pair_axis[5]=3"), (axes, dict(base=dict(table=None)), INVALID, "table"),
    (axes, dict(base=dict(q_pos=None)), INVALID, "q_pos"), (axes, dict(base=dict(eps=math.nan)), INVALID, "eps"),
    (axes, dict(base=dict(q_out_stride=(64, 64))), INVALID, "q_out overlaps"),
    (states, dict(dtype=0), UNSUPPORTED, "dtype"), (states, dict(dtype=4), INVALID, "dtype"), (states, dict(batch=-1), INVALID, "batch"),
    (states, dict(kv_rows=-1), INVALID, "kv_rows"), (states, dict(kv_heads=0), INVALID, "kv_heads"),
    (states, dict(head_dim=129), UNSUPPORTED, "head_dim"), (states, dict(kv_rows=1 << 30), CAPACITY, "2^27"),
    (states, dict(k8_stride=(0, 128, 64)), INVALID, "k8 overlaps"), (states, dict(v_scale_stride=(4, 1)), INVALID, "v_scale overlaps"),
    (states, dict(k_stride=(-1, 128, 64)), INVALID, "k has stride"), (states, dict(kv_mask=PTR, kv_mask_stride=-1), INVALID, "kv_mask"),
    (states, dict(kv_len=PTR + 2), INVALID, "kv_len"),
    (q8, dict(attn=dict(dtype=0)), UNSUPPORTED, "dtype"), (q8, dict(attn=dict(q_heads=3)), INVALID, "q_heads"),
    (q8, dict(attn=dict(scale=0.0)), INVALID, "scale"), (q8, dict(attn=dict(o_stride=(0, 256, 64))), INVALID, "o overlaps"),
    (q8, dict(k_scale_stride=(-2, 2)), INVALID, "k_scale has stride"),
]


@no_device
@pytest.mark.parametrize("make,bad,status,says", CASES, ids=lambda x: str(x)[:40])
def test_refusals(lib, make, bad, status, says):
    assert call(lib, make(**bad)) == status
    assert says in lib.pnerf_last_error().decode()


@no_device
def test_refusals_of_pointers(lib):
    def refused(st, says, status=INVALID):
        assert st == status and says in lib.pnerf_last_error().decode(), lib.pnerf_last_error()
    for make, names in ((layer_norm, ("x", "y")), (states, ("k", "v", "k_scale", "v_scale")), (axes, ("q", "k", "q_out", "k_out")),
                        (q8, ("q", "o", "k_scale", "v_scale"))):
        for n in names:
            refused(call(lib, make(), **{n: None}), f"{n} is NULL")
            refused(call(lib, make(), **{n: PTR + 1}), f"{n} is not aligned")
    for n in ("k8", "v8"):
        refused(call(lib, states(), **{n: None}), f"{n} is NULL")
        refused(call(lib, q8(), **{n: None}), f"{n} is NULL")
    refused(call(lib, layer_norm(), weight=PTR + 1), "weight is not aligned")
    refused(call(lib, layer_norm(), bias=PTR + 1), "bias is not aligned")
    refused(call(lib, q8(), lse=PTR + 2), "lse is not aligned")
    for fn, make, n in ((lib.pnerf_layer_norm_backward, layer_norm, 7), (lib.pnerf_rotate_axes_backward, axes, 8)):
        refused(fn(C.byref(make()), *[PTR] * n, None, 0, None), "NULL workspace")
        refused(fn(C.byref(make()), *[PTR] * n, PTR, 1, None), "workspace of 1 bytes", CAPACITY)
        refused(fn(C.byref(make()), *[PTR] * n, PTR + 8, 1 << 40, None), "16-byte aligned")
        refused(fn(None, *[PTR] * n, PTR, 1 << 40, None), "NULL params")
    refused(lib.pnerf_layer_norm_backward(C.byref(layer_norm(dres_stride=-1)), *[PTR] * 7, PTR, 1 << 40, None), "dres has stride")
    refused(lib.pnerf_layer_norm_backward(C.byref(layer_norm()), PTR, PTR, PTR, None, PTR, PTR, PTR + 1, PTR, 1 << 40, None), "dbias")
    # a rotation back names its own tensors and reads neither q nor k
    back = axes(norm=0)
    refused(lib.pnerf_rotate_axes_backward(C.byref(back), None, None, None, PTR, PTR, PTR, None, None, None, 0, None), "dq_out is NULL")
    refused(lib.pnerf_rotate_axes_backward(C.byref(back), None, None, PTR, PTR, PTR, PTR + 1, None, None, None, 0, None), "dk is not aligned")
    for fn, make in ((lib.pnerf_layer_norm_workspace, layer_norm), (lib.pnerf_rotate_axes_workspace, axes),
                     (lib.pnerf_cross_attention_q8_workspace, q8)):
        refused(fn(C.byref(make()), None), "NULL bytes")
        refused(fn(None, C.byref(C.c_int64())), "NULL params")
    refused(lib.pnerf_quantize_states(None, *[PTR] * 6, None), "NULL params")
    refused(lib.pnerf_cross_attention_q8(None, *[PTR] * 7, None, 0, None), "NULL params")


def gradients(*rows):
    a = (layers.Gradient * len(rows))()
    for e, (g, o, n, dt, odt) in zip(a, rows):
        e.grad, e.out, e.n, e.dtype, e.out_dtype = g, o, n, dt, odt
    return a


@no_device
def test_clip_refusals(lib):
    one = (PTR, PTR, 100, 0, 0)

    def clip(*rows, max_norm=1.0, eps=1e-6, norm=PTR * 4, ws=PTR * 8, nb=1 << 40, count=None):
        a = gradients(*rows)
        return lib.pnerf_clip_gradients(a, len(rows) if count is None else count, max_norm, eps, norm, ws, nb, None)

    def refused(st, says, status=INVALID):
        assert st == status and says in lib.pnerf_last_error().decode(), lib.pnerf_last_error()
    for kw, says in ((dict(max_norm=0.0), "max_norm"), (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=math.nan), "max_norm"),
                     (dict(eps=-1.0), "eps"), (dict(eps=math.inf), "eps"), (dict(norm=None), "norm is NULL"),
                     (dict(norm=PTR + 2), "norm is not aligned"), (dict(ws=None), "NULL workspace"), (dict(ws=PTR + 8), "16-byte"),
                     (dict(count=-1), "count"), (dict(count=65537), "count")):
        refused(clip(one, **kw), says)
    refused(clip(one, nb=100), "workspace of 100 bytes", CAPACITY)
    refused(lib.pnerf_clip_gradients(None, 1, 1.0, 0.0, PTR, PTR, 1 << 40, None), "gradients is NULL")
    for row, says in (((PTR, PTR, 4, 3, 3), "dtype=3"), ((PTR, PTR, 4, 0, 1), "out_dtype=1"), ((PTR, PTR, 4, 1, 2), "out_dtype=2"),
                      ((PTR, PTR, -1, 0, 0), "n=-1"), ((None, PTR, 4, 0, 0), "grad is NULL"), ((PTR, None, 4, 0, 0), "out is NULL"),
                      ((PTR + 2, PTR, 4, 0, 0), "grad is not aligned"), ((PTR, PTR + 2, 4, 1, 0), "out is not aligned")):
        refused(clip((PTR * 2, PTR * 2, 8, 0, 0), row), "gradient 1: " + says.split(": ")[-1])
    refused(clip((PTR, PTR, 1 << 42, 0, 0), one), "2^42", CAPACITY)
    # overlaps: two outputs, an output and another gradient, a widened output over its own gradient, the norm
    F = 100 * 4
    for rows in ([one, one], [one, (PTR + F - 4, PTR + F - 4, 9, 0, 0)], [(PTR, PTR * 2, 100, 0, 0), (PTR * 3, PTR + 40, 4, 0, 0)],
                 [(PTR, PTR, 100, 1, 0)], [(PTR, PTR + 4, 100, 0, 0)], [(PTR, PTR * 2, 8, 0, 0), (PTR, PTR * 2 + 16, 8, 0, 0)]):
        refused(clip(*rows), "overlaps")
    refused(clip(one, norm=PTR + 40), "overlaps")
    n = C.c_int64()
    refused(lib.pnerf_clip_gradients_workspace(1, None), "NULL bytes")
    refused(lib.pnerf_clip_gradients_workspace(-1, C.byref(n)), "count")


@no_device
def test_clip_takes_the_workspace_asked_for(lib):
    n = C.c_int64()
    for count in (0, 1, 95, 96, 97, 98, 500, 65536):
        assert lib.pnerf_clip_gradients_workspace(count, C.byref(n)) == pnerf.OK
        rows = gradients(*((PTR + 64 * i, PTR + 64 * i, 16, 0, 0) for i in range(count)))
        st = lib.pnerf_clip_gradients(rows, count, 1.0, 0.0, PTR // 2, PTR // 4 + 8, n.value, None)
        assert st == INVALID and "16-byte" in lib.pnerf_last_error().decode()
        st = lib.pnerf_clip_gradients(rows, count, 1.0, 0.0, PTR // 2, PTR // 4, n.value - 1, None)
        assert st == CAPACITY


@no_device
def test_calls_take_the_workspace_asked_for(lib):
    rng = random.Random(3)

    def size(most):
        return rng.choice([1, rng.randint(1, 40), rng.randint(1, most), int(2 ** rng.uniform(0, most.bit_length() - 1))])
    for _ in range(1500):
        rows, W, pad = size(1 << 20), size(1 << 20), rng.choice([0, 0, 1, 8])
        p = layer_norm(dtype=rng.randint(0, 2), rows=rows, width=W)
        p.x_stride = p.y_stride = p.dy_stride = p.dres_stride = p.dx_stride = W + pad
        _takes(lib, lib.pnerf_layer_norm_backward, p, 7,
               lambda n: lib.pnerf_layer_norm_workspace(C.byref(p), C.byref(n)), (rows, W))
        Tq, Tk, Hq, Hk, D = size(20000), size(20000), rng.randint(1, 64), rng.randint(1, 16), rng.choice([32, 64, 100, 128, 256])
        a = axes(base=dict(dtype=rng.randint(0, 2), q_rows=Tq, k_rows=Tk, q_heads=Hq, k_heads=Hk, head_dim=D))
        for names, h in ((("q", "q_out", "dq_out", "dq"), Hq), (("k", "k_out", "dk_out", "dk"), Hk)):
            for n in names:
                getattr(a.base, n + "_stride")[:] = (h * D, D)
        _takes(lib, lib.pnerf_rotate_axes_backward, a, 8,
               lambda n: lib.pnerf_rotate_axes_workspace(C.byref(a), C.byref(n)), (Tq, Tk, Hq, Hk, D))
    n = C.c_int64(-1)
    assert lib.pnerf_rotate_axes_workspace(C.byref(axes(norm=0)), C.byref(n)) == pnerf.OK and n.value == 0


def test_binding_wants_device_tensors():
    x = torch.zeros(4, 8, dtype=torch.float16)
    for fn in (lambda: layers.layer_norm(x), lambda: layers.clip_gradients([x], 1.0), lambda: layers.quantize_states(x, x),
               lambda: layers.rotate_axes(x, None, None, None, None, b""), lambda: layers.cross_attention_q8(x, x, x, x, x)):
        with pytest.raises(TypeError, match="device tensors"):
            fn()


# ---------------------------------------------------------------- the compiler's word
# kernel (mangled-name fragment) -> minimum waves per SIMD
BUDGET = {
    "rotate_axes.hip": {"k_axes_fwd": 4, "k_axes_bwd": 4, "k_axes_any": 4},
    "layer_norm.hip": {"k_layer_norm": 2},
    "clip.hip": {"k_clip": 6},
    "quantize.hip": {"k_quantize": 6},
    "attention_q8.hip": {"k_attn_q8": 1},
}


@needs_hipcc
@pytest.mark.parametrize("src", sorted(BUDGET))
def test_kernels_do_not_spill(src, tmp_path):
    got = kr.remarks(src, tmp_path)
    for frag, waves in BUDGET[src].items():
        hits = [n for n in got if frag in n]
        assert hits, (src, frag, sorted(got))
        for n in hits:
            assert got[n].get("ScratchSize") == 0, (n, got[n])
            assert got[n].get("Occupancy", 0) >= waves, (n, got[n])


@needs_hipcc
def test_no_mfma_result_read_unpadded_after_a_branch(tmp_path):
    out = tmp_path / "k.s"
    src = "attention_q8.hip"
    cmd = [build.HIPCC, *build.flags(src), "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    asm = out.read_text()
    assert "v_mfma" in asm and "v_pk_fma_f32" not in asm and "v_pk_mul_f32" not in asm and "v_pk_add_f32" not in asm
    assert kr.unpadded_mfma_reads_after_branches(asm) == []
