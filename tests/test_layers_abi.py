"""The C ABI of the layer operators without a device: every function declared in
include/pnerf_layers.h is exported and bound, the struct layouts match, bad
arguments are refused on the host, workspaces are planned for any sizes; and
the kernels' registers and MFMA results, from the compiler."""
import ctypes as C
import os
import random
import re
import shutil
import subprocess

import pytest
import torch

from paper_2210_10108_amd import build, layers, pnerf

from . import test_kernel_resources as kr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pnerf_layers.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pnerf.LIB_PATH):
        build.build()
    return layers.lib()


def test_every_declared_function_is_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pnerf_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(layers._SIGS)
    out = subprocess.run(["nm", "-D", "--defined-only", pnerf.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    assert set(names) <= set(re.findall(r"\bT (pnerf_\w+)", out))


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"pnerf_attention_params": layers.AttentionParams,
               "pnerf_norm_rotate_params": layers.NormRotateParams, "pnerf_linear_params": layers.LinearParams}
    lines = []
    for c, py in structs.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f[0]} %zu\\n", offsetof({c}, {f[0]}));' for f in py._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) {%s\n'
                   'printf("dtypes %%d\\n", PNERF_F32 + 10 * PNERF_F16 + 100 * PNERF_BF16);\n'
                   'printf("acts %%d\\n", PNERF_ACT_NONE + 10 * PNERF_ACT_RELU + 100 * PNERF_ACT_GELU + '
                   '1000 * PNERF_ACT_SILU);\nreturn 0; }' % (HEADER, "\n".join(lines)))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", str(src), "-o", str(exe)], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    for c, py in structs.items():
        assert int(got[c]) == C.sizeof(py)
        for f in py._fields_:
            assert int(got[f"{c}.{f[0]}"]) == getattr(py, f[0]).offset, (c, f[0])
    assert int(got["dtypes"]) == layers.F32 + 10 * layers.F16 + 100 * layers.BF16
    a = layers.ACTIVATIONS
    assert int(got["acts"]) == a["none"] + 10 * a["relu"] + 100 * a["gelu"] + 1000 * a["silu"]


# ---------------------------------------------------------------- refusals
PTR = 1 << 20  # an address that is never read: every call below is refused on the host


def attention(**kw):
    p = layers.AttentionParams()
    p.dtype, p.batch, p.q_rows, p.kv_rows, p.q_heads, p.kv_heads, p.head_dim = 1, 2, 8, 16, 4, 2, 64
    p.scale = 0.125
    for n, s, h in (("q", 8, 4), ("k", 16, 2), ("v", 16, 2), ("o", 8, 4), ("do", 8, 4), ("dq", 8, 4),
                    ("dk", 16, 2), ("dv", 16, 2)):
        getattr(p, n + "_stride")[:] = (s * h * 64, h * 64, 64)
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def norm(**kw):
    p = layers.NormRotateParams()
    p.dtype, p.q_rows, p.k_rows, p.q_heads, p.k_heads = 2, 5, 7, 4, 2
    p.head_dim, p.rotary_dim, p.n_positions, p.eps = 64, 32, 10, 1e-6
    for n, h in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2), ("dq_out", 4), ("dk_out", 2), ("dq", 4), ("dk", 2)):
        getattr(p, n + "_stride")[:] = (h * 64, 64)
    p.q_weight = p.k_weight = p.table = p.q_pos = p.k_pos = PTR
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def linear(**kw):
    p = layers.LinearParams()
    p.dtype, p.activation, p.m, p.n, p.k = 2, 2, 6, 16, 8
    p.x_stride = p.dx_stride = 8
    p.w_stride = p.y_stride = p.z_stride = p.dy_stride = p.dw_stride = p.residual_stride = 16
    for k, v in kw.items():
        setattr(p, k, v)
    return p


INVALID, UNSUPPORTED, CAPACITY = pnerf.ERR_INVALID_ARG, pnerf.ERR_NOT_SUPPORTED, pnerf.ERR_CAPACITY
CASES = [
    (attention, dict(dtype=3), INVALID, "dtype"), (attention, dict(dtype=0), UNSUPPORTED, "dtype"),
    (attention, dict(batch=-1), INVALID, "batch"), (attention, dict(batch=65536), INVALID, "batch"),
    (attention, dict(q_rows=-1), INVALID, "q_rows"), (attention, dict(kv_rows=-1), INVALID, "kv_rows"),
    (attention, dict(q_heads=3), INVALID, "q_heads"), (attention, dict(kv_heads=0), INVALID, "kv_heads"),
    (attention, dict(q_heads=0), INVALID, "q_heads"), (attention, dict(head_dim=0), INVALID, "head_dim"),
    (attention, dict(head_dim=129), UNSUPPORTED, "head_dim"), (attention, dict(scale=0.0), INVALID, "scale"),
    (attention, dict(scale=float("nan")), INVALID, "scale"), (attention, dict(scale=float("inf")), INVALID, "scale"),
    (attention, dict(q_rows=1 << 30), CAPACITY, "2^27"), (attention, dict(kv_rows=1 << 30), CAPACITY, "2^27"),
    (attention, dict(q_stride=(512, -1, 64)), INVALID, "q has stride"),
    (attention, dict(o_stride=(0, 256, 64)), INVALID, "o overlaps"),
    (attention, dict(o_stride=(2048, 256, 63)), INVALID, "o overlaps"),
    (attention, dict(kv_mask=PTR, kv_mask_stride=-1), INVALID, "kv_mask"),
    (attention, dict(kv_len=PTR + 2), INVALID, "kv_len"), (attention, dict(q_len=PTR + 1), INVALID, "q_len"),
    (norm, dict(dtype=-1), INVALID, "dtype"), (norm, dict(q_rows=-1), INVALID, "q_rows"),
    (norm, dict(k_heads=0), INVALID, "k_heads"), (norm, dict(head_dim=0), INVALID, "head_dim"),
    (norm, dict(head_dim=257), UNSUPPORTED, "head_dim"), (norm, dict(rotary_dim=66), INVALID, "rotary_dim"),
    (norm, dict(rotary_dim=7), INVALID, "rotary_dim"), (norm, dict(interleaved=2), INVALID, "interleaved"),
    (norm, dict(n_positions=0), INVALID, "n_positions"), (norm, dict(eps=-1.0), INVALID, "eps"),
    (norm, dict(eps=float("nan")), INVALID, "eps"), (norm, dict(table=None), INVALID, "table"),
    (norm, dict(table=PTR + 2), INVALID, "table"), (norm, dict(k_pos=None), INVALID, "k_pos"),
    (norm, dict(q_pos=PTR + 1), INVALID, "q_pos"), (norm, dict(q_weight=PTR + 1), INVALID, "q_weight"),
    (norm, dict(q_rows=1 << 30), CAPACITY, "2^26"), (norm, dict(k_out_stride=(64, 64)), INVALID, "k_out overlaps"),
    (norm, dict(q_stride=(256, -64)), INVALID, "q has stride"),
    (linear, dict(dtype=5), INVALID, "dtype"), (linear, dict(dtype=0), UNSUPPORTED, "dtype"),
    (linear, dict(activation=4), INVALID, "activation"), (linear, dict(m=-1), INVALID, "m="),
    (linear, dict(n=0), INVALID, "n="), (linear, dict(k=0), INVALID, "k="),
    (linear, dict(m=1 << 25, n=1 << 25), CAPACITY, "2^34"), (linear, dict(m=1 << 28), CAPACITY, "2^27"), (linear, dict(y_stride=15), INVALID, "y overlaps"),
    (linear, dict(x_stride=-8), INVALID, "x has stride"),
]


def call(lib, p, **kw):
    ptr = dict.fromkeys(("q", "k", "v", "o", "x", "w", "y", "bias", "residual", "z"), PTR)
    ptr.update(kw)
    ws, nb = ptr.pop("workspace", None), ptr.pop("bytes", 0)
    r = C.byref(p)
    if isinstance(p, layers.AttentionParams):
        return lib.pnerf_cross_attention(r, ptr["q"], ptr["k"], ptr["v"], ptr["o"], None, ws, nb, None)
    if isinstance(p, layers.NormRotateParams):
        return lib.pnerf_norm_rotate(r, ptr["q"], ptr["k"], ptr["o"], ptr["o"], None)
    return lib.pnerf_linear(r, ptr["x"], ptr["w"], ptr["bias"], ptr["residual"], ptr["y"], ptr["z"], ws, nb, None)


no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that are not memory: no device may see them")


@no_device
@pytest.mark.parametrize("make,bad,status,says", CASES, ids=lambda x: str(x)[:40])
def test_refusals(lib, make, bad, status, says):
    assert call(lib, make(**bad)) == status
    assert says in lib.pnerf_last_error().decode()


@no_device
def test_refusals_of_pointers(lib):
    def refused(st, says, status=INVALID):
        assert st == status and says in lib.pnerf_last_error().decode()
    for name in ("q", "k", "v", "o"):
        refused(call(lib, attention(), **{name: None}), f"{name} is NULL")
        refused(call(lib, attention(), **{name: PTR + 1}), f"{name} is not aligned")
    for name in ("x", "w", "y"):
        refused(call(lib, linear(), **{name: None}), f"{name} is NULL")
        refused(call(lib, linear(), **{name: PTR + 1}), f"{name} is not aligned")
    refused(call(lib, linear(), bias=PTR + 1), "bias is not aligned")
    refused(call(lib, norm(), q=None), "q is NULL")
    refused(call(lib, norm(), o=PTR + 1), "not aligned")
    for fn, make, n in ((lib.pnerf_cross_attention_backward, attention, 9), (lib.pnerf_linear_backward, linear, 7),
                        (lib.pnerf_norm_rotate_backward, norm, 8)):
        refused(fn(C.byref(make()), *[PTR] * n, None, 0, None), "NULL workspace")
        refused(fn(C.byref(make()), *[PTR] * n, PTR, 1, None), "workspace of 1 bytes", CAPACITY)
        refused(fn(C.byref(make()), *[PTR] * n, PTR + 8, 1 << 40, None), "16-byte aligned")
        refused(fn(None, *[PTR] * n, PTR, 1 << 40, None), "NULL params")
    args = [PTR] * 9
    args[4] = None
    refused(lib.pnerf_cross_attention_backward(C.byref(attention()), *args, PTR, 1 << 40, None), "lse is NULL")
    refused(lib.pnerf_cross_attention_backward(C.byref(attention(dk_stride=(0, 128, 64))), *[PTR] * 9, PTR, 1 << 40,
                                               None), "dk overlaps")
    refused(lib.pnerf_linear_backward(C.byref(linear()), PTR, PTR, None, PTR, PTR, PTR, PTR, PTR, 1 << 40, None),
            "z is NULL")
    for fn, make in ((lib.pnerf_cross_attention_workspace, attention), (lib.pnerf_linear_workspace, linear)):
        refused(fn(C.byref(make()), 0, None), "NULL bytes")
        refused(fn(None, 0, C.byref(C.c_int64())), "NULL params")
    refused(lib.pnerf_norm_rotate_workspace(C.byref(norm()), None), "NULL bytes")


def test_workspaces_of_any_sizes(lib):
    # host arithmetic only: no size makes it overflow, divide by zero or ask for less than nothing
    rng = random.Random(1)

    def size(most, least=0):
        return rng.choice([least, 1, rng.randint(least, 64), rng.randint(least, most),
                           min(most, int(2 ** rng.uniform(0, 31)))])
    n = C.c_int64()
    ok = 0
    for _ in range(20000):
        kv = max(1, size(64))
        p = attention(dtype=rng.choice([1, 2]), batch=size(65535), q_rows=size(1 << 27), kv_rows=size(1 << 27),
                      kv_heads=kv, q_heads=kv * rng.randint(1, 8), head_dim=rng.randint(1, 128))
        st = lib.pnerf_cross_attention_workspace(C.byref(p), rng.randint(0, 1), C.byref(n))
        assert st in (pnerf.OK, CAPACITY) and (st or 0 <= n.value < 1 << 50)
        ok += st == pnerf.OK
        p = linear(dtype=rng.choice([1, 2]), activation=rng.randint(0, 3), m=size(1 << 30), n=max(1, size(1 << 30)),
                   k=max(1, size(1 << 30)))
        p.x_stride = p.w_stride = p.dy_stride = size(1 << 30)
        st = lib.pnerf_linear_workspace(C.byref(p), rng.randint(0, 1), C.byref(n))
        assert st in (pnerf.OK, CAPACITY) and (st or 0 <= n.value < 1 << 50)
        ok += st == pnerf.OK
        p = norm(q_rows=size(1 << 26), k_rows=size(1 << 26), q_heads=max(1, size(64)), k_heads=max(1, size(64)),
                 head_dim=rng.randint(1, 256), rotary_dim=0)
        st = lib.pnerf_norm_rotate_workspace(C.byref(p), C.byref(n))
        assert st in (pnerf.OK, CAPACITY) and (st or 0 <= n.value < 1 << 30)
        ok += st == pnerf.OK
    assert ok > 10000


def test_binding_wants_device_tensors():
    x = torch.zeros(4, 8, dtype=torch.float16)
    with pytest.raises(TypeError, match="device tensors"):
        layers.linear(x, torch.zeros(8, 8, dtype=torch.float16))
    with pytest.raises(TypeError, match="device tensors"):
        layers.cross_attention(None, x, x)


# ---------------------------------------------------------------- the compiler's word
needs_hipcc = pytest.mark.skipif(not shutil.which(build.HIPCC) and not os.path.exists(build.HIPCC),
                                 reason="hipcc not installed")
# kernel (mangled-name fragment) -> minimum waves per SIMD
BUDGET = {
    "attention.hip": {"k_attn_fwdINS_4BF16ELi128": 2, "k_attn_fwdINS_3F16ELi128": 2, "k_attn_fwdINS_4BF16ELi64": 3,
                      "k_attn_few": 1, "k_attn_any": 1},
    "attention_bwd.hip": {"k_attn_dqINS_4BF16ELi128ELb1": 2, "k_attn_dqINS_3F16ELi128ELb1": 2,
                          "k_attn_dkvINS_4BF16ELi128ELb1": 2, "k_attn_dkvINS_3F16ELi128ELb1": 2,
                          "k_attn_dkvINS_4BF16ELi64ELb1": 3, "k_attn_dkv": 1},
    # fragments of the template arguments: the tiles of 256 x 256 and 128 x 128
    "linear.hip": {"k_product": 2, "k_product_few": 4},
    "norm_rotate.hip": {"k_norm_fwd": 7, "k_norm_bwd": 5},
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
@pytest.mark.parametrize("src", ["attention.hip", "attention_bwd.hip", "linear.hip"])
def test_no_mfma_result_read_unpadded_after_a_branch(src, tmp_path):
    out = tmp_path / "k.s"
    cmd = [build.HIPCC, *build.flags(src), "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    asm = out.read_text()
    assert "v_mfma" in asm and "v_pk_fma_f32" not in asm and "v_pk_mul_f32" not in asm and "v_pk_add_f32" not in asm
    assert kr.unpadded_mfma_reads_after_branches(asm) == []


# ---------------------------------------------------------------- workspaces and their calls
def _contiguous(p, **tensors):
    for name, sizes in tensors.items():
        stride, s = [], 1
        for n in reversed(sizes):
            s *= max(n, 1)
            stride.append(s)
        getattr(p, name + "_stride")[:] = tuple(reversed(stride))


def _takes(lib, fn, p, n_tensors, workspace_of, what):
    """The call takes as many bytes as it was said to need, wherever its tensors
    lie (a workspace 8 bytes off stops it before anything would be launched)."""
    n = C.c_int64(-1)
    assert workspace_of(n) == pnerf.OK, (what, lib.pnerf_last_error())
    for at in (PTR, PTR + 4):
        st = fn(C.byref(p), *[at] * n_tensors, PTR + 8 if n.value else None, n.value, None)
        says = lib.pnerf_last_error().decode()
        assert st not in (pnerf.OK, CAPACITY), (what, at, n.value, says)
        assert "16-byte aligned" in says if n.value else "NULL workspace" not in says, (what, at, says)


@no_device
@pytest.mark.parametrize("D", [32, 64, 128, 256, 100])
def test_norm_calls_take_the_workspace_asked_for(lib, D):
    rng = random.Random(D)
    cases = [(T, T, h, g) for T in (1, 513, 1025, 1030, 2011, 4100, 4999) for h, g in
             ((1, 1), (3, 1), (6, 2), (12, 4), (24, 8), (28, 4), (56, 8), (32, 8))]
    cases += [(1001, 3003, 8, 8), (1, 100000, 1, 1), (100000, 1, 7, 1), (5000, 0, 3, 1)]
    cases += [(rng.randint(1, 20000), rng.randint(0, 20000), rng.randint(1, 64), rng.randint(1, 16)) for _ in range(400)]
    for Tq, Tk, Hq, Hk in cases:
        p = norm(dtype=rng.randint(0, 2), q_rows=Tq, k_rows=Tk, q_heads=Hq, k_heads=Hk, head_dim=D, rotary_dim=0)
        _contiguous(p, **{n: (Hq, D) for n in ("q", "q_out", "dq_out", "dq")},
                    **{n: (Hk, D) for n in ("k", "k_out", "dk_out", "dk")})
        _takes(lib, lib.pnerf_norm_rotate_backward, p, 8,
               lambda n: lib.pnerf_norm_rotate_workspace(C.byref(p), C.byref(n)), (Tq, Tk, Hq, Hk, D))


@no_device
def test_attention_and_linear_calls_take_the_workspace_asked_for(lib):
    rng = random.Random(7)

    def size(most):
        return rng.choice([1, rng.randint(1, 40), rng.randint(1, most), int(2 ** rng.uniform(0, most.bit_length() - 1))])
    for _ in range(1500):
        B, Sq, Sk, Hk, D = size(64), size(8000), size(20000), rng.randint(1, 16), rng.randint(1, 128)
        Hq = Hk * rng.randint(1, 8)
        p = attention(dtype=rng.randint(1, 2), batch=B, q_rows=Sq, kv_rows=Sk, q_heads=Hq, kv_heads=Hk, head_dim=D)
        _contiguous(p, **{n: (Sq, Hq, D) for n in ("q", "o", "do", "dq")}, **{n: (Sk, Hk, D) for n in ("k", "v", "dk", "dv")})
        for fn, back, n in ((lib.pnerf_cross_attention, 0, 5), (lib.pnerf_cross_attention_backward, 1, 9)):
            _takes(lib, fn, p, n, lambda b: lib.pnerf_cross_attention_workspace(C.byref(p), back, C.byref(b)),
                   (back, B, Sq, Sk, Hq, Hk, D))
        M, N, K, pad = size(9000), size(9000), size(9000), rng.choice([0, 0, 1, 8])
        p = linear(dtype=rng.randint(1, 2), activation=rng.randint(0, 3), m=M, n=N, k=K)
        p.x_stride = p.dx_stride = K + pad
        p.w_stride = p.y_stride = p.z_stride = p.dy_stride = p.dw_stride = p.residual_stride = N + pad
        for fn, back, n in ((lib.pnerf_linear, 0, 6), (lib.pnerf_linear_backward, 1, 7)):
            _takes(lib, fn, p, n, lambda b: lib.pnerf_linear_workspace(C.byref(p), back, C.byref(b)), (back, M, N, K, pad))
