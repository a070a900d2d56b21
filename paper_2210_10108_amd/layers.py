"""Python binding of the layer operators (C ABI in include/pnerf_layers.h).

Argument marshalling only, as in `pnerf`: every operator runs in libpnerf.so,
torch provides device memory and the stream.  Tensors may have any strides as
long as their last dimension is contiguous; outputs that are not passed in are
torch.empty_like their input where they have its shape, else contiguous.  A call
enqueues its kernels on `stream` (default: the device's current stream) and
returns.  Outputs and workspaces that it allocates are torch's memory of that
stream, and inputs used on another stream than the current one are recorded on
it, so tensors may be dropped while the work is queued; what the streams wait
for is the caller's, as everywhere in torch.  No call makes an autograd graph,
whatever requires_grad says: every operator has its *_backward function.
"""
from __future__ import annotations

import ctypes as C
import math

from . import pnerf

F32, F16, BF16 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


class AttentionParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("batch", C.c_int32), ("q_rows", C.c_int32),
                ("kv_rows", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("scale", C.c_float),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3),
                ("do_stride", C.c_int64 * 3), ("dq_stride", C.c_int64 * 3),
                ("dk_stride", C.c_int64 * 3), ("dv_stride", C.c_int64 * 3),
                ("q_len", C.c_void_p), ("kv_len", C.c_void_p), ("kv_mask", C.c_void_p),
                ("kv_mask_stride", C.c_int64)]


class NormRotateParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("q_rows", C.c_int32), ("k_rows", C.c_int32),
                ("q_heads", C.c_int32), ("k_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("n_positions", C.c_int32),
                ("eps", C.c_float),
                ("q_stride", C.c_int64 * 2), ("k_stride", C.c_int64 * 2),
                ("q_out_stride", C.c_int64 * 2), ("k_out_stride", C.c_int64 * 2),
                ("dq_out_stride", C.c_int64 * 2), ("dk_out_stride", C.c_int64 * 2),
                ("dq_stride", C.c_int64 * 2), ("dk_stride", C.c_int64 * 2),
                ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("table", C.c_void_p),
                ("q_pos", C.c_void_p), ("k_pos", C.c_void_p)]


class LinearParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("activation", C.c_int32), ("m", C.c_int32),
                ("n", C.c_int32), ("k", C.c_int32),
                ("x_stride", C.c_int64), ("w_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("y_stride", C.c_int64), ("z_stride", C.c_int64), ("dy_stride", C.c_int64),
                ("dx_stride", C.c_int64), ("dw_stride", C.c_int64)]


_P, _I64, _I32 = C.c_void_p, C.c_int64, C.c_int32
# name -> argtypes; every function declared in include/pnerf_layers.h (each returns a status)
_SIGS = {
    "pnerf_cross_attention_workspace": [_P, _I32, _P],
    "pnerf_cross_attention": [_P] * 7 + [_I64, _P],
    "pnerf_cross_attention_backward": [_P] * 11 + [_I64, _P],
    "pnerf_norm_rotate": [_P] * 6,
    "pnerf_norm_rotate_workspace": [_P, _P],
    "pnerf_norm_rotate_backward": [_P] * 10 + [_I64, _P],
    "pnerf_linear_workspace": [_P, _I32, _P],
    "pnerf_linear": [_P] * 8 + [_I64, _P],
    "pnerf_linear_backward": [_P] * 9 + [_I64, _P],
}

_lib = None


def lib() -> C.CDLL:
    """libpnerf.so with the signatures of the layer operators."""
    global _lib
    if _lib is None:
        L = pnerf.lib()
        for name, args in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = C.c_int
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != pnerf.OK:
        raise pnerf.PnerfError(status, lib().pnerf_last_error().decode())


class _Call:
    """One call: its device, data type and stream.  (A call takes about 10 us of
    the host's time, more than the smallest take on the device: what is usual is
    looked at first, and told apart only where it is not.)"""
    __slots__ = ("index", "dtype", "code", "stream", "raw")

    def __init__(self, first, stream):
        import torch
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            raise TypeError("operands must be device tensors")
        self.index, self.dtype = first.get_device(), first.dtype
        self.code = _dtypes().get(self.dtype)
        if self.code is None:
            raise TypeError(f"unsupported data type {self.dtype}")
        current = torch._C._cuda_getCurrentRawStream(self.index)
        self.stream, self.raw = None, current  # stream: only where it is another one
        if stream is not None:
            if stream.device.index != self.index:
                raise ValueError(f"stream on {stream.device}, tensors on cuda:{self.index}")
            if stream.cuda_stream != current:
                self.stream, self.raw = stream, stream.cuda_stream

    def tensor(self, t, name, shape, dtype=None, contiguous=False):
        """Checks a tensor and returns its address (None for None)."""
        if t is None:
            return None
        if t.dtype is not (dtype or self.dtype):
            raise TypeError(f"{name} must be {dtype or self.dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.get_device() != self.index:  # -1 on the host
            raise TypeError(f"{name} must be on cuda:{self.index}")
        if not t.is_contiguous():
            if contiguous:
                raise ValueError(f"{name} must be contiguous")
            if t.stride(-1) != 1 and shape[-1] > 1:
                raise ValueError(f"the last dimension of {name} must be contiguous")
        if self.stream is not None:
            t.record_stream(self.stream)
        return t.data_ptr()

    def new(self, like, shape=None, dtype=None):
        """An output (as `like`, or of another shape) or workspace: memory of the
        call's stream, which the current one may read as well."""
        import torch
        if self.stream is None:
            return torch.empty_like(like) if shape is None else like.new_empty(shape, dtype=dtype)
        with torch.cuda.stream(self.stream):
            t = torch.empty_like(like) if shape is None else like.new_empty(shape, dtype=dtype)
        t.record_stream(torch.cuda.current_stream(self.index))
        return t

    def out(self, t, like, name, strides):
        """The output t, or one like `like`; its strides go into the call's params."""
        if t is None:
            t = self.new(like)
            at = t.data_ptr()
        else:
            at = self.tensor(t, name, like.shape)
        if strides is not None:
            strides[:] = t.stride()[:-1]
        return t, at

    def workspace(self, like, nbytes):
        """(address, bytes, the tensor) of a workspace."""
        if not nbytes:
            return None, 0, None
        import torch
        t = self.new(like, (nbytes,), torch.uint8)
        return t.data_ptr(), nbytes, t

    def run(self, fn, *args):
        import torch
        if torch._C._cuda_getDevice() == self.index:
            status = fn(*args, self.raw)
        else:
            with torch.cuda.device(self.index):
                status = fn(*args, self.raw)
        if status != pnerf.OK:
            _check(status)


_DTYPES = None


def _dtypes():
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
    return _DTYPES


# ---------------------------------------------------------------- attention
def _attention(call, q, k, v, q_len, kv_len, kv_mask, scale):
    import torch
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must have 4 dimensions: batch, rows, heads, head width")
    B, Sq, Hq, D = q.shape
    Sk, Hkv = k.shape[1:3]
    p = AttentionParams()
    p.dtype, p.batch, p.q_rows, p.kv_rows = call.code, B, Sq, Sk
    p.q_heads, p.kv_heads, p.head_dim = Hq, Hkv, D
    p.scale = (1.0 / math.sqrt(D) if D else 1.0) if scale is None else scale
    p.q_stride[:] = q.stride()[:3]
    p.k_stride[:] = k.stride()[:3]
    p.v_stride[:] = v.stride()[:3]
    p.q_len = call.tensor(q_len, "q_len", (B,), torch.int32, True)
    p.kv_len = call.tensor(kv_len, "kv_len", (B,), torch.int32, True)
    if kv_mask is not None:
        if kv_mask.dtype not in (torch.bool, torch.uint8):
            raise TypeError(f"kv_mask must be torch.bool or torch.uint8, got {kv_mask.dtype}")
        p.kv_mask = call.tensor(kv_mask, "kv_mask", (B, Sk), kv_mask.dtype)
        p.kv_mask_stride = kv_mask.stride(0)
    kv = (B, Sk, Hkv, D)
    return p, call.tensor(q, "q", q.shape), call.tensor(k, "k", kv), call.tensor(v, "v", kv)


def cross_attention(q, k, v, q_len=None, kv_len=None, kv_mask=None, scale=None, o=None,
                    return_lse: bool = False, stream=None):
    """pnerf_cross_attention.  q [B, Sq, Hq, D], k and v [B, Sk, Hkv, D] (float16
    or bfloat16, Hq a multiple of Hkv, D at most 128); q_len and kv_len int32 [B];
    kv_mask bool or uint8 [B, Sk], nonzero where a key may be read; scale defaults
    to 1 / sqrt(D).  Returns o [B, Sq, Hq, D], or (o, lse) with lse float32
    [B, Hq, Sq], which the backward pass needs."""
    import torch
    call = _Call(q, stream)
    p, qp, kp, vp = _attention(call, q, k, v, q_len, kv_len, kv_mask, scale)
    o, op = call.out(o, q, "o", p.o_stride)
    lse = lp = None
    if return_lse:
        lse = call.new(q, (p.batch, p.q_heads, p.q_rows), torch.float32)
        lp = lse.data_ptr()
    n = C.c_int64()
    ref = C.byref(p)
    _check(lib().pnerf_cross_attention_workspace(ref, 0, C.byref(n)))
    ws, nb, _keep = call.workspace(q, n.value)
    call.run(_lib.pnerf_cross_attention, ref, qp, kp, vp, op, lp, ws, nb)
    return (o, lse) if return_lse else o


def cross_attention_backward(do, q, k, v, o, lse, q_len=None, kv_len=None, kv_mask=None, scale=None,
                             dq=None, dk=None, dv=None, stream=None):
    """pnerf_cross_attention_backward: (dq, dk, dv) for do = dL/do, with o and lse
    as cross_attention(..., return_lse=True) gave them and its other arguments."""
    import torch
    call = _Call(q, stream)
    p, qp, kp, vp = _attention(call, q, k, v, q_len, kv_len, kv_mask, scale)
    op, dop = call.tensor(o, "o", q.shape), call.tensor(do, "do", q.shape)
    lp = call.tensor(lse, "lse", (p.batch, p.q_heads, p.q_rows), torch.float32, True)
    p.o_stride[:], p.do_stride[:] = o.stride()[:3], do.stride()[:3]
    dq, dqp = call.out(dq, q, "dq", p.dq_stride)
    dk, dkp = call.out(dk, k, "dk", p.dk_stride)
    dv, dvp = call.out(dv, v, "dv", p.dv_stride)
    n = C.c_int64()
    ref = C.byref(p)
    _check(lib().pnerf_cross_attention_workspace(ref, 1, C.byref(n)))
    ws, nb, _keep = call.workspace(q, n.value)
    call.run(_lib.pnerf_cross_attention_backward, ref, qp, kp, vp, op, lp, dop, dqp, dkp, dvp, ws, nb)
    return dq, dk, dv


# ---------------------------------------------------------------- norm and rotation
def _norm(call, q, k, q_weight, k_weight, table, q_pos, k_pos, eps, interleaved):
    import torch
    p = NormRotateParams()
    p.dtype, p.eps, p.interleaved = call.code, eps, int(interleaved)
    p.head_dim = D = q.shape[-1]
    if table is not None:
        if table.dim() != 3 or table.shape[1] != 2:
            raise ValueError(f"table has shape {tuple(table.shape)}, expected (positions, 2, pairs)")
        p.n_positions, p.rotary_dim = table.shape[0], 2 * table.shape[2]
        p.table = call.tensor(table, "table", table.shape, torch.float32, True)
    if q.dim() != 3:
        raise ValueError("q must have 3 dimensions: rows, heads, head width")
    qp = call.tensor(q, "q", q.shape)
    p.q_rows, p.q_heads, _ = q.shape
    p.q_stride[:] = q.stride()[:2]
    p.q_weight = call.tensor(q_weight, "q_weight", (D,), None, True)
    p.q_pos = call.tensor(q_pos, "q_pos", q.shape[:1], torch.int32, True)
    if k is None:
        return p, qp, None
    if k.dim() != 3 or k.shape[2] != D:
        raise ValueError(f"k has shape {tuple(k.shape)}, expected (rows, heads, {D})")
    kp = call.tensor(k, "k", k.shape)
    p.k_rows, p.k_heads, _ = k.shape
    p.k_stride[:] = k.stride()[:2]
    p.k_weight = call.tensor(k_weight, "k_weight", (D,), None, True)
    p.k_pos = call.tensor(k_pos, "k_pos", k.shape[:1], torch.int32, True)
    return p, qp, kp


def norm_rotate(q, k, q_weight, k_weight, table, q_pos, k_pos, eps: float = 1e-6,
                interleaved: bool = False, q_out=None, k_out=None, stream=None):
    """pnerf_norm_rotate.  q [Tq, Hq, D] and k [Tk, Hk, D] (or k None: queries
    alone), weights [D] or None; table float32 [positions, 2, pairs] (cosines,
    sines) or None (no rotation), positions int32 [Tq] and [Tk].  Returns
    (q_out, k_out); an output may be its input."""
    call = _Call(q, stream)
    p, qp, kp = _norm(call, q, k, q_weight, k_weight, table, q_pos, k_pos, eps, interleaved)
    q_out, qo = call.out(q_out, q, "q_out", p.q_out_stride)
    ko = None
    if k is None:
        k_out = None
    else:
        k_out, ko = call.out(k_out, k, "k_out", p.k_out_stride)
    call.run(lib().pnerf_norm_rotate, C.byref(p), qp, kp, qo, ko)
    return q_out, k_out


def norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, table, q_pos, k_pos,
                         eps: float = 1e-6, interleaved: bool = False, dq=None, dk=None, stream=None):
    """pnerf_norm_rotate_backward: (dq, dk, dq_weight, dk_weight) for the
    gradients of the outputs; dk and dk_weight are None where k is, a weight's
    gradient where the weight is.  dq may be dq_out, dk may be dk_out."""
    call = _Call(q, stream)
    p, qp, kp = _norm(call, q, k, q_weight, k_weight, table, q_pos, k_pos, eps, interleaved)

    gq, gk, dkp, dqw, dkw, wqp, wkp = call.tensor(dq_out, "dq_out", q.shape), *(None,) * 6
    p.dq_out_stride[:] = dq_out.stride()[:2]
    dq, dqp = call.out(dq, q, "dq", p.dq_stride)
    if q_weight is not None:
        dqw, wqp = call.out(None, q_weight, "", None)
    if k is None:
        dk = None
    else:
        gk = call.tensor(dk_out, "dk_out", k.shape)
        p.dk_out_stride[:] = dk_out.stride()[:2]
        dk, dkp = call.out(dk, k, "dk", p.dk_stride)
        if k_weight is not None:
            dkw, wkp = call.out(None, k_weight, "", None)
    n = C.c_int64()
    ref = C.byref(p)
    _check(lib().pnerf_norm_rotate_workspace(ref, C.byref(n)))
    ws, nb, _keep = call.workspace(q, n.value)
    call.run(_lib.pnerf_norm_rotate_backward, ref, qp, kp, gq, gk, dqp, dkp, wqp, wkp, ws, nb)
    return dq, dk, dqw, dkw


# ---------------------------------------------------------------- linear
def _linear(call, x, w, activation):
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x and w must have 2 dimensions")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation {activation!r}: one of {', '.join(ACTIVATIONS)}")
    (M, K), N = x.shape, w.shape[1]
    p = LinearParams()
    p.dtype, p.activation, p.m, p.n, p.k = call.code, ACTIVATIONS[activation], M, N, K
    p.x_stride, p.w_stride = x.stride(0), w.stride(0)
    return p, call.tensor(x, "x", (M, K)), call.tensor(w, "w", (K, N))


def linear(x, w, bias=None, residual=None, activation: str = "none", y=None,
           return_preact: bool = False, stream=None):
    """pnerf_linear: act(x @ w + bias) + residual for x [M, K], w [K, N] (float16
    or bfloat16), bias [N], residual [M, N]; activation "none", "relu", "gelu"
    or "silu".  y may be the residual.  Returns y, or (y, z) with
    return_preact, z = x @ w + bias as linear_backward takes it."""
    call = _Call(x, stream)
    p, xp, wp = _linear(call, x, w, activation)
    shape = (p.m, p.n)
    bp = call.tensor(bias, "bias", (p.n,), None, True)
    rp = call.tensor(residual, "residual", shape)
    if residual is not None:
        p.residual_stride = residual.stride(0)
    if y is None:
        y = call.new(x, shape)
        yp, p.y_stride = y.data_ptr(), p.n
    else:
        yp, p.y_stride = call.tensor(y, "y", shape), y.stride(0)
    z = zp = None
    if return_preact:
        z = call.new(x, shape)
        zp, p.z_stride = z.data_ptr(), p.n
    n = C.c_int64()
    ref = C.byref(p)
    _check(lib().pnerf_linear_workspace(ref, 0, C.byref(n)))
    ws, nb, _keep = call.workspace(x, n.value)
    call.run(_lib.pnerf_linear, ref, xp, wp, bp, rp, yp, zp, ws, nb)
    return (y, z) if return_preact else y


def linear_backward(dy, x, w, z=None, activation: str = "none", bias: bool = True, dx=None, dw=None,
                    stream=None):
    """pnerf_linear_backward: (dx, dw, db) for dy = dL/dy; db is None without
    bias.  z as linear(..., return_preact=True) gave it (None will do when the
    activation is "none").  The residual's gradient is dy itself."""
    call = _Call(x, stream)
    p, xp, wp = _linear(call, x, w, activation)
    shape = (p.m, p.n)
    gp = call.tensor(dy, "dy", shape)
    p.dy_stride = dy.stride(0)
    zp = call.tensor(z, "z", shape)
    if z is not None:
        p.z_stride = z.stride(0)
    dx, dxp = call.out(dx, x, "dx", None)
    dw, dwp = call.out(dw, w, "dw", None)
    p.dx_stride, p.dw_stride = dx.stride(0), dw.stride(0)
    db = call.new(x, (p.n,)) if bias else None
    dbp = None if db is None else db.data_ptr()
    n = C.c_int64()
    ref = C.byref(p)
    _check(lib().pnerf_linear_workspace(ref, 1, C.byref(n)))
    ws, nb, _keep = call.workspace(x, n.value)
    call.run(_lib.pnerf_linear_backward, ref, xp, wp, zp, gp, dxp, dwp, dbp, ws, nb)
    return dx, dw, db
