"""Python binding of the transformer operators of liberase.so (the C ABI in
include/erase_ops.h): rotary positions, layer norm and dropout, each with its
backward pass, on device tensors.

Argument marshalling only: every operator runs in the HIP kernels behind the C
ABI; PyTorch provides device memory and streams.  There is no fallback and no
autograd: the backward passes are calls of their own.  Each function enqueues
on ``stream`` (a torch stream of the tensors' device; default: that device's
current stream), returns without waiting, and allocates the outputs that
``out`` does not give.  Inputs written on another stream, and outputs read on one,
are ordered by the caller, as with torch's own operations.
"""
from __future__ import annotations

import ctypes
import struct
from ctypes import POINTER, c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from . import erase
from .erase import BF16, ERR_INVALID_ARG, ERR_SHAPE, ERR_WORKSPACE, F32, OK, EraseError

LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "by_parts": 3}


class RopeSpec(ctypes.Structure):
    """erase_rope_spec: which frequencies a table holds."""
    _fields_ = [("rot_dim", c_int32), ("scaling", c_int32), ("base", c_double), ("factor", c_double),
                ("original_length", c_double), ("fast", c_double), ("slow", c_double)]


class RopeConfig(ctypes.Structure):
    """erase_rope_config: shape of one rotation."""
    _fields_ = [("dtype", c_int32), ("layout", c_int32), ("batch", c_int32), ("seq", c_int32), ("q_heads", c_int32),
                ("k_heads", c_int32), ("head_dim", c_int32), ("rot_dim", c_int32), ("q_stride", c_int64 * 3),
                ("k_stride", c_int64 * 3), ("qo_stride", c_int64 * 3), ("ko_stride", c_int64 * 3),
                ("pos_stride", c_int64), ("start", c_int64)]


class NormConfig(ctypes.Structure):
    """erase_norm_config: shape of a layer norm and its backward pass."""
    _fields_ = [("rows", c_int64), ("cols", c_int32), ("dtype", c_int32), ("eps", c_float), ("x_ld", c_int64),
                ("y_ld", c_int64), ("dy_ld", c_int64), ("dx_ld", c_int64), ("res_ld", c_int64)]


class DropoutConfig(ctypes.Structure):
    """erase_dropout_config: shape, probability and place in the random stream."""
    _fields_ = [("rows", c_int64), ("cols", c_int64), ("dtype", c_int32), ("p", c_double), ("seed", c_uint64),
                ("offset", c_uint64), ("x_ld", c_int64), ("res_ld", c_int64), ("y_ld", c_int64)]


# The same three as packed bytes, for the calls themselves: a Structure with its
# arrays costs 2 us more than one pack, of 8 to 12 us for a whole call.
_ROPE, _NORM, _DROPOUT = struct.Struct("8i14q"), struct.Struct("qiif5q"), struct.Struct("qqidQQ3q")
_UNPACKABLE = (struct.error, OverflowError)  # a number that its field does not hold
assert (_ROPE.size, _NORM.size, _DROPOUT.size) == tuple(map(ctypes.sizeof, (RopeConfig, NormConfig, DropoutConfig)))

# every entry point of include/erase_ops.h with its ctypes signature
SIGNATURES = {
    "erase_rope_frequencies": (c_int32, [POINTER(RopeSpec), POINTER(c_double), POINTER(c_double)]),
    "erase_rope_table_bytes": (c_int32, [POINTER(RopeSpec), POINTER(c_size_t)]),
    "erase_rope_table": (c_int32, [POINTER(RopeSpec), c_void_p, c_void_p]),
    "erase_rope": (c_int32, [c_void_p] * 8),
    "erase_rope_backward": (c_int32, [c_void_p] * 8),
    "erase_layer_norm": (c_int32, [c_void_p] * 8),
    "erase_layer_norm_backward_scratch_bytes": (c_int32, [c_void_p, POINTER(c_size_t)]),
    "erase_layer_norm_backward": (c_int32, [c_void_p] * 11 + [c_size_t, c_void_p]),
    "erase_dropout": (c_int32, [c_void_p] * 6),
    "erase_dropout_backward": (c_int32, [c_void_p] * 5),
}

_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = erase.lib()
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise EraseError(status, where)


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
# the raw handle and number behind torch.cuda.current_stream() and current_device(), without an object a call
_current_stream = (getattr(torch._C, "_cuda_getCurrentRawStream", None)
                   or (lambda d: torch.cuda.current_stream(d).cuda_stream))
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _dtype(where: str, name: str, t) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise EraseError(ERR_INVALID_ARG, where, f"{name} must be float32 or bfloat16")
    return dt


def _on(where: str, *tensors) -> int:
    """The GPU that holds every tensor (None: not given)."""
    dev = tensors[0].get_device()
    if dev < 0:
        raise EraseError(ERR_INVALID_ARG, where, "tensors must be on the GPU")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise EraseError(ERR_INVALID_ARG, where, "tensors are on different devices")
    return dev


def _like(where: str, name: str, t, dtype, shape):
    if t.dtype != dtype or t.shape != shape:
        raise EraseError(ERR_SHAPE if t.dtype == dtype else ERR_INVALID_ARG, where,
                         f"{name} must have the type {dtype} and the shape {list(shape)}")


def _vector(where: str, name: str, t, n: int):
    if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous()):
        raise EraseError(ERR_INVALID_ARG, where, f"{name} must be a contiguous float32 tensor of {n}")


def _run(where: str, fn, dev: int, stream, *args):
    """fn(*args, stream handle) with dev as the current device."""
    if stream is None:
        handle = _current_stream(dev)
    elif stream.device.index == dev:
        handle = stream.cuda_stream
    else:
        raise EraseError(ERR_INVALID_ARG, where, "stream is not one of the tensors' GPU")
    if dev == _current_device():
        status = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, handle)
    if status != OK:
        raise EraseError(status, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _empty(shape, dtype, device, stream):
    """Memory of the stream that will use it: a block of another stream's could
    still be read or written there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def _rope_spec(rot_dim, base, scaling, factor, original_length, fast, slow) -> RopeSpec:
    if scaling not in SCALINGS:
        raise EraseError(ERR_INVALID_ARG, "rope", f"scaling must be one of {sorted(SCALINGS)}")
    return spec_of("rope", rot_dim, SCALINGS[scaling], base, factor, original_length, fast, slow)


def spec_of(where, rot_dim, scaling, base, factor, original_length, fast, slow) -> RopeSpec:
    """An erase_rope_spec of numbers (its field would take rot_dim modulo 2^32)."""
    if not -1 << 31 <= rot_dim < 1 << 31:
        raise EraseError(ERR_SHAPE, where, "rot_dim must be even, 2..1024")
    return RopeSpec(rot_dim, scaling, base, factor, original_length, fast, slow)


def rope_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_length=0.0, fast=32.0, slow=1.0):
    """(angles per position of the rot_dim / 2 pairs, amplitude) on the host (erase_rope_frequencies)."""
    spec = _rope_spec(rot_dim, base, scaling, factor, original_length, fast, slow)
    n, amp = c_size_t(0), c_double(0)
    _check(lib().erase_rope_table_bytes(ctypes.byref(spec), ctypes.byref(n)), "erase_rope_frequencies")
    freq = (c_double * (rot_dim // 2))()
    _check(lib().erase_rope_frequencies(ctypes.byref(spec), freq, ctypes.byref(amp)), "erase_rope_frequencies")
    return list(freq), amp.value


class RopeTable:
    """A device table of erase_rope_table: read only, for any number of calls."""

    def __init__(self, spec: RopeSpec, data):
        if data.dtype != torch.int64 or data.numel() < spec.rot_dim // 2 + 1 or not data.is_contiguous():
            raise EraseError(ERR_INVALID_ARG, "RopeTable", "data must be rot_dim / 2 + 1 contiguous int64")
        self.rot_dim, self.data = spec.rot_dim, data


def rope_table(rot_dim, base=10000.0, scaling="none", factor=1.0, original_length=0.0, fast=32.0, slow=1.0, device=None,
               stream=None) -> RopeTable:
    """The table of a rotation (erase_rope_spec's fields) on `device` (default: the
    current GPU), filled on `stream`.  As with any tensor, a caller who uses it on
    another stream orders that stream after this one (by an event or a
    synchronisation): the calls themselves do not wait."""
    spec = _rope_spec(rot_dim, base, scaling, factor, original_length, fast, slow)
    n = c_size_t(0)
    _check(lib().erase_rope_table_bytes(ctypes.byref(spec), ctypes.byref(n)), "erase_rope_table_bytes")
    dev = None if device is None else torch.device(device)
    if dev is not None and dev.type != "cuda":  # the fill would write to a host address
        raise EraseError(ERR_INVALID_ARG, "erase_rope_table", "device must be a GPU")
    if not torch.cuda.is_available():
        raise RuntimeError("no HIP device available: the operators run only on the GPU")
    if dev is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    data = _empty(n.value // 8, torch.int64, dev, stream)
    _run("erase_rope_table", lib().erase_rope_table, data.get_device(), stream, ctypes.byref(spec), data.data_ptr())
    return RopeTable(spec, data)


def _heads(where, name, t):
    """Strides of [batch][seq][heads][head_dim] with contiguous columns."""
    st = t.stride()
    if len(st) != 4 or (st[3] != 1 and t.shape[3] > 1):
        raise EraseError(ERR_SHAPE, where, f"{name} must be [batch][seq][heads][head_dim] with contiguous columns")
    return st


def _rotate(where, fn, q, k, table, positions, start, layout, out, stream):
    lay = LAYOUTS.get(layout)
    if lay is None:
        raise EraseError(ERR_INVALID_ARG, where, f"layout must be one of {sorted(LAYOUTS)}")
    qs = _heads(where, "q", q)
    B, T, Hq, D = shape = q.shape
    dt = _dtype(where, "q", q)
    Hk, ks = 0, (0, 0, 0, 0)
    if k is not None:
        ks = _heads(where, "k", k)
        Bk, Tk, Hk, Dk = kshape = k.shape
        if k.dtype != q.dtype or Bk != B or Tk != T or Dk != D:
            raise EraseError(ERR_SHAPE, where, "k must have q's type, batch, length and head size")
    pos_stride = 0
    if positions is not None:
        ps = positions.stride()
        if positions.dtype != torch.int32 or positions.shape != shape[:2] or (T > 1 and ps[1] != 1):
            raise EraseError(ERR_INVALID_ARG, where, "positions must be int32 [batch][seq] with unit stride along seq")
        pos_stride = ps[0]
    if out is None:
        qo = _empty(shape, q.dtype, q.device, stream)
        ko = None if k is None else _empty(kshape, k.dtype, k.device, stream)
    else:
        qo, ko = out
        if qo is None or (ko is None) != (k is None):
            raise EraseError(ERR_INVALID_ARG, where, "out must give a tensor exactly where there is an input")
        _like(where, "out[0]", qo, q.dtype, shape)
        if k is not None:
            _like(where, "out[1]", ko, q.dtype, kshape)
    dev = _on(where, q, k, table.data, positions, qo, ko)
    qos = _heads(where, "out[0]", qo)
    kos = ks if k is None else _heads(where, "out[1]", ko)
    try:
        cfg = _ROPE.pack(dt, lay, B, T, Hq, Hk, D, table.rot_dim, *qs[:3], *ks[:3], *qos[:3], *kos[:3], pos_stride, start)
    except _UNPACKABLE as e:
        raise EraseError(ERR_SHAPE, where, str(e)) from None
    _run(where, fn, dev, stream, cfg, q.data_ptr(), _ptr(k), qo.data_ptr(), _ptr(ko), _ptr(positions), table.data.data_ptr())
    return qo, ko


def rope(q, k, table, positions=None, start=0, layout="half", out=None, stream=None):
    """Queries q [batch][seq][heads][head_dim] and keys k (fewer heads, or None)
    rotated by their positions (erase_rope): position start + t, or `positions`
    int32 [batch][seq].  `table` is rope_table()'s; its rot_dim columns of every
    head turn, pairs (i, i + rot_dim / 2) with layout "half" and (2 i, 2 i + 1)
    with "interleaved".  Strides are free but for contiguous columns; ``out`` may
    be (q, k) themselves.  Returns (q_out, k_out)."""
    return _rotate("erase_rope", lib().erase_rope, q, k, table, positions, start, layout, out, stream)


def rope_backward(dq, dk, table, positions=None, start=0, layout="half", out=None, stream=None):
    """Gradients at q and k from those at rope()'s outputs (erase_rope_backward);
    arguments as for rope()."""
    return _rotate("erase_rope_backward", lib().erase_rope_backward, dq, dk, table, positions, start, layout, out, stream)


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------
def _matrix(where: str, name: str, t) -> int:
    """The row pitch of [rows][cols] with unit column stride."""
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and t.shape[1] > 1):
        raise EraseError(ERR_SHAPE, where, f"{name} must be [rows][cols] with unit column stride")
    return st[0]


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """Layer norm of the rows of x [rows][cols] (erase_layer_norm), weight and
    bias float32 [cols] or None.  Returns (y, mean, rstd), the float32 statistics
    [rows] for the backward pass.  ``out`` gives the three; its statistics may be
    None (not computed), its y may be x."""
    where = "erase_layer_norm"
    ld = _matrix(where, "x", x)
    dt = _dtype(where, "x", x)
    R, C = shape = x.shape
    _vector(where, "weight", weight, C)
    _vector(where, "bias", bias, C)
    if out is None:
        y = _empty((R, C), x.dtype, x.device, stream)
        mean, rstd = _empty((2, R), torch.float32, x.device, stream)
    else:
        y, mean, rstd = out
        _like(where, "out[0]", y, x.dtype, shape)
        _vector(where, "out[1]", mean, R)
        _vector(where, "out[2]", rstd, R)
    dev = _on(where, x, weight, bias, y, mean, rstd)
    try:
        cfg = _NORM.pack(R, C, dt, eps, ld, _matrix(where, "out[0]", y), 0, 0, 0)
    except _UNPACKABLE as e:
        raise EraseError(ERR_SHAPE, where, str(e)) from None
    _run(where, lib().erase_layer_norm, dev, stream, cfg, x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), _ptr(mean),
         _ptr(rstd))
    return y, mean, rstd


def _norm_scratch_bytes(cfg: bytes) -> int:
    n = c_size_t(0)
    _check(lib().erase_layer_norm_backward_scratch_bytes(cfg, ctypes.byref(n)), "erase_layer_norm_backward_scratch_bytes")
    return n.value


def layer_norm_backward_scratch(x):
    """Scratch of layer_norm_backward() for tensors of x's shape and type; one for
    every call in flight."""
    where = "erase_layer_norm_backward"
    _matrix(where, "x", x)
    try:
        cfg = _NORM.pack(x.shape[0], x.shape[1], _dtype(where, "x", x), 0.0, 0, 0, 0, 0, 0)
    except _UNPACKABLE as e:
        raise EraseError(ERR_SHAPE, where, str(e)) from None
    return torch.empty(_norm_scratch_bytes(cfg), dtype=torch.uint8, device=x.device)


def layer_norm_backward(dy, x, weight, mean, rstd, residual=None, need_input=True, need_weight=True, need_bias=True,
                        out=None, scratch=None, stream=None):
    """Gradients (dx, dweight, dbias) of layer_norm() (erase_layer_norm_backward)
    from dy and the forward's x, weight, mean and rstd; `residual` (a gradient of
    x's shape, or None) is added to dx.  What is not needed is returned as None.
    ``out`` gives the three (dx may be dy or residual), ``scratch``
    layer_norm_backward_scratch()'s memory (allocated unless given)."""
    where = "erase_layer_norm_backward"
    ld = _matrix(where, "x", x)
    dt = _dtype(where, "x", x)
    R, C = shape = x.shape
    _like(where, "dy", dy, x.dtype, shape)
    _vector(where, "weight", weight, C)
    _vector(where, "mean", mean, R)
    _vector(where, "rstd", rstd, R)
    dx, dw, db = (None, None, None) if out is None else out
    if not need_input:
        dx = None
    elif dx is None:
        dx = _empty((R, C), x.dtype, x.device, stream)
    else:
        _like(where, "out[0]", dx, x.dtype, shape)
    if not need_weight:
        dw = None
    elif dw is None:
        dw = _empty(C, torch.float32, x.device, stream)
    else:
        _vector(where, "out[1]", dw, C)
    if not need_bias:
        db = None
    elif db is None:
        db = _empty(C, torch.float32, x.device, stream)
    else:
        _vector(where, "out[2]", db, C)
    if residual is not None:
        _like(where, "residual", residual, x.dtype, shape)
    try:
        cfg = _NORM.pack(R, C, dt, 0.0, ld, 0, _matrix(where, "dy", dy),
                    0 if dx is None else _matrix(where, "out[0]", dx),
                    0 if residual is None else _matrix(where, "residual", residual))
    except _UNPACKABLE as e:
        raise EraseError(ERR_SHAPE, where, str(e)) from None
    if scratch is None:
        if need_weight or need_bias:
            scratch = _empty(_norm_scratch_bytes(cfg), torch.uint8, x.device, stream)
    elif not scratch.is_contiguous():
        raise EraseError(ERR_WORKSPACE, where, "scratch must be contiguous")
    dev = _on(where, x, dy, weight, mean, rstd, residual, dx, dw, db, scratch)
    _run(where, lib().erase_layer_norm_backward, dev, stream, cfg, x.data_ptr(), dy.data_ptr(), _ptr(weight),
         _ptr(mean), _ptr(rstd), _ptr(residual), _ptr(dx), _ptr(dw), _ptr(db), _ptr(scratch),
         0 if scratch is None else scratch.nbytes)
    return dx, dw, db


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
def _drop(where, fn, x, p, seed, offset, residual, step, out, stream):
    ld = _matrix(where, "x", x)
    dt = _dtype(where, "x", x)
    R, C = shape = x.shape
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise EraseError(ERR_INVALID_ARG, where, "seed and offset must be 64-bit unsigned numbers")
    if step is not None and (step.dtype not in (torch.int64, torch.uint64) or step.numel() != 1):
        raise EraseError(ERR_INVALID_ARG, where, "step must be one int64 or uint64 on the device")
    if out is None:
        out = _empty(shape, x.dtype, x.device, stream)
    else:
        _like(where, "out", out, x.dtype, shape)
    lr = 0
    if residual is not None:
        _like(where, "residual", residual, x.dtype, shape)
        lr = _matrix(where, "residual", residual)
    dev = _on(where, x, residual, step, out)
    try:
        cfg = _DROPOUT.pack(R, C, dt, p, seed, offset, ld, lr, _matrix(where, "out", out))
    except _UNPACKABLE as e:
        raise EraseError(ERR_SHAPE, where, str(e)) from None
    if fn == "erase_dropout":
        _run(where, lib().erase_dropout, dev, stream, cfg, x.data_ptr(), _ptr(residual), out.data_ptr(), _ptr(step))
    else:
        _run(where, lib().erase_dropout_backward, dev, stream, cfg, x.data_ptr(), out.data_ptr(), _ptr(step))
    return out


def dropout(x, p, seed, offset=0, residual=None, step=None, out=None, stream=None):
    """residual + dropout of x [rows][cols] with probability p (erase_dropout):
    the mask is a function of (seed, offset + step, row, column).  `step` is an
    int64 or uint64 [1] on the device (or None), read when the launch runs.
    ``out`` may be x or residual.  Returns y."""
    return _drop("erase_dropout", "erase_dropout", x, p, seed, offset, residual, step, out, stream)


def dropout_backward(dy, p, seed, offset=0, step=None, out=None, stream=None):
    """The gradient at dropout()'s x from that at its output, for the same p, seed,
    offset and step (erase_dropout_backward).  ``out`` may be dy."""
    return _drop("erase_dropout_backward", "erase_dropout_backward", dy, p, seed, offset, None, step, out, stream)
