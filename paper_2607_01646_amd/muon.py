"""Python binding of the orthogonalised optimizer step (include/ckpt_muon.h).
Argument marshalling only, as in `ops`, whose notes on streams and allocations
hold here too.

    ck.wait_captured(snap, lo, hi)                    # the gate, for these matrices' fragments
    ckpt_muon(params, masters, momentums, grads, lr=3e-4, weight_decay=0.1)
    x, = ckpt_orthogonalize([update])                 # the orthogonalisation alone
"""
import ctypes as C
import math

import torch

from .ckpt import CKPT_OK, _native_module, lib
from .ops import CKPT_TYPE_F32, _check, _handle, _listed, _on, _plain, _rows, _type

__all__ = ["ckpt_matrix", "ckpt_muon", "ckpt_muon_args", "ckpt_muon_matrix", "ckpt_newton_schulz", "ckpt_orthogonalize"]

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class ckpt_newton_schulz(C.Structure):
    _fields_ = [("steps", C.c_uint32), ("reserved", C.c_uint32), ("a", C.c_double), ("b", C.c_double),
                ("c", C.c_double), ("eps", C.c_double), ("piece_bytes", C.c_uint64)]


class ckpt_matrix(C.Structure):
    _fields_ = [("input", C.c_void_p), ("in_stride", C.c_uint64), ("out", C.c_void_p), ("out_stride", C.c_uint64),
                ("rows", C.c_uint64), ("cols", C.c_uint64)]


class ckpt_muon_matrix(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("momentum", C.c_void_p), ("grad", C.c_void_p),
                ("rows", C.c_uint64), ("cols", C.c_uint64), ("scale", C.c_double)]


class ckpt_muon_args(C.Structure):
    _fields_ = [("param_dtype", C.c_uint32), ("grad_dtype", C.c_uint32), ("nesterov", C.c_uint32),
                ("reserved", C.c_uint32), ("lr", C.c_double), ("momentum", C.c_double), ("weight_decay", C.c_double),
                ("grad_scale", C.c_void_p), ("ns", ckpt_newton_schulz)]


_lib = None
_native = None
_RULES = {"rms": 0, "spectral": 1}
_NAMES = ("param", "master", "momentum", "grad")


def _module():
    """(the native module or None, addresses of the entry points)."""
    global _native
    if _native is None:
        L = _ops()
        _native = (_native_module(), [C.cast(getattr(L, n), C.c_void_p).value for n in
                                      ("ckpt_orthogonalize_workspace", "ckpt_orthogonalize", "ckpt_muon_workspace",
                                       "ckpt_muon")])
    return _native


def _ops():
    global _lib
    if _lib is None:
        L = lib()
        vp, u64, u32, i32, P = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int32, C.POINTER
        sig = {
            "ckpt_orthogonalize_workspace": [P(ckpt_matrix), u32, P(ckpt_newton_schulz), P(u64)],
            "ckpt_orthogonalize": [P(ckpt_matrix), u32, u32, P(ckpt_newton_schulz), i32, vp, u64, vp],
            "ckpt_muon_workspace": [P(ckpt_muon_matrix), u32, P(ckpt_muon_args), P(u64)],
            "ckpt_muon": [P(ckpt_muon_matrix), u32, P(ckpt_muon_args), i32, vp, u64, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = i32
        _lib = L
    return _lib


def _ns(steps, coefficients, eps, piece_bytes):
    a, b, c = coefficients
    if not 0 <= steps <= 64:
        raise ValueError("%r steps: 1 to 64" % (steps,))
    return ckpt_newton_schulz(steps, 0, a, b, c, eps, piece_bytes)


def _scale(scale, rows, cols):
    if scale == "rms":
        return 0.2 * math.sqrt(max(rows, cols))
    if scale == "spectral":
        return math.sqrt(max(1.0, rows / cols)) if cols else 1.0
    if isinstance(scale, str):
        raise ValueError("scale is 'rms', 'spectral' or a number, not %r" % scale)
    return float(scale)


def ckpt_orthogonalize(matrices, steps=5, coefficients=COEFFICIENTS, eps=1e-7, piece_bytes=0, out=None, stream=None):
    """The matrices (one type, bf16 or fp32; rows of any spacing) with their
    singular values taken to about 1: each is divided by its 2-norm + eps and
    goes `steps` times through a x + b x^3 + c x^5 of its singular values.  A
    list of new tensors, or `out` (which may be the matrices themselves).
    piece_bytes bounds the workspace (0 = 4 GiB, at least one matrix's)."""
    matrices = _listed(matrices)
    native, at = _native or _module()
    if native is not None and out is None and matrices and isinstance(matrices[0], torch.Tensor) and matrices[0].is_cuda:
        a, b, c = coefficients
        with _on(stream, matrices[0]):
            got = native.orthogonalize(at[0], at[1], matrices, steps, a, b, c, eps, piece_bytes, _handle(stream, matrices[0]))
        if got is not None:
            if got[0] != CKPT_OK:
                _check(got[0])
            return got[1]
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    ns = _ns(steps, coefficients, eps, piece_bytes)
    if out is not None:
        out = _listed(out)
        if len(out) != len(matrices):
            raise ValueError("%d matrices, %d results" % (len(matrices), len(out)))
    if not matrices:
        return [] if out is None else out
    kind = _type(matrices[0], "matrix 0")
    device = matrices[0].device
    arr = (ckpt_matrix * len(matrices))()
    with _on(stream, matrices[0]):
        results = []
        for i, t in enumerate(matrices):
            if _type(t, "matrix %d" % i) != kind or t.dim() != 2 or t.device != device:
                raise ValueError("matrix %d is %s %s on %s" % (i, t.dtype, tuple(t.shape), t.device))
            x = torch.empty(t.shape, dtype=t.dtype, device=device) if out is None else out[i]
            if _type(x, "result %d" % i) != kind or x.shape != t.shape or x.device != device:
                raise ValueError("result %d is %s %s on %s" % (i, x.dtype, tuple(x.shape), x.device))
            results.append(x)
            a = arr[i]
            a.rows, a.cols = t.shape
            if t.numel():
                a.input, a.out = t.data_ptr(), x.data_ptr()
                a.in_stride, a.out_stride = _rows(t, "matrix %d" % i)[2], _rows(x, "result %d" % i)[2]
        L, need = _ops(), C.c_uint64()
        _check(L.ckpt_orthogonalize_workspace(arr, len(matrices), C.byref(ns), C.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(L.ckpt_orthogonalize(arr, len(matrices), kind, C.byref(ns), device.index, work.data_ptr(), need.value,
                                    _handle(stream, matrices[0])))
    return results if out is None else out


def ckpt_muon(params, masters, momentums, grads, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale="rms",
              steps=5, coefficients=COEFFICIENTS, eps=1e-7, grad_scale=None, piece_bytes=0, stream=None):
    """The step of matrices whose update is orthogonalised, in place and list
    by list: fp32 masters and momentums, params (bf16, or fp32 in full
    precision) rounded from the masters, grads (bf16 or fp32).  A parameter of
    more than 2 dimensions is the matrix of its first one; the others have its
    shape or are flat.  `scale` multiplies lr: 'rms' 0.2 sqrt(max(rows, cols)),
    which makes an update about as large as AdamW's; 'spectral'
    sqrt(max(1, rows / cols)); or a number.  One list may be a bucket, behind
    Checkpointer.wait_captured of the same range on the same stream."""
    params, masters, momentums, grads = map(_listed, (params, masters, momentums, grads))
    native, at = _native or _module()
    if native is not None and params and isinstance(params[0], torch.Tensor) and params[0].is_cuda and \
            (scale in _RULES if isinstance(scale, str) else isinstance(scale, float)):
        a, b, c = coefficients
        with _on(stream, params[0]):
            rc = native.muon(at[2], at[3], params, masters, momentums, grads, lr, momentum, nesterov, weight_decay,
                             _RULES.get(scale, 2), 0.0 if isinstance(scale, str) else scale, steps, a, b, c, eps,
                             grad_scale, piece_bytes, _handle(stream, params[0]))
        if rc is not None:
            if rc != CKPT_OK:
                _check(rc)
            return
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    lists = (params, masters, momentums, grads)
    n = len(params)
    if any(len(x) != n for x in lists):
        raise ValueError("lists of %s matrices" % ", ".join(str(len(x)) for x in lists))
    ns = _ns(steps, coefficients, eps, piece_bytes)
    if n == 0:
        return
    pt, gt = _type(params[0], "param 0"), _type(grads[0], "grad 0")
    kinds = (pt, CKPT_TYPE_F32, CKPT_TYPE_F32, gt)
    device = params[0].device
    arr = (ckpt_muon_matrix * n)()
    for i, row in enumerate(zip(*lists)):
        shape = row[0].shape
        if row[0].dim() < 2:
            raise ValueError("param %d is no matrix: %s" % (i, tuple(shape)))
        for t, kind, name in zip(row, kinds, _NAMES):
            if _type(t, "%s %d" % (name, i)) != kind or t.numel() != shape.numel() or not t.is_contiguous() or \
                    (t.shape != shape and t.dim() != 1) or t.device != device:
                raise ValueError("%s %d: %s %s, strides %s, on %s" % (name, i, t.dtype, tuple(t.shape), t.stride(), t.device))
            if shape.numel():
                setattr(arr[i], name, t.data_ptr())
        arr[i].rows, arr[i].cols = shape[0], shape[1:].numel()
        arr[i].scale = _scale(scale, arr[i].rows, arr[i].cols)
    args = ckpt_muon_args(pt, gt, bool(nesterov), 0, lr, momentum, weight_decay,
                          _plain(grad_scale, "grad_scale", torch.float32, 1) if grad_scale is not None else None, ns)
    with _on(stream, params[0]):
        L, need = _ops(), C.c_uint64()
        _check(L.ckpt_muon_workspace(arr, n, C.byref(args), C.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(L.ckpt_muon(arr, n, C.byref(args), device.index, work.data_ptr(), need.value, _handle(stream, params[0])))

