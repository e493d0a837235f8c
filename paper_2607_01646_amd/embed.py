"""Python binding of the vocabulary table's lookup and gradient
(include/ckpt_embed.h).  Argument marshalling only, as in `ops`, whose notes
on streams and allocations hold here too.

    x = ckpt_embedding(table, ids, scale=dim ** 0.5)
    ...                                                  # the model: d_x from d_hidden of the head's loss
    ckpt_embedding_grad(d_x, ids, vocab, scale=dim ** 0.5, add_to=r.d_weight)   # a table that is the head, too
"""
import ctypes as C

import torch

from .ckpt import CKPT_OK, _native_module, lib
from .ops import _TYPES, _check, _handle, _on, _rows, _type

__all__ = ["ckpt_embed_args", "ckpt_embedding", "ckpt_embedding_grad"]


class ckpt_embed_args(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("table_dtype", C.c_uint32), ("tokens", C.c_uint64), ("dim", C.c_uint64),
                ("vocab", C.c_uint64), ("ids", C.c_void_p), ("ignore_index", C.c_int64), ("scale", C.c_double),
                ("rows", C.c_void_p), ("rows_stride", C.c_uint64), ("table", C.c_void_p), ("table_stride", C.c_uint64),
                ("add", C.c_uint32), ("reserved", C.c_uint32)]


_lib = None
_native = None


def _module():
    """(the native module or None, addresses of the entry points)."""
    global _native
    if _native is None:
        L = _ops()
        _native = (_native_module(), [C.cast(getattr(L, n), C.c_void_p).value for n in
                                      ("ckpt_embedding", "ckpt_embedding_grad_workspace", "ckpt_embedding_grad")])
    return _native


def _ops():
    global _lib
    if _lib is None:
        L = lib()
        vp, u64, i32, P = C.c_void_p, C.c_uint64, C.c_int32, C.POINTER
        sig = {
            "ckpt_embedding": [P(ckpt_embed_args), i32, vp],
            "ckpt_embedding_grad_workspace": [P(ckpt_embed_args), P(u64)],
            "ckpt_embedding_grad": [P(ckpt_embed_args), i32, vp, u64, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = i32
        _lib = L
    return _lib


def _ids(ids, device):
    if not isinstance(ids, torch.Tensor) or not ids.is_cuda or ids.dtype != torch.int64:
        raise ValueError("ids is not a device tensor of torch.int64")
    if not ids.is_contiguous() or ids.device != device:
        raise ValueError("ids: contiguous values on %s are wanted (strides %s, on %s)" % (device, ids.stride(), ids.device))
    return ids.data_ptr() if ids.numel() else None


def ckpt_embedding(table, ids, scale=1.0, ignore_index=-100, stream=None):
    """scale * table[ids]: rows [..., dim] of table [vocab, dim] (bf16 or fp32,
    rows of any spacing) at ids [...] (int64), rounded once.  A token whose id
    is ignore_index has a row of zeros; one with another id outside [0, vocab)
    a row of NaN."""
    native, at = _native or _module()
    if native is not None and isinstance(table, torch.Tensor) and table.is_cuda:
        with _on(stream, table):
            got = native.embedding(at[0], table, ids, scale, ignore_index, _handle(stream, table))
        if got is not None:
            if got[0] != CKPT_OK:
                _check(got[0])
            return got[1]
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    a = ckpt_embed_args()
    a.dtype = a.table_dtype = _type(table, "table")
    if table.dim() != 2:
        raise ValueError("table %s" % (tuple(table.shape),))
    a.vocab, a.dim, a.table_stride = _rows(table, "table")
    a.ids, a.tokens = _ids(ids, table.device), ids.numel()
    a.ignore_index, a.scale = ignore_index, scale
    with _on(stream, table):
        rows = torch.empty((*ids.shape, table.shape[1]), dtype=table.dtype, device=table.device)
        a.table, a.rows, a.rows_stride = table.data_ptr(), rows.data_ptr() if rows.numel() else None, a.dim
        _check(_ops().ckpt_embedding(C.byref(a), table.device.index, _handle(stream, table)))
    return rows


def ckpt_embedding_grad(d_rows, ids, vocab, scale=1.0, ignore_index=-100, dtype=None, add_to=None, stream=None):
    """The table's gradient [vocab, dim] of ckpt_embedding's rows' [..., dim]:
    for each word scale times the sum of its tokens' rows, in fp32, rounded
    once to `dtype` (the rows' by default).  With add_to [vocab, dim] (bf16 or
    fp32) it is added to what is there, in place, and add_to is returned; rows
    that no token has stay as they are.  Tokens with ignore_index or an id
    outside [0, vocab) are not read."""
    native, at = _native or _module()
    if native is not None and isinstance(d_rows, torch.Tensor) and d_rows.is_cuda and dtype is None:
        with _on(stream, d_rows):
            got = native.embedding_grad(at[1], at[2], d_rows, ids, vocab, scale, ignore_index, add_to,
                                        _handle(stream, d_rows))
        if got is not None:
            if got[0] != CKPT_OK:
                _check(got[0])
            return got[1]
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    a = ckpt_embed_args()
    a.dtype = _type(d_rows, "d_rows")
    a.ids = _ids(ids, d_rows.device)
    if d_rows.dim() < 1 or ids.shape != d_rows.shape[:-1]:
        raise ValueError("d_rows %s for ids %s" % (tuple(d_rows.shape), tuple(ids.shape)))
    _, a.dim, a.rows_stride = _rows(d_rows, "d_rows")
    a.tokens, a.vocab = ids.numel(), vocab
    a.ignore_index, a.scale = ignore_index, scale
    a.rows = d_rows.data_ptr() if d_rows.numel() else None
    if add_to is not None and dtype not in (None, add_to.dtype):
        raise ValueError("dtype %s, add_to %s" % (dtype, add_to.dtype))
    if dtype is not None and dtype not in _TYPES:
        raise ValueError("dtype %s: bfloat16 or float32 is wanted" % (dtype,))
    with _on(stream, d_rows):
        if add_to is None:
            table = torch.empty((vocab, d_rows.shape[-1]), dtype=dtype or d_rows.dtype, device=d_rows.device)
        else:
            table, a.add = add_to, 1
        a.table_dtype = _type(table, "add_to")
        if table.shape != (vocab, d_rows.shape[-1]) or table.device != d_rows.device:
            raise ValueError("add_to %s on %s" % (tuple(table.shape), table.device))
        _, _, a.table_stride = _rows(table, "add_to")
        a.table = table.data_ptr()
        L, need = _ops(), C.c_uint64()
        _check(L.ckpt_embedding_grad_workspace(C.byref(a), C.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device=d_rows.device)
        _check(L.ckpt_embedding_grad(C.byref(a), d_rows.device.index, work.data_ptr(), need.value, _handle(stream, d_rows)))
    return table
