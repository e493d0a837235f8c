"""Python binding of the training-step operators (include/ckpt_ops.h): the
vocabulary head's losses with their gradients, and the clipped AdamW step over
a rank's fragments.  Argument marshalling only, as in `ckpt`; workspaces and
results come from torch's caching allocator, on the stream that the work runs
on.  With `stream` the allocator does not learn that the call's tensors are
used there: inputs have to be ready for that stream and to live until its work
has run, and results are another stream's only behind it (`wait_stream`,
`record_stream`), as for any work on a stream of its own.

    r = ckpt_linear_ce(hidden, lm_head, targets, grad=True)
    hidden.backward(r.d_hidden)                      # the rest of the model
    norm = ckpt_grad_norm(grads, max_norm=1.0)       # norm[0], and the clip's factor norm[1]
    ck.wait_captured(snap, lo, hi)                   # the gate before the optimizer step
    ckpt_adamw(params, masters, exp_avgs, exp_avg_sqs, grads, step=k, lr=3e-4, grad_scale=norm[1:])
"""
import contextlib
import ctypes as C
from typing import NamedTuple, Optional

import torch

from .ckpt import CKPT_OK, CkptError, _native_module, ckpt_tensor, lib, tensor_bytes

__all__ = ["CKPT_GRAD_NORM_SCRATCH", "CKPT_LOSS_MEAN", "CKPT_LOSS_SUM", "CKPT_TYPE_BF16", "CKPT_TYPE_F32", "LinearLoss",
           "ckpt_adamw", "ckpt_adamw_fragment", "ckpt_grad_norm", "ckpt_linear_ce", "ckpt_linear_distill",
           "ckpt_linear_loss_args"]

CKPT_TYPE_BF16 = 1
CKPT_TYPE_F32 = 2
CKPT_LOSS_MEAN = 0
CKPT_LOSS_SUM = 1
CKPT_GRAD_NORM_SCRATCH = 16384

_TYPES = {torch.bfloat16: CKPT_TYPE_BF16, torch.float32: CKPT_TYPE_F32}
_REDUCTIONS = {"mean": CKPT_LOSS_MEAN, "sum": CKPT_LOSS_SUM}


class ckpt_linear_loss_args(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("reduction", C.c_uint32), ("tokens", C.c_uint64), ("dim", C.c_uint64),
                ("vocab", C.c_uint64), ("hidden", C.c_void_p), ("hidden_stride", C.c_uint64), ("weight", C.c_void_p),
                ("weight_stride", C.c_uint64), ("target", C.c_void_p), ("ignore_index", C.c_int64),
                ("token_weight", C.c_void_p), ("topk", C.c_uint32), ("teacher_dtype", C.c_uint32),
                ("teacher_index", C.c_void_p), ("teacher_index_stride", C.c_uint64), ("teacher_logits", C.c_void_p),
                ("teacher_logits_stride", C.c_uint64), ("temperature", C.c_float), ("alpha", C.c_float),
                ("grad_scale", C.c_void_p), ("piece_bytes", C.c_uint64), ("loss", C.c_void_p),
                ("token_loss", C.c_void_p), ("lse", C.c_void_p), ("d_hidden", C.c_void_p),
                ("d_hidden_stride", C.c_uint64), ("d_weight", C.c_void_p), ("d_weight_stride", C.c_uint64)]


class ckpt_adamw_fragment(C.Structure):
    _fields_ = [("param", C.c_void_p), ("master", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
                ("grad", C.c_void_p), ("numel", C.c_uint64)]


class LinearLoss(NamedTuple):
    loss: torch.Tensor  # scalar, fp32
    token_loss: torch.Tensor  # fp32, the tokens' shape; 0 where a token does not count
    lse: torch.Tensor  # fp32 log-sum-exp (distillation, alpha > 0: at the temperature)
    d_hidden: Optional[torch.Tensor]
    d_weight: Optional[torch.Tensor]


_lib = None
_native = None
_HERE = contextlib.nullcontext()


def _module():
    """(the native module or None, addresses of the entry points)."""
    global _native
    if _native is None:
        L = _ops()
        _native = (_native_module(), {n: C.cast(getattr(L, n), C.c_void_p).value for n in
                                      ("ckpt_linear_loss_workspace", "ckpt_linear_loss", "ckpt_grad_norm",
                                       "ckpt_adamw")})
    return _native


def _handle(stream, tensor):
    """hipStream_t handle of a torch stream, an int handle, or (None) torch's current stream on the tensor's device."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(tensor.get_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _ops():
    global _lib
    if _lib is None:
        L = lib()
        vp, u64, u32, i32, f64 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int32, C.c_double
        P = C.POINTER
        sig = {
            "ckpt_linear_loss_workspace": [P(ckpt_linear_loss_args), P(u64)],
            "ckpt_linear_loss": [P(ckpt_linear_loss_args), i32, vp, u64, vp],
            "ckpt_grad_norm": [P(ckpt_tensor), u32, u32, C.c_float, vp, vp, i32, vp],
            "ckpt_adamw": [P(ckpt_adamw_fragment), u32, u32, u32, u64, f64, f64, f64, f64, f64, vp, i32, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = i32
        _lib = L
    return _lib


def _check(rc):
    if rc != CKPT_OK:
        raise CkptError(rc, (lib().ckpt_last_error(None) or b"").decode())


def _type(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s is not a device tensor" % what)
    if t.dtype not in _TYPES:
        raise ValueError("%s is %s: bfloat16 or float32 is wanted" % (what, t.dtype))
    return _TYPES[t.dtype]


def _rows(t, what):
    """A tensor whose last dimension is contiguous, as rows: (rows, columns, row stride).  Leading dimensions have to
    be evenly spaced."""
    cols = t.shape[-1]
    rows = t.numel() // cols if cols else 0
    if rows <= 1 or t.is_contiguous():
        if cols > 1 and t.stride(-1) != 1:
            raise ValueError("%s: the last dimension is not contiguous (strides %s)" % (what, t.stride()))
        return rows, cols, cols
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError("%s: the last dimension is not contiguous (strides %s)" % (what, t.stride()))
    dims = [k for k in range(t.dim() - 1) if t.shape[k] > 1]
    for a, b in zip(dims, dims[1:]):
        if t.stride(a) != t.stride(b) * t.shape[b]:
            raise ValueError("%s: rows are not evenly spaced (strides %s)" % (what, t.stride()))
    return rows, cols, t.stride(dims[-1])


def _on(stream, tensor):
    """The context in which the outputs and the workspace of work on `stream` are allocated.  A handle is a stream of
    the tensor's device, which need not be the current one."""
    if stream is None:
        return _HERE
    return torch.cuda.stream(torch.cuda.ExternalStream(stream, tensor.device) if isinstance(stream, int) else stream)


def _listed(x):
    return x if type(x) is list or type(x) is tuple else list(x)


def _plain(t, what, dtype, n):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype:
        raise ValueError("%s is not a device tensor of %s" % (what, dtype))
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: %d contiguous values are wanted (shape %s, strides %s)" %
                         (what, n, tuple(t.shape), t.stride()))
    return t.data_ptr() if n else None


def _each_token(t, what, dtype, shape):
    """A value for each token: of the tokens' shape, or flat.  Another shape of as many values may be another order."""
    p = _plain(t, what, dtype, shape.numel())
    if t.dim() != 1 and [k for k in t.shape if k != 1] != [k for k in shape if k != 1]:
        raise ValueError("%s %s for tokens %s" % (what, tuple(t.shape), tuple(shape)))
    return p


def _linear_loss(hidden, weight, target, teacher, temperature, alpha, token_weight, ignore_index, reduction, grad,
                 grad_scale, piece_bytes, stream):
    native, at = _native or _module()
    if native is not None and isinstance(hidden, torch.Tensor) and hidden.is_cuda and reduction in _REDUCTIONS:
        with _on(stream, hidden):
            got = native.linear_loss(at["ckpt_linear_loss_workspace"], at["ckpt_linear_loss"], hidden, weight, target,
                                     None if teacher is None else teacher[0], None if teacher is None else teacher[1],
                                     temperature, alpha, token_weight, ignore_index, _REDUCTIONS[reduction], grad,
                                     grad_scale, piece_bytes, _handle(stream, hidden))
        if got is not None:
            _check(got[0])
            return LinearLoss(*got[1:])
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    a = ckpt_linear_loss_args()
    a.dtype = _type(hidden, "hidden")
    if _type(weight, "weight") != a.dtype:
        raise ValueError("hidden is %s, weight is %s" % (hidden.dtype, weight.dtype))
    if hidden.dim() < 1 or weight.dim() != 2 or hidden.shape[-1] != weight.shape[1]:
        raise ValueError("hidden %s against weight %s" % (tuple(hidden.shape), tuple(weight.shape)))
    if hidden.device != weight.device:
        raise ValueError("hidden on %s, weight on %s" % (hidden.device, weight.device))
    if reduction not in _REDUCTIONS:
        raise ValueError("reduction is 'mean' or 'sum', not %r" % (reduction,))
    a.reduction = _REDUCTIONS[reduction]
    shape = hidden.shape[:-1]
    n = shape.numel()
    _, a.dim, a.hidden_stride = _rows(hidden, "hidden")
    a.tokens = n
    a.vocab, _, a.weight_stride = _rows(weight, "weight")
    a.hidden, a.weight = hidden.data_ptr(), weight.data_ptr()
    if target is not None:
        a.target = _each_token(target, "target", torch.int64, shape)
    a.ignore_index = ignore_index
    if token_weight is not None:
        a.token_weight = _each_token(token_weight, "token_weight", torch.float32, shape)
    a.temperature, a.alpha = temperature, alpha
    if teacher is not None:
        index, logits = teacher
        a.teacher_dtype = _type(logits, "teacher_logits")
        if not isinstance(index, torch.Tensor) or not index.is_cuda or index.dtype != torch.int64:
            raise ValueError("teacher_index is not a device tensor of torch.int64")
        if index.shape != logits.shape or index.shape[:-1] != shape or index.shape[-1] < 1:
            raise ValueError("teacher_index %s and teacher_logits %s for tokens %s" %
                             (tuple(index.shape), tuple(logits.shape), tuple(shape)))
        _, a.topk, a.teacher_index_stride = _rows(index, "teacher_index")
        _, _, a.teacher_logits_stride = _rows(logits, "teacher_logits")
        a.teacher_index, a.teacher_logits = index.data_ptr(), logits.data_ptr()
    if grad_scale is not None:
        a.grad_scale = _plain(grad_scale, "grad_scale", torch.float32, 1)
    a.piece_bytes = piece_bytes
    d_hidden = d_weight = None
    with _on(stream, hidden):
        out = torch.empty(2 * n + 1, dtype=torch.float32, device=hidden.device)
        a.loss = out.data_ptr()
        a.token_loss = a.loss + 4
        a.lse = a.token_loss + 4 * n
        if grad:
            d_hidden = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device)
            d_weight = torch.empty(weight.shape, dtype=weight.dtype, device=weight.device)
            a.d_hidden, a.d_weight = d_hidden.data_ptr(), d_weight.data_ptr()
            a.d_hidden_stride = a.d_weight_stride = a.dim
        need = C.c_uint64()
        L = _ops()
        _check(L.ckpt_linear_loss_workspace(C.byref(a), C.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device=hidden.device)
        _check(L.ckpt_linear_loss(C.byref(a), hidden.device.index, work.data_ptr(), need.value, _handle(stream, hidden)))
    return LinearLoss(out[0], out[1:n + 1].view(shape), out[n + 1:].view(shape), d_hidden, d_weight)


def ckpt_linear_ce(hidden, weight, target, token_weight=None, ignore_index=-100, reduction="mean", grad=False,
                   grad_scale=None, piece_bytes=0, stream=None):
    """Softmax cross entropy of hidden [..., dim] weight^T [vocab, dim]
    against target [...] (int64), without holding the logits of more tokens
    than piece_bytes allows (0 = 2 GiB).  target and token_weight (fp32) have
    the tokens' shape or are flat.  bf16 or fp32.  grad: also d_hidden
    and d_weight, of grad_scale (a device scalar; None = 1) times the loss.
    A token counts unless its target is ignore_index or its token_weight 0;
    hidden is not read where it does not."""
    return _linear_loss(hidden, weight, target, None, 1.0, 0.0, token_weight, ignore_index, reduction, grad,
                        grad_scale, piece_bytes, stream)


def ckpt_linear_distill(hidden, weight, teacher_index, teacher_logits, target=None, temperature=1.0, alpha=1.0,
                        token_weight=None, ignore_index=-100, reduction="mean", grad=False, grad_scale=None,
                        piece_bytes=0, stream=None):
    """Distillation from a teacher's top logits: alpha T^2 KL(q || p^T) +
    (1 - alpha) cross entropy, q the softmax of teacher_logits [..., topk] / T
    over the words teacher_index [..., topk] (int64; below 0 = absent), p^T
    the student's over the whole vocabulary.  target is needed where alpha <
    1; lse is that of p^T (alpha = 0: as ckpt_linear_ce's, which the call then
    is).  The other arguments are ckpt_linear_ce's."""
    return _linear_loss(hidden, weight, target, (teacher_index, teacher_logits), temperature, alpha, token_weight,
                        ignore_index, reduction, grad, grad_scale, piece_bytes, stream)


def ckpt_grad_norm(grads, max_norm=0.0, stream=None):
    """fp32 [2]: the 2-norm of all gradients together (one type, bf16 or
    fp32), and the factor min(1, max_norm / (norm + 1e-6)) that clips them to
    max_norm (1 where max_norm is 0), for ckpt_adamw's grad_scale."""
    grads = _listed(grads)
    if not grads:
        raise ValueError("no gradients")
    native, at = _native or _module()
    if native is not None and isinstance(grads[0], torch.Tensor) and grads[0].is_cuda:
        with _on(stream, grads[0]):
            got = native.grad_norm(at["ckpt_grad_norm"], grads, max_norm, _handle(stream, grads[0]))
        if got is not None:
            _check(got[0])
            return got[1]
    kind = _type(grads[0], "gradient 0")
    arr = (ckpt_tensor * len(grads))()
    for i, t in enumerate(grads):
        if _type(t, "gradient %d" % i) != kind:
            raise ValueError("gradient %d is %s, gradient 0 is %s" % (i, t.dtype, grads[0].dtype))
        arr[i].nbytes = tensor_bytes(t)
        arr[i].dev_ptr = t.data_ptr() if arr[i].nbytes else None
    device = grads[0].device
    with _on(stream, grads[0]):
        out = torch.empty(2, dtype=torch.float32, device=device)
        scratch = torch.empty(CKPT_GRAD_NORM_SCRATCH, dtype=torch.uint8, device=device)
        _check(_ops().ckpt_grad_norm(arr, len(grads), kind, max_norm, out.data_ptr(), scratch.data_ptr(), device.index,
                                     _handle(stream, grads[0])))
    return out


def ckpt_adamw(params, masters, exp_avgs, exp_avg_sqs, grads, step, lr, beta1=0.9, beta2=0.999, eps=1e-8,
               weight_decay=0.0, grad_scale=None, stream=None):
    """AdamW in place over a rank's fragments, list by list: fp32 masters and
    moments, params (bf16, or fp32 in full precision) rounded from the masters,
    grads (bf16 or fp32).  One list of fragments may be a bucket, behind
    Checkpointer.wait_captured of the same range on the same stream."""
    params, masters, exp_avgs, exp_avg_sqs, grads = map(_listed, (params, masters, exp_avgs, exp_avg_sqs, grads))
    native, at = _native or _module()
    if native is not None and params and isinstance(params[0], torch.Tensor) and params[0].is_cuda:
        rc = native.adamw(at["ckpt_adamw"], params, masters, exp_avgs, exp_avg_sqs, grads, step, lr, beta1, beta2, eps,
                          weight_decay, grad_scale, _handle(stream, params[0]))
        if rc is not None:
            if rc != CKPT_OK:
                _check(rc)
            return
    # Arguments that the native module leaves to this code, and those refused; every call where there is none.
    lists = (params, masters, exp_avgs, exp_avg_sqs, grads)
    n = len(lists[0])
    if any(len(x) != n for x in lists):
        raise ValueError("lists of %s fragments" % ", ".join(str(len(x)) for x in lists))
    if n == 0:
        return
    pt, gt = _type(lists[0][0], "param 0"), _type(lists[4][0], "grad 0")
    kinds = (pt, CKPT_TYPE_F32, CKPT_TYPE_F32, CKPT_TYPE_F32, gt)
    names = ("param", "master", "exp_avg", "exp_avg_sq", "grad")
    arr = (ckpt_adamw_fragment * n)()
    for i, row in enumerate(zip(*lists)):
        numel = row[0].numel()
        for t, kind, name in zip(row, kinds, names):
            if _type(t, "%s %d" % (name, i)) != kind or t.numel() != numel or not t.is_contiguous():
                raise ValueError("%s %d: %s %s, strides %s" % (name, i, t.dtype, tuple(t.shape), t.stride()))
            if numel:
                setattr(arr[i], name, t.data_ptr())
        arr[i].numel = numel
    scale = _plain(grad_scale, "grad_scale", torch.float32, 1) if grad_scale is not None else None
    _check(_ops().ckpt_adamw(arr, n, pt, gt, step, lr, beta1, beta2, eps, weight_decay, scale,
                             lists[0][0].device.index, _handle(stream, lists[0][0])))
