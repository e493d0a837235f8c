"""The training-step operators without a GPU: exported symbols, the binding's
structures against the header's, argument checks that need no device, and the
bound on the workspace (CPU only)."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2607_01646_amd as P
from paper_2607_01646_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ckpt_ops.h")


def test_library_exports_every_declared_operator():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\bckpt_status (ckpt_[a-z_]+)\s*\(", src)))
    assert names == ["ckpt_adamw", "ckpt_grad_norm", "ckpt_linear_loss", "ckpt_linear_loss_workspace"]
    assert all(hasattr(P.lib(), f) for f in names)


@pytest.mark.parametrize("name", ["ckpt_linear_loss_args", "ckpt_adamw_fragment"])
def test_structures_match_the_header(name, tmp_path):
    struct = getattr(ops, name)
    fields = [f for f, _ in struct._fields_]
    c = tmp_path / "s.c"
    c.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ckpt_ops.h"\nint main(void) {\n' +
                 "".join('printf("%%zu\\n", offsetof(%s, %s));\n' % (name, f) for f in fields) +
                 'printf("%%zu\\n%%d\\n", sizeof(%s), CKPT_GRAD_NORM_SCRATCH);\nreturn 0; }\n' % name)
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(c), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(struct, f).offset for f in fields] + [C.sizeof(struct), P.CKPT_GRAD_NORM_SCRATCH]


def need(**kw):
    a = ops.ckpt_linear_loss_args(dtype=P.CKPT_TYPE_BF16, tokens=8192, dim=4096, vocab=32000, hidden_stride=4096,
                                  weight_stride=4096, target=256, temperature=1, alpha=1)
    for k, v in kw.items():
        setattr(a, k, v)
    n = C.c_uint64()
    return ops._ops().ckpt_linear_loss_workspace(C.byref(a), C.byref(n)), n.value


def test_the_workspace_is_bounded_by_the_piece():
    grads = dict(d_hidden=256, d_weight=256)
    for dtype in (P.CKPT_TYPE_BF16, P.CKPT_TYPE_F32):
        sizes = [need(dtype=dtype, tokens=n, piece_bytes=256 << 20, **grads) for n in (1 << 16, 1 << 20, 1 << 24)]
        assert all(rc == P.CKPT_OK for rc, _ in sizes)
        # beyond a piece only a weight a row
        assert sizes[1][1] - sizes[0][1] <= 4 * ((1 << 20) - (1 << 16)) + 256
        assert sizes[2][1] - sizes[1][1] <= 4 * ((1 << 24) - (1 << 20)) + 256
    # without gradients the cross entropy holds no logits at all
    rc, n = need(tokens=8192)
    assert rc == P.CKPT_OK and n < 8192 * 32000 // 4


@pytest.mark.parametrize("kw", [
    dict(dtype=0), dict(dtype=9), dict(reduction=2), dict(tokens=1 << 31), dict(dim=0), dict(dim=1 << 31),
    dict(vocab=0), dict(vocab=1 << 31), dict(topk=1025), dict(target=0), dict(d_hidden=256), dict(d_weight=256),
    dict(topk=4), dict(topk=4, teacher_dtype=P.CKPT_TYPE_BF16, temperature=0),
    dict(topk=4, teacher_dtype=P.CKPT_TYPE_BF16, temperature=math.nan),
    dict(topk=4, teacher_dtype=P.CKPT_TYPE_BF16, alpha=1.5), dict(topk=4, teacher_dtype=P.CKPT_TYPE_BF16, alpha=math.nan),
    dict(topk=4, teacher_dtype=P.CKPT_TYPE_BF16, alpha=0.5, target=0)])
def test_sizes_and_numbers_that_are_refused(kw):
    rc, _ = need(**kw)
    assert rc == P.CKPT_EINVAL and P.ckpt_last_error(None)


def test_null_arguments():
    n = C.c_uint64()
    assert ops._ops().ckpt_linear_loss_workspace(None, C.byref(n)) == P.CKPT_EINVAL
    a = ops.ckpt_linear_loss_args()
    assert ops._ops().ckpt_linear_loss_workspace(C.byref(a), None) == P.CKPT_EINVAL
    assert ops._ops().ckpt_grad_norm(None, 3, P.CKPT_TYPE_F32, 0.0, None, None, 0, None) == P.CKPT_EINVAL
    assert ops._ops().ckpt_adamw(None, 3, P.CKPT_TYPE_F32, P.CKPT_TYPE_F32, 1, 1e-3, 0.9, 0.9, 0, 0, None, 0,
                                 None) == P.CKPT_EINVAL


def test_host_tensors_are_refused():
    h, w = torch.zeros(4, 8), torch.zeros(10, 8)
    y = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="hidden"):
        P.ckpt_linear_ce(h, w, y)
    with pytest.raises(ValueError, match="gradient 0"):
        P.ckpt_grad_norm([h])
    with pytest.raises(ValueError, match="param 0"):
        P.ckpt_adamw([h], [h], [h], [h], [h], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="fragments"):
        P.ckpt_adamw([h], [h], [h], [h], [], step=1, lr=1e-3)
