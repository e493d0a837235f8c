"""The training-step operators without a GPU: exported symbols, the binding's
structures against the header's, argument checks that need no device, and the
bound on the workspace (CPU only)."""
import ctypes as C
import functools
import math
import os
import re
import subprocess
import tempfile

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
    # nor does what it keeps for its tokens grow beyond a piece, up to the most tokens there can be
    sizes = [need(tokens=n, piece_bytes=64 << 20)[1] for n in (1 << 20, (1 << 31) - 1)]
    assert sizes[1] - sizes[0] <= 4 * ((1 << 31) - (1 << 20)) + 256


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


def test_a_stream_handle_belongs_to_the_tensors_device(monkeypatch):
    """What is allocated for work on a stream given as a handle comes from that stream's pool, on the tensor's device,
    whichever device is current."""
    seen = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: seen.append((handle, device)) or "s")
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)

    class On1:
        device = torch.device("cuda", 1)

    assert ops._on(1234, On1()) == "s" and seen == [(1234, torch.device("cuda", 1))]
    assert ops._on("a stream", On1()) == "a stream" and ops._on(None, On1()) is ops._HERE


@functools.lru_cache(None)
def kernels(name):
    """The gfx950 assembly of a kernel file."""
    from paper_2607_01646_amd import build as B

    with tempfile.TemporaryDirectory() as d:
        return assembly(B, name, os.path.join(d, "k.s"))


def assembly(B, name, out):
    cmd = [B.HIPCC] + [f for f in B.DEVICE_FLAGS if f != "-fPIC"] + [
        "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "--cuda-device-only", "-S", os.path.join(B.CSRC, name),
        "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        return f.read()


@pytest.mark.parametrize("name", ["loss_kernels.hip", "optim_kernels.hip"])
def test_kernels_keep_their_registers_and_use_no_packed_fp32(name):
    """No vector register goes to memory (the products' loops wait for their loads by count: a spill among them would
    be waited for too), and no packed fp32 arithmetic is made."""
    text = kernels(name)
    spills = [int(x) for x in re.findall(r"\.vgpr_spill_count:\s*(\d+)", text)]
    assert spills and not any(spills)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)


def test_products_wait_for_no_load_that_is_to_stay_in_flight():
    """In the loops of the largest products nothing but the barrier at which the waves meet waits for the loads made
    since the last one; with four buffers not even that."""
    text = kernels("loss_kernels.hip")
    bodies = re.findall(r"^(_ZN4ckpt\w*product_kernel\w*Li256ELi256E\w*):\s(.*?)s_endpgm", text, re.S | re.M)
    assert len(bodies) == 3
    for name, body in bodies:
        lines = [x.strip() for x in body.split("\n") if x.strip() and not x.strip().startswith(";")]
        labels = {x.split(":")[0]: i for i, x in enumerate(lines) if x.startswith(".L")}
        loops = []
        for i, x in enumerate(lines):
            m = re.match(r"s_c?branch\w*\s+(\.L\w+)", x)
            if m and labels.get(m.group(1), i) < i:
                loops.append(lines[labels[m.group(1)]:i])
        loop = max(loops, key=lambda l: sum("mfma" in x for x in l))
        assert sum("mfma" in x for x in loop) >= 64
        flying = waits = 0
        for x, after in zip(loop + loop, loop[1:] + loop + loop[:1]):
            if x.startswith("buffer_load") and x.endswith("lds"):
                flying += 1
            elif x.startswith("s_waitcnt") and "vmcnt(0)" in x:
                waits += 1
                assert "Li32ELi4E" not in name and (flying == 0 or after.startswith("s_barrier")), (name, x, after)
            elif x.startswith("s_barrier"):
                flying = 0
        assert waits or "Li32ELi4E" in name
