"""The vocabulary table's and the orthogonalised step's operators without a GPU:
exported symbols, the binding's structures against the headers', argument
checks that need no device, bounds on the workspaces, and the kernels' code
(CPU only)."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2607_01646_amd as P
from paper_2607_01646_amd import embed, muon
from test_ops_host import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INCLUDE = os.path.join(ROOT, "include")


@pytest.mark.parametrize("header, functions", [
    ("ckpt_embed.h", ["ckpt_embedding", "ckpt_embedding_grad", "ckpt_embedding_grad_workspace"]),
    ("ckpt_muon.h", ["ckpt_muon", "ckpt_muon_workspace", "ckpt_orthogonalize", "ckpt_orthogonalize_workspace"])])
def test_library_exports_every_declared_operator(header, functions):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, header)).read(), flags=re.S)
    assert sorted(set(re.findall(r"\bckpt_status (ckpt_[a-z_]+)\s*\(", src))) == functions
    assert all(hasattr(P.lib(), f) for f in functions)


@pytest.mark.parametrize("header, struct, rename", [
    ("ckpt_embed.h", embed.ckpt_embed_args, {}), ("ckpt_muon.h", muon.ckpt_newton_schulz, {}),
    ("ckpt_muon.h", muon.ckpt_matrix, {"input": "in"}), ("ckpt_muon.h", muon.ckpt_muon_matrix, {}),
    ("ckpt_muon.h", muon.ckpt_muon_args, {})])
def test_structures_match_the_header(header, struct, rename, tmp_path):
    fields = [f for f, _ in struct._fields_]
    c = tmp_path / "s.c"
    c.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) {\n' % header +
                 "".join('printf("%%zu\\n", offsetof(%s, %s));\n' % (struct.__name__, rename.get(f, f)) for f in fields) +
                 'printf("%%zu\\n", sizeof(%s));\nreturn 0; }\n' % struct.__name__)
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", INCLUDE, str(c), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(struct, f).offset for f in fields] + [C.sizeof(struct)]


def test_the_package_takes_the_operators_names():
    for module in (embed, muon):
        public = {k for k, x in vars(module).items() if k.startswith("ckpt_") and getattr(x, "__module__", "") == module.__name__}
        assert public == set(module.__all__) and all(getattr(P, k) is getattr(module, k) for k in public)
    assert not hasattr(P, "math") and not hasattr(P, "COEFFICIENTS")


# ---- the table ----


def need_grad(**kw):
    """Status and workspace bytes of a gradient."""
    a = embed.ckpt_embed_args(dtype=P.CKPT_TYPE_BF16, table_dtype=P.CKPT_TYPE_BF16, tokens=8192, dim=4096, vocab=32000, ids=256,
                              ignore_index=-100, scale=1.0, rows=256, rows_stride=4096, table=256, table_stride=4096)
    for k, v in kw.items():
        setattr(a, k, v)
    n = C.c_uint64()
    return embed._ops().ckpt_embedding_grad_workspace(C.byref(a), C.byref(n)), n.value


@pytest.mark.parametrize("kw", [dict(dtype=0), dict(dtype=3), dict(table_dtype=0), dict(tokens=1 << 31), dict(dim=0),
                                dict(dim=(1 << 22) + 1), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(scale=math.nan),
                                dict(scale=math.inf), dict(scale=1e39), dict(add=2), dict(reserved=1)])
def test_table_arguments_that_are_refused(kw):
    assert need_grad(**kw)[0] == P.CKPT_EINVAL and P.ckpt_last_error(None)


@pytest.mark.parametrize("tokens", [0, 1, 128, 129, 4096, 8192, 65536, 1 << 20, (1 << 31) - 1])
@pytest.mark.parametrize("dim, vocab", [(1, 1), (64, 256), (4096, 32000), (1 << 22, 3), (8, 1 << 22)])
def test_the_gradients_workspace(tokens, dim, vocab):
    """Places and words of the tokens, the words' beginnings, and two fp32 sums for each of at most 1024 (or twice as few
    as there are tokens in eights) chunks; none for few tokens."""
    rc, n = need_grad(tokens=tokens, dim=dim, vocab=vocab)
    assert rc == P.CKPT_OK
    if 0 < tokens <= 128:
        assert n == 0
        return
    chunks = min(-(-tokens // 8), 1024 * 4)
    assert n <= 8 * tokens + 4 * (vocab + 1) + chunks * (8 * (dim + 8) + 8) + 6 * 256
    assert n >= 8 * tokens


def test_table_null_arguments():
    n, a = C.c_uint64(), embed.ckpt_embed_args()
    assert embed._ops().ckpt_embedding(None, 0, None) == P.CKPT_EINVAL
    assert embed._ops().ckpt_embedding_grad_workspace(None, C.byref(n)) == P.CKPT_EINVAL
    assert embed._ops().ckpt_embedding_grad_workspace(C.byref(a), None) == P.CKPT_EINVAL
    assert embed._ops().ckpt_embedding_grad(None, 0, None, 0, None) == P.CKPT_EINVAL
    a = embed.ckpt_embed_args(dtype=P.CKPT_TYPE_BF16, table_dtype=P.CKPT_TYPE_F32, tokens=1, dim=1, vocab=1, scale=1.0)
    assert embed._ops().ckpt_embedding(C.byref(a), 0, None) == P.CKPT_EINVAL  # a lookup has one type
    a.table_dtype, a.add = P.CKPT_TYPE_BF16, 1
    assert embed._ops().ckpt_embedding(C.byref(a), 0, None) == P.CKPT_EINVAL  # and adds to nothing


# ---- the orthogonalised step ----


def newton_schulz(**kw):
    ns = muon.ckpt_newton_schulz(5, 0, *muon.COEFFICIENTS, 1e-7, 0)
    for k, v in kw.items():
        setattr(ns, k, v)
    return ns


def need_orth(shapes, **kw):
    arr = (muon.ckpt_matrix * max(len(shapes), 1))()
    for m, (r, c) in zip(arr, shapes):
        m.rows, m.cols = r, c
    n, ns = C.c_uint64(), newton_schulz(**kw)
    return muon._ops().ckpt_orthogonalize_workspace(arr, len(shapes), C.byref(ns), C.byref(n)), n.value


@pytest.mark.parametrize("kw", [dict(steps=0), dict(steps=65), dict(reserved=1), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-31),
                                dict(eps=2.0), dict(eps=math.nan), dict(a=math.nan), dict(b=math.inf), dict(a=3.0, b=3.0),
                                dict(a=2.1, b=0.0, c=0.0), dict(a=4.0, b=-7.5, c=4.5, steps=2), dict(a=9.0, b=-18.0, c=9.5), dict(a=1.2, b=0.0, c=0.0, steps=8)])
def test_polynomials_and_numbers_that_are_refused(kw):
    assert need_orth([(10, 20)], **kw)[0] == P.CKPT_EINVAL and P.ckpt_last_error(None)


@pytest.mark.parametrize("kw", [dict(), dict(steps=1), dict(steps=64, a=1.5, b=-0.5, c=0.0), dict(a=1.875, b=-1.25, c=0.375, steps=20),
                                dict(a=4.0, b=-7.5, c=4.5, steps=1), dict(eps=1e-30), dict(eps=1.0)])
def test_others_are_not(kw):
    assert need_orth([(10, 20)], **kw)[0] == P.CKPT_OK


def up(x, a):
    return -(-x // a) * a


def bytes_of(r, c):
    s, l = min(r, c), max(r, c)
    tiles = -(-r // 16) * -(-c // 256)
    if s <= 16:  # sums of 16 x 16 products for runs of 256 places, and what comes of them, in 64 bits
        return 2048 + 2048 * min(-(-l // 256), 512)
    return 2 * up(4 * s * up(l, 64), 256) + 3 * up(4 * s * up(s, 64), 256) + up(8 * tiles, 256)


@pytest.mark.parametrize("piece", [0, 1, 1 << 20, 64 << 20, 1 << 30])
def test_the_workspace_is_bounded_by_the_piece(piece):
    """What the largest matrix takes, or the piece; nothing for small and empty ones."""
    shapes = [(4096, 4096), (1000, 77), (64, 256), (256, 64), (0, 10), (300, 0), (65, 65), (11008, 4096)] * 9
    rc, n = need_orth(shapes, piece_bytes=piece)
    largest = max(bytes_of(*s) for s in shapes)
    assert rc == P.CKPT_OK and largest <= n <= max(piece or 4 << 30, largest)
    assert need_orth([(64, 256), (17, 17), (200, 64), (5, 0)]) == (P.CKPT_OK, 0)
    assert need_orth([(1, 5), (700000, 16), (64, 64)]) == (P.CKPT_OK, bytes_of(1, 5) + bytes_of(700000, 16))
    assert need_orth([(16, 900)], a=1.5, b=-0.5, c=0.0, steps=64) == (P.CKPT_OK, 2 * 4 * 16 * 960 + 3 * 4 * 16 * 64 + 256)
    assert need_orth([]) == (P.CKPT_OK, 0)
    assert need_orth([(300, 200)]) == (P.CKPT_OK, bytes_of(300, 200))


def test_sizes_that_are_refused():
    assert need_orth([((1 << 22) + 1, 3)])[0] == P.CKPT_EINVAL
    assert need_orth([(1 << 22, 1 << 22)])[0] == P.CKPT_EINVAL
    assert need_orth([(1 << 22, 64)])[0] == P.CKPT_OK


def need_muon(**kw):
    m = (muon.ckpt_muon_matrix * 1)()
    m[0].rows, m[0].cols, m[0].scale = 100, 200, kw.pop("scale", 1.0)
    a = muon.ckpt_muon_args(P.CKPT_TYPE_BF16, P.CKPT_TYPE_BF16, 1, 0, 1e-3, 0.95, 0.1, None, newton_schulz())
    for k, v in kw.items():
        setattr(a, k, v)
    n = C.c_uint64()
    return muon._ops().ckpt_muon_workspace(m, 1, C.byref(a), C.byref(n)), n.value


@pytest.mark.parametrize("kw", [dict(param_dtype=0), dict(grad_dtype=7), dict(nesterov=2), dict(reserved=1), dict(momentum=1.0),
                                dict(momentum=-0.1), dict(momentum=math.nan), dict(lr=math.nan), dict(lr=math.inf),
                                dict(weight_decay=math.inf), dict(lr=1e30, weight_decay=1e30), dict(scale=math.nan),
                                dict(scale=1e42), dict(lr=1e20, scale=1e20), dict(ns=newton_schulz(steps=0))])
def test_step_arguments_that_are_refused(kw):
    assert need_muon(**kw)[0] == P.CKPT_EINVAL and P.ckpt_last_error(None)


def test_step_workspace_is_the_orthogonalisations():
    assert need_muon() == (P.CKPT_OK, bytes_of(100, 200))


def test_muon_null_arguments():
    n, ns, a = C.c_uint64(), newton_schulz(), muon.ckpt_muon_args()
    L = muon._ops()
    assert L.ckpt_orthogonalize_workspace(None, 1, C.byref(ns), C.byref(n)) == P.CKPT_EINVAL
    assert L.ckpt_orthogonalize_workspace(None, 0, None, C.byref(n)) == P.CKPT_EINVAL
    assert L.ckpt_orthogonalize_workspace(None, 0, C.byref(ns), None) == P.CKPT_EINVAL
    assert L.ckpt_muon_workspace(None, 1, C.byref(a), C.byref(n)) == P.CKPT_EINVAL
    assert L.ckpt_muon_workspace(None, 0, None, C.byref(n)) == P.CKPT_EINVAL
    assert L.ckpt_muon(None, 0, None, 0, None, 0, None) == P.CKPT_EINVAL
    assert L.ckpt_orthogonalize(None, 0, 9, C.byref(ns), 0, None, 0, None) == P.CKPT_EINVAL


def test_host_tensors_are_refused():
    x = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="table"):
        P.ckpt_embedding(x, ids)
    with pytest.raises(ValueError, match="d_rows"):
        P.ckpt_embedding_grad(x, ids, 10)
    with pytest.raises(ValueError, match="matrix 0"):
        P.ckpt_orthogonalize([x])
    with pytest.raises(ValueError, match="param 0"):
        P.ckpt_muon([x], [x], [x], [x], lr=1e-3)
    with pytest.raises(ValueError, match="matrices"):
        P.ckpt_muon([x], [x], [x], [], lr=1e-3)
    with pytest.raises(ValueError, match="results"):
        P.ckpt_orthogonalize([x], out=[])
    assert P.ckpt_orthogonalize([]) == [] and P.ckpt_muon([], [], [], [], lr=1e-3) is None


# ---- the kernels' code ----


@pytest.mark.parametrize("name", ["muon_kernels.hip", "embed_kernels.hip"])
def test_kernels_keep_their_registers(name):
    """No vector register goes to memory (the products' loops wait for their loads by count), no packed fp32 arithmetic is
    made, and every access is known to be of global memory or of LDS (others are waited for with both)."""
    text = kernels(name)
    spills = [int(x) for x in re.findall(r"\.vgpr_spill_count:\s*(\d+)", text)]
    assert spills and not any(spills)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    assert not re.search(r"\bflat_(load|store)", text)


def test_products_wait_for_no_load_that_is_to_stay_in_flight():
    """In the loops of the large products nothing but the barrier at which the waves meet waits for the loads made since the
    last one."""
    text = kernels("muon_kernels.hip")
    bodies = re.findall(r"^(_ZN4ckpt\w*(?:tri|apply)_kernelI\w*Li(?:256|128)ELi256E\w*):\s(.*?)s_endpgm", text, re.S | re.M)
    assert len(bodies) == 6
    for name, body in bodies:
        lines = [x.strip() for x in body.split("\n") if x.strip() and not x.strip().startswith(";")]
        labels = {x.split(":")[0]: i for i, x in enumerate(lines) if x.startswith(".L")}
        loops = []
        for i, x in enumerate(lines):
            m = re.match(r"s_c?branch\w*\s+(\.L\w+)", x)
            if m and labels.get(m.group(1), i) < i:
                loops.append(lines[labels[m.group(1)]:i])
        loops = [l for l in loops if sum("mfma" in x for x in l) >= 64]
        assert loops
        for loop in loops:
            flying = waits = 0
            for x, after in zip(loop + loop, loop[1:] + loop + loop[:1]):
                if x.startswith("buffer_load") and x.endswith("lds"):
                    flying += 1
                elif x.startswith("s_waitcnt") and "vmcnt(0)" in x:
                    waits += 1
                    assert flying == 0 or after.startswith("s_barrier"), (name, x, after)
                elif x.startswith("s_barrier"):
                    flying = 0
            assert waits or "Li32ELi3E" in name  # three buffers: the meeting leaves a step's loads in flight, too
