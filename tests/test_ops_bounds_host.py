"""What the training-step operators check and bound on the host, without a GPU
(CPU only)."""
import ctypes as C

import pytest

import paper_2607_01646_amd as P
from paper_2607_01646_amd import ops


def need(**kw):
    """Status and workspace bytes of a call."""
    a = ops.ckpt_linear_loss_args(dtype=P.CKPT_TYPE_BF16, tokens=8192, dim=4096, vocab=32000, hidden_stride=4096,
                                  weight_stride=4096, target=256, temperature=1, alpha=1)
    for k, v in kw.items():
        setattr(a, k, v)
    n = C.c_uint64()
    return ops._ops().ckpt_linear_loss_workspace(C.byref(a), C.byref(n)), n.value


TEACHER = dict(topk=4, teacher_dtype=P.CKPT_TYPE_F32, teacher_index_stride=4, teacher_logits_stride=4)
GRADS = dict(d_hidden=256, d_weight=256, d_hidden_stride=4096, d_weight_stride=4096)


@pytest.mark.parametrize("kw", [
    dict(tokens=(1 << 23) + 1, hidden_stride=1 << 40),  # 2^64 bytes to the last row: its own bytes would be left
    dict(tokens=(1 << 25) + 1, hidden_stride=1 << 38),
    dict(tokens=(1 << 22) + 1, hidden_stride=1 << 40, dtype=P.CKPT_TYPE_F32),
    dict(tokens=(1 << 30) + 1, hidden_stride=(1 << 33) + 1),
    dict(hidden_stride=1 << 63),
    dict(weight_stride=1 << 60),
    dict(tokens=(1 << 21) + 1, **{**TEACHER, "teacher_index_stride": 1 << 40}),
    dict(tokens=(1 << 22) + 1, **{**TEACHER, "teacher_logits_stride": 1 << 40}),
    dict(tokens=(1 << 23) + 1, **{**GRADS, "d_hidden_stride": 1 << 40}),
    dict(**{**GRADS, "d_weight_stride": 1 << 60}),
])
def test_strides_that_wrap_are_refused(kw):
    """Rows so far apart that their distance in bytes does not fit 64 bits: what is left of it must not be taken for the
    operand's size."""
    rc, _ = need(**kw)
    assert rc == P.CKPT_EINVAL and "rows" in P.ckpt_last_error(None)


@pytest.mark.parametrize("kw", [
    dict(tokens=(1 << 23) - 1, hidden_stride=1 << 40), dict(tokens=(1 << 31) - 1, hidden_stride=1 << 20),
    dict(tokens=1, hidden_stride=1 << 63), dict(tokens=0, hidden_stride=1 << 63), dict(vocab=1, weight_stride=1 << 63),
    dict(vocab=1 << 22, dim=1 << 22, weight_stride=1 << 22), dict(d_hidden_stride=1 << 63, d_weight_stride=1 << 63),
    dict(teacher_index_stride=1 << 63), dict(**TEACHER, **GRADS)])
def test_strides_that_do_not_wrap_or_are_not_used_are_not(kw):
    assert need(**kw)[0] == P.CKPT_OK


def up(x, a):
    return (x + a - 1) // a * a


KINDS = {"ce": {}, "distill": TEACHER, "distill at 2": dict(TEACHER, temperature=2)}


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("dtype", [P.CKPT_TYPE_BF16, P.CKPT_TYPE_F32])
@pytest.mark.parametrize("dim, vocab", [(8192, 32000), (2048, 8192), (1024, 32000), (512, 8192), (640, 50304), (4096, 128256),
                                        (64, 256)])
@pytest.mark.parametrize("tokens", [300, 2047, 8192, 65536])
def test_what_is_held_for_the_tokens_is_within_the_piece(tokens, dim, vocab, dtype, kind):
    """Everything but the head's copy and the sum of its gradient, and a weight a token, is within piece_bytes, or what
    256 tokens take where that is more (with gradients)."""
    kw = dict(KINDS[kind], tokens=tokens, dim=dim, vocab=vocab, hidden_stride=dim, weight_stride=dim, dtype=dtype,
              d_hidden=256, d_weight=256, d_hidden_stride=dim, d_weight_stride=dim)
    fp32 = dtype == P.CKPT_TYPE_F32
    planes = 3 if fp32 else 1
    words = up(vocab, 64)
    token = 2 * planes * (words + dim) + (0 if kind == "ce" and not fp32 else 4 * words) + 12 * (words // 64) + 4
    for piece in (1, 1 << 20, 16 << 20, 64 << 20, 256 << 20, 1 << 30, 0):
        rc, total = need(piece_bytes=piece, **kw)
        assert rc == P.CKPT_OK
        head = (6 * vocab * dim if fp32 else 0) + 4 * tokens
        held = max(piece or 2 << 30, 256 * token)
        if total - head > held + 16 * 256:  # more than one piece: the head's gradient is summed over them
            head += 4 * vocab * dim
        assert total - head <= held + 16 * 256, (piece, total - head, held)


@pytest.mark.parametrize("temperature", [1e-39, 2.9e-39, 1e-45, 1.9e19, 1e30, 3.4e38])
def test_temperatures_whose_inverse_or_square_is_infinite_are_refused(temperature):
    """0 times an infinite 1/T, or an infinite T^2 times 0, would make a finite row NaN."""
    assert need(**dict(TEACHER, temperature=temperature))[0] == P.CKPT_EINVAL


@pytest.mark.parametrize("temperature", [3e-39, 1e-30, 0.01, 1.0, 1e4, 1.8e19])
def test_other_temperatures_are_not(temperature):
    assert need(**dict(TEACHER, temperature=temperature))[0] == P.CKPT_OK


def test_the_package_takes_the_operators_names_and_no_others():
    """What ops.py imports for itself (typing, contextlib) is not the package's."""
    assert not any(hasattr(P, name) for name in ("NamedTuple", "Optional", "contextlib"))
    assert all(hasattr(P, name) for name in ops.__all__)
    public = {k for k, x in vars(ops).items() if k.startswith(("ckpt_", "CKPT_")) and getattr(x, "__module__", ops.__name__) == ops.__name__}
    from paper_2607_01646_amd import ckpt
    assert public - set(vars(ckpt)) <= set(ops.__all__)
