"""The vocabulary head's losses at values that are no numbers, at the ends of
fp32's planes and over large vocabularies, against the definition in 64 bits
(needs an MI355X; through the C ABI)."""
import math
from types import SimpleNamespace

import pytest
import torch

from ops_util import check, definition, inputs, within

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

BF, F32 = torch.bfloat16, torch.float32


def distill(x, **kw):
    return P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target, **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("temperature, alpha", [(1.0, 1.0), (2.0, 1.0), (2.0, 0.5), (0.5, 1.0)])
@pytest.mark.parametrize("tokens", [3, 70, 300])
def test_nan_in_a_hidden_state_shows_in_distillation(tokens, temperature, alpha, grad, dtype):
    x = inputs(tokens, 64, 300, dtype, seed=tokens, topk=5)
    x.hidden[1, 7] = math.nan
    kw = dict(temperature=temperature, alpha=alpha)
    r = distill(x, grad=grad, **kw)
    odd = torch.arange(tokens, device="cuda") == 1
    assert torch.equal(r.lse.isnan(), odd) and torch.equal(r.token_loss.isnan(), odd) and r.loss.isnan()
    if grad:
        assert torch.equal(r.d_hidden.isnan().all(1), odd) and torch.equal(r.d_hidden.isnan().any(1), odd)
        assert r.d_weight.isnan().all()
    y = SimpleNamespace(**{k: t if k == "weight" else t[~odd] for k, t in vars(x).items()})
    ref = definition(y.hidden, y.weight, y.target, y.teacher_index, y.teacher_logits, **kw)
    check(P.LinearLoss(ref.loss, r.token_loss[~odd], r.lse[~odd], None, None), ref, grad=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("temperature, alpha", [(1.0, 1.0), (2.0, 1.0), (2.0, 0.5), (0.5, 1.0)])
@pytest.mark.parametrize("tokens", [3, 70, 300])
@pytest.mark.parametrize("vocab, first, last", [(65, 64, 65), (300, 64, 128)])
def test_words_that_are_nan_show_in_every_row(vocab, first, last, tokens, temperature, alpha, grad, dtype):
    """A whole run of words whose statistics are joined (64, or what the vocabulary's end leaves) is NaN, and neither a
    label nor a teacher's word is among them."""
    x = inputs(tokens, 64, vocab, dtype, seed=vocab, topk=5)
    x.weight[first:last] = math.nan
    x.target %= 64
    x.teacher_index %= 64
    r = distill(x, grad=grad, temperature=temperature, alpha=alpha)
    assert r.lse.isnan().all() and r.token_loss.isnan().all() and r.loss.isnan()
    if grad:
        assert r.d_hidden.isnan().all() and r.d_weight.isnan().all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens", [3, 24, 25, 70, 300])
@pytest.mark.parametrize("kind", ["ce", "distill"])
def test_words_left_out_by_an_infinite_weight(kind, tokens, dtype):
    """Entries of -inf against a positive coordinate of every hidden state, and of +inf against a negative one: logits of
    -inf, whatever the type and the number of tokens, and the loss and gradients of the other words."""
    x = inputs(tokens, 64, 300, dtype, seed=tokens, topk=5)
    x.hidden[:, 0] = x.hidden[:, 0].abs() + 0.5
    x.hidden[::2, 0] = 1.0
    x.hidden[:, 1] = -x.hidden[:, 1].abs() - 0.5
    out = torch.zeros(300, dtype=torch.bool, device="cuda")
    out[64:128] = True  # a whole run
    out[[5, 130, 299]] = True
    keep = (~out).nonzero().flatten()
    x.weight[out, 0] = -math.inf
    x.weight[299, :2] = torch.tensor([0.25, math.inf], device="cuda").to(dtype)
    y = SimpleNamespace(hidden=x.hidden, weight=x.weight[keep], target=x.target % keep.numel())
    x.target = keep[y.target]
    kw = dict(temperature=2.0, alpha=0.5) if kind == "distill" else {}
    if kind == "distill":
        y.teacher_index, y.teacher_logits = x.teacher_index % keep.numel(), x.teacher_logits
        x.teacher_index = keep[y.teacher_index]
        ref = definition(y.hidden, y.weight, y.target, y.teacher_index, y.teacher_logits, **kw)
        call = lambda grad: distill(x, grad=grad, **kw)  # noqa: E731
    else:
        ref = definition(y.hidden, y.weight, y.target)
        call = lambda grad: P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=grad)  # noqa: E731
    check(call(False), ref, grad=False)
    r = call(True)
    check(r, ref, grad=False)
    # 0 times the infinite entries: coordinates 0 and 1 of d_hidden are NaN by the formula
    within(r.d_hidden[:, 2:], ref.d_hidden[:, 2:], ref.b_d_hidden[:, 2:], "d_hidden")
    within(r.d_weight[keep], ref.d_weight, ref.b_d_weight, "d_weight")
    assert not r.d_weight[out].any()


@pytest.mark.parametrize("sign", [1, -1])
def test_fp32_products_drop_no_more_than_they_say(sign):
    """One product a logit, of values with many ones in their significand, as three bf16 planes each.  The products of
    planes left out are 2^-24 (1 + 2^-9) of the value at most; the others are added from the smallest, so what their
    sums round is a unit in the last place of the largest, 2^-23, and 2^-8 of that for the next.  With one word the
    log-sum-exp is the logit."""
    g = torch.Generator().manual_seed(0)
    bits = (0x3F800000 + torch.randint(0, 1 << 23, (300,), generator=g)).int()
    bits[:8] = torch.tensor([0x3F80FFFF, 0x3F817FFF, 0x3F818000, 0x3F80FF80, 0x3FFFFFFF, 0x3F807F7F, 0x3F80FEFF, 0x3F800001])
    values = bits.view(F32).cuda()
    hidden = (sign * values)[:, None]
    for w in values[:8].tolist():
        r = P.ckpt_linear_ce(hidden, torch.full((1, 1), w, device="cuda"), torch.zeros(300, dtype=torch.int64, device="cuda"))
        want = hidden[:, 0].double() * w
        within(r.lse, want, 4 * 2.0 ** -24 * want.abs(), "logits")


def test_fp32_operands_near_the_ends_of_their_range():
    """Values whose rounding to bf16 would be beyond fp32, and small ones: the same bound (below it a product's smaller
    planes are no normal numbers)."""
    most = torch.finfo(F32).max
    hidden = torch.tensor([most, -most, most * (1 - 2.0 ** -9), 3.39e38, 1e-30, -1e-30, 1.0], device="cuda").repeat(10)[:, None]
    target = torch.zeros(70, dtype=torch.int64, device="cuda")
    for w in (0.4999, 2.0 ** -60, 2.0 ** -100 * 1.7):
        r = P.ckpt_linear_ce(hidden, torch.full((1, 1), w, device="cuda"), target)
        want = hidden[:, 0].double() * torch.tensor(w, device="cuda").double()
        within(r.lse, want, 8 * 2.0 ** -24 * want.abs() + 2.0 ** -126, "logits")


# More than the statistics that a row's workgroup keeps in registers (512 runs of 64 words), and more than it keeps
# factors of (8192): the words of the runs behind those are the likely ones.
@pytest.mark.parametrize("tokens, dim, vocab", [(300, 64, 32769), (300, 64, 50301), (70, 64, 50301), (260, 64, 524289)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_vocabularies(tokens, dim, vocab, dtype):
    x = inputs(tokens, dim, vocab, dtype, seed=vocab, masked=0.1)
    x.weight[32768:] *= 8 if vocab > 32769 else 30
    x.weight[524288:] *= 4
    ref = definition(x.hidden, x.weight, x.target)
    tail = (ref.lse - torch.logsumexp(x.hidden.double() @ x.weight[:32768].double().t(), 1))[ref.lse != 0]
    assert (tail > 1).sum() > tail.numel() // 4  # they matter
    check(P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True), ref)


@pytest.mark.parametrize("tokens", [70, 300])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_distillation_over_a_large_vocabulary(tokens, dtype):
    x = inputs(tokens, 64, 50301, dtype, seed=7, topk=9, masked=0.1)
    x.weight[32768:] *= 8
    kw = dict(temperature=2.0, alpha=0.5)
    ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, **kw)
    check(distill(x, grad=True, **kw), ref)
    check(distill(x, **kw), ref, grad=False)
