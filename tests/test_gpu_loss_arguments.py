"""Shapes of what the vocabulary head's losses are given for each token (needs
an MI355X; through the C ABI)."""
import pytest
import torch

from ops_util import check, definition, inputs

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P


def test_targets_and_weights_in_another_order_are_refused():
    """As many values as there are tokens, but of another shape: [sequence, batch] for hidden [batch, sequence, dim]."""
    x = inputs(12, 64, 100, torch.bfloat16, masked=0.2, topk=3)
    hidden, weight = x.hidden.view(3, 4, 64), torch.rand(3, 4, device="cuda") + 0.5
    target = x.target.view(3, 4)
    index, logits = x.teacher_index.view(3, 4, 3), x.teacher_logits.view(3, 4, 3)
    for t in (target.t().contiguous(), target.view(2, 6), target.view(6, 1, 2)):
        with pytest.raises(ValueError, match="target"):
            P.ckpt_linear_ce(hidden, x.weight, t)
        with pytest.raises(ValueError, match="target"):
            P.ckpt_linear_distill(hidden, x.weight, index, logits, target=t, alpha=0.5)
        with pytest.raises(ValueError, match="token_weight"):
            P.ckpt_linear_ce(hidden, x.weight, target, token_weight=torch.ones_like(t, dtype=torch.float32))
    with pytest.raises(ValueError, match="target"):
        P.ckpt_linear_ce(x.hidden, x.weight, target)
    ref = definition(x.hidden, x.weight, x.target, token_weight=weight.view(-1))
    for t in (target, x.target, target[None], target[:, None]):  # the tokens' order, whatever the dimensions of one
        check(P.ckpt_linear_ce(hidden, x.weight, t, token_weight=weight.view(t.shape), grad=True), ref)
        check(P.ckpt_linear_ce(hidden[:, None], x.weight, t, token_weight=weight.view(t.shape), grad=True), ref)


def test_one_token_has_no_shape_of_its_own():
    x = inputs(1, 64, 100, torch.float32)
    ref = definition(x.hidden, x.weight, x.target)
    for t in (x.target, x.target[0], x.target[None]):
        r = P.ckpt_linear_ce(x.hidden[0], x.weight, t, grad=True)
        assert r.token_loss.shape == () and r.d_hidden.shape == (64,)
        check(r, ref)
