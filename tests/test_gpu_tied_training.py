"""The table's and the orthogonalised step's operators together with the
others and the snapshots, as a training loop uses them
(examples/train_tied.py; needs an MI355X)."""
import math
import os
import sys

import pytest
import torch

from muon_util import orthogonal

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

if torch.cuda.is_available():
    import train_tied


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [100, 700])
def test_a_lost_state_is_restored_and_the_run_ends_as_if_it_never_was(dtype, tokens):
    kw = dict(steps=7, tokens=tokens, dim=96, ffn=200, vocab=300, dtype=dtype)
    got, losses = train_tied.run(lose=5, **kw)  # the snapshot is of step 4
    want, plain = train_tied.run(**kw)
    assert losses == plain and all(math.isfinite(x) for x in losses)
    for x, y in zip(got, want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def plain_gradients(model, ids, target):
    """The same model in 64 bits through torch's autograd."""
    table, up, down = [w.double().requires_grad_() for w in model.param]
    there = ids >= 0
    x = torch.where(there[:, None], table[ids.clamp(min=0)] * model.scale, 0.0)
    hidden = x + torch.relu(x @ up.t()) @ down.t()
    loss = torch.nn.functional.cross_entropy(hidden @ table.t(), target)
    loss.backward()
    return loss.detach(), [table.grad, up.grad, down.grad]


@pytest.mark.parametrize("tokens", [100, 700])
def test_gradients_and_the_step_against_plain_torch(tokens):
    """One path through all operators in fp32.  The gradients pass two products and a softmax in fp32, each of at most 700
    terms: sqrt(700) roundings of 2^-24 times the terms' size, some 1e-5 of the gradient's norm at the most."""
    model = train_tied.Model(300, 96, 200, torch.float32)
    ids, target = train_tied.batch(0, tokens, 300)
    loss, grads = model.gradients(ids, target)
    want_loss, want = plain_gradients(model, ids, target)
    assert abs(float(loss) - float(want_loss)) < 1e-5
    for g, w in zip(grads, want):
        assert float((g.double() - w).norm()) < 2e-5 * float(w.norm())
    before = [w.clone() for w in model.master]
    model.update(grads, 1, 1e-3)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    clip = min(1.0, 1 / (norm + 1e-6))
    for k in (1, 2):
        u = grads[k].double() * clip * (0.05 * 0.95 + 0.05)  # nesterov, from a momentum of zero
        x = orthogonal(u)
        step = before[k].double() * (1 - 1e-3 * 0.01) - 1e-3 * 0.2 * math.sqrt(max(u.shape)) * x
        # an update's elements are about lr 0.2: 1e-4 of that, and the master's own rounding
        assert float((model.master[k].double() - step).abs().max()) < 2e-8 + float(step.abs().max()) * 2.0 ** -23


def test_the_loss_along_a_gradient():
    """Differences of the loss along the table's gradient, which has both of its uses in it: a step of h changes it by
    2 h |g|^2, but for the third order and the losses' own 2^-24."""
    model = train_tied.Model(120, 64, 100, torch.float32)
    ids, target = train_tied.batch(3, 200, 120)
    loss, grads = model.gradients(ids, target)
    for k in range(3):
        g = grads[k].double()
        h = 1e-2 / float(g.norm())
        values = []
        for sign in (1, -1):
            twin = train_tied.Model(120, 64, 100, torch.float32)
            twin.param[k] = (twin.param[k].double() + sign * h * g).float()
            values.append(float(plain_gradients(twin, ids, target)[0]))
        slope = (values[0] - values[1]) / (2 * h)
        assert abs(slope / float(g.square().sum()) - 1) < 2e-2, k
