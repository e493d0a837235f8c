"""The operators together with the snapshots, as a training loop uses them
(examples/train_head.py; needs an MI355X)."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

if torch.cuda.is_available():
    import train_head


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("teacher", [False, True])
def test_a_lost_state_is_restored_and_the_run_ends_as_if_it_never_was(teacher, dtype):
    kw = dict(steps=7, teacher=teacher, tokens=300, dim=192, vocab=1000, dtype=dtype)
    got, losses = train_head.run(lose=5, **kw)  # the snapshot is of step 4
    want, plain = train_head.run(**kw)
    assert losses == plain
    for x, y in zip(got, want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert losses[-1] < losses[0]  # it learns


def test_the_step_against_plain_torch():
    """One path through all operators in fp32, against torch's own loss, clip and AdamW in 64 bits."""
    got, losses = train_head.run(steps=3, tokens=200, dim=96, vocab=300, dtype=torch.float32)
    w = train_head.Head(300, 96, torch.float32).master.double().requires_grad_()
    opt = torch.optim.AdamW([w], lr=1e-2, betas=(0.9, 0.95), weight_decay=0.01)
    for step in range(3):
        hidden, target, _, _ = train_head.batch(step, 200, 96, 300, 8, torch.float32)
        loss = torch.nn.functional.cross_entropy(hidden.double() @ w.t(), target)
        opt.zero_grad()
        loss.backward()
        torch.nn.utils.clip_grad_norm_([w], 1.0)
        opt.step()
        assert abs(losses[step] - float(loss.detach())) < 1e-5
    # a step moves a weight by at most about lr; Adam divides by the gradient's own size, so where that is near its
    # rounding the step may differ by a part of lr
    assert (got[1].double() - w).abs().max() < 1e-2 * 0.05
    assert (got[1].double() - w).norm() / w.norm() < 1e-4
