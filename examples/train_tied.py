"""Trains a small model whose head is its vocabulary table, with snapshots of its state, loses the state and goes on.

The table's rows go through one block, x + relu(x up^T) down^T, to the head.  Each step is the path that the operators
make: the lookup, the head's loss with both gradients, the block's gradients (torch's autograd), the lookup's gradient
added to the head's, the clip, the gate on the snapshot in flight, AdamW for the table and the orthogonalised step for the
block's matrices.  At --lose the live state is overwritten, the newest committed snapshot is restored and the lost steps are
taken again: every operator gives the same bits for the same inputs, so the run ends in exactly the state of one that was
never interrupted.

    python examples/train_tied.py --steps 12 --lose 7
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_01646_amd as P  # noqa: E402
import workloads as W  # noqa: E402


class Model:
    """table [vocab, dim] with its fp32 master copy and Adam moments, up [ffn, dim] and down [dim, ffn] with theirs and one
    momentum each: fragments in the order of a rank's shard."""

    def __init__(self, vocab, dim, ffn, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def new(*shape):
            return torch.randn(shape, generator=g, device="cuda") * 0.02

        self.master = [new(vocab, dim), new(ffn, dim), new(dim, ffn)]
        self.param = [w.to(dtype) for w in self.master]
        self.moment = [torch.zeros_like(w) for w in self.master]
        self.square = torch.zeros_like(self.master[0])  # the table's alone
        self.scale = dim ** 0.5

    def fragments(self):
        out = [self.param[0], self.master[0], self.moment[0], self.square]
        for k in (1, 2):
            out += [self.param[k], self.master[k], self.moment[k]]
        return out

    def dtypes(self):
        return [W.DT_FP32 if t.dtype == torch.float32 else W.DT_BF16 for t in self.fragments()]

    def classes(self):
        matrix = [W.CLS_PARAM, W.CLS_MASTER, W.CLS_ADAM_M]
        return matrix + [W.CLS_ADAM_V] + matrix * 2

    def gradients(self, ids, target):
        """(loss, gradients of table, up and down)."""
        table, up, down = self.param
        x = P.ckpt_embedding(table, ids, scale=self.scale).requires_grad_()
        up, down = up.detach().requires_grad_(), down.detach().requires_grad_()
        hidden = x + torch.relu(x @ up.t()) @ down.t()
        r = P.ckpt_linear_ce(hidden.detach(), table, target, grad=True)
        hidden.backward(r.d_hidden)
        P.ckpt_embedding_grad(x.grad, ids, table.shape[0], scale=self.scale, add_to=r.d_weight)
        return r.loss, [r.d_weight, up.grad, down.grad]

    def update(self, grads, step, lr):
        scale = P.ckpt_grad_norm(grads, max_norm=1.0)[1:]
        P.ckpt_adamw(self.param[:1], self.master[:1], self.moment[:1], [self.square], grads[:1], step=step, lr=lr, beta2=0.95,
                     weight_decay=0.01, grad_scale=scale)
        P.ckpt_muon(self.param[1:], self.master[1:], self.moment[1:], grads[1:], lr=lr, weight_decay=0.01, grad_scale=scale)


def batch(step, tokens, vocab):
    """The step's ids and the words that follow them: made from the step alone, as a data loader would."""
    g = torch.Generator(device="cuda").manual_seed(1000 + step)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    target = (ids * 7 + 3) % vocab
    pad = torch.rand(tokens, generator=g, device="cuda") < 0.1
    return ids.masked_fill(pad, -100), target.masked_fill(pad, -100)


def run(steps=12, lose=None, tokens=512, dim=256, ffn=512, vocab=1000, dtype=torch.bfloat16, lr=3e-3, every=2,
        log=lambda *a: None):
    """Trains, with a snapshot before the first step and after every `every`; returns (the state's fragments, the loss
    of each step)."""
    model = Model(vocab, dim, ffn, dtype)
    losses = [None] * steps
    with P.Checkpointer(model.fragments(), model.dtypes(), model.classes(), chunk_bytes=1 << 20, direct=True) as ck:
        snap = ck.snapshot(step=0)
        step = 0
        while step < steps:
            if step == lose:
                lose = None
                ck.wait_committed(snap)
                torch.cuda.synchronize()
                for t in model.fragments():
                    t.view(torch.uint8).fill_(0xA5)
                bad = ck.restore()
                assert bad == [], "restore reported bad chunks %s" % bad
                step = ck.latest()[1]
                log("state lost, restored: back at step %d" % step)
                continue
            loss, grads = model.gradients(*batch(step, tokens, vocab))
            ck.wait_captured(snap)  # the snapshot of the state before this step
            model.update(grads, step + 1, lr)
            losses[step] = float(loss)
            log("step %3d  loss %.4f" % (step, losses[step]))
            step += 1
            if step % every == 0:
                ck.wait_committed(snap)
                snap = ck.snapshot(step=step)
        ck.wait_committed(snap)
        torch.cuda.synchronize()
    return model.fragments(), losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--lose", type=int, default=7)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--ffn", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--fp32", action="store_true")
    a = ap.parse_args()
    kw = dict(steps=a.steps, tokens=a.tokens, dim=a.dim, ffn=a.ffn, vocab=a.vocab,
              dtype=torch.float32 if a.fp32 else torch.bfloat16)
    got, losses = run(lose=a.lose, log=print, **kw)
    want, plain = run(**kw)
    same = all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, want)) and losses == plain
    print("the interrupted run's state and losses are %s" % ("those of a run never interrupted, bit for bit" if same else
                                                             "NOT those of a run never interrupted"))
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
