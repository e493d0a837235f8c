"""Trains the vocabulary head of a small model, with snapshots of its state, loses the state and goes on.

Each step is the path that the operators make: the loss and both gradients (cross entropy, or distillation from a
teacher's top logits with --teacher), the clip, the gate on the snapshot in flight, AdamW over the head's four
fragments, and every second step the next snapshot.  At --lose the live state is overwritten, as a replaced GPU's would be; the newest
committed snapshot is restored and the lost steps are taken again.  Every operator gives the same bits for the same
inputs, so the run ends in exactly the state of one that was never interrupted:

    python examples/train_head.py --steps 12 --lose 7 --teacher
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_01646_amd as P  # noqa: E402
import workloads as W  # noqa: E402


class Head:
    """lm_head [vocab, dim] with its fp32 master copy and Adam moments: fragments in the order of a rank's shard."""

    def __init__(self, vocab, dim, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.master = torch.randn(vocab, dim, generator=g, device="cuda") * 0.02
        self.weight = self.master.to(dtype)
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)

    def fragments(self):
        return [self.weight, self.master, self.m, self.v]

    def dtypes(self):
        return [W.DT_BF16 if self.weight.dtype == torch.bfloat16 else W.DT_FP32, W.DT_FP32, W.DT_FP32, W.DT_FP32]


def batch(step, tokens, dim, vocab, topk, dtype):
    """The step's hidden states, labels and teacher entries: made from the step alone, as a data loader would."""
    g = torch.Generator(device="cuda").manual_seed(1000 + step)
    hidden = torch.randn(tokens, dim, generator=g, device="cuda")
    # a word that the hidden state tells: its largest of the first `vocab` coordinates, so that there is something to learn
    target = hidden[:, :min(dim, vocab)].argmax(1)
    target[torch.rand(tokens, generator=g, device="cuda") < 0.1] = -100  # padding
    words = torch.randint(0, vocab, (tokens, topk), generator=g, device="cuda")
    words[:, 0] = target.clamp(min=0)
    logits = torch.randn(tokens, topk, generator=g, device="cuda")
    logits[:, 0] += 8
    return hidden.to(dtype), target, words, logits.to(dtype)


def run(steps=12, lose=None, teacher=False, tokens=512, dim=512, vocab=8192, topk=8, dtype=torch.bfloat16, lr=1e-2,
        every=2, log=lambda *a: None):
    """Trains, with a snapshot before the first step and after every `every`; returns (the state's fragments, the loss
    of each step)."""
    head = Head(vocab, dim, dtype)
    losses = [None] * steps
    classes = [W.CLS_PARAM, W.CLS_MASTER, W.CLS_ADAM_M, W.CLS_ADAM_V]
    with P.Checkpointer(head.fragments(), head.dtypes(), classes, chunk_bytes=1 << 20, direct=True) as ck:
        snap = ck.snapshot(step=0)
        step = 0
        while step < steps:
            if step == lose:
                lose = None
                ck.wait_committed(snap)
                torch.cuda.synchronize()
                for t in head.fragments():
                    t.view(torch.uint8).fill_(0xA5)
                bad = ck.restore()
                assert bad == [], "restore reported bad chunks %s" % bad
                step = ck.latest()[1]
                log("state lost, restored: back at step %d" % step)
                continue
            hidden, target, words, logits = batch(step, tokens, dim, vocab, topk, dtype)
            if teacher:
                r = P.ckpt_linear_distill(hidden, head.weight, words, logits, target=target, temperature=2.0, alpha=0.5,
                                          grad=True)
            else:
                r = P.ckpt_linear_ce(hidden, head.weight, target, grad=True)
            norm = P.ckpt_grad_norm([r.d_weight], max_norm=1.0)
            ck.wait_captured(snap)  # the snapshot of the state before this step
            P.ckpt_adamw([head.weight], [head.master], [head.m], [head.v], [r.d_weight], step=step + 1, lr=lr, beta2=0.95,
                         weight_decay=0.01, grad_scale=norm[1:])
            losses[step] = float(r.loss)
            log("step %3d  loss %.4f  gradient norm %.4f" % (step, losses[step], float(norm[0])))
            step += 1
            if step % every == 0:
                ck.wait_committed(snap)
                snap = ck.snapshot(step=step)
        ck.wait_committed(snap)
        torch.cuda.synchronize()
    return head.fragments(), losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--lose", type=int, default=7)
    ap.add_argument("--teacher", action="store_true")
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=8192)
    ap.add_argument("--fp32", action="store_true")
    a = ap.parse_args()
    kw = dict(steps=a.steps, teacher=a.teacher, tokens=a.tokens, dim=a.dim, vocab=a.vocab,
              dtype=torch.float32 if a.fp32 else torch.bfloat16)
    got, losses = run(lose=a.lose, log=print, **kw)
    want, plain = run(**kw)
    same = all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, want)) and losses == plain
    print("the interrupted run's state and losses are %s" % ("those of a run never interrupted, bit for bit" if same else
                                                             "NOT those of a run never interrupted"))
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
