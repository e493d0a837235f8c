"""The training-step operators' definitions in 64 bits, with bounds on what a
computation in 32 bits (and bf16 where the types are) may be off, element by
element, from the formulas alone."""
import math
from types import SimpleNamespace

import torch

IGNORE = -100
U32 = 2.0 ** -24  # unit roundoff of fp32
UBF = 2.0 ** -8  # of bf16


def inputs(tokens, dim, vocab, dtype, seed=0, topk=0, masked=0.0, device="cuda"):
    g = torch.Generator(device="cpu").manual_seed(seed)
    hidden = torch.randn(tokens, dim, generator=g)
    weight = torch.randn(vocab, dim, generator=g) / math.sqrt(dim)
    target = torch.randint(0, vocab, (tokens,), generator=g)
    target[torch.rand(tokens, generator=g) < masked] = IGNORE
    d = dict(hidden=hidden.to(device).to(dtype), weight=weight.to(device).to(dtype), target=target.to(device))
    if topk:
        index = torch.stack([torch.randperm(vocab, generator=g)[:topk] for _ in range(tokens)]) if tokens else \
            torch.zeros(0, topk, dtype=torch.int64)
        d["teacher_index"] = index.to(device)
        d["teacher_logits"] = (2 * torch.randn(tokens, topk, generator=g)).to(device).to(dtype)
    return SimpleNamespace(**d)


def definition(hidden, weight, target=None, teacher_index=None, teacher_logits=None, temperature=1.0, alpha=1.0,
               token_weight=None, ignore_index=IGNORE, reduction="mean", grad_scale=1.0):
    """Values and bounds, row by row as the formulas say: loss, token_loss,
    lse, d_hidden, d_weight, and b_* for each."""
    dtype = hidden.dtype
    n, d = hidden.shape
    vocab = weight.shape[0]
    teach = teacher_index is not None and alpha > 0
    hard = (1 - alpha) if teach else 1.0
    t = temperature if teach else 1.0
    tw = torch.ones(n, dtype=torch.float64, device=hidden.device) if token_weight is None else token_weight.double()
    has_label = torch.zeros(n, dtype=torch.bool, device=hidden.device)
    if target is not None and hard > 0:
        has_label = target != ignore_index
    has_teacher = torch.zeros_like(has_label)
    if teach:
        there = (teacher_index >= 0) & (teacher_logits != -math.inf)
        has_teacher = there.any(1)
    counts = (has_label | has_teacher) & (tw != 0)
    h = torch.where(counts[:, None], hidden.double(), 0.0)
    w = weight.double()
    l = h @ w.t()
    # error of a logit: dim products and sums in fp32 (the planes of an fp32 operand drop below 2^-24 of a product)
    e_l = (d + 16) * U32 * (h.abs() @ w.abs().t()).amax(1) if vocab else torch.zeros(n)
    lse1 = torch.logsumexp(l, 1)
    lset = torch.logsumexp(l / t, 1)
    tiny = 32 * U32
    b_lse = e_l / t + tiny * (1 + lset.abs() + l.abs().amax(1) / t)
    b_lse1 = e_l + tiny * (1 + lse1.abs() + l.abs().amax(1))
    token = torch.zeros(n, dtype=torch.float64, device=h.device)
    b_token = torch.zeros_like(token)
    dl = torch.zeros_like(l)
    e_dl = torch.zeros_like(l)
    label = torch.where(has_label, target, 0) if target is not None else torch.zeros(n, dtype=torch.int64, device=h.device)
    rows = torch.arange(n, device=h.device)
    if hard > 0:
        token = token + hard * has_label * (lse1 - l[rows, label])
        b_token = b_token + hard * has_label * (b_lse1 + e_l + tiny * (lse1.abs() + l[rows, label].abs()))
        p = (l - lse1[:, None]).exp() * has_label[:, None]
        one = torch.zeros_like(l)
        one[rows, label] = has_label.double()
        dl = dl + hard * (p - one)
        e_dl = e_dl + hard * (p * (2 * (e_l + b_lse1)[:, None] + tiny * (1 + (l - lse1[:, None]).abs())) + tiny * one)
    if teach:
        x = torch.where(there, teacher_logits.double() / t, -math.inf)
        x = torch.where(has_teacher[:, None], x, 0.0)
        log_q = torch.log_softmax(x, 1)
        q = log_q.exp() * there
        at = torch.where(there, teacher_index, 0)
        log_p = l.gather(1, at) / t - lset[:, None]
        terms = torch.where(q > 0, q * (log_q - log_p), 0.0)
        token = token + alpha * t * t * terms.sum(1)
        spread = (torch.where(there, log_q.abs() + x.abs().clamp(max=1e30), 0.0) + log_p.abs()).amax(1)
        b_token = b_token + alpha * t * t * has_teacher * (
            2 * (e_l / t + b_lse) + (tiny + 4 * teacher_index.shape[1] * U32) * (1 + spread) * (1 + spread))
        pt = (l / t - lset[:, None]).exp() * has_teacher[:, None]
        qs = torch.zeros_like(l).scatter_add_(1, at, q)
        dl = dl + alpha * t * (pt - qs)
        e_dl = e_dl + alpha * t * (pt * (2 * (e_l / t + b_lse)[:, None] + tiny * (1 + (l / t - lset[:, None]).abs()))
                                   + qs * (tiny * (1 + spread[:, None]) + 4 * teacher_index.shape[1] * U32))
    token = token * counts
    b_token = b_token * counts
    each = tw * counts
    total = each.sum()
    over = (1 / total if bool(counts.any()) else 0.0) if reduction == "mean" else 1.0
    loss = (token * each).sum() * over
    b_loss = (b_token * each.abs()).sum() * over + 4 * U32 * loss.abs()
    dl = dl * each[:, None]
    e_dl = e_dl * each.abs()[:, None]
    if dtype == torch.bfloat16:
        e_dl = e_dl + UBF * dl.abs()
    scale = over * grad_scale
    k1, k2 = (vocab + 16) * U32, (n + 16) * U32
    dh, dw = scale * (dl @ w), scale * (dl.t() @ h)
    out = UBF if dtype == torch.bfloat16 else 4 * U32
    b_dh = abs(scale) * (e_dl @ w.abs() + k1 * (dl.abs() @ w.abs())) + out * dh.abs()
    b_dw = abs(scale) * (e_dl.t() @ h.abs() + k2 * (dl.t().abs() @ h.abs())) + out * dw.abs()
    return SimpleNamespace(loss=loss, b_loss=b_loss, token_loss=token, b_token_loss=b_token,
                           lse=(lset if teach else lse1) * counts, b_lse=(b_lse if teach else b_lse1) * counts,
                           d_hidden=dh, b_d_hidden=b_dh, d_weight=dw, b_d_weight=b_dw)


def within(got, want, bound, what):
    got = got.double().reshape(want.shape)
    bad = ~((got - want).abs() <= bound + 1e-30)
    if bool(bad.any()):
        k = int(bad.reshape(-1).nonzero()[0])
        raise AssertionError("%s: %d of %d outside, first %d: got %r, want %r, bound %r" % (
            what, int(bad.sum()), bad.numel(), k, float(got.reshape(-1)[k]), float(want.reshape(-1)[k]),
            float(torch.broadcast_to(bound, want.shape).reshape(-1)[k])))


def check(r, ref, grad=True):
    for name in ("loss", "token_loss", "lse") + (("d_hidden", "d_weight") if grad else ()):
        within(getattr(r, name), getattr(ref, name), getattr(ref, "b_" + name), name)
