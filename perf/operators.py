"""The training-step operators whose time is watched: the vocabulary head's losses with their gradients, and the
clipped optimizer step that the snapshot's gate protects against.

  op ce       softmax cross entropy of hidden [tokens, dim] against weight [vocab, dim]: loss, token losses and
              log-sum-exp; with `grad` also the gradients of both
  op distill  distillation from a teacher's `topk` logits a token at `temperature`, mixed with the cross entropy by
              `alpha`, with both gradients
  op adamw    gradient norm, clip and AdamW over a rank's fragments: parameter, fp32 master copy, both moments

The mean of a loss is over the tokens that count: a target of -100 does not, nor does a token whose weight is zero.
"""
import math
import random

import numpy as np
import torch

own = False

IGNORE = -100
BETA1, BETA2, EPS, DECAY, LR, MAX_NORM = 0.9, 0.95, 1e-8, 0.1, 3e-4, 1.0


def listed():
    return [
        # The smallest call: a toy model's head and one short sequence. Its time is launches and host work.
        dict(name="ce-toy", op="ce", grad=True, type="bf16", tokens=64, dim=64, vocab=256, masked=0.1, weighted=False),
        # Scoring one token against a 7B model's head: the head is read once, nothing else is large.
        dict(name="ce-score-token", op="ce", grad=False, type="bf16", tokens=1, dim=4096, vocab=32000, masked=0.0,
             weighted=False),
        # One sequence of a small GPT.
        dict(name="ce-gpt", op="ce", grad=True, type="bf16", tokens=512, dim=512, vocab=8192, masked=0.1,
             weighted=False),
        # A packed batch of a 1.3B GPT: odd numbers of tokens and words, and a weight for each token.
        dict(name="ce-ragged", op="ce", grad=True, type="bf16", tokens=2047, dim=2048, vocab=50301, masked=0.2,
             weighted=True),
        # The step of a 7B model on one GPU: two sequences of 4096.
        dict(name="ce-llama", op="ce", grad=True, type="bf16", tokens=8192, dim=4096, vocab=32000, masked=0.05,
             weighted=False),
        # Training in full precision.
        dict(name="ce-f32", op="ce", grad=True, type="f32", tokens=2048, dim=2048, vocab=8192, masked=0.1,
             weighted=False),
        # A small student.
        dict(name="distill-gpt", op="distill", grad=True, type="bf16", tokens=250, dim=512, vocab=8192, masked=0.1,
             weighted=False, topk=16, temperature=2.0, alpha=0.5),
        # A 7B student and a teacher's 64 best words a token, with the labels mixed in.
        dict(name="distill-llama", op="distill", grad=True, type="bf16", tokens=4096, dim=4096, vocab=32000,
             masked=0.05, weighted=False, topk=64, temperature=2.0, alpha=0.7),
        # A student in full precision that learns from the teacher alone.
        dict(name="distill-f32", op="distill", grad=True, type="f32", tokens=1023, dim=1024, vocab=8192, masked=0.1,
             weighted=True, topk=32, temperature=1.0, alpha=1.0),
        # The optimizer step of a toy model: 16 parameter tensors, launches and host work.
        dict(name="adamw-toy", op="adamw", type="bf16", layout="gpt", layers=1, hidden=64, vocab=256, seq=64),
        # A distributed optimizer's flat buffers in full precision: fragments start and end anywhere.
        dict(name="adamw-views", op="adamw", type="f32", layout="views", frags=500, params=60_000_000),
        # One rank of a 65B model under TP=8 x PP=8.
        dict(name="adamw-llama-rank", op="adamw", type="bf16", layout="llama", layers=10, hidden=8192, ffn=22016, tp=8),
    ]


def _log_between(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng: random.Random):
    op = rng.choice(["ce", "ce", "ce", "distill", "distill", "adamw"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "adamw":
        if rng.random() < 0.5:
            frags = _log_between(rng, 1, 1000)
            return dict(op=op, type=kind, layout="views", frags=frags,
                        params=_log_between(rng, 100 * frags, 300_000_000))
        return dict(op=op, type=kind, layout="gpt", layers=rng.randint(1, 8), hidden=8 * _log_between(rng, 8, 128),
                    vocab=_log_between(rng, 256, 50304), seq=_log_between(rng, 64, 2048))
    unit = rng.choice([1, 64, 64])  # one head in three has a width of any size
    most = 8192 * 4096 * 32000 // (1 if kind == "bf16" else 4)
    while True:
        tokens = 1 if rng.random() < 0.1 else _log_between(rng, 2, 8192)
        dim = max(1, _log_between(rng, 64, 8192) // unit) * unit
        vocab = _log_between(rng, 256, 50304)
        if tokens * dim * vocab <= most:
            break
    c = dict(op=op, grad=op == "distill" or rng.random() < 0.8, type=kind, tokens=tokens, dim=dim, vocab=vocab,
             masked=rng.choice([0.0, 0.1, 0.5]), weighted=rng.random() < 0.3)
    if op == "distill":
        c.update(topk=_log_between(rng, 1, 64), temperature=rng.choice([1.0, 2.0, 4.0]),
                 alpha=rng.choice([0.5, 0.9, 1.0]))
    return c


# ---- inputs ----


def _fragments(case):
    """Element counts of the parameters, and each one's offset in a flat buffer of all (elements)."""
    if case["layout"] == "views":
        n, total = case["frags"], case["params"]
        r = np.random.Generator(np.random.PCG64(n * 1000003 + total))  # the layout belongs to the case
        raw = np.exp(r.uniform(math.log(64.0), math.log(4e6), n))
        counts = [max(1, int(x)) for x in raw * (total / raw.sum())]
        unit = 1
    else:
        h = case["hidden"]
        if case["layout"] == "gpt":
            layer = [h, h, 3 * h * h, 3 * h, h * h, h, h, h, 4 * h * h, 4 * h, 4 * h * h, h]
            counts = [case["vocab"] * h, case["seq"] * h] + layer * case["layers"] + [h, h]
        else:
            tp, f = case["tp"], case["ffn"] // case["tp"]
            counts = [h, h // tp * h, h // tp * h, h // tp * h, h * h // tp, h, f * h, f * h, f * h] * case["layers"]
        unit = 128  # as an allocator aligns them
    ends = np.cumsum([-(-c // unit) * unit for c in counts]).tolist()
    return counts, [0] + ends[:-1], ends[-1]


def _normal(gen, shape, scale):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    s = {"case": case}
    if case["op"] == "adamw":
        counts, offsets, total = _fragments(case)
        flat = {"master": _normal(gen, total, 0.02), "m": _normal(gen, total, 1e-3),
                "v": _normal(gen, total, 1e-3).square_(), "grad": _normal(gen, total, 1e-3).to(dtype)}
        used = torch.zeros(total, dtype=torch.bool, device="cuda")
        for c, o in zip(counts, offsets):
            used[o:o + c] = True
        for t in flat.values():
            t.mul_(used)  # the space between fragments
        flat["param"] = flat["master"].to(dtype)
        s["flat"] = flat
        s["lists"] = {k: [t[o:o + c] for c, o in zip(counts, offsets)] for k, t in flat.items()}
        s["step"] = 1000
        return s
    n, d, v = case["tokens"], case["dim"], case["vocab"]
    weight = _normal(gen, (v, d), 0.02)
    target = torch.randint(0, v, (n,), generator=gen, device="cuda")
    # A trained model's states: near enough to the right word to raise its logit by 0 to 12.
    near = weight[target]
    lift = 12 * torch.rand((n, 1), generator=gen, device="cuda") / near.square().sum(1, keepdim=True)
    s["hidden"] = (_normal(gen, (n, d), 1.0) + lift * near).to(dtype)
    s["weight"] = weight.to(dtype)
    target[torch.rand(n, generator=gen, device="cuda") < case["masked"]] = IGNORE
    s["target"] = target
    s["token_weight"] = None
    if case["weighted"]:
        w = torch.rand(n, generator=gen, device="cuda").add_(0.5)
        w[torch.rand(n, generator=gen, device="cuda") < 0.1] = 0.0
        s["token_weight"] = w
    if case["op"] == "distill":
        k = case["topk"]
        # The teacher's best words: one is the label, the others are spread over the vocabulary, all distinct.
        first = torch.where(target >= 0, target, 0)[:, None]
        stride = v // k
        rest = torch.randint(0, stride, (n, k), generator=gen, device="cuda") + stride * torch.arange(k, device="cuda")
        index = torch.where(rest // stride == torch.div(first, stride, rounding_mode="floor"), first, rest)
        logits = _normal(gen, (n, k), 2.0) + 6 * (index == first)
        absent = torch.rand((n, k), generator=gen, device="cuda") < 0.05  # fewer than topk were kept
        absent |= (torch.rand((n, 1), generator=gen, device="cuda") < 0.02)  # or none for this token
        s["teacher_index"] = torch.where(absent, -1, index)
        s["teacher_logits"] = logits.to(dtype)
    return s


# ---- one pass ----


def run(s):
    case = s["case"]
    if own:
        import paper_2607_01646_amd as P
        if case["op"] == "adamw":
            L = s["lists"]
            s["step"] += 1
            norm = P.ckpt_grad_norm(L["grad"], max_norm=MAX_NORM)
            P.ckpt_adamw(L["param"], L["master"], L["m"], L["v"], L["grad"], step=s["step"], lr=LR, beta1=BETA1,
                         beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=norm[1:])
            f = s["flat"]
            return {"norm": norm[0], "param": f["param"], "master": f["master"], "m": f["m"], "v": f["v"]}
        if case["op"] == "ce":
            r = P.ckpt_linear_ce(s["hidden"], s["weight"], s["target"], token_weight=s["token_weight"],
                                 ignore_index=IGNORE, grad=case["grad"])
        else:
            r = P.ckpt_linear_distill(s["hidden"], s["weight"], s["teacher_index"], s["teacher_logits"],
                                      target=s["target"], temperature=case["temperature"], alpha=case["alpha"],
                                      token_weight=s["token_weight"], ignore_index=IGNORE, grad=case["grad"])
        out = {"loss": r.loss, "token_loss": r.token_loss, "lse": r.lse}
        if case["grad"]:
            out.update(d_hidden=r.d_hidden, d_weight=r.d_weight)
        return out
    return _plain_adamw(s) if case["op"] == "adamw" else _plain_loss(s)


def _plain_adamw(s):
    f = s["flat"]
    s["step"] += 1
    g = f["grad"].float()
    norm = (g * g).sum().sqrt()
    g = g * (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    f["m"].mul_(BETA1).add_(g * (1 - BETA1))
    f["v"].mul_(BETA2).add_(g * g * (1 - BETA2))
    top = f["m"] / (1 - BETA1 ** s["step"])
    down = (f["v"] / (1 - BETA2 ** s["step"])).sqrt() + EPS
    f["master"].mul_(1 - LR * DECAY).sub_(top / down * LR)
    f["param"].copy_(f["master"])
    return {"norm": norm, "param": f["param"], "master": f["master"], "m": f["m"], "v": f["v"]}


def _lse(x):
    top = x.amax(1, keepdim=True)
    return (x - top).exp().sum(1).log() + top[:, 0]


def _plain_loss(s):
    case, dtype = s["case"], s["hidden"].dtype
    h, w = s["hidden"].float(), s["weight"].float()
    logits = h @ w.t()
    n = logits.shape[0]
    rows = torch.arange(n, device=h.device)
    labelled = s["target"] >= 0
    label = torch.where(labelled, s["target"], 0)
    t = case.get("temperature", 1.0)
    alpha = case["alpha"] if case["op"] == "distill" else 0.0
    weight = torch.ones(n, device=h.device) if s["token_weight"] is None else s["token_weight"]
    hard = labelled * (1 - alpha)
    plain_lse = _lse(logits)
    token_loss = hard * (plain_lse - logits[rows, label])
    counts, lse = labelled & (alpha < 1), plain_lse
    if alpha:
        lse = _lse(logits / t)
        held = s["teacher_index"] >= 0
        at = torch.where(held, s["teacher_index"], 0)
        teacher = torch.where(held, s["teacher_logits"].float() / t, float("-inf"))
        soft = held.any(1)
        teacher = torch.where(soft[:, None], teacher, 0.0)
        log_q = teacher - _lse(teacher)[:, None]
        q = log_q.exp() * held
        log_p = logits.gather(1, at) / t - lse[:, None]
        token_loss = token_loss + alpha * t * t * (q * (torch.where(held, log_q, 0.0) - log_p)).sum(1)
        counts = counts | soft
    counts = counts & (weight != 0)
    token_loss = token_loss * counts
    lse = lse * counts
    total = (weight * counts).sum()
    scale = torch.where(total > 0, 1 / total, 0.0)
    out = {"loss": (token_loss * weight).sum() * scale, "token_loss": token_loss, "lse": lse}
    if not case["grad"]:
        return out
    d = (logits - plain_lse[:, None]).exp()
    d[rows, label] -= 1.0
    d *= hard[:, None]
    if alpha:
        d += (alpha * t) * soft[:, None] * (logits / t - lse[:, None]).exp()
        d.scatter_add_(1, at, -alpha * t * q)
    d *= (weight * counts * scale)[:, None]
    out["d_hidden"] = (d @ w).to(dtype)
    out["d_weight"] = (d.t() @ h).to(dtype)
    return out


# ---- what a pass cannot do without ----


def work(case):
    e = 2 if case["type"] == "bf16" else 4
    if case["op"] == "adamw":
        n = sum(_fragments(case)[0])
        return {"bytes": n * (e + 12 + 12 + e), "flops": 17 * n}
    n, d, v = case["tokens"], case["dim"], case["vocab"]
    data = n * d * e + v * d * e + 8 * n + 8 * n
    if case["weighted"]:
        data += 4 * n
    if case["op"] == "distill":
        data += n * case["topk"] * (8 + e)
    units = 1
    if case["grad"]:
        data += n * d * e + v * d * e
        units = 3
    return {"bytes": data, "flops": 2 * n * d * v * units}


# ---- the definition in 64 bits ----


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        f = s["flat"]
        step = s["step"] + 1
        grad = f["grad"].double()
        norm = torch.linalg.vector_norm(grad)
        grad *= min(1.0, MAX_NORM / (float(norm) + 1e-6))
        m = torch.lerp(grad, f["m"].double(), BETA1)
        v = torch.lerp(grad.square(), f["v"].double(), BETA2)
        update = m.div(1 - BETA1 ** step).div_(v.div(1 - BETA2 ** step).sqrt_().add_(EPS))
        master = f["master"].double()
        master -= LR * (update + DECAY * master)
        return {"norm": norm, "param": master, "master": master, "m": m, "v": v}
    n = case["tokens"]
    h, w = s["hidden"].double(), s["weight"].double()
    logits = torch.mm(h, w.t())
    target = s["target"]
    each = torch.ones(n, dtype=torch.float64, device="cuda") if s["token_weight"] is None else s["token_weight"].double()
    t, alpha = case.get("temperature", 1.0), (case["alpha"] if case["op"] == "distill" else 0.0)
    log_p = torch.log_softmax(logits, 1)
    a_label = (target != IGNORE).double() * (1 - alpha)
    label = target.clamp(min=0)[:, None]
    token_loss = -a_label * log_p.gather(1, label)[:, 0]
    lse = torch.logsumexp(logits, 1)
    counted = a_label > 0
    back = log_p.exp_()
    back.scatter_add_(1, label, -torch.ones_like(label, dtype=torch.float64))
    back *= a_label[:, None]
    if alpha:
        lse = torch.logsumexp(logits / t, 1)
        absent = s["teacher_index"] < 0
        some = ~absent.all(1)
        q = torch.softmax(s["teacher_logits"].double().div(t).masked_fill(absent, -math.inf), 1)
        q = torch.nan_to_num(q, nan=0.0)
        at = s["teacher_index"].clamp(min=0)
        log_s = torch.log_softmax(logits / t, 1)
        cross = -(q * log_s.gather(1, at)).sum(1)
        token_loss += alpha * t ** 2 * (torch.special.xlogy(q, q).sum(1) + cross)
        soft = log_s.exp_() * some[:, None]
        soft.scatter_add_(1, at, -q)
        back += alpha * t * soft
        counted |= some
    counted &= each != 0
    each = each * counted
    share = each / each.sum() if bool(counted.any()) else each
    token_loss = torch.where(counted, token_loss, 0.0)
    out = {"loss": (share * token_loss).sum(), "token_loss": token_loss, "lse": torch.where(counted, lse, 0.0)}
    if case["grad"]:
        back *= share[:, None]
        out["d_hidden"] = torch.mm(back, w)
        out["d_weight"] = torch.mm(back.t(), h)
    return out
