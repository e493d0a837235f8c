"""The training-step operators beyond those of `operators.py` whose time is watched: the vocabulary table's lookup with its
gradient, and the optimizer step that orthogonalises a matrix's update.

  op embed       rows of table [vocab, dim] at `tokens` ids, times a scale
  op embed_grad  the table's gradient from the rows' gradients; with `tied` added to a gradient that is there (the head's)
  op muon        momentum, Newton-Schulz orthogonalisation and update of matrices: parameter, fp32 master copy, momentum
  op orth        the orthogonalisation alone

A token whose id is -100 is padding: its row is zero, and it gives no gradient.
"""
import random

import torch

own = False

IGNORE = -100
A, B, C, STEPS, EPS = 3.4445, -4.7750, 2.0315, 5, 1e-7
MOMENTUM, DECAY, LR = 0.95, 0.1, 3e-4


def listed():
    return [
        # One token of a 7B model's table, as at each step of a generation: latency.
        dict(name="embed-token", op="embed", type="bf16", tokens=1, dim=4096, vocab=32000, masked=0.0),
        # Two sequences of 4096 of a 7B model.
        dict(name="embed-llama", op="embed", type="bf16", tokens=8192, dim=4096, vocab=32000, masked=0.05),
        # A table in full precision with rows of an odd width, and an odd number of tokens.
        dict(name="embed-f32-odd", op="embed", type="f32", tokens=2047, dim=1001, vocab=50301, masked=0.1),
        # The gradient of a toy model's table from one short sequence: launches.
        dict(name="embed-grad-toy", op="embed_grad", type="bf16", tokens=64, dim=64, vocab=256, masked=0.1, tied=False),
        # A 7B model's table: most of the time is writing the rows that no token has.
        dict(name="embed-grad-llama", op="embed_grad", type="bf16", tokens=8192, dim=4096, vocab=32000, masked=0.05,
             tied=False),
        # A 1.3B GPT whose head is its table: a packed batch, added to the head's gradient.
        dict(name="embed-grad-tied", op="embed_grad", type="bf16", tokens=16383, dim=2048, vocab=50304, masked=0.2,
             tied=True),
        # The optimizer step of a toy model's layer: four small matrices.
        dict(name="muon-toy", op="muon", type="bf16", layout="gpt", layers=1, hidden=64),
        # All matrices of a small GPT.
        dict(name="muon-gpt", op="muon", type="bf16", layout="gpt", layers=4, hidden=512),
        # One layer of a 7B model.
        dict(name="muon-llama-layer", op="muon", type="bf16", layout="llama", layers=1, hidden=4096, ffn=11008, tp=1),
        # One layer of a rank of a 65B model under TP=8, in full precision.
        dict(name="muon-f32-rank", op="muon", type="f32", layout="llama", layers=1, hidden=8192, ffn=22016, tp=8),
        # An update by itself, for an optimizer of the user's own; odd sizes.
        dict(name="orth-odd", op="orth", type="bf16", rows=777, cols=1003),
        # A tall update in full precision.
        dict(name="orth-f32-tall", op="orth", type="f32", rows=8192, cols=2048),
    ]


def _log_between(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng: random.Random):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "muon", "muon", "orth"])
    kind = rng.choice(["bf16", "bf16", "f32"])
    if op in ("embed", "embed_grad"):
        unit = rng.choice([1, 64, 64])  # one table in three has a width of any size
        c = dict(op=op, type=kind, tokens=1 if rng.random() < 0.1 else _log_between(rng, 2, 65536),
                 dim=max(1, _log_between(rng, 64, 8192) // unit) * unit, vocab=_log_between(rng, 256, 128256),
                 masked=rng.choice([0.0, 0.1, 0.5]))
        if op == "embed_grad":
            c["tied"] = rng.random() < 0.4
        return c
    if op == "orth":
        return dict(op=op, type=kind, rows=_log_between(rng, 1, 8192), cols=_log_between(rng, 1, 8192))
    if rng.random() < 0.5:
        return dict(op=op, type=kind, layout="gpt", layers=rng.randint(1, 5), hidden=8 * _log_between(rng, 8, 128))
    h = 64 * _log_between(rng, 4, 64)
    return dict(op=op, type=kind, layout="llama", layers=1, hidden=h, ffn=h * 8 // 3 // 64 * 64, tp=rng.choice([1, 2, 8]))


# ---- inputs ----


def _shapes(case):
    if case["op"] == "orth":
        return [(case["rows"], case["cols"])]
    h = case["hidden"]
    if case["layout"] == "gpt":
        layer = [(3 * h, h), (h, h), (4 * h, h), (h, 4 * h)]
    else:
        q, f = h // case["tp"], case["ffn"] // case["tp"]
        layer = [(q, h), (q, h), (q, h), (h, q), (f, h), (f, h), (h, f)]
    return layer * case["layers"]


def _normal(gen, shape, scale):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale)


def _gradient(gen, shape):
    """A matrix's gradient: few directions that most tokens share, over noise."""
    k = 1 + min(shape) // 8
    return (_normal(gen, (shape[0], k), k ** -0.5) @ _normal(gen, (k, shape[1]), 1.0)).add_(_normal(gen, shape, 0.5)).mul_(1e-3)


def _ids(gen, case):
    """Words as often as in text: the n-th most frequent about 1/n of the most frequent, at any place of the table."""
    n, v = case["tokens"], case["vocab"]
    often = (v + 1.0) ** torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    word = (often.long() - 1).clamp_(0, v - 1)
    ids = torch.randperm(v, generator=gen, device="cuda")[word]
    ids[torch.rand(n, generator=gen, device="cuda") < case["masked"]] = IGNORE
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    s = {"case": case}
    if case["op"] in ("embed", "embed_grad"):
        n, d, v = case["tokens"], case["dim"], case["vocab"]
        s["ids"] = _ids(gen, case)
        s["scale"] = float(d) ** 0.5
        if case["op"] == "embed":
            s["table"] = _normal(gen, (v, d), 0.02).to(dtype)
        else:
            s["d_out"] = _normal(gen, (n, d), 1e-3).to(dtype)
            if case["tied"]:
                s["d_table"] = _normal(gen, (v, d), 1e-2).to(dtype)
        return s
    shapes = _shapes(case)
    s["grad"] = [_gradient(gen, x).to(dtype) for x in shapes]
    if case["op"] == "muon":
        s["master"] = [_normal(gen, x, 0.02) for x in shapes]
        s["param"] = [w.to(dtype) for w in s["master"]]
        s["momentum"] = [_gradient(gen, x) for x in shapes]
    return s


# ---- one pass ----


def run(s):
    case = s["case"]
    if own:
        import paper_2607_01646_amd as P
        if case["op"] == "embed":
            return P.ckpt_embedding(s["table"], s["ids"], scale=s["scale"], ignore_index=IGNORE)
        if case["op"] == "embed_grad":
            return P.ckpt_embedding_grad(s["d_out"], s["ids"], case["vocab"], scale=s["scale"], ignore_index=IGNORE,
                                         add_to=s.get("d_table"))
        if case["op"] == "orth":
            return P.ckpt_orthogonalize(s["grad"])
        P.ckpt_muon(s["param"], s["master"], s["momentum"], s["grad"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY)
        return {k: s[k] for k in ("param", "master", "momentum")}
    if case["op"] == "embed":
        there = s["ids"] >= 0
        rows = s["table"][torch.where(there, s["ids"], 0)].float() * s["scale"]
        return torch.where(there[:, None], rows, 0.0).to(s["table"].dtype)
    if case["op"] == "embed_grad":
        there = s["ids"] >= 0
        rows = torch.where(there[:, None], s["d_out"].float(), 0.0)
        total = torch.zeros(case["vocab"], case["dim"], device=rows.device)
        total.index_add_(0, torch.where(there, s["ids"], 0), rows)
        total *= s["scale"]
        if not case["tied"]:
            return total.to(s["d_out"].dtype)
        s["d_table"].copy_(total.add_(s["d_table"]))
        return s["d_table"]
    if case["op"] == "orth":
        return [_plain_orthogonal(g.float()).to(g.dtype) for g in s["grad"]]
    for param, master, momentum, grad in zip(s["param"], s["master"], s["momentum"], s["grad"]):
        g = grad.float() * (1 - MOMENTUM)
        momentum.mul_(MOMENTUM).add_(g)
        x = _plain_orthogonal(momentum * MOMENTUM + g)
        master.mul_(1 - LR * DECAY).sub_(x * (LR * 0.2 * max(x.shape) ** 0.5))
        param.copy_(master)
    return {k: s[k] for k in ("param", "master", "momentum")}


def _plain_orthogonal(u):
    x = u / (u.square().sum(dtype=torch.float64).sqrt() + EPS).float()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    for _ in range(STEPS):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.t() if tall else x


# ---- what a pass cannot do without ----


def work(case):
    e = 2 if case["type"] == "bf16" else 4
    if case["op"] in ("embed", "embed_grad"):
        n, d, v = case["tokens"], case["dim"], case["vocab"]
        counted = n * (1 - case["masked"])
        # distinct words among n of this distribution: a word of rank r is met n / (r log v) times
        rank = torch.arange(1, v + 1, dtype=torch.float64)
        distinct = float((1 - (-(counted * (torch.log1p(1 / rank) / torch.log(torch.tensor(v + 1.0))))).exp()).sum())
        if case["op"] == "embed":
            return {"bytes": 8 * n + (distinct + n) * d * e, "flops": counted * d}
        rows = 2 * distinct if case["tied"] else v
        return {"bytes": 8 * n + (counted + rows) * d * e, "flops": counted * d}
    data = flops = 0
    for r, c in _shapes(case):
        s, l = min(r, c), max(r, c)
        # a step: A = X X^T and A A are symmetric, half of each is computed; then the product with X
        flops += STEPS * (s * s * l + s * s * s + 2 * s * s * l)
        data += r * c * (2 * e if case["op"] == "orth" else e + 8 + 8 + e)
    return {"bytes": data, "flops": flops}


# ---- the definition in 64 bits ----


def _definite(u):
    """The same polynomials from the other side: of the short dimension's Gram matrix, on the matrix stood upright."""
    y = (u if u.shape[0] >= u.shape[1] else u.t()).contiguous()
    y = y / (torch.linalg.vector_norm(y) + EPS)
    one = torch.eye(y.shape[1], dtype=torch.float64, device=y.device)
    for _ in range(STEPS):
        gram = torch.mm(y.t(), y)
        y = torch.mm(y, torch.addmm(A * one + B * gram, gram, gram, alpha=C))
    return y if u.shape[0] >= u.shape[1] else y.t()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["ids"] != IGNORE)[:, 0]
        out[at] = torch.index_select(s["table"], 0, s["ids"][at]).double() * s["scale"]
        return out
    if case["op"] == "embed_grad":
        at = torch.nonzero(s["ids"] != IGNORE)[:, 0]
        order = at[torch.argsort(s["ids"][at], stable=True)]
        word = s["ids"][order]
        out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
        if order.numel():
            words, count = torch.unique_consecutive(word, return_counts=True)
            owner = torch.repeat_interleave(torch.arange(words.numel(), device="cuda"), count)
            sums = torch.zeros(words.numel(), case["dim"], dtype=torch.float64, device="cuda")
            sums.index_add_(0, owner, s["d_out"][order].double())
            out[words] = sums * s["scale"]
        if case["tied"]:
            out += s["d_table"].double()
        return out
    if case["op"] == "orth":
        return [_definite(g.double()) for g in s["grad"]]
    out = {"param": [], "master": [], "momentum": []}
    for w, m, g in zip(s["master"], s["momentum"], s["grad"]):
        g = g.double()
        m = torch.lerp(g, m.double(), MOMENTUM)
        x = _definite(torch.lerp(g, m, MOMENTUM))
        w = w.double() * (1 - LR * DECAY) - (LR * 0.2 * max(w.shape) ** 0.5) * x
        out["param"].append(w)
        out["master"].append(w)
        out["momentum"].append(m)
    return out
