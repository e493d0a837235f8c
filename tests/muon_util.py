"""The orthogonalised step's definition in 64 bits, and how far a computation
may be off whose operands are held in 22 bits and whose sums are in fp32."""
import math
from types import SimpleNamespace

import torch

from ops_util import U32, UBF

A, B, C, EPS = 3.4445, -4.7750, 2.0315, 1e-7
U22 = 2.0 ** -22  # of two planes of fp16: half a step of the second, 2^-11 of half a step of the first


def _short(u):
    return u if u.shape[0] <= u.shape[1] else u.t()


def orthogonal(u, steps=5, coefficients=(A, B, C), eps=EPS, noise=None):
    """X of the definition; with `noise` (a generator) every value that the operator rounds is moved by as much as its
    rounding may move it: operands by 2^-22 of themselves and half of fp16's smallest step at their scale of 2^12, sums of k
    products by sqrt(k) roundings of fp32, each of a partial sum, which the factors' norms bound (and 2^-22 of it, the product
    of planes that is left out)."""
    a, b, c = coefficients
    x = _short(u.double())

    def rounded(t):
        return t if noise is None else t + (U22 * t.abs() + 2.0 ** -37) * _signs(t, noise)

    def product(p, q):
        r = p @ q
        if noise is None:
            return r
        return r + (math.sqrt(p.shape[1]) * U32 + U22) * _signs(r, noise) * p.norm(dim=1)[:, None] * q.norm(dim=0)[None, :]

    x = rounded(x / (x.norm() + eps))
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for k in range(steps):
        g = rounded(product(x, x.t().contiguous()))
        x = product(rounded(a * one + b * g + c * product(g, g)), x)
        if k + 1 < steps:
            x = rounded(x)
    return (x if u.shape[0] <= u.shape[1] else x.t()).contiguous()


def _signs(t, gen):
    return torch.randint(0, 2, t.shape, generator=gen, device=t.device).double() * 2 - 1


def bounds(u, **kw):
    """(X, bound on the 2-norm of its error, bound on an element's): 4 times what roundings of random sign make in the worst of
    three draws, in norm, and 8 times the largest element's."""
    want = orthogonal(u, **kw)
    gen = torch.Generator(device=u.device).manual_seed(1)
    off = [orthogonal(u, noise=gen, **kw) - want for _ in range(3)]
    return want, 4 * max(float(d.norm()) for d in off), 8 * max(float(d.abs().max()) for d in off)


def check_orthogonal(got, u, what="", **kw):
    want, norm, most = bounds(u, **kw)
    out = UBF if got.dtype == torch.bfloat16 else U32
    off = got.double() - want
    assert float(off.norm()) <= norm + out * float(want.norm()), "%s: norm of the error %.3g of %.3g, bound %.3g" % (
        what, float(off.norm()), float(want.norm()), norm + out * float(want.norm()))
    bad = off.abs() > most + 2 * out * want.abs()
    assert not bool(bad.any()), "%s: %d elements off" % (what, int(bad.sum()))


def step(param, master, momentum, grad, lr, beta, nesterov, wd, scale, c=1.0, **kw):
    """One step in 64 bits, and bounds: some ten roundings in fp32 on the way to each value, and lr * scale times X's error."""
    shape = param.shape
    g = grad.double().reshape(shape) * c
    m = beta * momentum.double().reshape(shape) + (1 - beta) * g
    u = beta * m + (1 - beta) * g if nesterov else m
    flat = u.reshape(shape[0], -1)
    x, norm, most = bounds(flat, **kw)
    x = x.reshape(shape)
    f = lr * scale
    w = master.double().reshape(shape) * (1 - lr * wd) - f * x
    few = 12 * U32
    b_m = few * (beta * momentum.double().reshape(shape).abs() + (1 - beta) * g.abs())
    # the update's own roundings reach X as a perturbation of as many ulps, which its error model's first rounding has 4 of
    b_w = few * (master.double().reshape(shape).abs() + abs(f) * x.abs()) + abs(f) * 4 * most
    p = b_w + (UBF * w.abs() if param.dtype == torch.bfloat16 else 0)
    return SimpleNamespace(master=(w, b_w), momentum=(m, b_m), param=(w, p), x=x, norm=norm)
