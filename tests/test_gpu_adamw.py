"""The gradient norm and AdamW over fragments against the definition in 64
bits (needs an MI355X; through the C ABI)."""
import math

import pytest
import torch

from ops_util import U32, UBF, within

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

BF, F32 = torch.bfloat16, torch.float32
EDGES = [1, 2, 3, 4, 5, 7, 0, 255, 1023, 1024, 2047, 2048, 2049, 4095, 4097, 8191, 8192, 8193, 20_000, 0]


def fragments(sizes, param, grad, seed=0, gap=0):
    """Lists of views into flat buffers, `gap` elements apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(sizes) + gap * len(sizes) + 1
    flat = [torch.randn(total, generator=g, device="cuda") * s for s in (0.02, 1e-3, 1e-3, 1e-2)]
    flat[2].square_()
    flat = [flat[0].to(param), flat[0], flat[1], flat[2], flat[3].to(grad)]
    lists, at = [[] for _ in flat], gap
    for n in sizes:
        for k, t in enumerate(flat):
            lists[k].append(t[at:at + n])
        at += n + gap
    return lists, flat


def adamw(param, master, m, v, grad, step, lr, b1, b2, eps, wd, c):
    """One step in 64 bits, and how far fp32 may be off: some ten roundings on
    the way to each value."""
    g = grad.double() * c
    m2 = b1 * m.double() + (1 - b1) * g
    v2 = b2 * v.double() + (1 - b2) * g * g
    up = (m2 / (1 - b1 ** step)) / ((v2 / (1 - b2 ** step)).sqrt() + eps)
    w = master.double() * (1 - lr * wd) - lr * up
    few = 12 * U32
    b_m = few * (b1 * m.double().abs() + (1 - b1) * g.abs())
    b_up = few * up.abs() + lr * 0 + (b_m / (1 - b1 ** step)) / ((v2 / (1 - b2 ** step)).sqrt() + eps)
    b_w = few * (master.double().abs() + lr * up.abs()) + lr * b_up
    p = w if param.dtype == F32 else w
    return dict(master=(w, b_w), m=(m2, b_m), v=(v2, few * v2), param=(p, b_w + (UBF * w.abs() if param.dtype == BF else 0)))


@pytest.mark.parametrize("param", [BF, F32])
@pytest.mark.parametrize("grad", [BF, F32])
@pytest.mark.parametrize("gap", [0, 1, 7, 64])
def test_adamw(param, grad, gap):
    lists, flat = fragments(EDGES, param, grad, gap=gap)
    old = [t.clone() for t in flat]
    used = torch.zeros(flat[0].numel(), dtype=torch.bool, device="cuda")
    at = gap
    for n in EDGES:
        used[at:at + n] = True
        at += n + gap
    c = torch.tensor([0.37], device="cuda")
    kw = dict(step=3, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    P.ckpt_adamw(*lists, grad_scale=c, **kw)
    want = adamw(*old, 3, 1e-3, 0.9, 0.95, 1e-8, 0.1, float(c))
    for k, name in enumerate(("param", "master", "m", "v")):
        value, bound = want[name]
        within(flat[k][used], value[used], bound[used], name)
        assert torch.equal(flat[k][~used], old[k][~used]), name  # what lies between the fragments
    assert torch.equal(flat[4], old[4])
    assert torch.equal(flat[0][used], flat[1][used].to(param))  # the parameter is the master copy, rounded


def test_adamw_defaults_and_first_step():
    lists, flat = fragments([5000], F32, F32)
    for t in flat[2:4]:
        t.zero_()
    old = [t.clone() for t in flat]
    P.ckpt_adamw(*lists, step=1, lr=1e-3)
    want = adamw(*old, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0)
    for k, name in enumerate(("param", "master", "m", "v")):
        within(flat[k][:5000], want[name][0][:5000], want[name][1][:5000], name)


def test_more_fragments_than_a_launch_takes():
    sizes = [(37 * k) % 501 for k in range(700)]
    lists, flat = fragments(sizes, BF, BF, gap=1)
    alone, one = fragments(sizes, BF, BF, gap=1)
    P.ckpt_adamw(*lists, step=7, lr=1e-3, weight_decay=0.01)
    for row in zip(*alone):
        P.ckpt_adamw(*[[t] for t in row], step=7, lr=1e-3, weight_decay=0.01)
    assert all(torch.equal(a, b) for a, b in zip(flat, one))
    norm = P.ckpt_grad_norm(lists[4], max_norm=1e-3)
    want = torch.cat(lists[4]).double().norm()
    within(norm[0], want, 4 * U32 * want, "norm")
    within(norm[1], 1e-3 / (want + 1e-6), 4 * U32 * (1e-3 / (want + 1e-6)), "factor")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [[1], [0, 0], [3, 0, 8192, 1], EDGES, [3_000_001]])
def test_grad_norm(sizes, dtype):
    lists, flat = fragments(sizes, BF, dtype, gap=3)
    every = torch.cat(lists[4]).double()
    want = every.norm()
    for most in (0.0, float(want) / 3, float(want) * 3 + 1):
        r = P.ckpt_grad_norm(lists[4], max_norm=most)
        within(r[0], want, 4 * U32 * want, "norm")
        factor = min(1.0, most / (float(want) + 1e-6)) if most > 0 else 1.0
        assert abs(float(r[1]) - factor) <= 4 * U32 * factor
        assert torch.equal(r, P.ckpt_grad_norm(lists[4], max_norm=most))


def test_grad_norm_of_squares_beyond_fp32():
    big = torch.full((5000,), 1e30, device="cuda")
    small = torch.full((5000,), 1e-30, device="cuda")
    assert abs(float(P.ckpt_grad_norm([big])[0]) / (1e30 * math.sqrt(5000)) - 1) < 1e-6
    assert abs(float(P.ckpt_grad_norm([small])[0]) / (1e-30 * math.sqrt(5000)) - 1) < 1e-6


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_gradients_that_are_no_numbers_show(value):
    lists, flat = fragments([100, 3000], BF, BF)
    lists[4][1][5] = value
    r = P.ckpt_grad_norm(lists[4], max_norm=1.0)
    assert not torch.isfinite(r[0]) and not (r[1] > 0)  # inf: factor 0; NaN: NaN


def test_many_elements():
    """More than 2^31 elements in one fragment."""
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.5, dtype=BF, device="cuda")
    g[-1] = 3.0
    r = P.ckpt_grad_norm([g])
    want = math.sqrt((n - 1) * 0.25 + 9)
    assert abs(float(r[0]) / want - 1) < 4 * U32
    p = torch.zeros(n, dtype=BF, device="cuda")
    w, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    P.ckpt_adamw([p], [w], [m], [v], [g], step=1, lr=0.5, eps=0.0)
    ends = torch.tensor([0, 1, 12345, (1 << 31) - 1, 1 << 31, n - 2, n - 1], device="cuda")
    assert torch.allclose(w[ends], torch.full((7,), -0.5, device="cuda"), rtol=1e-5)
    assert torch.equal(p[ends], w[ends].to(BF)) and abs(float(m[-1]) - 0.3) < 1e-6 and abs(float(v[-1]) - 0.009) < 1e-6
    assert float(w.sum(dtype=torch.float64)) == pytest.approx(-0.5 * n, rel=1e-5)


def test_another_stream_and_a_graph():
    lists, flat = fragments(EDGES, BF, BF, gap=1)
    twin, same = fragments(EDGES, BF, BF, gap=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    norm = P.ckpt_grad_norm(lists[4], max_norm=0.1, stream=s)
    P.ckpt_adamw(*lists, step=2, lr=1e-3, grad_scale=norm[1:], stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n2 = P.ckpt_grad_norm(twin[4], max_norm=0.1)
        P.ckpt_adamw(*twin, step=2, lr=1e-3, grad_scale=n2[1:])
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        if k:
            n = P.ckpt_grad_norm(lists[4], max_norm=0.1)
            P.ckpt_adamw(*lists, step=2, lr=1e-3, grad_scale=n[1:])
            torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat, same)), k


def test_refusals():
    lists, flat = fragments([10, 20], BF, F32)
    before = [t.clone() for t in flat]
    p, w, m, v, g = lists

    def refuse(error, *x, **kw):
        with pytest.raises(error):
            P.ckpt_adamw(*x, **{**dict(step=1, lr=1e-3), **kw})

    refuse(ValueError, p[:1], w, m, v, g)
    refuse(ValueError, [p[1], p[0]], w, m, v, g)
    refuse(ValueError, p, [x.double() for x in w], m, v, g)
    refuse(ValueError, p, w, m, v, [g[0], g[1].to(BF)])
    refuse(ValueError, [x.half() for x in p], w, m, v, g)
    refuse(ValueError, [x.cpu() for x in p], w, m, v, g)
    refuse(ValueError, p, w, m, v, [g[0], torch.zeros(40, device="cuda")[::2]])
    refuse(ValueError, p, w, m, v, g, grad_scale=torch.ones(2, device="cuda"))
    for kw in (dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(eps=-1.0), dict(lr=math.nan),
               dict(eps=math.inf), dict(weight_decay=math.inf)):
        refuse(P.CkptError, p, w, m, v, g, **kw)
    with pytest.raises(ValueError):
        P.ckpt_grad_norm([])
    with pytest.raises(ValueError):
        P.ckpt_grad_norm([g[0], p[0]])
    with pytest.raises(P.CkptError):
        P.ckpt_grad_norm(g, max_norm=math.nan)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat, before))
    P.ckpt_adamw([], [], [], [], [], step=1, lr=1e-3)
