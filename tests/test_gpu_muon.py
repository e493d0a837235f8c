"""The orthogonalisation and the optimizer step with it against the definition
in 64 bits (needs an MI355X; through the C ABI)."""
import math

import pytest
import torch

from muon_util import check_orthogonal, orthogonal, step
from ops_util import U32, within

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

BF, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, 1), (1, 7), (7, 1), (1, 5000), (3000, 1), (2, 1033), (16, 16), (5000, 16), (15, 257), (200000, 3), (2, 3), (31, 33), (63, 65), (64, 64), (65, 64), (64, 256), (130, 70), (127, 513),
          (300, 1000), (1000, 300), (512, 512), (257, 2049)]


def matrix(shape, dtype=F32, seed=0, few=False, scale=1e-2):
    g = torch.Generator(device="cuda").manual_seed(seed + 7919 * shape[0] + shape[1])
    x = torch.randn(shape, generator=g, device="cuda")
    if few:  # some directions, and little beside them
        k = max(1, min(shape) // 16)
        x = torch.randn(shape[0], k, generator=g, device="cuda") @ torch.randn(k, shape[1], generator=g, device="cuda") + 0.1 * x
    return (x * scale).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize(shape, dtype):
    x = matrix(shape, dtype)
    old = x.clone()
    y, = P.ckpt_orthogonalize([x])
    assert y.dtype == dtype and y.shape == x.shape and torch.equal(x, old)
    check_orthogonal(y, x, str(shape))


@pytest.mark.parametrize("shape", [(64, 64), (200, 900), (900, 200), (512, 512)])
def test_few_directions(shape):
    x = matrix(shape, few=True)
    check_orthogonal(P.ckpt_orthogonalize([x])[0], x, str(shape))


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e12, 1e30])
def test_sizes_of_the_values(scale):
    """Below eps the norm does not show; squares beyond fp32 do not matter."""
    x = matrix((70, 130), scale=1.0) * scale
    check_orthogonal(P.ckpt_orthogonalize([x])[0], x, str(scale))


def test_one_element_beside_zeros():
    x = torch.zeros(300, 200, device="cuda")
    x[17, 131] = -3.0
    y, = P.ckpt_orthogonalize([x])
    check_orthogonal(y, x)
    y[17, 131] = 0
    assert not y.any()


def test_thin_matrices_are_as_exact_as_64_bits_let_them():
    """Short sides up to 16 are rounded once, at the end.  What 64 bits leave grows by a step's factor, 3.45, twice for every
    step but one: 16 * 2^-53 * 3.45^8, 4e-11."""
    for shape in ((1, 300), (3, 5), (16, 700), (900, 11)):
        for few in (False, True):
            x = matrix(shape, few=few)
            y, = P.ckpt_orthogonalize([x])
            want = orthogonal(x)
            assert bool(((y.double() - want).abs() <= 2 * U32 * want.abs() + 1e-9).all()), shape
    # with so many steps that the Gram matrix of U would not do
    for shape in ((5, 400), (1, 700), (900, 1), (3000, 16)):
        x = matrix(shape)
        y, = P.ckpt_orthogonalize([x], steps=64, coefficients=(1.5, -0.5, 0.0))
        check_orthogonal(y, x, steps=64, coefficients=(1.5, -0.5, 0.0))


def test_thin_zeros_and_what_is_no_number():
    good, zero = matrix((7, 300)), torch.zeros(300, 9, device="cuda")
    bad = [matrix((4, 600)), matrix((600, 4)), matrix((1, 5))]
    bad[0][2, 599], bad[1][0, 0], bad[2][0, 4] = math.nan, math.inf, -math.inf
    out = P.ckpt_orthogonalize([bad[0], good, zero, bad[1], bad[2]])
    assert all(bool(out[k].isnan().all()) for k in (0, 3, 4)) and not out[2].any()
    assert torch.equal(out[1], P.ckpt_orthogonalize([good])[0])


def test_long_rows_alone_and_among_others():
    """Gram matrices of few long rows are summed by many workgroups, and by fewer in a call of many: to the same bits."""
    for shape, n in (((448, 4096), 32), ((65, 5001), 40), ((3000, 130), 64), ((509, 2600), 20)):
        x = [matrix(shape, scale=k + 1) for k in range(2)]
        alone = [P.ckpt_orthogonalize([y])[0] for y in x]
        check_orthogonal(alone[1], x[1])
        among = P.ckpt_orthogonalize([x[k % 2] for k in range(n)] + [matrix((300, 300))])
        assert all(torch.equal(among[k], alone[k % 2]) for k in range(n)), shape


def test_zeros_and_what_is_no_number():
    """In one call: each matrix goes by itself."""
    good = matrix((80, 200))
    zero = torch.zeros(100, 90, device="cuda")
    bad = [matrix((70, 80)), matrix((80, 70)), matrix((64, 64))]
    bad[0][3, 5], bad[1][69, 0], bad[2][0, 0] = math.nan, math.inf, -math.inf
    out = P.ckpt_orthogonalize([bad[0], good, zero, bad[1], bad[2]])
    assert all(bool(out[k].isnan().all()) for k in (0, 3, 4))
    assert not out[2].any()
    assert torch.equal(out[1], P.ckpt_orthogonalize([good])[0])


def test_a_matrix_does_not_depend_on_the_others():
    """Groups by the workspace's bound, launches of 32, and sizes of tiles that the number of matrices decides."""
    shapes = SHAPES + [(96, 64)] * 40 + [(700, 800)] * 8
    x = [matrix(s, seed=k) for k, s in enumerate(shapes)]
    alone = [P.ckpt_orthogonalize([t])[0] for t in x]
    for piece in (0, 1, 4 << 20):
        for a, b in zip(P.ckpt_orthogonalize(x, piece_bytes=piece), alone):
            assert torch.equal(a, b), (piece, tuple(a.shape))
    assert P.ckpt_orthogonalize([]) == []


@pytest.mark.parametrize("count", [2, 3, 4, 6, 16, 24])
def test_every_size_of_tiles(count):
    """So many matrices of the same sides that each size of tiles is the quickest for some launch: a matrix's result is that
    of its own call, which is checked."""
    x = [matrix((1000, 1100) if k % 2 else (1100, 1000), BF if count == 4 else F32, seed=k) for k in range(count)]
    out = P.ckpt_orthogonalize(x)
    for a, b in zip(out, x):
        assert torch.equal(a, P.ckpt_orthogonalize([b])[0])
    for k in range(2):
        check_orthogonal(out[k], x[k])


def test_more_parts_of_a_norm_than_a_workgroup_adds_up():
    """Above 1024 tiles of 16 x 256: a launch for the norm, beside matrices that need none."""
    x = [matrix((40, 110)), matrix((70, 70000)), matrix((70000, 65)), matrix((300, 300))]
    out = P.ckpt_orthogonalize(x)
    for a, b in zip(out, x):
        assert torch.equal(a, P.ckpt_orthogonalize([b])[0])
        check_orthogonal(a, b, str(tuple(b.shape)))


def test_without_the_native_module(monkeypatch):
    """The binding's own code does what the native one does."""
    from paper_2607_01646_amd import muon
    lists, _ = state([(33, 65), (96, 3, 5), (200, 70)], BF, BF)
    twin = [[t.clone() for t in x] for x in lists]
    x = [matrix((90, 70)), matrix((70, 300))]
    want = P.ckpt_orthogonalize(x)
    P.ckpt_muon(*lists, lr=1e-2, scale=0.7, weight_decay=0.1)
    monkeypatch.setattr(muon, "_native", (None, muon._module()[1]))
    P.ckpt_muon(*twin, lr=1e-2, scale=0.7, weight_decay=0.1)
    assert all(torch.equal(a, b) for c, d in zip(lists, twin) for a, b in zip(c, d))
    assert all(torch.equal(a, b) for a, b in zip(P.ckpt_orthogonalize(x), want))


def test_the_step_follows_differences_of_its_definition():
    """Along a direction: X of U + h D against X of U, which the definition's polynomial gives in 64 bits."""
    u, d = matrix((96, 160)), matrix((96, 160), seed=1)
    more, less = P.ckpt_orthogonalize([u + 0.5 * d, u - 0.5 * d])
    want = orthogonal(u + 0.5 * d) - orthogonal(u - 0.5 * d)
    # each to its own bound, and these are 1e3 times smaller than the difference
    assert float(((more - less).double() - want).norm()) < 1e-4 * float(want.norm())


def test_strided_rows_and_results_in_place():
    wide = matrix((150, 1000))
    parts = [wide[:, :300], wide[:, 301:307], wide[10:20, 400:401], wide[5:6, 500:], wide[::2, 600:700]]
    want = [P.ckpt_orthogonalize([p.contiguous()])[0] for p in parts]
    for a, b in zip(P.ckpt_orthogonalize(parts), want):
        assert torch.equal(a, b)
    old = wide.clone()
    mask = torch.ones_like(wide, dtype=torch.bool)
    got = P.ckpt_orthogonalize(parts, out=parts)
    for a, b, p in zip(got, want, parts):
        assert a is p and torch.equal(a, b)
    for m in (mask[:, :300], mask[:, 301:307], mask[10:20, 400:401], mask[5:6, 500:], mask[::2, 600:700]):
        m.fill_(False)
    assert torch.equal(wide[mask], old[mask])  # what lies between


@pytest.mark.parametrize("steps, coefficients", [(1, (3.4445, -4.7750, 2.0315)), (2, (3.4445, -4.7750, 2.0315)),
                                                 (10, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))])
def test_other_polynomials(steps, coefficients):
    x = matrix((120, 333))
    y, = P.ckpt_orthogonalize([x], steps=steps, coefficients=coefficients)
    check_orthogonal(y, x, steps=steps, coefficients=coefficients)


def state(shapes, param, grad, seed=0, gap=0):
    """Lists of views into flat buffers, `gap` elements apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(math.prod(s) for s in shapes) + gap * (len(shapes) + 1)
    flat = [torch.randn(total, generator=g, device="cuda") * s for s in (0.02, 1e-3, 1e-3)]
    flat = [flat[0].to(param), flat[0], flat[1], flat[2].to(grad)]
    lists, at = [[] for _ in flat], gap
    for s in shapes:
        n = math.prod(s)
        for k, t in enumerate(flat):
            lists[k].append(t[at:at + n].view(s))
        at += n + gap
    return lists, flat


@pytest.mark.parametrize("param, grad, nesterov, gap", [(BF, BF, True, 0), (BF, F32, True, 1), (F32, BF, False, 7),
                                                        (F32, F32, True, 3), (BF, BF, False, 1)])
def test_muon(param, grad, nesterov, gap):
    shapes = [(1, 1), (5, 1), (1, 300), (33, 65), (130, 70), (64, 64), (0, 5), (96, 3, 5), (200, 513), (7, 0)]
    lists, flat = state(shapes, param, grad, gap=gap)
    old = [t.clone() for t in flat]
    before = [[t.clone() for t in x] for x in lists]
    used = torch.zeros(flat[0].numel(), dtype=torch.bool, device="cuda")
    at = gap
    for s in shapes:
        used[at:at + math.prod(s)] = True
        at += math.prod(s) + gap
    c = torch.tensor([0.37], device="cuda")
    P.ckpt_muon(*lists, lr=2e-2, momentum=0.9, nesterov=nesterov, weight_decay=0.1, grad_scale=c)
    for i, s in enumerate(shapes):
        if math.prod(s) == 0:
            continue
        scale = 0.2 * math.sqrt(max(s[0], math.prod(s[1:])))
        want = step(*[x[i] for x in before], 2e-2, 0.9, nesterov, 0.1, scale, float(c))
        for k, name in enumerate(("param", "master", "momentum")):
            value, bound = getattr(want, name)
            within(lists[k][i], value, bound, "%s %s" % (name, s))
        assert torch.equal(lists[0][i], lists[1][i].to(param))  # the parameter is the master copy, rounded
    for k in range(4):
        assert torch.equal(flat[k][~used], old[k][~used])  # what lies between the fragments
    assert torch.equal(flat[3], old[3])


def test_the_update_itself():
    """Without decay and with masters of zero the step is -lr scale X: X to its own bound, not the masters' rounding."""
    for scale, number in (("spectral", math.sqrt(300 / 200)), ("rms", 0.2 * math.sqrt(300)), (0.5, 0.5)):
        lists, _ = state([(300, 200)], F32, F32)
        for t in lists[:3]:
            t[0].zero_()
        P.ckpt_muon(*lists, lr=1.0, momentum=0.0, nesterov=False, scale=scale)
        check_orthogonal(-lists[1][0] / number, lists[3][0], str(scale))
        assert torch.equal(lists[2][0], lists[3][0])


def test_a_parameter_that_is_its_master_copy_and_flat_lists():
    lists, _ = state([(40, 60), (70, 20)], F32, F32)
    twin = [[t.clone() for t in x] for x in lists]
    P.ckpt_muon(*lists, lr=1e-2)
    P.ckpt_muon(twin[1], [t for t in twin[1]], [t.view(-1) for t in twin[2]], [t.view(-1) for t in twin[3]], lr=1e-2)
    for k in (1, 2):
        assert all(torch.equal(a, b) for a, b in zip(lists[k], twin[k]))


@pytest.mark.parametrize("shapes", [[(64, 64), (33, 200), (200, 33), (300, 300)], [(5, 300), (80, 6000), (3000, 16), (4096, 500), (1, 1000)]])
def test_another_stream_and_a_graph(shapes):
    lists, flat = state(shapes, BF, BF, gap=1)
    twin, same = state(shapes, BF, BF, gap=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.ckpt_muon(*lists, lr=1e-2, stream=s)
    s.synchronize()
    x = [t.float() for t in lists[3]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.ckpt_muon(*twin, lr=1e-2)
        y = P.ckpt_orthogonalize(x)
    want = P.ckpt_orthogonalize(x)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        if k:
            P.ckpt_muon(*lists, lr=1e-2)
            torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat, same)), k
        assert all(torch.equal(a, b) for a, b in zip(y, want)), k


def test_rows_of_4_million():
    """The longest rows there may be: sums of 2^22 squares, and more tiles of the first launches than 2^16."""
    x = matrix((66, 1 << 22))
    for t in (x, x.t().contiguous()):
        y, = P.ckpt_orthogonalize([t])
        got = (y if t is x else y.t()).double()
        g = x.double() @ x.double().t()
        # X = F U with F of U's Gram matrix alone: 66 x 66 in 64 bits
        n = float(g.diagonal().sum().sqrt()) + 1e-7
        f, a = torch.eye(66, dtype=torch.float64, device="cuda") / n, g / n ** 2
        for _ in range(5):
            b = 3.4445 * torch.eye(66, dtype=torch.float64, device="cuda") - 4.7750 * a + 2.0315 * a @ a
            f, a = b @ f, b @ a @ b
        want = f @ x.double()
        # 5 steps of 3 roundings of 2^-22 and sums of 2^-23 a square, grown by the steps' factors (at most 3.4 a step, 2 in all here)
        assert float((got - want).norm()) < 2e-5 * float(want.norm())


def test_calls_on_two_streams_at_once():
    shapes = [(300, 500), (64, 64), (1, 900), (129, 130)]
    lists, flat = state(shapes, BF, F32)
    twin, same = state(shapes, BF, F32)
    x = [matrix((600, 700)), matrix((40, 200))]
    want = P.ckpt_orthogonalize(x)
    for _ in range(3):
        P.ckpt_muon(*twin, lr=1e-2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        P.ckpt_muon(*lists, lr=1e-2, stream=streams[0])
        got.append(P.ckpt_orthogonalize(x, stream=streams[1].cuda_stream))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat, same))
    assert all(torch.equal(a, b) for y in got for a, b in zip(y, want))


def test_refusals():
    lists, flat = state([(10, 20), (30, 5)], BF, F32)
    before = [t.clone() for t in flat]
    p, w, m, g = lists

    def refuse(error, *x, **kw):
        with pytest.raises(error):
            P.ckpt_muon(*x, **{**dict(lr=1e-3), **kw})

    refuse(ValueError, p[:1], w, m, g)
    refuse(ValueError, [p[1], p[0]], w, m, g)
    refuse(ValueError, [p[0].view(-1), p[1]], w, m, g)
    refuse(ValueError, p, [w[0].view(20, 10), w[1]], m, g)
    refuse(ValueError, p, [x.double() for x in w], m, g)
    refuse(ValueError, p, w, m, [g[0], g[1].to(BF)])
    refuse(ValueError, [x.cpu() for x in p], w, m, g)
    refuse(ValueError, p, w, m, [g[0], torch.zeros(60, 5, device="cuda")[::2]])
    refuse(ValueError, p, w, m, g, grad_scale=torch.ones(2, device="cuda"))
    refuse(ValueError, p, w, m, g, scale="other")
    refuse(ValueError, p, w, m, g, steps=65)
    for kw in (dict(steps=0), dict(momentum=1.0), dict(momentum=-0.1), dict(eps=0.0), dict(eps=math.nan), dict(lr=math.nan),
               dict(weight_decay=math.inf), dict(scale=math.inf), dict(coefficients=(3.0, 3.0, 3.0)),
               dict(coefficients=(math.nan, 0.0, 0.0))):
        refuse(P.CkptError, p, w, m, g, **kw)
    refuse(P.CkptError, p, w, m, g, lr=1e30, scale=1e30)
    refuse(P.CkptError, [p[0], p[0]], [w[0], w[0]], [m[0], m[0]], [g[0], g[0]])  # one matrix twice
    refuse(P.CkptError, p, w, w, g)
    with pytest.raises(ValueError):
        P.ckpt_orthogonalize([g[0], p[1]])
    with pytest.raises(ValueError):
        P.ckpt_orthogonalize([g[0].t()])
    with pytest.raises(ValueError):
        P.ckpt_orthogonalize(g, out=[g[0]])
    with pytest.raises(P.CkptError):
        P.ckpt_orthogonalize([g[0], g[1]], out=[torch.empty_like(g[0]), g[0].view(-1)[:150].view(30, 5)])  # over the other's input
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat, before))
    P.ckpt_muon([], [], [], [], lr=1e-3)
