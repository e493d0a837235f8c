"""How exact the orthogonalised step is: one arithmetic for every type and both
entry points, as near to 64 bits as products in fp32, and the step's own
outputs on all sizes of tiles (needs an MI355X; through the C ABI)."""
import pytest
import torch

from muon_util import A, B, C, EPS, check_orthogonal, orthogonal, step
from ops_util import within
from test_gpu_muon import BF, F32, matrix, state

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

# On both sides of every way that a matrix's own sides choose (16, 64 x 256, 448) and of the lengths of its sums in parts
# (384, 640, 1024).
SHAPES = [(9, 300), (33, 33), (64, 256), (21, 153), (40, 300), (300, 70), (96, 5000), (384, 390), (300, 700), (448, 448),
          (450, 449), (512, 700), (640, 700), (700, 641), (777, 1003), (1003, 900), (1100, 1024), (1025, 1030)]


@pytest.mark.parametrize("shape", SHAPES)
def test_the_step_takes_the_orthogonalisation_s_own_bits(shape):
    """From masters and momentum of zero, without decay and with lr scale 1, the master copy is -X and nothing is rounded: X
    is that of ckpt_orthogonalize in fp32, whatever the types of gradient and parameter."""
    for grad_type in (F32, BF):
        grad = matrix(shape, grad_type)
        x, = P.ckpt_orthogonalize([grad.float()])
        for param_type in (F32, BF):
            master, momentum = torch.zeros_like(x), torch.zeros_like(x)
            param = torch.ones_like(x).to(param_type)
            P.ckpt_muon([param], [master], [momentum], [grad], lr=1.0, momentum=0.0, nesterov=False, scale=1.0)
            assert torch.equal(master, -x), (grad_type, param_type)
            assert torch.equal(param, (-x).to(param_type)) and torch.equal(momentum, grad.float())


@pytest.mark.parametrize("shape", SHAPES)
def test_a_bf16_result_is_the_fp32_one_rounded(shape):
    x = matrix(shape, BF)
    assert torch.equal(P.ckpt_orthogonalize([x])[0], P.ckpt_orthogonalize([x.float()])[0].to(BF))


def in_fp32(u):
    """The definition with torch's products in fp32."""
    x = u / (u.square().sum(dtype=torch.float64).sqrt() + EPS).float()
    x = x if x.shape[0] <= x.shape[1] else x.t().contiguous()
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x if u.shape[0] <= u.shape[1] else x.t()


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("shape", [(17, 40), (21, 153), (33, 33), (40, 300), (64, 256), (65, 300), (96, 160), (300, 130),
                                   (257, 2049), (384, 400), (448, 448), (449, 600), (520, 1100), (777, 1003), (1100, 1024)])
def test_as_exact_as_products_in_fp32(shape, few):
    """Both against 64 bits, over eight matrices.  Each rounds its operands once: a value in fp32 by 0.29 steps of 2^-23 in the
    mean square, one in two planes of fp16 by that and 0.24 of 2^-22 more (the first leaves half a step of 2^-10 at most,
    evenly, of which the second's half step is 2^-22 in half of the cases, 2^-23 in a quarter, ..): 1.9 times as much
    together.  The sums are rounded by no more than in fp32: once for 16 values of k and product of planes, 3 or 4 of those,
    where fp32 products round at least once for 4 values, and in parts of 128 besides."""
    off = [0.0, 0.0]
    for seed in range(8):
        u = matrix(shape, few=few, seed=seed)
        want = orthogonal(u)
        for k, x in enumerate((P.ckpt_orthogonalize([u])[0], in_fp32(u))):
            off[k] += float((x.double() - want).square().sum())
    assert off[0] ** 0.5 <= 2 * off[1] ** 0.5, "%.3g, in fp32 %.3g" % (off[0] ** 0.5, off[1] ** 0.5)


def test_short_sides_beside_the_ways_limits_in_one_call():
    """A launch's matrices go one way: those on either side of a limit keep the bits of their own calls, in any order."""
    shapes = [(449, 600), (447, 600), (600, 448), (385, 500), (450, 449), (383, 500), (500, 384), (640, 641), (17, 600),
              (1025, 1026), (65, 449), (448, 449), (1024, 1023)]
    x = [matrix(s, BF if k % 3 == 0 else F32) for k, s in enumerate(shapes)]
    for kind in (BF, F32):
        mine = [t for t in x if t.dtype == kind]
        alone = [P.ckpt_orthogonalize([t])[0] for t in mine]
        for order in (1, -1):
            for piece in (0, 8 << 20):
                out = P.ckpt_orthogonalize(mine[::order], piece_bytes=piece)
                assert all(torch.equal(a, b) for a, b in zip(out[::order], alone))


def test_matrices_that_overlap_row_by_row_are_refused():
    wide = matrix((150, 1000))
    old = wide.clone()
    a, b = wide[:, :300], wide[:, 299:500]
    new = [torch.empty_like(t) for t in (a, b)]
    for x, out in (([a, b], [a, b]),  # a column of both is written
                   ([a, a], [a, a]),  # one matrix twice
                   ([a, b], [new[0], a[:, :201]]),  # over the other's input
                   ([a], [wide.view(-1)[:75000].view(150, 500)[:, :300]]),  # in place, but with other rows
                   ([a], [wide.view(-1)[100:45100].view(150, 300)]),  # contiguous, over the strided ones
                   ([a, new[0]], [wide[:, 500:800], wide[:, 700:]])):
        with pytest.raises(P.CkptError, match="overlap"):
            P.ckpt_orthogonalize(x, out=out)
    torch.cuda.synchronize()
    assert torch.equal(wide, old)
    # what reads the same, and what lies between the rows of others, does not
    want = P.ckpt_orthogonalize([a.contiguous(), wide[:, 300:600].contiguous(), wide[1::2, 600:].contiguous()])
    twice = P.ckpt_orthogonalize([a, a, b])
    assert torch.equal(twice[0], want[0]) and torch.equal(twice[1], want[0])
    parts = [a, wide[:, 300:600], wide[1::2, 600:]]
    for x, y in zip(P.ckpt_orthogonalize(parts, out=parts), want):
        assert torch.equal(x, y)
    assert torch.equal(wide[::2, 600:], old[::2, 600:])


def test_a_scale_that_lies_in_what_is_written_is_refused():
    p, w, m, g = (torch.ones(40, 300, device="cuda") for _ in range(4))
    for t in (p, w, m):
        with pytest.raises(P.CkptError, match="overlap"):
            P.ckpt_muon([p], [w], [m], [g], lr=1e-2, grad_scale=t.view(-1)[-1:])
    torch.cuda.synchronize()
    assert all(bool((t == 1).all()) for t in (p, w, m))
    P.ckpt_muon([p], [w], [m], [g], lr=1e-2, grad_scale=g.view(-1)[:1])  # beside what is only read


def check_step(lists, before, i, lr, wd, scale, what):
    want = step(*[x[i] for x in before], lr, 0.9, True, wd, scale)
    for k, name in enumerate(("param", "master", "momentum")):
        value, bound = getattr(want, name)
        within(lists[k][i], value, bound, "%s of %s" % (name, what))


@pytest.mark.parametrize("param, grad", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("shape", [(390, 500), (448, 900), (900, 448), (520, 1100), (1100, 520), (777, 1003), (1003, 777),
                                   (1100, 1200)])
def test_the_step_of_larger_matrices_against_64_bits(shape, param, grad):
    """With decay, and from masters of zero with a large lr, where X is all that there is."""
    for lr, wd, scale, zero in ((2e-2, 0.1, 0.2 * max(shape) ** 0.5, False), (1.0, 0.0, 0.7, True)):
        lists, _ = state([shape], param, grad, gap=1)
        if zero:
            lists[0][0].zero_()
            lists[1][0].zero_()
        before = [[t.clone() for t in x] for x in lists]
        P.ckpt_muon(*lists, lr=lr, momentum=0.9, weight_decay=wd, scale=scale)
        check_step(lists, before, 0, lr, wd, scale, shape)
        assert torch.equal(lists[0][0], lists[1][0].to(param))


@pytest.mark.parametrize("shape, count", [((1000, 1100), 4), ((1000, 1100), 24), ((1088, 1152), 8), ((2176, 2200), 2)])
def test_the_step_on_larger_tiles_against_64_bits(shape, count):
    """So many matrices, every other one tall, that tiles of 128 x 256 and 256 x 256 are the quickest for their products."""
    shapes = [shape if k % 2 else shape[::-1] for k in range(count)]
    lists, _ = state(shapes, BF, BF)
    before = [[t.clone() for t in x] for x in lists]
    P.ckpt_muon(*lists, lr=2e-2, momentum=0.9, weight_decay=0.1, scale=5.0)
    for i in (0, count - 1):
        check_step(lists, before, i, 2e-2, 0.1, 5.0, shapes[i])
    for i in range(count):
        one = [[x[i]] for x in before]
        P.ckpt_muon(*one, lr=2e-2, momentum=0.9, weight_decay=0.1, scale=5.0)
        assert all(torch.equal(a[0], b[i]) for a, b in zip(one, lists)), i


@pytest.mark.parametrize("count", [1, 2, 3, 5, 6, 7, 8])
@pytest.mark.parametrize("side", [1025, 1088, 1152, 1153])
def test_tiles_past_the_last_row_of_a_symmetric_product(side, count):
    """Short sides of up to half a tile of 256 more than whole ones: of the last row's two tiles of 128 x 256 one begins past
    the matrix.  With 5 to 8 matrices those tiles are the quickest for X X^T and its polynomials."""
    x = [matrix((side, side + 64) if k % 2 else (side + 64, side), seed=k) for k in range(count)]
    out = P.ckpt_orthogonalize(x)
    check_orthogonal(out[-1], x[-1])
    for a, b in zip(out, x):
        assert torch.equal(a, P.ckpt_orthogonalize([b])[0])


@pytest.mark.parametrize("share", [1e-2, 1e-4, 1e-7, 1e-12])
@pytest.mark.parametrize("shape", [(9, 300), (64, 256), (70, 130), (777, 1003), (2100, 1300)])
def test_norms_far_below_eps(shape, share):
    """X is small then.  A value of X in planes is off by 2^-37 at most where they hold no 22 bits of it (half of fp16's
    smallest step, of 2^12 times the value), and what was rounded grows by 3.4445 a step: 2^-37 (3.4445 + .. + 3.4445^5) for
    each value, beside the roundings that any X has.  Short sides up to 16 have none of that."""
    u = matrix(shape, scale=1.0)
    u = u / u.norm() * (EPS * share)
    x, = P.ckpt_orthogonalize([u])
    want = orthogonal(u)
    grown = 0.0 if min(shape) <= 16 else 2.0 ** -37 * sum(A ** k for k in range(1, 6)) * (shape[0] * shape[1]) ** 0.5
    assert float((x.double() - want).norm()) <= grown + 5e-6 * float(want.norm())
