"""The vocabulary head's losses and their gradients against the definition in
64 bits (needs an MI355X; through the C ABI)."""
import math

import pytest
import torch

from ops_util import IGNORE, check, definition, inputs

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

BF, F32 = torch.bfloat16, torch.float32
# lengths around every tile's edge, widths that need no copy of the operands (multiples of 64) and that do
SIZES = [(1, 64, 1), (1, 1, 1), (1, 128, 1000), (2, 63, 65), (31, 192, 129), (33, 65, 64), (64, 64, 256), (65, 130, 257),
         (127, 200, 383), (129, 128, 128), (255, 8, 511), (257, 320, 1025), (300, 515, 2049), (700, 64, 300)]


# sizes that take the larger tiles, products cut along the words, and both launches of the gradients
LARGE = [(257, 2048, 8192), (1025, 512, 12001), (513, 1088, 4100), (2100, 640, 3000), (4097, 128, 20000), (700, 4096, 9000)]


def bits(r):
    return [x.view(torch.int16) if x.dtype == BF else x.view(torch.int32) for x in r if x is not None]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, dim, vocab", SIZES)
def test_cross_entropy(tokens, dim, vocab, dtype):
    x = inputs(tokens, dim, vocab, dtype, seed=tokens, masked=0.2)
    ref = definition(x.hidden, x.weight, x.target)
    check(P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True), ref)
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target)
    check(r, ref, grad=False)
    assert r.d_hidden is None and r.d_weight is None


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, dim, vocab", LARGE)
def test_larger_sizes(tokens, dim, vocab, dtype):
    x = inputs(tokens, dim, vocab, dtype, seed=tokens, masked=0.2, topk=5)
    check(P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True), definition(x.hidden, x.weight, x.target))
    ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, temperature=2.0, alpha=0.5)
    check(P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target, temperature=2.0,
                                alpha=0.5, grad=True), ref)


@pytest.mark.parametrize("tokens", [1, 40, 256])
def test_few_tokens_gradients_are_as_exact_as_their_type(tokens):
    """Up to 256 tokens the gradient of the logits keeps 16 bits: what is left is the outputs' own rounding."""
    x = inputs(tokens, 256, 700, BF, seed=3, topk=5)
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target, temperature=2.0,
                              alpha=0.5, grad=True)
    ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, temperature=2.0, alpha=0.5)
    for got, want in ((r.d_hidden, ref.d_hidden), (r.d_weight, ref.d_weight)):
        # half a unit of bf16, and 2^-13 of the tensor's size for two planes of 8 bits and the sums
        assert ((got.double().reshape(want.shape) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -13 * want.abs().max()).all()


def test_a_wide_range_of_logits():
    """Confident rows: logits hundreds apart, so that most probabilities vanish."""
    for dtype in (BF, F32):
        x = inputs(300, 128, 3000, dtype)
        x.hidden *= 40
        ref = definition(x.hidden, x.weight, x.target)
        check(P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True), ref)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("temperature, alpha", [(1.0, 1.0), (2.0, 0.5), (0.5, 0.9), (4.0, 1.0), (3.0, 0.0)])
@pytest.mark.parametrize("tokens, dim, vocab, topk", [(1, 64, 1, 1), (3, 70, 100, 100), (65, 64, 257, 7), (129, 200, 513, 64),
                                                      (200, 128, 2000, 300)])
def test_distillation(tokens, dim, vocab, topk, temperature, alpha, dtype):
    x = inputs(tokens, dim, vocab, dtype, seed=tokens + topk, topk=topk, masked=0.2)
    g = torch.Generator().manual_seed(1)
    absent = (torch.rand(tokens, topk, generator=g) < 0.2) | (torch.rand(tokens, 1, generator=g) < 0.1)
    x.teacher_index[absent.cuda()] = -1
    kw = dict(temperature=temperature, alpha=alpha)
    ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, **kw)
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target, grad=True, **kw)
    check(r, ref)
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target, **kw)
    check(r, ref, grad=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_words_given_twice_and_logits_of_minus_infinity(dtype):
    x = inputs(70, 64, 50, dtype, topk=12)
    x.teacher_index[:, 5] = x.teacher_index[:, 2]
    x.teacher_index[:, 7] = x.teacher_index[:, 2]
    x.teacher_logits[:, 3] = -math.inf
    x.teacher_logits[4] = -math.inf  # nothing left: the row does not count
    x.hidden[4] = math.nan
    ref = definition(x.hidden, x.weight, None, x.teacher_index, x.teacher_logits, temperature=2.0)
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, temperature=2.0, grad=True)
    check(r, ref)
    assert r.token_loss[4] == 0 and r.lse[4] == 0 and not r.d_hidden[4].any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [64, 70])
def test_rows_that_do_not_count_are_not_read(dim, dtype):
    x = inputs(100, dim, 300, dtype, masked=0.4)
    weight = torch.rand(100, device="cuda")
    weight[::7] = 0
    out = (x.target == IGNORE) | (weight == 0)
    x.hidden[out] = math.nan
    x.hidden[out.nonzero()[0]] = math.inf
    ref = definition(x.hidden, x.weight, x.target, token_weight=weight)
    for grad in (True, False):
        r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, token_weight=weight, grad=grad)
        check(r, ref, grad)
        assert not r.token_loss[out].any() and not r.lse[out].any()
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, token_weight=weight, grad=True)
    assert not r.d_hidden[out].any() and torch.isfinite(r.d_weight).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_row_counts(dtype):
    x = inputs(70, 64, 300, dtype)
    x.target[:] = IGNORE
    x.hidden[:] = math.nan
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    assert r.loss == 0 and not any(t.any() for t in r)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_tokens(dtype):
    x = inputs(0, 70, 300, dtype, topk=3)
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    assert r.loss == 0 and r.token_loss.shape == (0,) and r.d_hidden.shape == (0, 70)
    assert r.d_weight.shape == (300, 70) and not r.d_weight.any()
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits)
    assert r.loss == 0 and r.d_weight is None


@pytest.mark.parametrize("bad", [-1, 300, 1 << 40])
def test_a_target_that_is_no_word_shows(bad):
    x = inputs(70, 64, 300, BF)
    x.target[9] = bad
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    assert r.loss.isnan() and r.token_loss.isnan().nonzero().flatten().tolist() == [9]
    assert r.d_hidden[9].isnan().all() and r.d_weight.isnan().any()


def test_a_teacher_word_beyond_the_vocabulary_shows():
    x = inputs(70, 64, 300, BF, topk=4)
    x.teacher_index[9, 2] = 300
    r = P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, grad=True)
    assert r.loss.isnan() and r.token_loss.isnan().nonzero().flatten().tolist() == [9]
    assert r.d_hidden[9].isnan().all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinities_and_nan_in_rows_that_count_stay_in_them(dtype):
    x = inputs(70, 64, 300, dtype)
    x.hidden[3, 5] = math.nan
    x.hidden[66, 0] = math.inf
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target)
    odd = torch.zeros(70, dtype=torch.bool)
    odd[3] = odd[66] = True
    assert torch.equal(~torch.isfinite(r.token_loss.cpu()), odd) and not torch.isfinite(r.loss)
    keep = (~odd).nonzero().flatten().cuda()
    ref = definition(x.hidden[keep], x.weight, x.target[keep])
    got = P.LinearLoss(ref.loss, r.token_loss[keep], r.lse[keep], None, None)
    check(got, ref, grad=False)


def test_the_ignored_target_may_be_a_word():
    x = inputs(90, 64, 40, BF)
    x.target[::9] = 7
    ref = definition(x.hidden, x.weight, x.target, ignore_index=7)
    check(P.ckpt_linear_ce(x.hidden, x.weight, x.target, ignore_index=7, grad=True), ref)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_offsets_and_leading_dimensions(dtype):
    x = inputs(96, 128, 300, dtype, topk=5)
    ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, temperature=2.0, alpha=0.5)
    for off, pad in ((0, 64), (1, 0), (3, 5), (8, 8)):
        def spread(t):
            big = torch.full((t.shape[0] * (t.shape[1] + pad) + off,), 7, dtype=t.dtype, device="cuda")
            v = torch.as_strided(big, t.shape, (t.shape[1] + pad, 1), off)
            v.copy_(t)
            return v
        h, w, i, t = spread(x.hidden), spread(x.weight), spread(x.teacher_index), spread(x.teacher_logits)
        r = P.ckpt_linear_distill(torch.as_strided(h, (4, 24, 128), (24 * h.stride(0), h.stride(0), 1), off), w,
                                  i.unflatten(0, (4, 24)), t.unflatten(0, (4, 24)), target=x.target.view(4, 24),
                                  temperature=2.0, alpha=0.5, grad=True)
        assert r.token_loss.shape == (4, 24) and r.d_hidden.shape == (4, 24, 128)
        check(r, ref)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, dim, vocab", [(40, 256, 8200), (256, 1024, 8209), (2048, 2048, 8224), (2048, 2048, 8193)])
def test_nothing_beyond_the_vocabulary_is_read(tokens, dim, vocab, dtype):
    """A head whose rows are the first of a larger buffer, and whose words leave most of the products' last 64 values
    of k without a row: the rows behind it are NaN, which no zero of d_logits would take out of d_hidden."""
    x = inputs(tokens, dim, vocab, dtype, seed=vocab, masked=0.1)
    big = torch.full((vocab + 64, dim), math.nan, dtype=dtype, device="cuda")
    big[:vocab] = x.weight
    r = P.ckpt_linear_ce(x.hidden, big[:vocab], x.target, grad=True)
    check(r, definition(x.hidden, x.weight, x.target))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sum_scale_and_weights(dtype):
    x = inputs(130, 72, 200, dtype, masked=0.2)
    w = torch.rand(130, device="cuda") * 3
    scale = torch.tensor([128.0], device="cuda")
    for reduction in ("mean", "sum"):
        ref = definition(x.hidden, x.weight, x.target, token_weight=w, reduction=reduction, grad_scale=128.0)
        r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, token_weight=w, reduction=reduction, grad=True,
                             grad_scale=scale)
        check(r, ref)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("topk", [0, 6])
def test_pieces(dtype, topk):
    """Many pieces of 256 tokens, the last one ragged, against one."""
    x = inputs(256 * 3 + 41, 128, 500, dtype, topk=topk, masked=0.1)
    if topk:
        call = lambda **kw: P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits,  # noqa: E731
                                                  target=x.target, temperature=2.0, alpha=0.5, grad=True, **kw)
        ref = definition(x.hidden, x.weight, x.target, x.teacher_index, x.teacher_logits, temperature=2.0, alpha=0.5)
    else:
        call = lambda **kw: P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True, **kw)  # noqa: E731
        ref = definition(x.hidden, x.weight, x.target)
    whole, cut = call(), call(piece_bytes=1)
    check(whole, ref)
    check(cut, ref)
    assert torch.equal(whole.token_loss, cut.token_loss) and torch.equal(whole.loss, cut.loss)


def test_the_workspace_does_not_grow_with_the_tokens():
    x = inputs(20000, 64, 8192, BF)
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True, piece_bytes=64 << 20)
    peak = torch.cuda.max_memory_allocated() - before
    logits = 20000 * 8192 * 4
    assert peak < logits // 4, (peak, logits)
    one = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    assert torch.equal(r.token_loss, one.token_loss)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_same_inputs_give_the_same_bits(dtype):
    x = inputs(333, 192, 1111, dtype, topk=8, masked=0.1)
    call = lambda: P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target,  # noqa: E731
                                         temperature=2.0, alpha=0.5, grad=True)
    a = call()
    torch.empty(1 << 26, dtype=torch.uint8, device="cuda").fill_(0xFF)  # what the allocator hands out next holds something else
    for _ in range(3):
        b = call()
        assert all(torch.equal(p, q) for p, q in zip(bits(a), bits(b)))


@pytest.mark.parametrize("kind", ["ce", "distill"])
def test_gradient_against_differences(kind):
    """d(loss) along random directions, the loss in 64 bits at both ends."""
    x = inputs(40, 64, 120, F32, topk=6, masked=0.1)
    kw = dict(temperature=2.0, alpha=0.6) if kind == "distill" else {}
    teacher = (x.teacher_index, x.teacher_logits) if kind == "distill" else (None, None)
    if kind == "distill":
        r = P.ckpt_linear_distill(x.hidden, x.weight, *teacher, target=x.target, grad=True, **kw)
    else:
        r = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    for name in ("hidden", "weight"):
        at = getattr(x, name).double()
        way = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
        step = 1e-5
        ends = []
        for s in (step, -step):
            y = dict(hidden=x.hidden.double(), weight=x.weight.double())
            y[name] = at + s * way
            ends.append(float(definition(y["hidden"], y["weight"], x.target, *teacher, **kw).loss))
        slope = (ends[0] - ends[1]) / (2 * step)
        got = float((getattr(r, "d_" + name).double() * way).sum())
        # a third derivative of order 10 |way|^3 at most, and the gradient's own 32-bit error
        scale = float((getattr(r, "d_" + name).double().abs() * way.abs()).sum())
        assert abs(got - slope) <= 1e-5 * scale + 1e-6, (name, got, slope)


@pytest.mark.parametrize("grad", [True, False])
def test_another_stream(grad):
    x = inputs(300, 128, 2000, BF)
    want = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=grad)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=grad)
    other = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=grad, stream=s)
    handle = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=grad, stream=s.cuda_stream)
    s.synchronize()
    for r in (got, other, handle):
        assert all(torch.equal(a, b) for a, b in zip(bits(want), bits(r)))


def test_captured_into_a_graph():
    x = inputs(300, 128, 2000, BF, topk=4)
    call = lambda: P.ckpt_linear_distill(x.hidden, x.weight, x.teacher_index, x.teacher_logits, target=x.target,  # noqa: E731
                                         temperature=2.0, alpha=0.5, grad=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = call()
    for k in range(3):
        x.hidden.add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bits(r), bits(want))), k


def test_offsets_beyond_32_bits():
    """Rows 2^29 elements apart: byte offsets of 1 GiB a row, past 2^32 from the fifth on."""
    big = torch.zeros((8 << 29) + 64, dtype=BF, device="cuda")
    x = inputs(8, 64, 300, BF)
    far = torch.as_strided(big, (8, 64), (1 << 29, 1), 0)
    far.copy_(x.hidden)
    a = P.ckpt_linear_ce(x.hidden, x.weight, x.target, grad=True)
    b = P.ckpt_linear_ce(far, x.weight, x.target, grad=True)
    assert all(torch.equal(p, q) for p, q in zip(bits(a), bits(b)))
    c = P.ckpt_linear_ce(far, x.weight, x.target)
    assert torch.equal(c.token_loss, a.token_loss)
    far.copy_(x.weight[:8])
    a = P.ckpt_linear_ce(x.hidden, x.weight[:8], x.target % 8, grad=True)
    b = P.ckpt_linear_ce(x.hidden, far, x.target % 8, grad=True)
    assert all(torch.equal(p, q) for p, q in zip(bits(a), bits(b)))


def test_a_piece_of_logits_beyond_32_bits():
    """270000 tokens of 8192 words in one piece: logits and their gradients past 2^31 elements and 2^32 bytes."""
    n, d, v = 270_000, 64, 8192
    g = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn(n, d, generator=g, device="cuda").to(BF)
    w = (torch.randn(v, d, generator=g, device="cuda") / 8).to(BF)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    a = P.ckpt_linear_ce(h, w, t, grad=True, piece_bytes=16 << 30)
    last = slice(n - 100, n)
    ref = definition(h[last], w, t[last])
    b = P.ckpt_linear_ce(h[last], w, t[last], grad=True, grad_scale=torch.tensor([100 / n], device="cuda"))
    assert torch.equal(a.token_loss[last], b.token_loss)
    assert (a.d_hidden[last].double() - b.d_hidden.double()).abs().max() <= 2 ** -7 * b.d_hidden.double().abs().max()
    assert (b.token_loss.double() - ref.token_loss).abs().max() < 1e-3
    cut = P.ckpt_linear_ce(h, w, t, grad=True)
    assert torch.equal(cut.token_loss, a.token_loss)
    diff = (cut.d_weight.double() - a.d_weight.double()).norm() / a.d_weight.double().norm()
    assert diff < 2 * 2 ** -8


def test_refusals():
    x = inputs(8, 64, 100, BF, topk=3)
    ce = lambda **kw: P.ckpt_linear_ce(**{**dict(hidden=x.hidden, weight=x.weight, target=x.target), **kw})  # noqa: E731
    for kw in (dict(hidden=x.hidden.half()), dict(hidden=x.hidden.cpu()), dict(hidden=x.hidden.float()),
               dict(weight=x.weight[:, :32]), dict(weight=x.weight.t()), dict(hidden=x.hidden.t().contiguous().t()),
               dict(target=x.target[:7]), dict(target=x.target.int()), dict(target=x.target.cpu()),
               dict(token_weight=torch.ones(8, dtype=BF, device="cuda")), dict(reduction="none"),
               dict(grad_scale=torch.ones(2, device="cuda")), dict(hidden=x.hidden[0:0].new_empty(8, 0))):
        with pytest.raises(ValueError):
            ce(**kw)
    with pytest.raises(P.CkptError) as e:
        ce(target=None)
    assert e.value.code == P.CKPT_EINVAL and "target" in str(e.value)
    kd = lambda **kw: P.ckpt_linear_distill(**{**dict(hidden=x.hidden, weight=x.weight, teacher_index=x.teacher_index,  # noqa: E731
                                                      teacher_logits=x.teacher_logits, target=x.target), **kw})
    for kw in (dict(teacher_index=x.teacher_index.int()), dict(teacher_logits=x.teacher_logits[:, :2]),
               dict(teacher_logits=x.teacher_logits.half()), dict(teacher_index=x.teacher_index[:, :0],
                                                                  teacher_logits=x.teacher_logits[:, :0])):
        with pytest.raises(ValueError):
            kd(**kw)
    for kw in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan),
               dict(alpha=1.5), dict(alpha=-0.1), dict(alpha=math.nan), dict(target=None, alpha=0.5)):
        with pytest.raises(P.CkptError) as e:
            kd(**kw)
        assert e.value.code == P.CKPT_EINVAL
    check(kd(), definition(x.hidden, x.weight, None, x.teacher_index, x.teacher_logits), grad=False)  # none of it stuck


def test_refusals_of_the_c_entry():
    """Sizes, strides, alignment and memory, with plain pointers; nothing is enqueued."""
    import ctypes as C
    from paper_2607_01646_amd import ops

    x = inputs(8, 64, 100, BF)
    out = torch.zeros(64, device="cuda")
    work = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def args(**kw):
        a = ops.ckpt_linear_loss_args(dtype=P.CKPT_TYPE_BF16, tokens=8, dim=64, vocab=100, hidden=x.hidden.data_ptr(),
                                      hidden_stride=64, weight=x.weight.data_ptr(), weight_stride=64,
                                      target=x.target.data_ptr(), ignore_index=IGNORE, temperature=1, alpha=1,
                                      loss=out.data_ptr(), token_loss=out.data_ptr() + 4, lse=out.data_ptr() + 64)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    L = ops._ops()

    def call(a, ws=work.data_ptr(), size=work.numel(), device=0):
        return L.ckpt_linear_loss(C.byref(a), device, ws, size, None)

    assert call(args()) == P.CKPT_OK
    torch.cuda.synchronize()
    before = out.clone()
    host = torch.zeros(1 << 12)
    for kw in (dict(dtype=0), dict(dtype=3), dict(reduction=2), dict(tokens=1 << 31), dict(dim=0), dict(vocab=0),
               dict(vocab=1 << 31), dict(topk=1025), dict(hidden_stride=63), dict(weight_stride=1), dict(weight_stride=1 << 50),
               dict(hidden=0), dict(weight=0), dict(hidden=x.hidden.data_ptr() + 1), dict(loss=0), dict(lse=0),
               dict(token_loss=host.data_ptr()), dict(weight=host.data_ptr()), dict(tokens=1 << 30), dict(vocab=1 << 30),
               dict(d_hidden=x.hidden.data_ptr(), d_hidden_stride=64), dict(d_weight=x.weight.data_ptr(), d_weight_stride=64),
               dict(target=0), dict(grad_scale=host.data_ptr())):
        assert call(args(**kw)) == P.CKPT_EINVAL, kw
        assert P.ckpt_last_error(None)
    assert call(args(), ws=None) == P.CKPT_EINVAL
    assert call(args(), ws=work.data_ptr() + 16) == P.CKPT_EINVAL
    assert call(args(), size=100) == P.CKPT_EINVAL
    assert call(args(), device=99) == P.CKPT_EINVAL
    assert L.ckpt_linear_loss(None, 0, work.data_ptr(), work.numel(), None) == P.CKPT_EINVAL
    torch.cuda.synchronize()
    assert torch.equal(out, before)
