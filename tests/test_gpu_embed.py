"""The vocabulary table's lookup and its gradient against their definitions in
64 bits (needs an MI355X; through the C ABI)."""
import math

import pytest
import torch

from ops_util import U32, UBF, within

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P

BF, F32 = torch.bfloat16, torch.float32
IGNORE = -100


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def words(n, vocab, kind, seed=0):
    """ids: spread evenly, as in text (few words have most tokens), or one word."""
    g = gen(seed)
    if kind == "one":
        ids = torch.full((n,), vocab // 3, device="cuda")
    elif kind == "even":
        ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    else:
        ids = ((vocab + 1.0) ** torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).long().sub_(1).clamp_(0, vocab - 1)
        ids = torch.randperm(vocab, generator=g, device="cuda")[ids]
    return ids


def masked(ids, share=0.2, seed=1):
    ids[torch.rand(ids.shape, generator=gen(seed), device="cuda") < share] = IGNORE
    return ids


def unit(dtype):
    return UBF if dtype == BF else U32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n, dim, vocab", [(0, 64, 10), (1, 1, 1), (10, 2, 5), (10, 3, 5), (1, 4096, 300), (3, 7, 5), (64, 64, 256), (65, 513, 100),
                                           (300, 1000, 77), (5, 8191, 9), (9000, 320, 500), (2000, 2049, 1000)])
def test_lookup(n, dim, vocab, dtype):
    table = torch.randn(vocab, dim, generator=gen(n), device="cuda").to(dtype)
    ids = masked(words(n, vocab, "even"))
    if n > 2:
        ids[0], ids[1], ids[n - 1] = vocab - 1, 0, vocab - 1
    got = P.ckpt_embedding(table, ids, scale=0.3)
    there = ids != IGNORE
    want = torch.where(there[:, None], table.double()[ids.clamp(min=0)] * 0.3, 0.0)
    assert got.shape == (n, dim) and got.dtype == dtype
    within(got, want, (unit(dtype) + 2 * U32) * want.abs(), "rows")
    same = P.ckpt_embedding(table, ids)
    assert torch.equal(same[there], table[ids[there]])


def test_lookup_of_ids_that_are_no_words():
    table = torch.randn(50, 33, device="cuda")
    ids = torch.tensor([[0, 49, 50, -1], [IGNORE, 7, 1 << 40, -(1 << 62)]], device="cuda")
    got = P.ckpt_embedding(table, ids)
    assert got.shape == (2, 4, 33)
    assert torch.equal(got[0, :2], table[[0, 49]]) and torch.equal(got[1, 1], table[7]) and not got[1, 0].any()
    for k in ((0, 2), (0, 3), (1, 2), (1, 3)):
        assert got[k].isnan().all()
    got = P.ckpt_embedding(table, ids, ignore_index=7)  # a word of the table, too
    assert not got[1, 1].any() and got[1, 0].isnan().all() and torch.equal(got[0, 1], table[49])


def test_strides_and_values_that_are_no_numbers():
    wide = torch.randn(40, 1000, device="cuda").to(BF)
    wide[3, 20], wide[4, 21], wide[5, 22] = math.inf, -math.inf, math.nan
    for a, b in ((0, 1000), (1, 500), (3, 4), (17, 600)):
        table = wide[::2, a:b]
        ids = torch.arange(20, device="cuda").flip(0)
        assert torch.equal(P.ckpt_embedding(table, ids).view(torch.int16), table.flip(0).contiguous().view(torch.int16))
    wide = torch.randn(3, 5, 700, device="cuda")
    d = wide[..., 5:606]
    ids = torch.arange(15, device="cuda").view(3, 5) % 4
    want = torch.zeros(6, 601, dtype=torch.float64, device="cuda").index_add_(0, ids.view(-1), d.reshape(15, 601).double())
    within(P.ckpt_embedding_grad(d, ids, 6), want, 8 * U32 * want.abs().clamp(min=4), "table")


def reference(d, ids, vocab, scale, old=None):
    """Sums in 64 bits, and bounds: a word's sum of k rows in fp32, k + 4 roundings of partial sums."""
    d, ids = d.cpu(), ids.cpu()  # (adding to one row on the GPU takes seconds)
    there = (ids >= 0) & (ids < vocab) & (ids != IGNORE)
    want = torch.zeros(vocab, d.shape[1], dtype=torch.float64)
    size = want.clone()
    rows = d[there].double()
    want.index_add_(0, ids[there], rows)
    size.index_add_(0, ids[there], rows.abs())
    count = torch.bincount(ids[there], minlength=vocab).double().cuda()
    want, size = want.cuda(), size.cuda()
    want, bound = scale * want, abs(scale) * (count + 4)[:, None] * U32 * size
    if old is not None:
        want = want + old.double()
        bound = bound + U32 * want.abs()
    return want, bound, count


@pytest.mark.parametrize("rows, table", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)])
@pytest.mark.parametrize("kind", ["even", "text", "one"])
@pytest.mark.parametrize("n, dim, vocab", [(1, 1, 1), (10, 2, 5), (200, 3, 5), (1, 4096, 300), (3, 7, 5), (63, 64, 33), (64, 64, 256), (65, 513, 100),
                                           (128, 1030, 40), (129, 5000, 7), (1000, 1000, 77), (3000, 65, 1001),
                                           (5000, 320, 40000), (20000, 9, 3), (70000, 130, 2500)])
def test_gradient(n, dim, vocab, kind, rows, table):
    d = torch.randn(n, dim, generator=gen(n), device="cuda").to(rows)
    ids = masked(words(n, vocab, kind))
    d[ids == IGNORE] = math.nan  # not read
    want, bound, count = reference(d, ids, vocab, 0.7)
    got = P.ckpt_embedding_grad(d, ids, vocab, scale=0.7, dtype=table)
    assert got.shape == (vocab, dim) and got.dtype == table
    within(got, want, bound + unit(table) * want.abs(), "table")
    assert not got[count == 0].any()
    assert torch.equal(got, P.ckpt_embedding_grad(d, ids, vocab, scale=0.7, dtype=table))  # no order of its own

    old = torch.randn(vocab, dim, generator=gen(n + 1), device="cuda").to(table)
    want, bound, count = reference(d, ids, vocab, 0.7, old)
    got = old.clone()
    assert P.ckpt_embedding_grad(d, ids, vocab, scale=0.7, add_to=got) is got
    within(got, want, bound + unit(table) * want.abs(), "added to")
    assert torch.equal(got[count == 0], old[count == 0])


@pytest.mark.parametrize("n", [100, 1024, 66000])
def test_sums_in_fp32_and_in_order(n):
    """A word's tokens far apart and in several runs: whole numbers, whose sum is exact in fp32 in any order, and 1 + tiny."""
    ids = torch.arange(n, device="cuda") % 3
    d = (torch.arange(n, device="cuda") % 101).float()[:, None].repeat(1, 70)
    got = P.ckpt_embedding_grad(d.to(BF), ids, 4, dtype=F32)
    want = torch.zeros(4, 70, device="cuda").index_add_(0, ids, d)
    assert torch.equal(got, want)


@pytest.mark.parametrize("vocab", [255, 256, 257, 8192, 32000, 128256, 300000, 1 << 22])
def test_vocabularies(vocab):
    """Every sorting workgroup's first and last word."""
    n = 4096
    ids = words(n, vocab, "even", seed=vocab)
    ids[:4] = torch.tensor([0, vocab - 1, vocab // 2, 0], device="cuda")
    each = min(max(-(-vocab // 256), 32), 1000)
    edges = torch.arange(0, vocab, each, device="cuda")[:1000]
    ids[4:4 + edges.numel()] = edges
    ids[1500:1500 + edges.numel()] = (edges - 1).clamp(min=0)
    d = torch.randint(-8, 9, (n, 24), generator=gen(0), device="cuda").float()
    want = torch.zeros(vocab, 24, device="cuda").index_add_(0, ids, d)
    assert torch.equal(P.ckpt_embedding_grad(d, ids, vocab), want)


def test_nothing_to_sum():
    d = torch.full((30, 50), math.nan, device="cuda")
    ids = torch.full((30,), IGNORE, device="cuda")
    ids[::2] = 99
    ids[1] = -1
    old = torch.randn(12, 50, device="cuda")
    got = old.clone()
    assert not P.ckpt_embedding_grad(d, ids, 12).any()
    P.ckpt_embedding_grad(d, ids, 12, add_to=got)
    assert torch.equal(got, old)
    empty = torch.zeros(0, 50, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    assert not P.ckpt_embedding_grad(*empty, 12).any()
    P.ckpt_embedding_grad(*empty, 12, add_to=got)
    assert torch.equal(got, old)
    assert P.ckpt_embedding(old, empty[1]).shape == (0, 50)


def test_infinities_reach_their_words_alone():
    d = torch.ones(8, 20, device="cuda")
    ids = torch.tensor([1, 2, 1, 3, 3, 1, 0, 2], device="cuda")
    d[2], d[3], d[4] = math.inf, math.inf, -math.inf
    got = P.ckpt_embedding_grad(d, ids, 5)
    assert (got[1] == math.inf).all() and got[3].isnan().all()
    assert (got[0] == 1).all() and (got[2] == 2).all() and not got[4].any()


def test_strided_results():
    wide = torch.randn(60, 500, device="cuda").to(BF)
    old = wide.clone()
    ids = masked(words(333, 30, "text"))
    d = torch.randn(333, 101, device="cuda").to(BF)
    table = wide[::2, 7:108]
    want = table.clone()
    P.ckpt_embedding_grad(d, ids, 30, add_to=want)
    P.ckpt_embedding_grad(d, ids, 30, add_to=table)
    assert torch.equal(table, want)
    mask = torch.ones_like(wide, dtype=torch.bool)
    mask[::2, 7:108] = False
    assert torch.equal(wide[mask], old[mask])


def test_many_elements():
    """Rows beyond 2^31 elements and 2^32 bytes."""
    vocab, dim = 70000, 32768
    table = torch.zeros(vocab, dim, dtype=BF, device="cuda")
    table[vocab - 1], table[65537] = 3.0, 2.0
    ids = torch.full((66000,), vocab - 1, device="cuda")
    ids[0], ids[-1] = 65537, 65537
    rows = P.ckpt_embedding(table, ids)
    assert (rows[0] == 2).all() and (rows[-1] == 2).all() and (rows[1:-1] == 3).all()
    got = P.ckpt_embedding_grad(rows, ids, vocab, dtype=F32)
    assert (got[65537] == 4).all() and (got[vocab - 1] == 3 * 65998).all()
    assert float(got.sum(dtype=torch.float64)) == dim * (4 + 3 * 65998)


def test_many_tokens():
    """More than a launch of the lookup takes, of few words."""
    n = (1 << 26) + 77
    ids = torch.arange(n, device="cuda") % 5
    table = torch.tensor([[1.0, -2.0], [2.0, 3.0], [4.0, 0.5], [8.0, 0.0], [16.0, 1.0]], device="cuda").to(BF)
    rows = P.ckpt_embedding(table, ids)
    for at in (0, 1, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, n - 1):
        assert torch.equal(rows[at], table[at % 5])
    assert float(rows[:, 0].sum(dtype=torch.float64)) == float(table.double()[:, 0][ids[:5]].sum()) * (n // 5) + float(
        table.double()[:n % 5, 0].sum())
    got = P.ckpt_embedding_grad(rows, ids, 5, scale=2.0 ** -20, dtype=F32)
    count = torch.bincount(ids, minlength=5).double()
    want = table.double() * count[:, None] * 2.0 ** -20
    within(got, want, 1024 * U32 * want.abs(), "table")  # whole numbers up to 2^24 a chunk, and at most 1024 of those


def test_another_stream_and_a_graph():
    ids = masked(words(777, 200, "text"))
    table = torch.randn(200, 130, device="cuda").to(BF)
    want = P.ckpt_embedding(table, ids, scale=2.0)
    grad = P.ckpt_embedding_grad(want, ids, 200)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = P.ckpt_embedding(table, ids, scale=2.0, stream=s)
    b = P.ckpt_embedding_grad(want, ids, 200, stream=s)
    s.synchronize()
    assert torch.equal(a, want) and torch.equal(b, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = P.ckpt_embedding(table, ids, scale=2.0)
        b = P.ckpt_embedding_grad(a, ids, 200)
    for k in range(3):
        ids.copy_(masked(words(777, 200, "text", seed=k), seed=k + 5))
        graph.replay()
        torch.cuda.synchronize()
        want = P.ckpt_embedding(table, ids, scale=2.0)
        assert torch.equal(a, want) and torch.equal(b, P.ckpt_embedding_grad(want, ids, 200)), k


def test_the_gradient_is_the_lookups():
    """Differences of a weighted sum of the rows, in fp32 with steps that are exact in it."""
    g = gen(3)
    table = torch.randint(-8, 9, (20, 12), generator=g, device="cuda").float()
    ids = masked(words(50, 20, "text"))
    d = torch.randint(-8, 9, (50, 12), generator=g, device="cuda").float()
    grad = P.ckpt_embedding_grad(d, ids, 20, scale=2.0)
    value = lambda t: float((P.ckpt_embedding(t, ids, scale=2.0).double() * d.double()).sum())
    for v in range(20):
        for c in (0, 5, 11):
            more, less = table.clone(), table.clone()
            more[v, c] += 1
            less[v, c] -= 1
            assert (value(more) - value(less)) / 2 == float(grad[v, c])


def test_without_the_native_module(monkeypatch):
    """The binding's own code does what the native one does."""
    from paper_2607_01646_amd import embed
    ids = masked(words(500, 90, "text")).view(5, 100)
    table = torch.randn(90, 70, device="cuda").to(BF)
    rows = P.ckpt_embedding(table, ids, scale=3.0)
    grad = P.ckpt_embedding_grad(rows, ids, 90, scale=3.0)
    more = P.ckpt_embedding_grad(rows, ids, 90, add_to=grad.clone())
    monkeypatch.setattr(embed, "_native", (None, embed._module()[1]))
    assert torch.equal(P.ckpt_embedding(table, ids, scale=3.0), rows)
    assert torch.equal(P.ckpt_embedding_grad(rows, ids, 90, scale=3.0), grad)
    assert torch.equal(P.ckpt_embedding_grad(rows, ids, 90, add_to=grad.clone()), more)


def test_no_more_workspace_than_said_and_none_for_few():
    """The rows behind the last token, and what lies around the workspace, stay as they are."""
    import ctypes as C
    from paper_2607_01646_amd import embed
    for n in (100, 5000):
        d = torch.randn(n + 10, 200, device="cuda")
        ids = words(n, 300, "text")
        a = embed.ckpt_embed_args(dtype=P.CKPT_TYPE_F32, table_dtype=P.CKPT_TYPE_F32, tokens=n, dim=200, vocab=300,
                                  ids=ids.data_ptr(), ignore_index=IGNORE, scale=1.0, rows=d.data_ptr(), rows_stride=200)
        table = torch.full((302, 200), 7.0, device="cuda")
        a.table, a.table_stride = table[1].data_ptr(), 200
        need = C.c_uint64()
        assert embed._ops().ckpt_embedding_grad_workspace(C.byref(a), C.byref(need)) == P.CKPT_OK
        assert (need.value == 0) == (n == 100)
        work = torch.full((need.value + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        assert embed._ops().ckpt_embedding_grad(C.byref(a), 0, work[256:].data_ptr() if need.value else None, need.value,
                                                torch.cuda.current_stream().cuda_stream) == P.CKPT_OK
        torch.cuda.synchronize()
        assert (work[:256] == 0x5A).all() and (work[-256:] == 0x5A).all()
        assert (table[0] == 7).all() and (table[-1] == 7).all()
        assert torch.equal(table[1:-1], P.ckpt_embedding_grad(d[:n], ids, 300))
        if need.value:
            assert embed._ops().ckpt_embedding_grad(C.byref(a), 0, work[256:].data_ptr(), need.value - 1, None) == P.CKPT_EINVAL


def test_refusals():
    table = torch.randn(10, 8, device="cuda")
    ids = torch.tensor([1, 2], device="cuda")
    d = torch.randn(2, 8, device="cuda")
    for bad in (table.half(), table.cpu(), table[None], table[:, ::2]):
        with pytest.raises(ValueError):
            P.ckpt_embedding(bad, ids)
    for bad in (ids.int(), ids.cpu(), torch.arange(6, device="cuda")[::2]):
        with pytest.raises(ValueError):
            P.ckpt_embedding(table, bad)
        with pytest.raises(ValueError):
            P.ckpt_embedding_grad(torch.randn(bad.numel(), 8, device="cuda"), bad, 10)
    for kw in (dict(scale=math.nan), dict(scale=1e300)):
        with pytest.raises(P.CkptError):
            P.ckpt_embedding(table, ids, **kw)
        with pytest.raises(P.CkptError):
            P.ckpt_embedding_grad(d, ids, 10, **kw)
    with pytest.raises(P.CkptError):
        P.ckpt_embedding(table[:1].expand(10, 8), ids)
    with pytest.raises(P.CkptError):
        P.ckpt_embedding_grad(d, ids, 0)
    with pytest.raises(ValueError):
        P.ckpt_embedding_grad(d.half(), ids, 10)
    with pytest.raises(ValueError):
        P.ckpt_embedding_grad(d[None], ids, 10)
    for bad in (table[:9], table[:, :7], table.half(), table.cpu()):
        with pytest.raises(ValueError):
            P.ckpt_embedding_grad(d, ids, 10, add_to=bad)
    both = torch.randn(14, 8, device="cuda")
    with pytest.raises(P.CkptError):
        P.ckpt_embedding_grad(both[9:11], ids, 10, add_to=both[:10])
    with pytest.raises(ValueError):
        P.ckpt_embedding_grad(d, ids, 10, dtype=torch.float16)
    with pytest.raises(ValueError):
        P.ckpt_embedding_grad(d, ids, 10, dtype=BF, add_to=table)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n, dim, vocab", [(5, 7, 300), (100, 513, 333), (300, 1, 1000), (1000, 259, 500)])
def test_what_lies_beside_the_gradient_s_rows(n, dim, vocab, dtype):
    """Rows of the C call's table at any place and any distance: all of each is written, and nothing else."""
    import ctypes as C
    from paper_2607_01646_amd import embed
    d = torch.randn(n, dim, generator=gen(n), device="cuda").to(dtype)
    ids = masked(words(n, vocab, "text"))
    want = P.ckpt_embedding_grad(d, ids, vocab)
    for begin, more in ((0, 1), (1, 0), (3, 8), (5, 129), (64, 3)):
        whole = torch.full((begin + vocab * (dim + more) + 100,), 7.0, device="cuda").to(dtype)
        a = embed.ckpt_embed_args(dtype=P.CKPT_TYPE_BF16 if dtype == BF else P.CKPT_TYPE_F32, tokens=n, dim=dim, vocab=vocab,
                                  ids=ids.data_ptr(), ignore_index=IGNORE, scale=1.0, rows=d.data_ptr(), rows_stride=dim,
                                  table=whole.data_ptr() + begin * whole.element_size(), table_stride=dim + more)
        a.table_dtype = a.dtype
        need = C.c_uint64()
        assert embed._ops().ckpt_embedding_grad_workspace(C.byref(a), C.byref(need)) == P.CKPT_OK
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        assert embed._ops().ckpt_embedding_grad(C.byref(a), 0, work.data_ptr(), need.value,
                                                torch.cuda.current_stream().cuda_stream) == P.CKPT_OK
        rows = whole[begin:begin + vocab * (dim + more)].view(vocab, dim + more)
        assert torch.equal(rows[:, :dim], want)
        assert bool((rows[:, dim:] == 7).all()) and bool((whole[:begin] == 7).all()) and bool((whole[begin + vocab * (dim + more):] == 7).all())


@pytest.mark.parametrize("kind", ["text", "one"])
def test_more_tokens_of_a_word_than_its_sorting_waves_list(kind):
    n, dim, vocab = 150000, 17, 300000
    d = torch.randn(n, dim, generator=gen(n), device="cuda")
    ids = masked(words(n, vocab, kind))
    want, bound, count = reference(d, ids, vocab, 1.0)
    got = P.ckpt_embedding_grad(d, ids, vocab)
    within(got, want, bound + U32 * want.abs(), "table")
    assert torch.equal(got, P.ckpt_embedding_grad(d, ids, vocab))


def test_ids_that_lie_in_what_is_written():
    table = torch.zeros(10, 8, device="cuda")
    ids = table.view(torch.int64)[3, :2]
    with pytest.raises(P.CkptError, match="overlap"):
        P.ckpt_embedding_grad(torch.ones(2, 8, device="cuda"), ids, 10, add_to=table)
    assert not table.any()
    d = torch.zeros(2, 8, device="cuda")  # ids beside the rows that are only read
    assert not P.ckpt_embedding_grad(d, d.view(torch.int64)[0, :2], 10).any()
