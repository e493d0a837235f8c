"""The table's gradient where a word has many tokens: none is lost or counted
twice, and their order is the tokens' own (needs an MI355X; through the C
ABI)."""
import ctypes as C

import numpy as np
import pytest
import torch

from test_gpu_embed import BF, F32, IGNORE, gen, masked, words

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2607_01646_amd as P
    from paper_2607_01646_amd import embed


def digits(n, columns, dtype):
    """Rows that name their token: column c has digit c % 3 of it in base 64, from 1 on."""
    t = torch.arange(n, device="cuda")[:, None]
    return (t // 64 ** (torch.arange(columns, device="cuda") % 3) % 64 + 1).to(dtype)


@pytest.mark.parametrize("rows", [BF, F32])
@pytest.mark.parametrize("kind", ["text", "one"])
@pytest.mark.parametrize("n, dim, vocab", [(129, 70, 5), (4000, 1030, 40), (20000, 9, 3), (70000, 130, 2500), (150000, 17, 300000),
                                           (250000, 33, 900)])
def test_every_token_is_counted_once(n, dim, vocab, kind, rows):
    """Whole numbers up to 64: sums of up to 250000 of them are exact in fp32, in any order."""
    ids = masked(words(n, vocab, kind))
    d = digits(n, dim, rows)
    there = ids != IGNORE
    want = torch.zeros(vocab, dim, dtype=torch.int64).index_add_(0, ids[there].cpu(), d[there].long().cpu()).cuda()
    assert 2 * int(want.max()) + 3 < 1 << 24
    got = P.ckpt_embedding_grad(d, ids, vocab, dtype=F32)
    assert torch.equal(got, want.float())
    old = torch.full((vocab, dim), 3.0, device="cuda")
    P.ckpt_embedding_grad(d, ids, vocab, scale=2.0, add_to=old)
    assert torch.equal(old, (2 * want + 3).float())
    assert torch.equal(P.ckpt_embedding_grad(d, ids, vocab, dtype=BF), want.float().to(BF))


@pytest.mark.parametrize("kind", ["even", "text", "one"])
@pytest.mark.parametrize("n, vocab", [(129, 7), (1000, 77), (5000, 40000), (40000, 300), (150000, 300000)])
def test_tokens_are_sorted_by_word_and_keep_their_order(n, vocab, kind):
    """The words' beginnings and the tokens behind them, as the workspace holds them; the longest lists go over the ids twice."""
    ids = masked(words(n, vocab, kind))
    ids[::17] = vocab + 3  # no word
    d, table = torch.ones(n, 8, device="cuda"), torch.empty(vocab, 8, device="cuda")
    a = embed.ckpt_embed_args(dtype=P.CKPT_TYPE_F32, table_dtype=P.CKPT_TYPE_F32, tokens=n, dim=8, vocab=vocab,
                              ids=ids.data_ptr(), ignore_index=IGNORE, scale=1.0, rows=d.data_ptr(), rows_stride=8,
                              table=table.data_ptr(), table_stride=8)
    need = C.c_uint64()
    assert embed._ops().ckpt_embedding_grad_workspace(C.byref(a), C.byref(need)) == P.CKPT_OK
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    assert embed._ops().ckpt_embedding_grad(C.byref(a), 0, work.data_ptr(), need.value,
                                            torch.cuda.current_stream().cuda_stream) == P.CKPT_OK
    torch.cuda.synchronize()
    whole = lambda x: -(-x // 256) * 256
    at = whole(4 * (vocab + 1))
    start = work[:4 * (vocab + 1)].view(torch.int32)
    there = torch.nonzero((ids >= 0) & (ids < vocab))[:, 0]
    count = torch.bincount(ids[there], minlength=vocab)
    assert torch.equal(start.long(), torch.cat([count.new_zeros(1), count.cumsum(0)]))
    by_word = there[torch.argsort(ids[there], stable=True)]
    order = work[at:at + 4 * n].view(torch.int32)[:by_word.numel()]
    word = work[at + whole(4 * n):at + whole(4 * n) + 4 * n].view(torch.int32)[:by_word.numel()]
    assert torch.equal(order.long(), by_word) and torch.equal(word.long(), ids[by_word])


def in_order(rows):
    total = np.zeros(rows.shape[1], np.float32)
    for r in rows:
        total += r
    return total


@pytest.mark.parametrize("n", [1, 2, 63, 65, 100, 128])
def test_few_tokens_are_summed_in_their_order(n):
    """In fp32 and token by token: values of very different sizes, whose sum depends on their order."""
    ids = masked(words(n, 5, "text"))
    d = torch.randn(n, 70, generator=gen(n), device="cuda") * 4.0 ** torch.randint(-9, 10, (n, 1), generator=gen(n + 1), device="cuda")
    got = P.ckpt_embedding_grad(d, ids, 5).cpu().numpy()
    rows, of = d.cpu().numpy(), ids.cpu().numpy()
    for v in range(5):
        assert np.array_equal(got[v], in_order(rows[of == v])), v


@pytest.mark.parametrize("n, dim", [(129, 70), (3000, 20), (9000, 300)])
def test_many_tokens_are_summed_in_their_order(n, dim):
    """Run by run of the sorted tokens, each in its order, and the runs in theirs: so for one length of the runs, which the
    call's sizes decide, every word's sum has the bits of that order."""
    vocab = 11
    ids = masked(words(n, vocab, "text"))
    d = torch.randn(n, dim, generator=gen(n), device="cuda") * 4.0 ** torch.randint(-9, 10, (n, 1), generator=gen(n + 1), device="cuda")
    got = P.ckpt_embedding_grad(d, ids, vocab).cpu().numpy()
    there = torch.nonzero(ids >= 0)[:, 0]
    by_word = there[torch.argsort(ids[there], stable=True)].cpu().numpy()
    rows, of = d.cpu().numpy()[by_word], ids.cpu().numpy()[by_word]

    def by_runs(run):
        want = np.zeros((vocab, dim), np.float32)
        for v in np.unique(of):
            at = np.nonzero(of == v)[0]
            parts = [in_order(rows[at[at // run == k]]) for k in range(at[0] // run, at[-1] // run + 1)]
            want[v] = in_order(np.stack(parts))
        return want

    assert sum(np.array_equal(got, by_runs(8 << k)) for k in range(5)) == 1
