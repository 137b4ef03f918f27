"""Attention over a cache in 4 bits whose tables name no page inside of a request's length, as page_tables and page_fork write
them where free pages run out: keys and values of such slots are zeros, whatever the memory of a block held before (GPU)."""
import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


def with_holes(b, holes):
    """b's table on the GPU with entries that are no pages at `holes` [(request, page)]; for the reference they are a page of
    zeros."""
    table = b.table.clone()
    for i, (r, n) in enumerate(holes):
        table[r, n] = (-1, b.npages, 2 ** 31 - 1, -2 ** 31)[i % 4]
        b.table[r, n] = b.npages
    b.k, b.v = (torch.cat([x, torch.zeros_like(x[:1])]) for x in (b.k, b.v))
    return table.cuda()


# 1 and 8 tokens: the row kernel, of few rows and of 32; 100: the tensor cores
@pytest.mark.parametrize("tokens", [1, 8, 100])
@pytest.mark.parametrize("D,page,dtype", [(128, 16, BF16), (128, 32, FP16), (64, 48, BF16), (32, 64, FP16), (96, 16, FP16)])
def test_pages_that_are_not_there(slnr, tokens, D, page, dtype):
    """The first page, some in the middle, the last, every second one, all: those rows see zeros, the others what they did."""
    lens = [(tokens, 700)] * 4 + [(tokens, 333), (min(3, tokens), 500), (1, 130)]
    b = P.Batch4(slnr, lens, page, 8, 2, D, dtype, seed=D + tokens)
    n = -(-700 // page)
    holes = [(0, 0), (1, n // 2), (1, n // 2 + 1), (2, n - 1), (6, 130 // page)]
    holes += [(3, i) for i in range(0, n, 2)] + [(4, i) for i in range(-(-333 // page))]
    table = with_holes(b, holes)
    ref = b.attention(D ** -0.5)
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(table=table))
    b.check(got, ref)
    assert (got[0][4 * tokens:5 * tokens] == 0).all()
    for x, y in zip(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(table=table)), got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("tokens", [1, 8, 100])
def test_long_requests_of_which_pages_are_not_there(slnr, tokens):
    """Shares of many units, cut through the items; runs of pages, at the ends of a block's share too."""
    b = P.Batch4(slnr, [(1, 4000), (tokens, 9000)], 16, 4, 1, 64, seed=tokens)
    g = torch.Generator().manual_seed(1)
    some = torch.randperm(562, generator=g)[:300].tolist()
    table = with_holes(b, [(1, i) for i in some] + [(0, i) for i in range(20, 200)])
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(table=table)), b.attention(0.125))


@pytest.mark.parametrize("tokens", [1, 100])
def test_a_cache_without_pages(slnr, tokens):
    b = P.Batch4(slnr, [(tokens, 200)], 16, 4, 2, 64, FP16, seed=3)
    b.table[:], b.k, b.v = 0, 0 * b.k[:1].nan_to_num(), 0 * b.v[:1].nan_to_num()
    cache = slnr.PagedCache4(torch.empty((0, 2, 1, 18 * 64), dtype=torch.uint8, device="cuda"))
    b.check(slnr.paged_attention(b.q.cuda(), cache, b.tables()), b.attention(0.125))
