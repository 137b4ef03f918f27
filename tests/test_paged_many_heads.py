"""Key heads that many query heads share: a token's rows are a large part of a row tile, or several of them (GPU)."""
import pytest

torch = pytest.importorskip("torch")

import _paged as P  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


LENS = [(1, 300), (0, 4), (3, 70), (5, 2), (2, 700), (7, 7)]


@pytest.mark.parametrize("heads", [(65, 1), (96, 1), (128, 1), (200, 2), (256, 1), (300, 1), (512, 1)])
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.float16, 16)])
def test_all_pages(slnr, heads, dtype, D):
    b = P.Batch(LENS, 16, *heads, D, dtype, seed=heads[0])
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(D ** -0.5))


@pytest.mark.parametrize("heads", [(65, 1), (96, 1), (128, 1), (200, 2), (256, 1), (300, 1), (512, 1)])
@pytest.mark.parametrize("page", [16, 7, 64])  # 7: the row kernel, a token's rows in several blocks
def test_picked_pages(slnr, heads, page):
    b = P.Batch(LENS, page, *heads, 32, torch.bfloat16, seed=heads[0] + 1)
    picked = P.picks(b, 4, seed=page)
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
    b.check(got, b.attention(32 ** -0.5, picked))


@pytest.mark.parametrize("heads", [(96, 1), (300, 1), (256, 2)])
def test_selection(slnr, heads):
    """The sum of the group's query rows, in the heads' order."""
    from test_paged_tables import plain_select
    b = P.Batch([(1, 700), (3, 100), (2, 1)], 16, *heads, 64, torch.bfloat16, seed=5)
    codes = torch.randint(-127, 128, (b.npages, b.H, 64), generator=b.g).to(torch.int8)
    scales = torch.rand((b.npages, b.H), generator=b.g)
    got = slnr.page_select(b.q.cuda(), b.cache(codes=codes.cuda(), scales=scales.cuda()), b.tables(), 6, validate=True)
    assert torch.equal(got.cpu(), plain_select(b, codes, scales, 6, 1, 2))
