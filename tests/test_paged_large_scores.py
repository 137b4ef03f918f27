"""Scores so large that fp32 tells apart whole numbers only, or multiples of larger ones (GPU).

All scores of a row are equal, so the output is the mean of the values whatever their size: the weights may not leave the
range of the cache's type, and parts that are joined may not lose their sums beside the scores.  A log-sum-exp is off by
four roundings of its own size at most: the factor log2 e, its product with the score, the logarithm added, and ln 2.
"""
import math

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


@pytest.mark.parametrize("lens", [[(1, 300)], [(80, 300)]])
@pytest.mark.parametrize("q,k", [(1.0, 17.5), (-60.0, 60000.0), (60.0, 60000.0), (1000.0, 60000.0)])
def test_scores_of_any_size_in_fp16(slnr, lens, q, k):
    b = P.Batch(lens, 16, 4, 1, 16, torch.float16, seed=3)
    b.q = torch.full_like(b.q, q)
    b.k = torch.where(torch.isnan(b.k), b.k, torch.full_like(b.k, k))
    b.kd = b.k.cuda()
    out, lse = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=1.0)
    want, want_lse, mag = b.attention(1.0)  # equal scores: the mean of the values
    assert ((out.double().cpu() - want).abs() <= 2.5 * P.U[torch.float16] * mag).all()
    assert ((lse.double().cpu() - want_lse).abs() <= P.LSE_TOL + 2.0 ** -22 * want_lse.abs()).all()
    assert math.isfinite(float(lse.abs().max()))


@pytest.mark.parametrize("lens", [[(1, 300)], [(1, 9000)], [(80, 300)], [(90, 6000)]])
@pytest.mark.parametrize("q,k", [(60.0, 60000.0), (-1e10, 1e20), (1e10, 1e20)])
def test_scores_of_any_size_in_bf16(slnr, lens, q, k):
    b = P.Batch(lens, 16, 4, 1, 16, torch.bfloat16, seed=3)
    b.q = torch.full_like(b.q, q)
    b.k = torch.where(torch.isnan(b.k), b.k, torch.full_like(b.k, k))
    b.kd = b.k.cuda()
    out, lse = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=1.0)
    want, want_lse, mag = b.attention(1.0)  # equal scores: the mean of the values
    assert ((out.double().cpu() - want).abs() <= 2.5 * P.U[torch.bfloat16] * mag).all()
    assert ((lse.double().cpu() - want_lse).abs() <= P.LSE_TOL + 2.0 ** -22 * want_lse.abs()).all()
    assert math.isfinite(float(lse.abs().max()))
