"""Rows of one key that outweighs all others, and many small ones (GPU).

One key's score lies 17.5 above those of n others, so each of these weighs 2^-25.2 of it.  Together they make up what one
column of the output is: w n v, every other contribution to that column being zero.  The error that is allowed is
_paged.py's: a share of sum_j w_j |v_j|, which is that column itself.  It holds where a weight is rounded by a share of
itself, as it is in bf16 at any size and in fp16 while its product with the kernel's factor of 2^12 or more stays normal
(2^-25.2 2^12 > 2^-14).
"""
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


def batch(lens, page, Hq, H, dtype, at, seed=0):
    """Key `at` of each request scores 17.5 and has the value 1 in column 1; the others score 0, 64 in column 0."""
    b = P.Batch(lens, page, Hq, H, 16, dtype, seed=seed)
    real = ~torch.isnan(b.k)
    b.q = torch.zeros_like(b.q)
    b.q[..., 0] = 1
    b.k, b.v = (torch.where(real, torch.zeros_like(x), x) for x in (b.k, b.v))
    b.v[..., 0] = torch.where(real[..., 0], torch.full_like(b.v[..., 0], 64.0), b.v[..., 0])
    for r, (_, n) in enumerate(lens):
        page_at = int(b.table[r, at // page])
        b.k[page_at, at % page, :, 0] = 17.5
        b.v[page_at, at % page, :, 0], b.v[page_at, at % page, :, 1] = 0, 1
    b.kd, b.vd = b.k.cuda(), b.v.cuda()
    return b


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("at", [0, 5, 200])
@pytest.mark.parametrize("lens,heads", [([(1, 2000)], (4, 1)), ([(1, 2000)] * 200, (4, 1)), ([(8, 1500)], (2, 1)),
                                        ([(1, 9000)], (4, 2)), ([(70, 2100)], (4, 1)), ([(100, 3000), (40, 1200)], (1, 1))])
def test_small_weights(slnr, lens, heads, at, dtype):
    """Row kernel in one part, as a cluster and in parts that are joined; the tensor-core kernel with two tiles and one."""
    b = batch(lens, 16, *heads, dtype, at)
    ref = b.attention(1.0)
    assert float(ref[0][..., 0].min()) > 64 * 1000 * 2.0 ** -25.3
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=1.0), ref)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens", [[(1, 2000)], [(70, 2100)]])
def test_small_weights_of_picked_pages(slnr, lens, dtype):
    b = batch(lens, 16, 4, 1, dtype, 5)
    picked = torch.arange(120, dtype=torch.int32).expand(b.T, 1, 120).clone()
    b.check(slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), scale=1.0), b.attention(1.0, picked))
