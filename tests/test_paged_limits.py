"""The largest sizes of calls over a paged cache: what is refused, and what is not (no GPU needed: no call gets as far as a
launch)."""
import ctypes

import pytest

import paper_2205_11622_gb300 as slnr
from test_paged_abi import UNSUPPORTED, WORKSPACE, attention, cache, opts, pages, rows

MOST = 0x7FFF0000


@pytest.fixture(scope="module")
def lib():
    slnr.build()
    return slnr.lib()


def far(page_size, max_k):
    """A cache of few such pages, and requests whose tables name them again and again."""
    width = -(-max_k // page_size)
    return cache(npages=2 ** 30 // page_size, page_size=page_size), pages(max_k=max_k, width=width, table_stride=width)


@pytest.mark.parametrize("picked", [False, True])
@pytest.mark.parametrize("page_size,max_k,refused", [
    (1 << 20, MOST - 5, True),          # ends inside the last page, which ends past the limit
    (3 << 20, MOST - (1 << 20), True),
    (1 << 20, MOST - (1 << 20), False),
    (16, MOST, False), (16, MOST + 1, True), (1, 2 ** 31 - 1, True)])
def test_keys_of_a_request_in_whole_pages(lib, page_size, max_k, refused, picked):
    """Positions of a request's last page are computed as ints, past its last key too."""
    c, p = far(page_size, max_k)
    kw = dict(picked=0x7000, n=3) if picked and 3 * page_size < MOST else {}
    status = attention(lib, c=c, p=p, **kw)
    assert status == (UNSUPPORTED if refused else WORKSPACE), slnr.last_error()
    if refused:
        assert "max_k" in slnr.last_error()
        k = rows(tok=128)
        r = ctypes.byref
        assert lib.slnr_page_append(r(c), r(p), r(k), r(k), r(opts())) == UNSUPPORTED


@pytest.mark.parametrize("ntok,nreq,max_q,heads,refused", [
    (5_000_000, 10, 600_000, 8, False),       # long prompts: 78135 row tiles
    (70_000, 70_000, 40, 4, False),           # more requests than 65535, the bound on their tokens above one
    (2 ** 31 - 1, 1, 2 ** 20, 512, True),     # more row tiles than an int
    (2 ** 31 - 1, 5, 2 ** 31 - 1, 4, True)])  # rows of a request
@pytest.mark.parametrize("picked", [False, True])
def test_row_tiles_of_the_tensor_core_kernel(lib, ntok, nreq, max_q, heads, refused, picked):
    """None of its launches has row tiles along an axis that ends at 65535."""
    status = attention(lib, p=pages(ntok=ntok, nreq=nreq, max_q=max_q), heads=heads,
                       **(dict(picked=0x7000, n=3) if picked else {}))
    assert status == (UNSUPPORTED if refused else WORKSPACE), slnr.last_error()


def test_items_of_the_tensor_core_kernel(lib):
    """Row tiles times key heads are counted in an int."""
    c = cache(nheads=60_000, k_stride=(2048, 128, 0), v_stride=(2048, 128, 0))
    assert attention(lib, c=c, p=pages(ntok=50_000, nreq=50_000, max_q=80), heads=60_000) == UNSUPPORTED
    assert attention(lib, c=c, p=pages(ntok=30_000, nreq=30_000, max_q=80), heads=60_000) == WORKSPACE
