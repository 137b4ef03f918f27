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
