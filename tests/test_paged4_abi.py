"""The entry points of the 4-bit cache and of whole pages refuse bad arguments on the host, before any CUDA call (no GPU)."""
import ctypes

import pytest

import paper_2205_11622_gb300 as slnr
from test_paged_abi import NULL, OK, SHAPE, UNSUPPORTED, WORKSPACE, cache, opts, pages, rows

R = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    slnr.build()
    return slnr.lib()


def cache4(**kw):
    c = slnr.slnr_cache4(100, 16, 2, 64, 2 * 1152, 1152, 0x10000)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attention(lib, c=None, p=None, q=None, heads=8, dtype=0, scale=0.125, out=0x60000, o=None):
    return lib.slnr_paged_attention4(R(q or rows()), heads, R(c or cache4()), R(p or pages()), dtype, scale, out, None,
                                     R(o or opts()))


def append(lib, c=None, p=None, k=None, v=None, dtype=1):
    return lib.slnr_page_append4(R(c or cache4()), R(p or pages()), R(k or rows(tok=128)), R(v or rows(tok=128)), dtype, R(opts()))


def values(lib, c=None, ids=0x1000, n=3, k=0x20000, v=0x30000, dtype=0):
    return lib.slnr_page_values4(R(c or cache4()), ids, n, k, v, dtype, R(opts()))


BAD_CACHES = [(dict(npages=-1), SHAPE), (dict(page_size=0), SHAPE), (dict(nheads=0), SHAPE), (dict(head_dim=0), SHAPE),
              (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=8), UNSUPPORTED), (dict(head_dim=160), UNSUPPORTED),
              (dict(page_size=24), UNSUPPORTED), (dict(npages=1 << 28), UNSUPPORTED), (dict(page_stride=8), UNSUPPORTED),
              (dict(head_stride=-16), UNSUPPORTED), (dict(data=None), NULL), (dict(data=0x10008), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches(lib, bad, status):
    c = cache4(**bad)
    assert attention(lib, c=c) == status, slnr.last_error()
    assert append(lib, c=c) == status
    assert values(lib, c=c) == status
    assert lib.slnr_page_copy4(R(c), R(cache4()), 0x1000, 0x2000, 3, R(opts())) == status
    assert lib.slnr_page_copy4(R(cache4()), R(c), 0x1000, 0x2000, 3, R(opts())) == status


@pytest.mark.parametrize("bad,status", [
    (dict(nreq=-1), SHAPE), (dict(ntok=-1), SHAPE), (dict(max_k=129), SHAPE), (dict(table_stride=7), SHAPE),
    (dict(max_q=0), SHAPE), (dict(reserved=3), UNSUPPORTED), (dict(q_pos=None), NULL), (dict(k_len=None), NULL),
    (dict(table=None), NULL), (dict(req=None), NULL)])
def test_bad_pages(lib, bad, status):
    assert attention(lib, p=pages(**bad)) == status, slnr.last_error()
    assert append(lib, p=pages(**bad)) == status


def test_bad_attention_and_append_arguments(lib):
    assert attention(lib, heads=7) == SHAPE and attention(lib, heads=0) == SHAPE
    assert attention(lib, q=rows(p=None)) == NULL and attention(lib, q=rows(p=0x50004)) == UNSUPPORTED
    assert attention(lib, q=rows(tok=500)) == UNSUPPORTED
    assert attention(lib, scale=float("nan")) == SHAPE and attention(lib, scale=float("inf")) == SHAPE
    assert attention(lib, out=None) == NULL and attention(lib, out=0x60008) == UNSUPPORTED
    assert attention(lib, dtype=2) == UNSUPPORTED and attention(lib, dtype=-1) == UNSUPPORTED
    assert attention(lib, o=opts(reserved=1)) == UNSUPPORTED
    for max_q in (1, 4, 100):  # row kernel, wider rows, tensor cores
        assert attention(lib, p=pages(max_q=max_q)) == WORKSPACE and "workspace" in slnr.last_error()
        assert attention(lib, p=pages(max_q=max_q), o=opts(workspace=0x1010, workspace_bytes=1 << 30)) == WORKSPACE
    assert attention(lib, p=pages(nreq=0, ntok=0)) == OK  # nothing to do: nothing is launched
    assert append(lib, dtype=3) == UNSUPPORTED and append(lib, k=rows(p=None)) == NULL
    assert append(lib, v=rows(tok=100)) == UNSUPPORTED and append(lib, p=pages(slots=None)) == NULL
    assert append(lib, p=pages(nreq=0, ntok=0)) == OK
    assert append(lib, c=cache4(nheads=60_000), p=pages(ntok=2 ** 31 - 1, max_q=2 ** 31 - 1)) == UNSUPPORTED


def test_workspace_queries(lib):
    n = ctypes.c_size_t(0)
    query = lambda p, heads=8, c=None: lib.slnr_paged_attention4_workspace(R(c or cache4()), R(p), heads, R(opts()),  # noqa: E731
                                                                           R(n))
    sizes = []
    for max_q in (1, 4, 8, 100):
        assert query(pages(max_q=max_q)) == OK and n.value >= 256 and n.value % 256 == 0
        sizes.append(n.value)
    assert query(pages(q_pos=None, k_len=None, table=None, req=None), c=cache4(data=None)) == OK  # sizes alone
    assert n.value == sizes[1]
    assert query(pages(max_k=100_000, width=7000, table_stride=7000)) == OK and n.value == sizes[1]  # shares, not splits
    assert query(pages(max_k=129)) == SHAPE and query(pages(), 7) == SHAPE
    assert query(pages(), c=cache4(head_dim=80)) == UNSUPPORTED
    assert lib.slnr_paged_attention4_workspace(R(cache4()), R(pages()), 8, R(opts()), None) == NULL


def test_the_largest_calls(lib):
    """Rows, tiles and items of the tensor-core kernel are counted in ints; the row kernel's units in 64 bits."""
    for kw, heads, status in ((dict(ntok=2 ** 31 - 1, nreq=1, max_q=2 ** 20), 512, UNSUPPORTED),
                              (dict(ntok=2 ** 31 - 1, nreq=5, max_q=2 ** 31 - 1), 4, UNSUPPORTED),
                              (dict(ntok=5_000_000, nreq=10, max_q=600_000), 8, WORKSPACE),
                              (dict(ntok=2 ** 31 - 1, nreq=2 ** 31 - 1, max_q=1), 8, WORKSPACE)):
        assert attention(lib, p=pages(**kw), heads=heads) == status, slnr.last_error()
    most = 0x7FFF0000
    for max_k, status in ((most, WORKSPACE), (most + 1, UNSUPPORTED)):
        width = -(-max_k // 16)
        assert attention(lib, p=pages(max_k=max_k, width=width, table_stride=width)) == status


def test_bad_values_arguments(lib):
    assert values(lib, n=-1) == SHAPE and values(lib, ids=None, n=101) == SHAPE
    assert values(lib, k=None) == NULL and values(lib, v=None) == NULL
    assert values(lib, k=0x20008) == UNSUPPORTED and values(lib, dtype=2) == UNSUPPORTED
    assert values(lib, n=0, k=None, v=None) == OK
    assert values(lib, c=cache4(page_size=1 << 20, npages=1000, nheads=1000), n=1000) == UNSUPPORTED


def test_bad_copies(lib):
    def copy(to=None, source=None, src=0x1000, dst=0x2000, n=3, o=None):
        return lib.slnr_page_copy(R(to or cache()), R(source or cache()), src, dst, n, R(o or opts()))
    assert copy(n=-1) == SHAPE and copy(src=None) == NULL and copy(dst=None) == NULL and copy(n=0, src=None, dst=None) == OK
    assert copy(o=opts(reserved=1)) == UNSUPPORTED and copy(o=opts(validate=1)) == WORKSPACE
    for bad in (dict(page_size=32), dict(nheads=4), dict(head_dim=32), dict(dtype=1)):
        assert copy(source=cache(**bad)) == SHAPE, bad
    assert copy(source=cache(k=None, v=None)) == NULL  # keys on one side alone
    assert copy(to=cache(k=None, v=None, codes=None, scales=None), source=cache(k=None, v=None)) == NULL
    assert copy(to=cache(v=None)) == NULL and copy(to=cache(k=0x20008)) == UNSUPPORTED
    assert copy(source=cache(k_stride=(2048, 132, 64))) == UNSUPPORTED
    assert copy(to=cache(npages=0)) == OK and copy(source=cache(npages=0)) == OK  # no entry is a page
    assert lib.slnr_page_copy(None, R(cache()), 0x1000, 0x2000, 3, R(opts())) == NULL
    assert lib.slnr_page_copy(R(cache()), None, 0x1000, 0x2000, 3, R(opts())) == NULL
    big = cache(npages=1, page_size=1 << 30, nheads=64, head_dim=128)
    assert copy(to=big, source=big) == UNSUPPORTED  # more pieces of a page than an int
    c = cache4()
    for bad in (dict(page_size=32), dict(nheads=4), dict(head_dim=32)):
        assert lib.slnr_page_copy4(R(cache4(**bad)), R(c), 0x1000, 0x2000, 3, R(opts())) == SHAPE
    assert lib.slnr_page_copy4(R(c), R(c), None, 0x2000, 3, R(opts())) == NULL
    assert lib.slnr_page_copy4(R(c), R(c), None, None, 0, R(opts())) == OK
    assert lib.slnr_page_copy4(R(c), R(cache4(npages=0, data=None)), 0x1000, 0x2000, 3, R(opts())) == OK


def test_bad_sets(lib):
    def fork(nreq=3, lens=0x1000, table=0x2000, stride=8, width=8, page=16, parent=0x3000, n=4, free=0x4000, nfree=4, out=0x5000,
             out_lens=0x6000, src=0x7000, dst=0x8000, used=0x9000, o=None):
        return lib.slnr_page_fork(nreq, lens, table, stride, width, page, parent, n, free, nfree, out, out_lens, src, dst, used,
                                  R(o or opts()))

    def free(nreq=3, lens=0x1000, table=0x2000, stride=8, width=8, page=16, drop=0x3000, ndrop=2, npages=40, out=0x4000,
             count=0x5000, o=None):
        return lib.slnr_page_free(nreq, lens, table, stride, width, page, drop, ndrop, npages, out, count, R(o or opts()))

    def compact(nreq=3, lens=0x1000, table=0x2000, stride=8, width=8, page=16, npages=40, out=0x4000, src=0x5000, dst=0x6000,
                ids=0x7000, used=0x8000, o=None):
        return lib.slnr_page_compact(nreq, lens, table, stride, width, page, npages, out, src, dst, ids, used, R(o or opts()))

    for call in (fork, free, compact):
        for bad, status in [(dict(nreq=-1), SHAPE), (dict(width=-1), SHAPE), (dict(stride=7), SHAPE), (dict(page=0), SHAPE),
                            (dict(lens=None), NULL), (dict(table=None), NULL), (dict(o=opts(reserved=2)), UNSUPPORTED),
                            (dict(o=opts(validate=1)), WORKSPACE)]:
            assert call(**bad) == status, (call.__name__, bad, slnr.last_error())
    for bad, status in [(dict(n=-1), SHAPE), (dict(nfree=-1), SHAPE), (dict(n=65537), UNSUPPORTED), (dict(parent=None), NULL),
                        (dict(free=None), NULL), (dict(out=None), NULL), (dict(out_lens=None), NULL), (dict(src=None), NULL),
                        (dict(dst=None), NULL), (dict(used=None), NULL), (dict(out=0x2000), UNSUPPORTED)]:
        assert fork(**bad) == status, bad
    for bad, status in [(dict(npages=-1), SHAPE), (dict(npages=8388609), UNSUPPORTED), (dict(ndrop=-1), SHAPE),
                        (dict(drop=None), NULL), (dict(out=None), NULL), (dict(count=None), NULL)]:
        assert free(**bad) == status, bad
    for bad, status in [(dict(npages=-1), SHAPE), (dict(npages=8388609), UNSUPPORTED), (dict(out=None), NULL),
                        (dict(src=None), NULL), (dict(dst=None), NULL), (dict(ids=None), NULL), (dict(used=None), NULL),
                        (dict(out=0x2000), UNSUPPORTED)]:
        assert compact(**bad) == status, bad


def test_python_objects(lib):
    torch = pytest.importorskip("torch")
    good = torch.zeros((3, 2, 4, 18 * 64), dtype=torch.uint8)
    for bad in (good, good.float(), good[0], good[..., :100]):  # not on a GPU; another type; fewer axes; no width
        with pytest.raises(ValueError, match="data must be"):
            slnr.PagedCache4(bad)
    for kw in (dict(page_size=24), dict(page_size=0), dict(width=80), dict(width=256)):
        with pytest.raises(ValueError):
            slnr.PagedCache4.empty(**{**dict(npages=3, page_size=16, heads=2, width=64, device="cpu"), **kw})
