"""The paged cache's entry points refuse bad arguments on the host, before any CUDA call (no GPU needed)."""
import ctypes

import pytest

import paper_2205_11622_gb300 as slnr

OK, NULL, SHAPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 4, 5


@pytest.fixture(scope="module")
def lib():
    slnr.build()
    return slnr.lib()


def cache(**kw):
    c = slnr.slnr_cache(100, 16, 2, 64, 0, 0)
    c.k_stride[:] = c.v_stride[:] = (2048, 128, 64)
    c.k, c.v, c.codes, c.scales = 0x10000, 0x20000, 0x30000, 0x40000
    for k, v in kw.items():
        if k in ("k_stride", "v_stride"):
            getattr(c, k)[:] = v
        else:
            setattr(c, k, v)
    return c


def pages(**kw):
    p = slnr.slnr_pages(3, 5, 4, 100, 8, 0, 8, 0x1000, 0x2000, 0x3000, 0x4000, 0x5000)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def rows(p=0x50000, tok=512, head=64):
    return slnr.slnr_rows(p, tok, head)


def opts(**kw):
    o = slnr.slnr_opts(0, 0, 0, 0, None, None, 0)
    for k, v in kw.items():
        setattr(o, k, v)
    return o


def attention(lib, c=None, p=None, q=None, heads=8, scale=0.125, out=0x60000, o=None, picked=None, n=0):
    c, p, q, o = c or cache(), p or pages(), q or rows(), o or opts()
    r = ctypes.byref
    if n:
        return lib.slnr_selected_attention(r(q), heads, r(c), r(p), picked, n, scale, out, None, r(o))
    return lib.slnr_paged_attention(r(q), heads, r(c), r(p), scale, out, None, r(o))


BAD_CACHES = [(dict(npages=-1), SHAPE), (dict(page_size=0), SHAPE), (dict(nheads=0), SHAPE), (dict(head_dim=0), SHAPE),
              (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
              (dict(reserved=1), UNSUPPORTED), (dict(npages=1 << 28), UNSUPPORTED), (dict(k_stride=(2048, 132, 64)), UNSUPPORTED),
              (dict(v_stride=(2048, 128, -64)), UNSUPPORTED), (dict(k=None), NULL), (dict(v=0x20008), UNSUPPORTED)]
BAD_PAGES = [(dict(nreq=-1), SHAPE), (dict(ntok=-1), SHAPE), (dict(max_k=129), SHAPE), (dict(table_stride=7), SHAPE),
             (dict(max_q=0), SHAPE), (dict(nreq=0), SHAPE), (dict(reserved=3), UNSUPPORTED), (dict(q_pos=None), NULL),
             (dict(k_len=None), NULL), (dict(table=None), NULL), (dict(req=None), NULL)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches(lib, bad, status):
    assert attention(lib, c=cache(**bad)) == status, slnr.last_error()
    assert attention(lib, c=cache(**bad), picked=0x7000, n=3) == status
    k = rows(tok=128)
    assert lib.slnr_page_append(ctypes.byref(cache(**bad)), ctypes.byref(pages()), ctypes.byref(k), ctypes.byref(k),
                                ctypes.byref(opts())) == status


@pytest.mark.parametrize("bad,status", BAD_PAGES)
def test_bad_pages(lib, bad, status):
    assert attention(lib, p=pages(**bad)) == status, slnr.last_error()
    q = rows()
    assert lib.slnr_page_select(ctypes.byref(q), 8, ctypes.byref(cache()), ctypes.byref(pages(**bad)), 0x7000, 4, 1, 2,
                                ctypes.byref(opts())) == status


def test_bad_attention_arguments(lib):
    assert attention(lib, heads=7) == SHAPE
    assert attention(lib, heads=0) == SHAPE
    assert attention(lib, q=rows(p=None)) == NULL
    assert attention(lib, q=rows(p=0x50004)) == UNSUPPORTED
    assert attention(lib, q=rows(tok=500)) == UNSUPPORTED
    assert attention(lib, scale=float("nan")) == SHAPE
    assert attention(lib, scale=float("inf")) == SHAPE
    assert attention(lib, out=None) == NULL
    assert attention(lib, out=0x60008) == UNSUPPORTED
    assert attention(lib, o=opts(reserved=1)) == UNSUPPORTED
    assert attention(lib) == WORKSPACE and "workspace" in slnr.last_error()
    assert attention(lib, o=opts(workspace=0x1010, workspace_bytes=1 << 30)) == WORKSPACE
    assert attention(lib, picked=None, n=3) == NULL
    assert attention(lib, picked=0x7000, n=1025) == UNSUPPORTED
    assert lib.slnr_selected_attention(ctypes.byref(rows()), 8, ctypes.byref(cache()), ctypes.byref(pages()), 0x7000, 0,
                                       0.1, 0x60000, None, ctypes.byref(opts())) == SHAPE
    assert attention(lib, p=pages(nreq=0, ntok=0)) == OK  # nothing to do: nothing is launched


def test_bad_select_arguments(lib):
    call = lambda n, first, last, **kw: lib.slnr_page_select(  # noqa: E731
        ctypes.byref(rows()), 8, ctypes.byref(cache(**kw.get("c", {}))), ctypes.byref(pages(**kw.get("p", {}))),
        kw.get("out", 0x7000), n, first, last, ctypes.byref(opts()))
    assert call(0, 0, 1) == SHAPE
    assert call(4, -1, 2) == SHAPE
    assert call(4, 1, 0) == SHAPE
    assert call(4, 2, 3) == SHAPE
    assert call(1025, 1, 2) == UNSUPPORTED
    assert call(4, 1, 2, out=None) == NULL
    assert call(4, 1, 2, c=dict(codes=None)) == NULL
    assert call(4, 1, 2, c=dict(codes=0x30004)) == UNSUPPORTED
    assert call(4, 1, 2, p=dict(width=60000, table_stride=60000, max_k=60000 * 16)) == UNSUPPORTED
    assert call(4, 1, 2, p=dict(nreq=0, ntok=0)) == OK


def test_bad_table_arguments(lib):
    def call(nreq=2, table=0x3000, stride=8, width=8, free=0x4000, nfree=4, page=16, ntok=3, q_pos=0x5000, req=0x6000, o=None):
        return lib.slnr_page_tables(nreq, 0x1000, 0x2000, table, stride, width, free, nfree, page, ntok, q_pos, 0x7000, req,
                                    0x8000, 0x9000, ctypes.byref(o) if o else None)
    assert call() == NULL
    for bad, status in [(dict(nreq=-1), SHAPE), (dict(stride=7), SHAPE), (dict(page=0), SHAPE), (dict(nfree=-1), SHAPE),
                        (dict(table=None), NULL), (dict(free=None), NULL), (dict(q_pos=None), NULL), (dict(req=None), NULL)]:
        assert call(**bad, o=opts()) == status, bad
    assert call(o=opts(validate=1)) == WORKSPACE


def test_workspace_queries(lib):
    n = ctypes.c_size_t(0)
    r = ctypes.byref
    query = lambda p, c=None: lib.slnr_paged_attention_workspace(r(c or cache()), r(p), 8, r(opts()), r(n))  # noqa: E731
    assert query(pages()) == OK and n.value >= 256 and n.value % 256 == 0
    assert query(pages(q_pos=None, k_len=None, table=None, req=None)) == OK  # sizes alone
    few = n.value
    assert query(pages(max_k=100_000, width=7000, table_stride=7000)) == OK and n.value > few
    assert query(pages(max_k=129)) == SHAPE
    assert query(pages(), cache(head_dim=12)) == UNSUPPORTED
    assert lib.slnr_paged_attention_workspace(r(cache()), r(pages()), 8, r(opts()), None) == NULL
    assert lib.slnr_selected_attention_workspace(r(cache()), r(pages()), 8, 0, r(opts()), r(n)) == SHAPE
    assert lib.slnr_selected_attention_workspace(r(cache()), r(pages()), 8, 4, r(opts()), r(n)) == OK


def test_python_objects_refuse_cpu_tensors():
    torch = pytest.importorskip("torch")
    i = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        slnr.PageTables(table=i, q_pos=i[0], k_len=i[0], req=i[0], slots=None, max_q=1, max_k=1)
    k = torch.zeros((2, 4, 1, 8), dtype=torch.bfloat16)
    for bad in (dict(k=k, v=k), dict(k=k), dict(), dict(k=k.float(), v=k.float()), dict(codes=k, scales=None)):
        with pytest.raises(ValueError):
            slnr.PagedCache(**bad)
