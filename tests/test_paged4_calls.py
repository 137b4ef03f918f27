"""What the calls over a 4-bit cache and over whole pages check and hold before the library is called: with it and the GPU faked
(no GPU needed)."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2205_11622_gb300 as slnr  # noqa: E402
from paper_2205_11622_gb300 import paged  # noqa: E402
from test_paged_calls import ELSEWHERE, FIELDS, HERE, Tensor as Base  # noqa: E402


class Tensor(Base):
    is_cuda = True

    def split_with_sizes(self, sizes):
        return [Tensor((n,), device=self.device) for n in sizes]

    def view(self, *shape):
        return Tensor(shape, device=self.device)


@pytest.fixture
def fake(monkeypatch):
    launched = []
    library = SimpleNamespace(**{n: (lambda *a, n=n: launched.append(n) or 0) for n in slnr.SIGNATURES})
    monkeypatch.setattr(paged, "lib", lambda: library)
    monkeypatch.setattr(paged, "_device_now", lambda: 0)
    monkeypatch.setattr(paged, "_stream_now", lambda index: 0x10)
    monkeypatch.setattr(paged, "_empty", lambda shape, dtype, device, stream:
                        Tensor((shape,) if isinstance(shape, int) else shape, dtype, device))
    monkeypatch.setattr(paged, "_attention4_bytes", lambda *a: 0)
    return launched


def cache4(device=HERE):
    c = object.__new__(paged.PagedCache4)
    c.__dict__.update(data=Tensor((4, 1, 1, 576), torch.uint8, device), page_size=16, device=device,
                      _c=slnr.slnr_cache4(4, 16, 1, 32, 576, 576, 4096), _sizes=(4, 16, 1, 32))
    return c


def cache16(device=HERE):
    c = object.__new__(paged.PagedCache)
    c.__dict__.update({f: Tensor(device=device) for f in ("v", "codes", "scales")}, k=Tensor(dtype=torch.bfloat16, device=device),
                      page_size=4, device=device, _c=slnr.slnr_cache(4, 4, 1, 8, 0), _sizes=(4, 4, 1, 8, 0))
    return c


def tables(device=HERE):
    return paged.PageTables._of(slnr.slnr_pages(1, 2, 2, 16, 1), **{f: Tensor(device=device) for f in FIELDS}, max_q=2, max_k=16)


X = (2, 1, 32)


def calls(c, t, stream=None, held=None):
    """{entry point: call}; held: a list that gets the tensors that the call has to hold."""
    x = Tensor(X, torch.bfloat16)
    mine = [Tensor((3,), device=c.device) for _ in range(2)]
    if held is not None:
        held += [x, c.data, *(getattr(t, f) for f in FIELDS)]
    return {"slnr_page_append4": lambda: paged.page_append(c, t, x, x, stream=stream),
            "slnr_paged_attention4": lambda: paged.paged_attention(x, c, t, stream=stream)}, mine


@pytest.mark.parametrize("entry", ["slnr_page_append4", "slnr_paged_attention4"])
def test_tables_and_streams(fake, entry):
    """Tables on another GPU than the cache are refused; every tensor that a call may read is held on the stream it is given."""
    with pytest.raises(ValueError, match="tables are on cuda:1"):
        calls(cache4(), tables(ELSEWHERE))[0][entry]()
    assert fake == []
    stream, held = SimpleNamespace(cuda_stream=0x20), []
    calls(cache4(), tables(), stream, held)[0][entry]()
    assert fake == [entry]
    assert all(stream in x.recorded for x in held)


def test_caches_of_another_device(fake):
    with pytest.raises(ValueError, match="the tensors are on cuda:1, the current device is 0"):
        paged.page_values(cache4(ELSEWHERE), Tensor((3,), device=ELSEWHERE))
    with pytest.raises(ValueError, match="the source is on cuda:1"):
        paged.page_copy(cache4(), Tensor((3,)), Tensor((3,)), source=cache4(ELSEWHERE))
    with pytest.raises(ValueError, match="src must be"):
        paged.page_copy(cache16(), Tensor((3,), device=ELSEWHERE), Tensor((3,)))
    with pytest.raises(ValueError, match="one kind"):
        paged.page_copy(cache16(), Tensor((3,)), Tensor((3,)), source=cache4())
    assert fake == []


def test_copies_hold_both_caches(fake):
    stream = SimpleNamespace(cuda_stream=0x20)
    for make, entry in ((cache16, "slnr_page_copy"), (cache4, "slnr_page_copy4")):
        to, source, src, dst = make(), make(), Tensor((3,)), Tensor((3,))
        paged.page_copy(to, src, dst, source=source, stream=stream)
        names = ("data",) if make is cache4 else ("k", "v", "codes", "scales")
        for x in [src, dst] + [getattr(c, n) for c in (to, source) for n in names]:
            assert x.recorded == [stream]
        assert fake.pop() == entry


def test_a_4_bit_cache_has_no_summaries(fake):
    x = Tensor(X, torch.bfloat16)
    with pytest.raises(ValueError, match="summaries"):
        paged.page_select(x, cache4(), tables(), 4)
    with pytest.raises(ValueError, match="16-bit"):
        paged.selected_attention(x, cache4(), tables(), Tensor((2, 1, 3)))
    with pytest.raises(ValueError, match="PagedCache4"):
        paged.page_values(cache16())
    with pytest.raises(ValueError, match="dtype"):
        paged.page_values(cache4(), dtype=torch.float32)
    assert fake == []


def test_types_and_shapes_of_rows(fake):
    t = tables()
    for k, v in ((Tensor(X, torch.float32), Tensor(X, torch.float32)), (Tensor(X, torch.float16), Tensor(X, torch.bfloat16)),
                 (Tensor((3, 1, 32), torch.float16),) * 2, (Tensor((2, 2, 32), torch.float16),) * 2,
                 (Tensor((2, 1, 64), torch.float16),) * 2):
        with pytest.raises(ValueError):
            paged.page_append(cache4(), t, k, v)
    with pytest.raises(ValueError, match="float16|bf16"):
        paged.paged_attention(Tensor(X, torch.float32), cache4(), t)
    no_slots = tables()
    no_slots.__dict__["slots"] = None
    with pytest.raises(ValueError, match="slots"):
        paged.page_append(cache4(), no_slots, Tensor(X, torch.float16), Tensor(X, torch.float16))
    assert fake == []


class Table(Tensor):
    def stride(self, i=None):
        s = (self.shape[1] if len(self.shape) > 1 else 1, 1)
        return s if i is None else s[i]

    def dim(self):
        return len(self.shape)


def test_whole_pages(fake):
    """Each call's checks of its lists, and the stream that holds them."""
    stream, table, lens = SimpleNamespace(cuda_stream=0x20), Table((5, 7)), Tensor((5,))
    parent, free, drop = Tensor((9,)), Tensor((4,)), Tensor((2,))
    got = paged.page_fork(table, lens, parent, free, 16, stream=stream)
    assert [tuple(x.shape) for x in got] == [(9, 7), (9,), (9,), (9,), (1,)]
    assert [x.recorded for x in (table, lens, parent, free)] == [[stream]] * 4
    got = paged.page_free(table, lens, 33, 16, drop=drop, stream=stream)
    assert [tuple(x.shape) for x in got] == [(33,), (1,)] and drop.recorded == [stream]
    got = paged.page_compact(table, lens, 33, 16, stream=stream)
    assert [tuple(x.shape) for x in got] == [(5, 7), (16,), (16,), (33,), (1,)]
    assert fake == ["slnr_page_fork", "slnr_page_free", "slnr_page_compact"]
    bad = [lambda: paged.page_fork(table, Tensor((4,)), parent, free, 16), lambda: paged.page_fork(table, lens, parent, free, 0),
           lambda: paged.page_fork(table, lens, Tensor((3, 3)), free, 16),
           lambda: paged.page_fork(table, lens, parent, Tensor((4,), torch.int64), 16),
           lambda: paged.page_free(table, lens, -1, 16), lambda: paged.page_free(table, lens, 33, 16, drop=Tensor((2, 2))),
           lambda: paged.page_free(Table((5, 7), torch.int64), lens, 33, 16),
           lambda: paged.page_compact(table, Tensor((5,), device=ELSEWHERE), 33, 16),
           lambda: paged.page_compact(table, lens, -2, 16)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert len(fake) == 3
