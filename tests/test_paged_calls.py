"""What the calls over a paged cache check and hold before the library is called: with it and the GPU faked (no GPU needed)."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2205_11622_gb300 as slnr  # noqa: E402
from paper_2205_11622_gb300 import paged  # noqa: E402

HERE, ELSEWHERE = torch.device("cuda", 0), torch.device("cuda", 1)


class Tensor:
    """As much of a tensor as the calls look at; notes the streams that it is recorded on."""

    def __init__(self, shape=(1,), dtype=torch.int32, device=HERE):
        self.shape, self.dtype, self.device, self.recorded = torch.Size(shape), dtype, device, []

    def stride(self):
        return tuple(8 for _ in self.shape[1:]) + (1,)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return 1 << 20

    def record_stream(self, stream):
        self.recorded.append(stream)


FIELDS = ("table", "q_pos", "k_len", "req", "slots")


@pytest.fixture
def calls(monkeypatch):
    """calls(device of the tables, stream) -> (tables, {entry point: call}) on a faked library."""
    launched = []
    fake = SimpleNamespace(**{n: (lambda *a, n=n: launched.append(n) or 0) for n in slnr.SIGNATURES})
    monkeypatch.setattr(paged, "lib", lambda: fake)
    monkeypatch.setattr(paged, "_device_now", lambda: 0)
    monkeypatch.setattr(paged, "_stream_now", lambda index: 0x10)
    monkeypatch.setattr(paged, "_empty", lambda shape, dtype, device, stream: Tensor(shape, dtype, device))
    monkeypatch.setattr(paged, "_attention_bytes", lambda *a: 0)

    def make(device, stream):
        tables = paged.PageTables._of(slnr.slnr_pages(1, 2, 2, 4, 1), **{f: Tensor(device=device) for f in FIELDS}, max_q=2,
                                      max_k=4)
        cache = object.__new__(paged.PagedCache)
        c = slnr.slnr_cache(4, 4, 1, 8, 0)
        cache.__dict__.update({f: Tensor() for f in ("v", "codes", "scales")}, k=Tensor(dtype=torch.bfloat16), page_size=4,
                              device=HERE, _c=c, _sizes=(4, 4, 1, 8, 0))
        x = Tensor((2, 1, 8), torch.bfloat16)
        return launched, tables, {
            "slnr_page_append": lambda: paged.page_append(cache, tables, x, x, stream=stream),
            "slnr_page_select": lambda: paged.page_select(x, cache, tables, 4, stream=stream),
            "slnr_paged_attention": lambda: paged.paged_attention(x, cache, tables, stream=stream),
            "slnr_selected_attention": lambda: paged.selected_attention(x, cache, tables, Tensor((2, 1, 3)), stream=stream)}
    return make


ENTRIES = ("slnr_page_append", "slnr_page_select", "slnr_paged_attention", "slnr_selected_attention")


@pytest.mark.parametrize("entry", ENTRIES)
def test_tables_of_another_device(calls, entry):
    """Tables beside the cache are taken, tables on another GPU refused: the kernels follow their addresses."""
    launched, _, on = calls(HERE, None)
    on[entry]()
    assert launched == [entry]
    _, _, off = calls(ELSEWHERE, None)
    with pytest.raises(ValueError, match="tables are on cuda:1"):
        off[entry]()
    assert launched == [entry]


@pytest.mark.parametrize("entry", ENTRIES)
def test_tables_are_held_on_the_stream_of_the_call(calls, entry):
    """Every tensor of the tables that a call may read is recorded on the stream that it is given: a caller may drop the
    tables while the call is pending there, and each may be an allocation of its own."""
    stream = SimpleNamespace(cuda_stream=0x20)
    launched, tables, on = calls(HERE, stream)
    on[entry]()
    assert launched == [entry]
    for name in FIELDS:
        assert getattr(tables, name).recorded == [stream], name
