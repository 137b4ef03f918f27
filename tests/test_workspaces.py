"""Which device buffer a call is given: by the bookkeeping alone, with the library and the GPU faked (no GPU needed)."""
import contextlib
import threading
import time
import weakref
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2205_11622_gb300 as slnr  # noqa: E402
from paper_2205_11622_gb300 import paged  # noqa: E402

STREAM = 0x10


class Library:
    """Entry points that note the workspace that they are given."""

    def __init__(self):
        self.given = []

    def __getattr__(self, name):
        def entry(*args):
            o = args[-1]._obj
            self.given.append((o.workspace, o.workspace_bytes))
            return 0
        return entry


@pytest.fixture
def machine(monkeypatch):
    """A fake of the library, of the device's memory and of the current stream; .capturing is the stream's state."""
    m = Library()
    m.capturing = False
    empty = torch.empty
    for mod in (slnr, paged):
        monkeypatch.setattr(mod, "lib", lambda: m)
    monkeypatch.setattr(slnr, "_lib", m)
    monkeypatch.setattr(slnr, "_default_ws", {})
    monkeypatch.setattr(paged, "_default_ws", slnr._default_ws, raising=False)
    monkeypatch.setattr(slnr, "_last_ws", [None])
    monkeypatch.setattr(paged, "_last_ws", slnr._last_ws)
    monkeypatch.setattr(slnr, "_ws_bytes", lambda name, shape, sizes, *_: sizes[0])
    monkeypatch.setattr(slnr, "_stream_ptr", lambda stream: STREAM)
    monkeypatch.setattr(paged, "_device_now", lambda: 0)
    monkeypatch.setattr(paged, "_stream_now", lambda index: STREAM)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: m.capturing)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    return m


def paged_call(need, workspace=None):
    paged._call("slnr_paged_attention", (), 0, need, False, workspace, None, ())


def expression_call(need, workspace=None):
    slnr._run("slnr_spmm_gemm", slnr.slnr_csr(4, 4, 4, None, None, None), (), (need,), "fused", True, False, workspace, None)


@pytest.fixture(params=[paged_call, expression_call])
def call(request):
    return request.param


def shared():
    return slnr._default_ws[0, STREAM].buf.data_ptr()


def test_calls_of_a_stream_share_a_buffer(machine, call):
    for need in (1000, 5000, 4000):
        call(need)
    one, two, three = machine.given
    assert one[1] == 1000 and two[1] >= 5000 and three == two and two[0] == shared()


def test_a_captured_call_has_a_buffer_of_its_own(machine, call):
    """A graph holds the address: the stream's buffer, which later calls grow and share, is not given to it."""
    call(1000)
    machine.capturing = True
    call(1000)
    call(5000)
    machine.capturing = False
    eager, captured, larger = machine.given
    assert captured[0] != eager[0] and larger[0] != eager[0] and larger[1] >= 5000
    assert shared() == eager[0] and slnr._default_ws[0, STREAM].buf.numel() == eager[1]


def test_a_callers_workspace_keeps_what_a_captured_call_was_given(machine, call):
    """It grows with later calls, but the buffer that a graph holds the address of stays allocated."""
    ws = slnr.Workspace()
    machine.capturing = True
    call(1000, ws)
    machine.capturing = False
    held = ws.buf
    address = held.data_ptr()
    assert machine.given[-1][0] == address
    call(50000, ws)
    assert machine.given[-1][0] != address and ws.buf is not held
    alive = weakref.ref(held)
    del held
    slnr._last_ws[0] = None
    assert alive() is not None and alive().data_ptr() == address


def test_an_uncaptured_workspace_frees_what_it_outgrew(machine, call):
    ws = slnr.Workspace()
    call(1000, ws)
    old = weakref.ref(ws.buf)
    call(50000, ws)
    assert old() is None


class Bare:
    """A caller's workspace with get() alone."""

    def __init__(self):
        self.held = []

    def get(self, need):
        self.held.append(torch.empty(need, dtype=torch.uint8))
        return self.held[-1]


@pytest.mark.parametrize("workspace", [None, slnr.Workspace, Bare])
def test_threads_of_a_stream_do_not_share_a_buffer_at_once(machine, call, workspace):
    """A call is several launches that hand their results on in the workspace: those of two threads that use one stream
    (all threads do, by default) may not mix."""
    ws = workspace() if workspace else None
    inside, mixed, calls = [], [], []

    def entry(*args):
        inside.append(1)
        time.sleep(0.002)  # as a foreign call without the interpreter's lock
        if len(inside) > 1:
            mixed.append(len(inside))
        calls.append(args[-1]._obj.workspace)
        inside.pop()
        return 0

    machine.slnr_paged_attention = machine.slnr_spmm_gemm = entry
    threads = [threading.Thread(target=lambda i=i: [call(1000 + 500 * i + k, ws) for k in range(5)]) for i in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(calls) == 30 and not mixed


def test_a_refused_call_leaves_the_workspace_usable(machine, call):
    machine.slnr_paged_attention = machine.slnr_spmm_gemm = lambda *args: 2
    machine.slnr_last_error = lambda: b"refused"
    for _ in range(2):
        with pytest.raises(slnr.SlnrError) as e:
            call(1000)
        assert e.value.status == 2


def test_a_captured_stream_that_is_given(machine, monkeypatch):
    """The stream of the call counts, not the current one: captured there, or captured here."""
    side = SimpleNamespace(cuda_stream=0x20)
    made, states = [], {0x20: 0}

    def state_of(s, out):
        out._obj.value = states[s]
        return 0

    machine.cudaStreamIsCapturing = state_of
    monkeypatch.setattr(slnr, "_stream_ptr", lambda stream: stream.cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: made.append(s) or contextlib.nullcontext())
    run = lambda: slnr._run("slnr_spmm_gemm", slnr.slnr_csr(4, 4, 4, None, None, None), (), (1000,), "fused", True, False,  # noqa: E731
                            None, side)
    run()
    run()
    assert machine.given[0] == machine.given[1] and made == [side]  # its memory is that stream's; made once
    states[0x20] = 1
    run()
    assert machine.given[2][0] != machine.given[0][0] and made == [side, side]
    paged._call("slnr_paged_attention", (), 0, 1000, False, None, side, ())
    assert machine.given[3][0] != machine.given[0][0]
    states[0x20], machine.capturing = 0, True
    run()
    paged._call("slnr_paged_attention", (), 0, 1000, False, None, side, ())
    assert machine.given[0] == machine.given[4] == machine.given[5]
    states[0x20] = 2  # a capture that something made void
    run()
    assert machine.given[6][0] != machine.given[0][0]
