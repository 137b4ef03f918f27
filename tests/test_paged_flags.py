"""The flag word after calls over a paged cache that set none (GPU)."""
import ctypes

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


def call(slnr, b, selected=False, **kw):
    if selected:
        return slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), P.picks(b, 3).cuda(), **kw)
    return slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), **kw)


@pytest.mark.parametrize("selected", [False, True])
@pytest.mark.parametrize("lens", [[(1, 40)], [(0, 5), (1, 700)], [(1, 9000), (1, 3)]])  # one block, a cluster, two launches
def test_no_flag_on_memory_that_held_others(slnr, lens, selected):
    b, ws = P.Batch(lens, 16, 4, 2, 64, seed=80), slnr.Workspace()
    ws.get(64 << 20).fill_(255)
    call(slnr, b, selected, workspace=ws)
    assert slnr.device_flags() == 0 and slnr.device_flags(ws) == 0


def test_a_timeout_is_not_reported_again(slnr):
    """A chunk whose waits gave up, then a single token: its flags are its own.  A call without tokens has none to set."""
    chunk, one, none = (P.Batch([n], 16, 4, 1, 64, seed=81) for n in ((200, 1500), (1, 50), (0, 50)))
    lib = slnr.lib()
    assert lib.slnr_set_wait_limit(ctypes.c_int64(100)) == 0
    try:
        call(slnr, chunk)
        assert slnr.device_flags() & 16
    finally:
        assert lib.slnr_set_wait_limit(ctypes.c_int64(0)) == 0
    call(slnr, one)
    assert slnr.device_flags() == 0
    ws = slnr.Workspace()
    ws.get(4096).fill_(255)
    for validate in (False, True):
        call(slnr, none, workspace=ws, validate=validate)
        assert slnr.device_flags() == 0
