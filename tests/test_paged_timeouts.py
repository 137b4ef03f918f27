"""Rows of calls whose device-side waits gave up: NaN or right, never what the output's memory held (GPU)."""
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


@pytest.mark.parametrize("selected", [False, True])
@pytest.mark.parametrize("lens", [[(200, 1500)], [(100, 1500), (20, 20)], [(90, 90), (300, 700), (70, 4000)]])
def test_rows_without_validation(slnr, lens, selected):
    """Items of two row tiles and of one, whole ones and such that shares cut; limits from none to more than a step takes."""
    b = P.Batch(lens, 16, 4, 2, 64, seed=90)
    picked = P.picks(b, 40, seed=91) if selected else None
    ref = b.attention(0.125, picked)
    out, lse = torch.empty_like(b.q, device="cuda"), torch.empty(b.q.shape[:2], device="cuda")
    args = (b.q.cuda(), b.cache(), b.tables()) + ((picked.cuda(),) if selected else ())
    call = slnr.selected_attention if selected else slnr.paged_attention
    lib = slnr.lib()
    gave_up = 0
    for limit in (1, 100, 1000, 3000, 10000, 30000, 100000, 0):
        out.fill_(7)
        lse.fill_(7)
        assert lib.slnr_set_wait_limit(ctypes.c_int64(limit)) == 0
        try:
            call(*args, out=out, lse=lse)
            flags = slnr.device_flags()
        finally:
            assert lib.slnr_set_wait_limit(ctypes.c_int64(0)) == 0
        bad = torch.isnan(lse).cpu()
        assert torch.equal(torch.isnan(out).all(-1).cpu(), bad) and torch.equal(torch.isnan(out).any(-1).cpu(), bad)
        assert not bad.any() or flags & 16, limit
        gave_up += int(bad.sum())
        good = ~bad
        want, want_lse, mag = (x[good] for x in ref)
        b.check((out.cpu()[good], lse.cpu()[good]), (want, want_lse, mag), f"limit {limit}")
    assert gave_up > 0 and not bad.any()
