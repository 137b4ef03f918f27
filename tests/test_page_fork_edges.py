"""page_fork of requests whose tables or lengths are not whole: entries that are no pages, lengths past a row's end (GPU)."""
import pytest

torch = pytest.importorskip("torch")

from _paged4 import i32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


def test_a_last_page_that_is_none_is_not_copied(slnr):
    """Where free pages ran out before, a request's last entry is -1: no child of it takes a page, as there is nothing to copy."""
    table = i32([[3, 4, -1], [5, 6, 7], [-1, 9, 9], [-5, 8, 8]])
    lens = i32([40, 33, 7, 1])
    new, new_lens, src, dst, used = slnr.page_fork(table, lens, i32([0, 0, 1, 2, 1, 2, 0, 3, 3]), i32([20, 21, 22]), 16)
    assert new_lens.tolist() == [40, 40, 33, 7, 33, 7, 40, 1, 1]
    assert src.tolist() == [-1, -1, -1, -1, 7, -1, -1, -1, -1] and dst.tolist() == [-1, -1, -1, -1, 20, -1, -1, -1, -1]
    assert used.item() == 1
    got = new.tolist()
    assert [got[i] for i in (0, 1, 6)] == [[3, 4, -1]] * 3 and got[2] == [5, 6, 7] and got[4] == [5, 6, 20]
    for i in (3, 5, 7, 8):  # a full row would be no page either
        assert got[i][0] < 0 and got[i][1:] == [-1, -1]


def test_lengths_past_a_rows_end_are_the_rows(slnr):
    table = i32([[3, 4], [5, 6], [7, 8]])
    parent = i32([0, 1, 1, 2, 0])
    new, lens, src, dst, used = slnr.page_fork(table, i32([33, 2 ** 31 - 1, -4]), parent, i32([9]), 16)
    assert lens.tolist() == [32, 32, 32, 0, 32] and used.item() == 0
    assert new.tolist() == [[3, 4], [5, 6], [5, 6], [-1, -1], [3, 4]]
    assert (src == -1).all() and (dst == -1).all()
    # pages that together hold more slots than an int counts: no length is past the end
    for n in (2 ** 31 - 1, 2 ** 30):
        assert slnr.page_fork(table, i32([n] * 3), parent, i32([9]), 2 ** 30)[1].tolist() == [n] * 5
    assert slnr.page_fork(table[:, :0], i32([5, 6, 7]), parent, i32([9]), 16)[1].tolist() == [0] * 5
    with pytest.raises(slnr.SlnrError, match="SLNR_ERR_INDEX"):
        slnr.page_fork(table, i32([33, 2, 3]), parent, i32([9]), 16, validate=True)
