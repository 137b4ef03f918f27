"""Lengths that no cache holds: results are defined where the definition reaches, and nothing outside the arrays is read or
written (GPU)."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("page", [1, 16])
def test_keys_past_the_largest_int(slnr, page):
    """One request's keys and new tokens together pass the largest int: its slots are -1, the next request has its own."""
    table = i32([[40, 41, 42, 43], [7, -1, -1, -1]])
    held = 1 if page == 1 else 16
    t, used = slnr.page_tables(i32([5, 2 * page]), i32([MOST, held]), table, i32([3, 9, 8]), page, 5 + 2 * page)
    assert t.slots.tolist() == [-1] * 5 + [3 * page + i for i in range(page)] + [9 * page + i for i in range(page)]
    assert t.req.tolist() == [0] * 5 + [1] * 2 * page and t.q_pos.tolist() == [0, 5, 5 + 2 * page]
    assert t.k_len.tolist() == [MOST, held + 2 * page] and used.tolist() == [2]
    assert table.tolist() == [[40, 41, 42, 43], [7, 3, 9, -1]]


def test_new_tokens_past_the_largest_int(slnr):
    """Sums of new tokens that pass the largest int: every slot is one of the free pages' or -1."""
    table = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    t, _ = slnr.page_tables(i32([MOST, 3, MOST, 9]), i32([0, 2, 5, 0]), table, i32([3, 1]), 4, 10)
    assert set(table.flatten().tolist()) <= {-1, 1, 3}
    assert all(s == -1 or s // 4 in (1, 3) for s in t.slots.tolist())


def test_negative_lengths_are_none(slnr):
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    t, used = slnr.page_tables(i32([-3, 4]), i32([-2 ** 31, -5]), table, i32([3, 1]), 4, 4)
    assert t.slots.tolist() == [12, 13, 14, 15] and t.req.tolist() == [1] * 4 and used.tolist() == [1]
    assert t.k_len.tolist() == [0, 4]
