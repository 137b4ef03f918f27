"""Block tables, slot maps, appended keys and page selection against plain definitions (GPU)."""
import math

import numpy as np
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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def plain_tables(new, old, table, free, s):
    table, free = table.clone(), list(free)
    taken, slots, req, q_pos = 0, [], [], [0]
    for r, (n, o) in enumerate(zip(new, old)):
        for i in range(-(-o // s), -(-(o + n) // s)):
            at = free[taken] if taken < len(free) and i < table.shape[1] else -1
            if i < table.shape[1]:
                table[r, i] = at
            taken += 1
        for p in range(o, o + n):
            at = int(table[r, p // s]) if p // s < table.shape[1] else -1
            slots.append(at * s + p % s if at >= 0 else -1)
            req.append(r)
        q_pos.append(q_pos[-1] + n)
    return table, q_pos, [n + o for n, o in zip(new, old)], req, slots, taken


def check_tables(slnr, new, old, s, width, nfree, seed=0, validate=True):
    g = torch.Generator().manual_seed(seed)
    R, T = len(new), sum(new)
    table = torch.full((R, width), -1, dtype=torch.int32)
    ids = torch.randperm(R * width + nfree + 1, generator=g).to(torch.int32)
    at = 0
    for r in range(R):
        for i in range(-(-old[r] // s)):
            table[r, i] = ids[at]
            at += 1
    free = ids[at:at + nfree]
    want = plain_tables(new, old, table, free.tolist(), s)
    t, used = slnr.page_tables(i32(new), i32(old), table.cuda(), free.cuda(), s, T, validate=validate)
    assert torch.equal(t.table.cpu(), want[0])
    for got, ref in zip((t.q_pos, t.k_len, t.req, t.slots), want[1:5]):
        assert got.tolist() == list(ref)
    assert used.tolist() == [want[5]]


@pytest.mark.parametrize("s", [1, 7, 16, 64])
@pytest.mark.parametrize("new,old", [([1], [0]), ([0], [0]), ([], []), ([1, 1, 1], [15, 16, 17]), ([0, 5, 0, 0, 40, 0], [3, 0, 64, 0, 63, 1]),
                                     ([1] * 70, list(range(70))), ([300, 1, 2049], [5, 0, 100])])
def test_tables(slnr, s, new, old):
    width = max([-(-(n + o) // s) for n, o in zip(new, old)] + [1])
    check_tables(slnr, new, old, s, width, nfree=sum(-(-n // s) + 1 for n in new) + 2)


def test_tables_many_requests(slnr):
    """More requests than one scan step takes, many without a new token."""
    rng = np.random.default_rng(0)
    new = [int(x) for x in rng.integers(0, 4, 2500) * (rng.random(2500) < 0.6)]
    old = [int(x) for x in rng.integers(0, 50, 2500)]
    check_tables(slnr, new, old, 16, 4, 2500)


def test_tables_without_enough_pages(slnr):
    """Pages past the free list, or past a row of the table: -1, and nothing is written outside."""
    check_tables(slnr, [40, 3, 20], [0, 10, 5], 16, 4, nfree=3, validate=False)
    check_tables(slnr, [90, 3], [0, 10], 16, 4, nfree=30, validate=False)
    with pytest.raises(slnr.SlnrError) as e:
        check_tables(slnr, [40, 3, 20], [0, 10, 5], 16, 4, nfree=3)
    assert e.value.status == 3
    with pytest.raises(slnr.SlnrError) as e:
        check_tables(slnr, [90, 3], [0, 10], 16, 4, nfree=30)
    assert e.value.status == 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,H,D,first", [(16, 2, 64, False), (64, 3, 128, True), (7, 1, 80, False), (1, 2, 8, False),
                                            (33, 5, 40, True)])
def test_append(slnr, dtype, page, H, D, first):
    """Appended rows land in their slots, nothing else changes, and filled pages get their summary.

    The mean in fp32 is off by (page + 2) 2^-24 of the mean of |k| at most, so a code stands for the 64-bit mean within
    half a step and that."""
    b = P.Batch([(1, 1), (0, 9), (page, page), (2 * page + 3, 3 * page + 2), (5, 2 * page + 3), (1, page), (3, 700)], page, H, H, D,
                dtype, seed=page, heads_first=first)
    old_k, old_v = b.k.clone(), b.v.clone()
    slots = [int(b.table[r, p // page]) * page + p % page for r, p in zip(b.req.tolist(), b.pos.tolist())]
    new_k, new_v = (torch.randn((b.T, H, D), generator=b.g).to(dtype) for _ in range(2))
    codes = torch.full((b.npages, H, D), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((b.npages, H), 99.0, device="cuda")
    wide = torch.full((b.T, H + 2, D + 8), math.nan, dtype=dtype, device="cuda")  # keys as a slice of a wider tensor
    wide[:, 1:H + 1, :D] = new_k.cuda()
    slnr.page_append(b.cache(codes=codes, scales=scales), b.tables(slots=i32(slots)), wide[:, 1:H + 1, :D], new_v.cuda(),
                     validate=True)
    filled = set()
    for t, slot in enumerate(slots):
        old_k[slot // page, slot % page], old_v[slot // page, slot % page] = new_k[t], new_v[t]
        if slot % page == page - 1:
            filled.add(slot // page)
    for got, want in ((b.kd, old_k), (b.vd, old_v)):
        assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))
    assert filled
    for pg in range(b.npages):
        if pg not in filled:
            assert (codes[pg] == 99).all() and (scales[pg] == 99).all()
            continue
        keys = old_k[pg].double()
        mean, err = keys.mean(0), (page + 2) * 2.0 ** -24 * keys.abs().mean(0)
        most = mean.abs().amax(-1)
        scale = scales[pg].cpu().double()
        assert ((scale * 127 - most).abs() <= err.amax(-1) + 1e-6 * most).all()
        off = (codes[pg].cpu().double() * scale[:, None] - mean).abs()
        assert (off <= scale[:, None] * (0.5 + 1e-4) + err).all()


def test_append_skips_negative_slots(slnr):
    b = P.Batch([(3, 3)], 4, 1, 1, 8)
    before = b.kd.clone()
    ones = torch.ones((3, 1, 8), dtype=torch.bfloat16, device="cuda")
    slnr.page_append(b.cache(), b.tables(slots=i32([-1, -1, -1])), ones, ones)
    assert torch.equal(b.kd.view(torch.int16), before.view(torch.int16))


def test_append_zero_keys(slnr):
    """A page of zeros: scale 0, codes 0."""
    b = P.Batch([(4, 4)], 4, 2, 2, 16)
    codes, scales = torch.full((b.npages, 2, 16), 5, dtype=torch.int8, device="cuda"), torch.ones((b.npages, 2), device="cuda")
    zero = torch.zeros((4, 2, 16), dtype=torch.bfloat16, device="cuda")
    pg = int(b.table[0, 0])
    slnr.page_append(b.cache(codes=codes, scales=scales), b.tables(slots=i32([pg * 4 + i for i in range(4)])), zero, zero)
    assert (codes[pg] == 0).all() and (scales[pg] == 0).all()


def plain_select(b, codes, scales, n, first, last):
    """The definition: whole-number sums, one rounded product, the lower page where scores are equal."""
    T, H, G, s = b.T, b.H, b.Hq // b.H, b.page
    out = torch.full((T, H, n), -1, dtype=torch.int32)
    u = b.q.float().numpy().reshape(T, H, G, b.D)
    for t in range(T):
        if b.pos[t] < 0:
            continue
        own = int(b.pos[t]) // s
        at = b.table[int(b.req[t]), :own + 1].long()
        for h in range(H):
            x = u[t, h, 0].copy()
            for g in range(1, G):
                x = x + u[t, h, g]
            most = np.abs(x).max()
            c = np.rint(x * (np.float32(127) * (np.float32(1) / most))).astype(np.int64) if most > 0 else np.zeros(b.D, np.int64)
            dot = codes[at, h].numpy().astype(np.int64) @ c
            score = dot.astype(np.float32) * scales[at, h].numpy()
            must = [p for p in range(own + 1) if p < first or p > own - last]
            rest = sorted((p for p in range(own + 1) if p not in must), key=lambda p: (-score[p], p))
            pages = sorted(must + rest[:n - len(must)])
            out[t, h, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,D", [((8, 2), 128), ((4, 4), 64), ((6, 2), 80), ((16, 1), 8), ((3, 3), 120), ((2, 1), 24)])
@pytest.mark.parametrize("n,first,last", [(1, 0, 1), (4, 1, 2), (7, 3, 4), (16, 0, 1), (60, 1, 2)])
def test_select(slnr, dtype, heads, D, n, first, last):
    """Few levels of codes and scales, so that equal scores abound; zero and negative-zero scores; short and empty requests."""
    b = P.Batch([(1, 900), (3, 3), (0, 50), (5, 2), (40, 333), (1, 16), (2, 17), (1, 640)], 16, *heads, D, dtype, seed=n)
    codes = torch.randint(-2, 3, (b.npages, b.H, D), generator=b.g).to(torch.int8)
    scales = torch.randint(0, 3, (b.npages, b.H), generator=b.g).float() * 0.5
    codes[::5] = 0
    b.q[0] = 0
    got = slnr.page_select(b.q.cuda(), b.cache(codes=codes.cuda(), scales=scales.cuda()), b.tables(), n, first=first,
                           last=last, validate=True)
    assert torch.equal(got.cpu(), plain_select(b, codes, scales, n, first, last))


def test_select_all_codes(slnr):
    """Codes over their whole range, 40 query tokens of one request and long ones, no keys in the cache."""
    b = P.Batch([(40, 1500), (1, 9000), (17, 130)], 4, 12, 4, 128, seed=3)
    codes = torch.randint(-127, 128, (b.npages, 4, 128), generator=b.g).to(torch.int8)
    scales = torch.rand((b.npages, 4), generator=b.g)
    cache = slnr.PagedCache(codes=codes.cuda(), scales=scales.cuda(), page_size=4)
    got = slnr.page_select(b.q.cuda(), cache, b.tables(), 31, validate=True)
    assert torch.equal(got.cpu(), plain_select(b, codes, scales, 31, 1, 2))


@pytest.mark.parametrize("lens", [[(1, 9000), (1, 5000), (1, 30), (0, 7)], [(1, 2800), (1, 400)] * 30, [(35, 9000), (2, 600)]])
@pytest.mark.parametrize("n", [19, 20, 60, 99, 100, 300])
@pytest.mark.parametrize("levels", [2, 127])
def test_select_many(slnr, lens, n, levels):
    """Single tokens of few and of many requests, and chunks, over hundreds of pages; few and many taken, with and without
    equal scores."""
    b = P.Batch(lens, 4, 8, 4, 128, seed=n)
    codes = torch.randint(-levels, levels + 1, (b.npages, 4, 128), generator=b.g).to(torch.int8)
    scales = torch.randint(0, levels + 1, (b.npages, 4), generator=b.g).float()
    cache = slnr.PagedCache(codes=codes.cuda(), scales=scales.cuda(), page_size=4)
    got = slnr.page_select(b.q.cuda(), cache, b.tables(), n, validate=True)
    assert torch.equal(got.cpu(), plain_select(b, codes, scales, n, 1, 2))


def test_select_long_requests(slnr):
    """So many pages that a block holds two tokens' scores, and one's."""
    for n in (20000, 40000):
        b = P.Batch([(5, n), (1, 700)], 1, 2, 1, 8, seed=4)
        codes = torch.randint(-127, 128, (b.npages, 1, 8), generator=b.g).to(torch.int8)
        scales = torch.rand((b.npages, 1), generator=b.g)
        cache = slnr.PagedCache(codes=codes.cuda(), scales=scales.cuda(), page_size=1)
        got = slnr.page_select(b.q.cuda(), cache, b.tables(), 20, validate=True)
        assert torch.equal(got.cpu(), plain_select(b, codes, scales, 20, 1, 2))


def test_select_scores_that_are_not_finite(slnr):
    """Scales of NaN and infinity: no page twice, the forced ones there, nothing outside."""
    b = P.Batch([(3, 900)], 16, 2, 1, 64, seed=5)
    codes = torch.randint(-9, 10, (b.npages, 1, 64), generator=b.g).to(torch.int8)
    scales = torch.rand((b.npages, 1), generator=b.g)
    scales[::3], scales[1::7] = math.nan, math.inf
    got = slnr.page_select(b.q.cuda(), b.cache(codes=codes.cuda(), scales=scales.cuda()), b.tables(), 9).cpu()
    for t in range(3):
        own = int(b.pos[t]) // 16
        pages = [p for p in got[t, 0].tolist() if p >= 0]
        assert pages == sorted(set(pages)) and pages[0] == 0 and pages[-2:] == [own - 1, own]


def test_append_refuses_more_tokens_than_keys(slnr):
    b = P.Batch([(3, 3)], 4, 1, 1, 8)
    ones = torch.ones((3, 1, 8), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(slnr.SlnrError) as e:
        slnr.page_append(b.cache(), b.tables(slots=i32([0, 1, 2]), k_len=i32([2])), ones, ones, validate=True)
    assert e.value.status == 3


def test_tables_on_another_stream_and_in_a_wider_table(slnr):
    """A table that is a slice of a wider one, on a stream of its own."""
    wide = torch.full((2, 30), 77, dtype=torch.int32, device="cuda")
    wide[:, 4:10] = -1
    new, old, free = i32([20, 3]), i32([0, 0]), i32([5, 3, 8, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    t, used = slnr.page_tables(new, old, wide[:, 4:10], free, 16, 23, stream=side)
    side.synchronize()
    assert wide[0].tolist() == [77] * 4 + [5, 3] + [-1] * 4 + [77] * 20
    assert wide[1].tolist() == [77] * 4 + [8] + [-1] * 5 + [77] * 20
    assert t.slots.tolist() == [5 * 16 + i for i in range(16)] + [48 + i for i in range(4)] + [128, 129, 130]
    assert used.tolist() == [3]
