"""Copies, forks, free pages and compaction against plain loops (GPU)."""
import random

import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402
from _paged4 import i32  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


def some_tables(rng, R, width, page, npages):
    """Tables of random lengths (some 0) over random pages; every third request shares its first pages with another."""
    lens = [min(rng.choice((0, 1, page, width * page, rng.randrange(width * page + 1))), width * page) for _ in range(R)]
    ids = list(range(npages))
    rng.shuffle(ids)
    table = [[rng.randrange(npages) for _ in range(width)] for _ in range(R)]  # entries past the lengths: any page
    for r in range(R):
        for i in range(-(-lens[r] // page)):
            if not ids:
                lens[r] = i * page
                break
            table[r][i] = ids.pop()
        if r % 3 == 2:
            n = min(lens[r], lens[r - 1]) // page // 2
            table[r][:n] = table[r - 1][:n]
    return lens, table, ids


def held(lens, table, page):
    return {table[r][i] for r in range(len(lens)) for i in range(-(-lens[r] // page))}


# requests, columns, page size, pages
SIZES = [(1, 1, 1, 1), (1, 0, 16, 3), (3, 4, 16, 40), (7, 300, 5, 3001), (65, 33, 64, 2500), (700, 9, 16, 7000),
         (2, 2000, 16, 100_000), (40, 600, 128, 600_001), (30, 100, 16, 1_100_003)]


@pytest.mark.parametrize("R,width,page,npages", SIZES)
@pytest.mark.parametrize("dropped", [None, 0, 1, 5])
def test_free(slnr, R, width, page, npages, dropped):
    rng = random.Random(R + npages)
    lens, table, _ = some_tables(rng, R, width, page, npages)
    drop = None if dropped is None else [rng.randrange(R) for _ in range(dropped)]  # the same one twice, too
    t = torch.full((R, width + 3), -5, dtype=torch.int32, device="cuda")
    t[:, 1:width + 1] = i32(table).reshape(R, width)
    at = i32(lens)
    free, count = slnr.page_free(t[:, 1:width + 1], at, npages, page, drop=None if drop is None else i32(drop), validate=True)
    for r in drop or ():
        lens[r] = 0
    assert at.tolist() == lens
    used = held(lens, table, page)
    want = [p for p in range(npages) if p not in used]
    assert count.item() == len(want)
    assert free.tolist() == want + [-1] * (npages - len(want))


def test_free_skips_what_is_none(slnr):
    """Entries and requests that are none are skipped; a length past a row's end is the row's."""
    table = i32([[3, -1, 9, 2], [5, 6, 7, 1], [4, 4, 4, 4]])
    lens = i32([60, 1000, -7])
    free, count = slnr.page_free(table, lens, 8, 16, drop=i32([-1, 3, 2 ** 31 - 1]))
    assert lens.tolist() == [60, 1000, -7] and free.tolist() == [0, 4, -1, -1, -1, -1, -1, -1] and count.item() == 2
    free, count = slnr.page_free(table, lens, 0, 16)
    assert free.numel() == 0 and count.item() == 0
    free, count = slnr.page_free(table[:0], lens[:0], 3, 16)
    assert free.tolist() == [0, 1, 2] and count.item() == 3
    with pytest.raises(slnr.SlnrError, match="SLNR_ERR_INDEX"):
        slnr.page_free(table, lens, 8, 16, validate=True)


@pytest.mark.parametrize("R,width,page,npages", SIZES)
def test_compact(slnr, R, width, page, npages):
    rng = random.Random(R * npages)
    lens, table, _ = some_tables(rng, R, width, page, npages)
    new, src, dst, ids, used = slnr.page_compact(i32(table).reshape(R, width), i32(lens), npages, page, validate=True)
    have = held(lens, table, page)
    U = len(have)
    movers = [p for p in sorted(have) if p >= U]
    holes = [p for p in range(U) if p not in have]
    assert len(movers) == len(holes) and used.item() == U
    pad = [-1] * (npages // 2 - len(movers))
    assert src.tolist() == movers + pad and dst.tolist() == holes + pad
    to = {p: p for p in have if p < U} | dict(zip(movers, holes))
    assert ids.tolist() == [to.get(p, -1) for p in range(npages)]
    want = [[to[table[r][i]] if i < -(-lens[r] // page) else -1 for i in range(width)] for r in range(R)]
    assert new.tolist() == want


@pytest.mark.parametrize("share", [0.0, 1.0])
def test_compact_of_none_and_of_all(slnr, share):
    n = 1000
    lens = i32([int(n * share) * 4])
    table = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None]
    new, src, dst, ids, used = slnr.page_compact(table, lens, n, 4)
    assert used.item() == n * share and (src == -1).all() and (dst == -1).all()
    assert torch.equal(new, table if share else torch.full_like(table, -1))
    assert ids.tolist() == (list(range(n)) if share else [-1] * n)


@pytest.mark.parametrize("R,width,page,npages", SIZES)
@pytest.mark.parametrize("n", [0, 1, 17, 1500])
@pytest.mark.parametrize("nfree", [0, 3, 3000])
def test_fork(slnr, R, width, page, npages, n, nfree):
    rng = random.Random(R + n + nfree)
    lens, table, _ = some_tables(rng, R, width, page, npages)
    parent = [rng.randrange(-1, R + 1) for _ in range(n)]
    free = [rng.randrange(npages) for _ in range(nfree)]
    new, new_lens, src, dst, used = slnr.page_fork(i32(table).reshape(R, width), i32(lens), i32(parent), i32(free), page)
    at, seen = 0, set()
    want, want_lens, want_src, want_dst = [], [], [], []
    for p in parent:
        have = 0 <= p < R
        L = lens[p] if have else 0
        need = -(-L // page)
        row = [table[p][i] if i < need else -1 for i in range(width)] if have else [-1] * width
        s = d = -1
        if have and L % page and p in seen:
            d = free[at] if at < nfree else -1
            s = row[need - 1] if d >= 0 else -1
            row[need - 1] = d
            at += 1
        seen.add(p)
        want.append(row)
        want_lens.append(L)
        want_src.append(s)
        want_dst.append(d)
    assert new.shape == (n, width) and new.tolist() == want and new_lens.tolist() == want_lens
    assert src.tolist() == want_src and dst.tolist() == want_dst and used.item() == at


def test_fork_of_many(slnr):
    """As many children as a call takes, of few and of many parents."""
    for R in (1, 3, 50_000):
        n, page = 65536, 4
        parent = torch.randint(0, R, (n,), generator=torch.Generator().manual_seed(R), dtype=torch.int32)
        table = torch.arange(2 * R, dtype=torch.int32).reshape(R, 2)
        free = torch.arange(n, dtype=torch.int32) + 1_000_000
        new, lens, src, dst, used = slnr.page_fork(table.cuda(), torch.full((R,), 6, dtype=torch.int32, device="cuda"),
                                                   parent.cuda(), free.cuda(), page)
        first = torch.full((R,), n).scatter_reduce_(0, parent.long(), torch.arange(n), "amin")
        copied = first[parent.long()] != torch.arange(n)
        want = torch.where(copied, 1_000_000 + torch.cumsum(copied, 0) - 1, -1)
        assert torch.equal(dst.cpu().long(), want) and used.item() == int(copied.sum())
        assert torch.equal(src.cpu(), torch.where(copied, table[parent.long(), 1], -1))
        assert torch.equal(new[:, 0].cpu(), table[parent.long(), 0])
        assert torch.equal(new[:, 1].cpu().long(), torch.where(copied, want, table[parent.long(), 1].long()))


def caches(slnr, kind, npages, page, H, D, dtype, g):
    """A cache of random contents, and its tensors."""
    if kind == "4 bits":
        x = torch.randint(0, 256, (npages, H, page // 16, 18 * D), generator=g, dtype=torch.uint8).cuda()
        return slnr.PagedCache4(x), [x]
    rnd = lambda *s: torch.randn(s, generator=g).to(dtype).cuda()  # noqa: E731
    if kind == "heads first":
        k, v = (rnd(npages, H, page, D).transpose(1, 2) for _ in range(2))
    elif kind == "apart":  # every second page, wider rows, k and v in one tensor
        kv = rnd(2 * npages, page, 2, H, D + 8)
        k, v = kv[::2, :, 0, :, :D], kv[::2, :, 1, :, 8:]
    else:
        k, v = rnd(npages, page, H, D), rnd(npages, page, H, D)
    codes = torch.randint(-127, 128, (npages, H, D), generator=g, dtype=torch.int8).cuda()
    scales = torch.rand((npages, H), generator=g).cuda()
    if kind == "summary":
        return slnr.PagedCache(codes=codes, scales=scales, page_size=page), [codes, scales]
    if kind == "no summary":
        return slnr.PagedCache(k=k, v=v), [k, v]
    return slnr.PagedCache(k=k, v=v, codes=codes, scales=scales), [k, v, codes, scales]


KINDS = ("packed", "heads first", "apart", "summary", "no summary", "4 bits")


@pytest.mark.parametrize("page,H,D", [(16, 1, 32), (7, 3, 8), (48, 8, 96), (64, 5, 128), (33, 2, 40)])
@pytest.mark.parametrize("kind", KINDS)
def test_copy(slnr, kind, page, H, D):
    if kind == "4 bits" and (page % 16 or D % 32):
        page, D = 32, 64
    g = torch.Generator().manual_seed(page + H)
    npages = 50
    cache, tensors = caches(slnr, kind, npages, page, H, D, FP16 if D == 96 else BF16, g)
    ids = torch.randperm(npages, generator=g).to(torch.int32)
    src, dst = ids[:20].clone(), ids[20:40].clone()
    src[3], dst[4] = -1, -1
    src[5], dst[6] = npages, npages + 7
    want = [x.clone() for x in tensors]
    on = (src >= 0) & (dst >= 0) & (src < npages) & (dst < npages)
    for w in want:
        w[dst[on].long().cuda()] = w[src[on].long().cuda()]
    slnr.page_copy(cache, src.cuda(), dst.cuda())
    for x, w in zip(tensors, want):
        assert torch.equal(x, w)
    # lists of which most say nothing
    long = torch.full((30_000,), -1, dtype=torch.int32)
    long_dst = long.clone()
    long[29_999], long_dst[29_999], long[100], long_dst[100] = int(ids[45]), int(ids[44]), int(ids[45]), int(ids[46])
    slnr.page_copy(cache, long.cuda(), long_dst.cuda(), validate=True)
    for x, w in zip(tensors, want):
        w[int(ids[44])] = w[int(ids[46])] = w[int(ids[45])]
        assert torch.equal(x, w)


def test_copy_between_caches(slnr):
    """Pages of a cache of one order to one of another; summaries go along where both have them."""
    g = torch.Generator().manual_seed(1)
    for a, b in (("packed", "heads first"), ("apart", "packed"), ("heads first", "no summary"), ("summary", "summary"),
                 ("4 bits", "4 bits")):
        (to, x), (source, y) = (caches(slnr, kind, n, 16, 3, 64, BF16, g) for kind, n in ((a, 9), (b, 30)))
        src, dst = [29, 0, 7], [2, 8, 0]
        slnr.page_copy(to, i32(src), i32(dst), source=source, validate=True)
        for p, q in zip(x, y):
            assert torch.equal(p[dst], q[src])


def test_a_pool_that_lives_long(slnr):
    """Requests come, grow, fork, end and are packed, over both kinds of caches of one table: what attention sees stays what
    was appended."""
    rng, g = random.Random(7), torch.Generator().manual_seed(7)
    page, H, D, npages, width = 16, 2, 64, 200, 12
    c16 = slnr.PagedCache(k=torch.zeros((npages, page, H, D), dtype=BF16, device="cuda"),
                          v=torch.zeros((npages, page, H, D), dtype=BF16, device="cuda"))
    c4 = slnr.PagedCache4.empty(npages, page, H, D)
    R = 6
    table, lens = torch.full((R, width), -1, dtype=torch.int32, device="cuda"), i32([0] * R)
    said = [torch.empty((0, 2, H, D), dtype=BF16) for _ in range(R)]
    free, _ = slnr.page_free(table, lens, npages, page)
    for step in range(25):
        new = [rng.choice((0, 1, 1, 5, 20)) if len(s) < width * page - 20 else 0 for s in said]
        T = sum(new)
        t, used = slnr.page_tables(i32(new), lens, table, free, page, T)
        kv = torch.randn((T, 2, H, D), generator=g).to(BF16)
        for c in (c16, c4):
            slnr.page_append(c, t, kv[:, 0].cuda(), kv[:, 1].cuda(), validate=T > 0)
        lens, at = t.k_len.clone(), 0
        for r, n in enumerate(new):
            said[r] = torch.cat([said[r], kv[at:at + n]])
            at += n
        free, count = slnr.page_free(table, lens, npages, page)
        if step % 3 == 1:  # beams: some go on twice, some end
            parent = [rng.randrange(R) for _ in range(R)]
            table, lens, src, dst, _ = slnr.page_fork(table, lens, i32(parent), free, page, validate=True)
            for c in (c16, c4):
                slnr.page_copy(c, src, dst, validate=True)
            said = [said[p] for p in parent]
        if step % 4 == 2:
            r = rng.randrange(R)
            slnr.page_free(table, lens, npages, page, drop=i32([r]))
            said[r] = said[r][:0]
        if step % 5 == 3:
            table, src, dst, ids, used = slnr.page_compact(table, lens, npages, page, validate=True)
            for c in (c16, c4):
                slnr.page_copy(c, src, dst, validate=True)
            assert int(table.max()) < used.item()
        free, count = slnr.page_free(table, lens, npages, page)
        assert lens.tolist() == [len(s) for s in said]
        at = table.cpu()
        k4, v4 = (x.cpu().double() for x in slnr.page_values(c4))
        for r, s in enumerate(said):
            j = torch.arange(len(s))
            where = at[r, j // page].long(), j % page
            assert torch.equal(c16.k.cpu()[where], s[:, 0]) and torch.equal(c16.v.cpu()[where], s[:, 1])
            assert torch.equal(k4[where], P.held(s[:, 0])) and torch.equal(v4[where], P.held(s[:, 1]))
