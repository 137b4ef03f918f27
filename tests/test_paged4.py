"""A cache in 4 bits: appends, values and attention against their definitions in 64 bits (GPU)."""
import math

import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402

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


def same(got, want):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def blocks(dtype, n, g):
    """Blocks of 16 values where a code or a scale could go wrong."""
    x = torch.randn((n, 16), generator=g) * torch.exp2(torch.randint(-20, 14, (n, 1), generator=g))
    x[0] = 0
    x[1] = 2.0 ** -24
    x[2] = torch.linspace(-1, 1, 16) * 2.0 ** -16        # scales below 2^-14
    x[3] = torch.arange(16) - 7.5                         # halves, of a scale of 1
    x[4] = (torch.arange(16) - 7.5) * 1.125               # and of one with a fraction
    x[5] = torch.where(torch.arange(16) == 3, 60000.0, 1.0)
    x[6] = torch.where(torch.arange(16) == 15, math.inf, 1.0)
    x[7] = torch.where(torch.arange(16) == 0, math.nan, -2.0)
    x[8] = -torch.finfo(dtype).max                        # bf16: past the largest value
    x[9] = torch.where(torch.arange(16) % 2 == 0, 7.0, -7.0)
    x[10] = torch.where(torch.arange(16) == 5, 0.0, -0.0)
    x[11] = torch.finfo(dtype).tiny
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D,H,page", [(32, 1, 16), (64, 3, 48), (96, 2, 16), (128, 8, 64), (128, 300, 16)])
def test_append_and_values(slnr, dtype, D, H, page):
    """Slots in any order, written twice, skipped; pages that no slot names keep their bytes."""
    g = torch.Generator().manual_seed(D + H)
    npages, T = 5, 2 * page + 7
    data = torch.randint(0, 256, (npages, H, page // 16, 18 * D), generator=g, dtype=torch.uint8).cuda()
    before, cache = data.clone(), slnr.PagedCache4(data)
    slots = torch.randperm(3 * page, generator=g)[:T].to(torch.int32)  # pages 0 .. 2
    slots[5] = -1
    slots[6] = npages * page  # past the last page
    k, v = (torch.cat([blocks(dtype, T * H * D // 16, g)]).reshape(T, H, D) for _ in range(2))
    tables = slnr.PageTables(table=P.i32([[0, 1, 2]]), q_pos=P.i32([0, T]), k_len=P.i32([T]), req=P.i32([0] * T),
                             slots=slots.cuda(), max_q=T, max_k=T)
    for _ in range(2):
        slnr.page_append(cache, tables, k.cuda(), v.cuda())
    assert torch.equal(data[3:], before[3:])
    got_k, got_v = slnr.page_values(cache, dtype=dtype)
    assert got_k.shape == (npages, page, H, D) and got_k.dtype == dtype
    on = (slots >= 0) & (slots < npages * page)
    at = slots[on].long()
    for got, x in ((got_k, k), (got_v, v)):
        same(got.reshape(-1, H, D).cpu()[at], P.held(x[on]))
    # what was not written stands for what it did
    other = torch.ones(npages * page, dtype=torch.bool)
    other[at] = False
    kept = slnr.page_values(slnr.PagedCache4(before), dtype=dtype)
    for got, old in zip((got_k, got_v), kept):
        a, b = (y.reshape(-1, H, D).cpu()[other] for y in (got, old))
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_every_largest_value(slnr, dtype):
    """Each finite number as the largest of a block, beside halves of its scale's steps and numbers next to them."""
    g = torch.Generator().manual_seed(2)
    m = torch.arange(0, 0x7f80 if dtype == BF16 else 0x7c00, dtype=torch.int16).view(dtype)
    step = P.held(torch.cat([m[:, None]] + [torch.zeros_like(m)[:, None]] * 15, 1))[:, :1] / 7  # the scale, or less of a step
    n = torch.randint(-7, 7, (len(m), 14), generator=g).double() + 0.5
    rest = (n * step).clamp(-m[:, None].double(), m[:, None].double()).to(dtype)
    rest[:, ::3] = (rest[:, ::3].view(torch.int16) + 1).view(dtype)
    rest = torch.where(rest.double().abs() <= m[:, None].double(), rest, torch.zeros_like(rest))
    x = torch.cat([m[:, None], rest, -m[:, None]], dim=1)
    page, H, D = 64, 2, 64
    per = H * D // 16
    T = -(-len(m) // per)
    x = torch.cat([x, torch.zeros((T * per - len(m), 16), dtype=dtype)]).reshape(T, H, D)
    npages = -(-T // page)
    k = torch.zeros((npages * page, H, D), dtype=dtype)
    k[:T] = x
    k = k.reshape(npages, page, H, D)
    cache = P.written(slnr, k, -k, torch.arange(npages, dtype=torch.int32)[None], [T], npages, page, H, D)
    for got, want in zip(slnr.page_values(cache, dtype=dtype), (x, -x)):
        same(got.reshape(-1, H, D)[:T], P.held(want))
    off = (P.held(x) - x.double()).abs().reshape(-1, 16)[:len(m)]
    scale = P.SCALES[P.np.searchsorted(P.SCALES * 7.5, m.double().numpy().clip(max=7.5 * P.MOST))]
    ordinary = m.double() <= 7.5 * P.MOST
    assert (off[ordinary] <= torch.from_numpy(scale)[ordinary][:, None] / 2).all()  # as the format promises


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_values_of_some_pages(slnr, dtype):
    """Pages in any order, twice, and entries that are none; the values are exact in both types."""
    g = torch.Generator().manual_seed(3)
    page, H, D = 32, 2, 64
    k, v = (torch.randn((4, page, H, D), generator=g).to(FP16) for _ in range(2))
    cache = P.written(slnr, k, v, torch.arange(4, dtype=torch.int32)[None], [4 * page], 4, page, H, D)
    at = P.i32([2, -1, 0, 2, 4])
    out = tuple(torch.full((5, page, H, D), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    got = slnr.page_values(cache, at, dtype=dtype, out=out)
    assert got[0] is out[0] and got[1] is out[1]
    for y, x in zip(got, (k, v)):
        want = P.held(x)
        same(y, torch.stack([want[2], 0 * want[0], want[0], want[2], 0 * want[0]]))
    assert slnr.page_values(cache, at[:0], dtype=dtype)[0].shape == (0, page, H, D)


def test_appended_rows_of_other_strides(slnr):
    g = torch.Generator().manual_seed(4)
    T, H, D, page = 19, 2, 96, 16
    wide = torch.randn((T, 3 * H, D + 8), generator=g).to(BF16).cuda()
    k, v = wide[:, :H, :D], wide[:, 2 * H:, 8:]
    whole = torch.full((7, 4, H, 2, 18 * D), 0x55, dtype=torch.uint8, device="cuda")
    cache = slnr.PagedCache4(whole[::2, 1, :, 1:])  # every second page, a slice of a wider one
    assert cache.page_size == page
    tables = slnr.PageTables(table=P.i32([[3, 1]]), q_pos=P.i32([0, T]), k_len=P.i32([T]), req=P.i32([0] * T),
                             slots=P.i32([3 * page + i if i < page else page + i - page for i in range(T)]), max_q=T, max_k=T)
    slnr.page_append(cache, tables, k, v, validate=True)
    for got, x in zip(slnr.page_values(cache, dtype=FP16), (k, v)):
        want = P.held(x.cpu())
        same(got[3], want[:page])
        same(got[1, :3], want[page:])
    rest = whole.clone()
    rest[::2, 1, :, 1:] = 0x55
    assert (rest == 0x55).all()


# (new tokens, keys): one token; none; fewer keys than tokens (the first tokens see nothing); no keys at all
EDGES = [(1, 1), (0, 40), (3, 3), (5, 2), (2, 0), (1, 130), (7, 63), (0, 0), (1, 64), (4, 65)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (6, 2), (16, 1)])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 32), (32, 48), (96, 16)])
def test_edges(slnr, dtype, heads, D, page):
    b = P.Batch4(slnr, EDGES, page, *heads, D, dtype, seed=D + page)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(D ** -0.5))


@pytest.mark.parametrize("lens", [[(1, 5000)], [(1, 5000), (1, 77), (1, 2049), (1, 0)], [(2, 3001), (1, 9)],
                                  [(9, 2500), (1, 1)], [(40, 1500)], [(70, 70), (3, 400), (1, 1)], [(129, 700), (130, 131)],
                                  [(300, 300)], [(257, 1000), (1, 3000)], [(1, 1)] * 700])
@pytest.mark.parametrize("heads,D,page,first", [((4, 1), 128, 16, False), ((8, 4), 64, 48, True), ((3, 3), 128, 64, True),
                                                ((4, 2), 96, 32, False), ((5, 1), 32, 16, True)])
def test_lengths(slnr, lens, heads, D, page, first):
    """Single tokens over many shares, short chunks, chunks: every row tile, and requests of different kinds together."""
    b = P.Batch4(slnr, lens, page, *heads, D, seed=len(lens), heads_first=first)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(D ** -0.5))


@pytest.mark.parametrize("heads", [(4, 2), (24, 1)])
def test_few_of_many_requests_have_tokens(slnr, heads):
    """Long runs of requests without new tokens, at the ends too, before and behind long and short ones."""
    g = torch.Generator().manual_seed(12)
    lens = [(0, int(torch.randint(0, 40, (1,), generator=g))) for _ in range(1500)]
    for r, n in ((31, 900), (32, 17), (64, 1), (500, 3000), (501, 0), (1130, 64), (1467, 333)):
        lens[r] = (1, n)
    b = P.Batch4(slnr, lens, 16, *heads, 64, seed=13)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(0.125))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads", [(7, 1), (12, 1), (32, 1), (33, 1), (64, 2), (512, 1)])
def test_many_query_heads(slnr, dtype, heads):
    """Row tiles of 8, 16 and 32, and the tensor-core kernel, by the number of rows alone."""
    b = P.Batch4(slnr, [(1, 333), (1, 16), (1, 17), (1, 0)], 16, *heads, 128, dtype, seed=heads[0])
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(128 ** -0.5))


@pytest.mark.parametrize("tokens", [3, 90])
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
def test_scales(slnr, scale, tokens):
    b = P.Batch4(slnr, [(tokens, 200), (1, 900)], 16, 4, 2, 64, FP16, seed=5)
    b.q = (b.q.float() * 0.25).to(FP16)  # keeps the scores' own error (which grows with the scale) below the tolerance
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=scale), b.attention(scale))


@pytest.mark.parametrize("tokens", [1, 200])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_cache_of_the_other_type(slnr, dtype, tokens):
    """Keys written in one type, queries of the other."""
    other = FP16 if dtype == BF16 else BF16
    b = P.Batch4(slnr, [(tokens, 300)], 16, 4, 1, 128, other, seed=6)
    b.dtype, b.q = dtype, b.q.to(dtype)
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables())
    assert got[0].dtype == dtype
    b.check(got, b.attention(128 ** -0.5))


@pytest.mark.parametrize("power", [-120, -40, 40, 120])
def test_queries_of_any_size(slnr, power):
    """bf16 queries far outside of fp16's range, the scale such that the scores are ordinary."""
    b = P.Batch4(slnr, [(2, 300)], 16, 4, 1, 128, BF16, seed=7)
    ref = b.attention(128 ** -0.5)
    b.q = (b.q.float() * 2.0 ** power).to(BF16)  # exact
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=128 ** -0.5 * 2.0 ** -power), ref)


@pytest.mark.parametrize("tokens", [1, 100])
def test_bad_pages_and_other_bounds(slnr, tokens):
    """Bounds wider than the batch; tables that are slices of wider ones."""
    b = P.Batch4(slnr, [(tokens, 500), (3, 20)], 16, 4, 2, 64, width=200, seed=10)
    ref = b.attention(0.125)
    wide = torch.full((2, 300), 7, dtype=torch.int32, device="cuda")
    wide[:, 5:205] = b.table.cuda()
    for max_q, max_k in ((tokens, 500), (tokens, 3200), (9 + tokens, 500), (200, 3200)):
        t = b.tables(max_q=max(max_q, 3), max_k=max_k, table=wide[:, 5:205])
        b.check(slnr.paged_attention(b.q.cuda(), b.cache(), t), ref, f"{max_q} {max_k}")


@pytest.mark.parametrize("tokens", [1, 100])
def test_values_that_are_not_finite(slnr, tokens):
    """A value of NaN reaches the rows of its request that see it, and no other request."""
    b = P.Batch4(slnr, [(tokens, 200), (tokens, 200)], 16, 2, 1, 64, seed=11)
    k, v = (torch.randn((b.npages, 16, 1, 64)).to(BF16) for _ in range(2))
    v[b.table[0, 3].long(), 5, 0, 17] = math.inf
    c = P.written(slnr, k, v, b.table, [200, 200], b.npages, 16, 1, 64)
    out, lse = slnr.paged_attention(b.q.cuda(), c, b.tables())
    assert torch.isnan(out[:tokens, :, 16:32]).all() and torch.isfinite(out[tokens:]).all() and torch.isfinite(lse).all()


def test_offsets_past_32_bits(slnr):
    """Pages 2^30 bytes apart."""
    b = P.Batch4(slnr, [(1, 60), (70, 90)], 16, 4, 2, 64, seed=9)
    stride = 1 << 30
    buf = torch.empty((b.npages - 1) * stride + (1 << 16), dtype=torch.uint8, device="cuda")
    assert buf.numel() > 1 << 33
    data = buf.as_strided((b.npages, 2, 1, 18 * 64), (stride, 18 * 64, 18 * 64, 1))
    data.copy_(b.c4.data)
    b.check(slnr.paged_attention(b.q.cuda(), slnr.PagedCache4(data), b.tables()), b.attention(0.125))
    other = slnr.PagedCache4.empty(b.npages, 16, 2, 64)
    i = torch.arange(b.npages, dtype=torch.int32, device="cuda")
    slnr.page_copy(other, i, i, source=slnr.PagedCache4(data))
    assert torch.equal(other.data, b.c4.data)
