"""Attention over a paged cache against its definition in 64 bits (GPU): all pages and picked ones."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")

import _paged as P  # noqa: E402

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


# (new tokens, keys): one token; none; fewer keys than tokens (the first tokens see nothing); no keys at all
EDGES = [(1, 1), (0, 40), (3, 3), (5, 2), (2, 0), (1, 130), (7, 63), (0, 0), (1, 64), (4, 65)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (6, 2), (16, 1)])
@pytest.mark.parametrize("D,page", [(128, 16), (64, 32), (80, 7), (8, 1), (40, 64), (96, 130)])
def test_edges(slnr, dtype, heads, D, page):
    b = P.Batch(EDGES, page, *heads, D, dtype, seed=D + page)
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True)
    b.check(got, b.attention(D ** -0.5))


@pytest.mark.parametrize("lens", [[(1, 5000)], [(1, 5000), (1, 77), (1, 2049), (1, 0)], [(2, 3001), (1, 9)],
                                  [(9, 2500), (1, 1)], [(40, 1500)], [(70, 70), (3, 400), (1, 1)], [(129, 700), (130, 131)],
                                  [(300, 300)], [(257, 1000), (1, 3000)]])
@pytest.mark.parametrize("heads,D,page,first", [((4, 1), 128, 16, False), ((8, 4), 64, 48, True), ((3, 3), 128, 64, True)])
def test_lengths(slnr, lens, heads, D, page, first):
    """Single tokens over many splits, short chunks, chunks: every row tile, and requests of different kinds together."""
    b = P.Batch(lens, page, *heads, D, seed=len(lens), heads_first=first)
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True)
    b.check(got, b.attention(D ** -0.5))


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
def test_scales(slnr, scale):
    """Any finite scale; with a large one a single key takes all the weight."""
    b = P.Batch([(3, 200), (1, 900)], 16, 4, 2, 64, FP16, seed=5)
    b.q = (b.q.float() * 0.25).to(FP16)  # keeps the scores' own error (which grows with the scale) below the tolerance
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=scale)
    b.check(got, b.attention(scale))


def test_large_scores(slnr):
    """Scores of some hundreds, rising and falling along the keys: the running maximum rescales what was summed."""
    for lens in ([(1, 700)], [(200, 700)]):
        b = P.Batch(lens, 16, 4, 1, 64, BF16, seed=6)
        ramp = torch.linspace(-30, 30, b.npages).roll(3)[:, None, None, None]
        b.k = torch.where(torch.isnan(b.k), b.k, ramp.to(BF16).expand_as(b.k))
        b.q = torch.ones_like(b.q)
        b.kd = b.k.cuda()
        got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=0.125)
        b.check(got, b.attention(0.125))


def test_lowest_values(slnr):
    """Keys at the type's lowest finite value: scores of -1e38 and below are finite or -inf, never NaN beside a finite one."""
    b = P.Batch([(1, 40)], 16, 2, 1, 64, BF16, seed=7)
    low = torch.finfo(BF16).min
    at = b.table[0, :3].long()
    b.k[at] = torch.where(torch.isnan(b.k[at]), b.k[at], torch.zeros_like(b.k[at]))
    b.k[at[1], 3, 0] = low / 64
    b.q = torch.full_like(b.q, 0.5)
    b.kd = b.k.cuda()
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables())
    b.check(got, b.attention(64 ** -0.5))


def test_inputs_of_other_strides(slnr):
    """Queries as a slice of a wider projection, a table that is a slice of a wider one, every second page of a cache."""
    b = P.Batch([(2, 300), (1, 41)], 16, 8, 2, 64, seed=8)
    wide = torch.full((b.T, 8 + 4, 64 + 8), math.nan, dtype=BF16, device="cuda")
    wide[:, 2:10, :64] = b.q.cuda()
    table = torch.full((2, 64), 7, dtype=torch.int32, device="cuda")
    table[:, 5:5 + b.width] = b.table.cuda()
    kv = torch.full((2 * b.npages, 16, 2, 2, 64), math.nan, dtype=BF16, device="cuda")
    kv[::2, :, :, 0], kv[::2, :, :, 1] = b.kd, b.vd
    cache = slnr.PagedCache(k=kv[::2, :, :, 0], v=kv[::2, :, :, 1])
    out = torch.empty((b.T, 8, 64), dtype=BF16, device="cuda")
    lse = torch.empty((b.T, 8), device="cuda")
    got = slnr.paged_attention(wide[:, 2:10, :64], cache, b.tables(table=table[:, 5:5 + b.width]), out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    b.check(got, b.attention(0.125))


def test_offsets_past_32_bits(slnr):
    """Pages 2^27 values apart: the last ones lie past 2^32 values (and 2^33 bytes) into the cache."""
    b = P.Batch([(1, 600), (70, 90)], 16, 4, 2, 64, seed=9)
    stride = 1 << 27
    buf = torch.empty((b.npages - 1) * stride + (1 << 16), dtype=BF16, device="cuda")
    assert buf.numel() > 1 << 32
    view = lambda o: buf.as_strided((b.npages, 16, 2, 64), (stride, 128, 64, 1), o)  # noqa: E731
    k, v = view(0), view(1 << 15)
    k.copy_(b.kd)
    v.copy_(b.vd)
    b.check(slnr.paged_attention(b.q.cuda(), slnr.PagedCache(k=k, v=v), b.tables()), b.attention(0.125))


def test_bounds_wider_than_the_batch(slnr):
    """max_q and max_k are bounds: larger ones change the split of the work, not the result's meaning."""
    b = P.Batch([(1, 500), (3, 20)], 16, 4, 2, 64, width=200, seed=10)
    ref = b.attention(0.125)
    for max_q, max_k in itertools.product((3, 9, 100), (500, 3200)):
        b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(max_q=max_q, max_k=max_k)), ref, f"{max_q} {max_k}")


@pytest.mark.parametrize("lens,heads", [([(9, 500), (1, 20)], (8, 2)), ([(33, 70), (0, 3), (40, 12), (64, 1030)], (2, 2)),
                                        ([(5, 4000), (7, 3)], (8, 1))])
@pytest.mark.parametrize("D", [64, 128])
def test_short_chunks_of_many_keys(slnr, lens, heads, D):
    """33 to 64 rows a request: the bound on the keys decides which kernel takes them."""
    b = P.Batch(lens, 16, *heads, D, width=(1 << 19) // 16 // heads[1] // len(lens) + 1, seed=D + len(lens))
    ref = b.attention(D ** -0.5)
    for max_k in (4000, 16 * b.width - 16, 16 * b.width):
        b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(max_k=max_k)), ref, f"{max_k}")


@pytest.mark.parametrize("lens", [[(1, 3000)], [(300, 900)]])
def test_same_call_same_bits(slnr, lens):
    b = P.Batch(lens, 16, 8, 2, 128, seed=11)
    args = (b.q.cuda(), b.cache(), b.tables())
    one, two = slnr.paged_attention(*args), slnr.paged_attention(*args)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_other_stream(slnr):
    """On a stream that is given, and on one that is current; each waits for nothing but what its caller ordered."""
    b = P.Batch([(1, 3000), (5, 70)], 16, 8, 2, 64, seed=12)
    ref, cache, tables, q = b.attention(0.125), b.cache(), b.tables(), b.q.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = slnr.paged_attention(q, cache, tables, stream=side)
    with torch.cuda.stream(side):
        also = slnr.paged_attention(q, cache, tables)
    side.synchronize()
    b.check(got, ref)
    b.check(also, ref)


def test_graph(slnr):
    """A captured call, replayed on new inputs in the same tensors."""
    b = P.Batch([(1, 3000), (1, 70)], 16, 8, 2, 64, seed=13)
    cache, tables, q = b.cache(), b.tables(), torch.zeros_like(b.q).cuda()
    slnr.paged_attention(q, cache, tables)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = slnr.paged_attention(q, cache, tables)
    q.copy_(b.q)
    graph.replay()
    torch.cuda.synchronize()
    b.check(got, b.attention(0.125))


def test_nothing_to_do(slnr):
    b = P.Batch([(0, 10), (0, 0)], 16, 4, 2, 64)
    out, lse = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables())
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    b = P.Batch([], 16, 4, 2, 64)
    out, lse = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables())
    assert out.shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (6, 2), (40, 1)])
@pytest.mark.parametrize("D,page,n", [(128, 16, 9), (64, 64, 4), (80, 7, 5), (8, 1, 33)])
def test_selected(slnr, dtype, heads, D, page, n):
    b = P.Batch([(1, 700), (0, 5), (3, 3), (5, 2), (9, 400), (2, 0), (1, 1)], page, *heads, D, dtype, seed=D + n)
    picked = P.picks(b, n, seed=n)
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
    b.check(got, b.attention(D ** -0.5, picked))


def test_selected_many_pages(slnr):
    """More picked pages than one block takes: splits joined, empty ones among them."""
    b = P.Batch([(1, 5000), (2, 5000)], 16, 8, 2, 128, seed=21)
    for n in (1, 100, 300):
        picked = P.picks(b, n, seed=n)
        picked[0, 0] = -1
        got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
        b.check(got, b.attention(128 ** -0.5, picked), f"{n} pages")


@pytest.mark.parametrize("heads,D,page", [((8, 2), 128, 64), ((4, 4), 64, 16), ((16, 1), 96, 32), ((6, 2), 64, 48)])
def test_selected_chunk(slnr, heads, D, page):
    """A chunk of tokens whose picks overlap, beside single tokens."""
    b = P.Batch([(150, 1200), (1, 300), (60, 60)], page, *heads, D, seed=22)
    picked = P.picks(b, 6, seed=23)
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
    b.check(got, b.attention(D ** -0.5, picked))


def test_selected_pages_past_the_token(slnr):
    """Picked pages that begin after the token hold nothing that it sees."""
    b = P.Batch([(4, 64)], 16, 2, 1, 64, seed=24)
    b.lens, b.k_len = [(4, 64)], torch.tensor([64], dtype=torch.int32)
    picked = torch.tensor([[[1, 3]], [[3, -1]], [[-1, -1]], [[0, 3]]], dtype=torch.int32)
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda())
    b.check(got, b.attention(0.125, picked))


def test_all_pages_picked_is_paged_attention(slnr):
    b = P.Batch([(5, 200), (1, 17)], 16, 4, 2, 64, seed=25)
    picked = torch.arange(b.width, dtype=torch.int32).expand(b.T, 2, b.width).clone()
    picked[picked > (b.pos // 16)[:, None, None]] = -1
    b.check(slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda()), b.attention(0.125))


def test_many_requests(slnr):
    """More requests, row tiles and items than one step of the plan takes; a chunk among single tokens."""
    lens = [(1, 1 + r % 19) for r in range(1300)] + [(0, 4)] * 40 + [(70, 90)] + [(1, 300)] * 3
    b = P.Batch(lens, 16, 2, 2, 16, seed=26)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(0.25))


@pytest.mark.parametrize("page", [16, 128, 256])
def test_selected_chunk_many_pages(slnr, page):
    """Pages far into a long request: the list of picked pages is made in several windows."""
    b = P.Batch([(20, 20000 if page == 16 else 9000), (3, 500)], page, 4, 1, 16, seed=27)
    picked = P.picks(b, 5, seed=28)
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
    b.check(got, b.attention(0.25, picked))


def test_selected_chunk_nothing_picked(slnr):
    """Row tiles whose tokens picked no page at all, beside others."""
    b = P.Batch([(64, 200), (64, 64)], 64, 4, 1, 64, seed=29)
    picked = torch.full((b.T, 1, 3), -1, dtype=torch.int32)
    picked[70:, 0, 1] = 0
    got = slnr.selected_attention(b.q.cuda(), b.cache(), b.tables(), picked.cuda(), validate=True)
    b.check(got, b.attention(0.125, picked))


def test_chunk_with_fewer_keys_than_tokens(slnr):
    """The first tokens of a chunk see nothing; a chunk without any key."""
    b = P.Batch([(200, 150), (90, 0), (80, 80)], 16, 4, 2, 64, seed=30)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), b.attention(0.125))


@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_chunk_scales(slnr, scale):
    b = P.Batch([(70, 400)], 16, 2, 1, 64, FP16, seed=31)
    b.q = (b.q.float() * 0.25).to(FP16)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), scale=scale), b.attention(scale))


def test_out_of_any_alignment(slnr):
    """An output on a 16-byte boundary that is none of 32, and widths whose rows are not whole sectors."""
    for D in (64, 40, 8):
        b = P.Batch([(90, 300)], 16, 2, 1, D, seed=D)
        room = torch.zeros(b.T * 2 * D + 8, dtype=BF16, device="cuda")
        out = room[8:].view(b.T, 2, D)
        got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), out=out)
        b.check(got, b.attention(D ** -0.5))
        assert (room[:8] == 0).all()


@pytest.mark.parametrize("selected", [False, True])
def test_chunk_graph_and_stream(slnr, selected):
    """The launches of a chunk, which wait for one another on the device, captured and replayed on another stream."""
    b = P.Batch([(100, 700), (1, 90)], 64, 4, 2, 64, seed=32)
    picked = P.picks(b, 4, seed=33)
    cache, tables, q, pd = b.cache(), b.tables(), torch.zeros_like(b.q).cuda(), picked.cuda()
    call = (lambda: slnr.selected_attention(q, cache, tables, pd)) if selected else \
        (lambda: slnr.paged_attention(q, cache, tables))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = call()
        q.copy_(b.q)
        for _ in range(3):
            graph.replay()
    side.synchronize()
    b.check(got, b.attention(0.125, picked if selected else None))


@pytest.mark.parametrize("selected", [False, True])
def test_calls_after_one_another_share_a_workspace(slnr, selected):
    """Calls of different sizes back to back on one workspace: none sees what another left there."""
    batches = [P.Batch(lens, 64, 4, 2, 64, seed=40 + i) for i, lens in
               enumerate([[(100, 700)], [(1, 3000)], [(300, 310), (2, 50)], [(70, 2000)], [(1, 5)], [(90, 90)]])]
    ws = slnr.Workspace()
    picked = [P.picks(b, 4, seed=50 + i) for i, b in enumerate(batches)]
    on_gpu = [(b.q.cuda(), b.cache(), b.tables(), p.cuda()) for b, p in zip(batches, picked)]
    torch.cuda.synchronize()
    got = [slnr.selected_attention(q, c, t, p, workspace=ws) if selected else slnr.paged_attention(q, c, t, workspace=ws)
           for _ in range(2) for q, c, t, p in on_gpu]
    for i, b in enumerate(batches):
        ref = b.attention(0.125, picked[i] if selected else None)
        b.check(got[i], ref, f"call {i}")
        b.check(got[i + len(batches)], ref, f"call {i} again")


def test_short_wait_limit_reports_timeout(slnr):
    """The tensor-core kernel's bounded waits: with a limit far below a step's time a validated call returns
    SLNR_ERR_TIMEOUT, and the next call with the default limit is right."""
    import ctypes
    b = P.Batch([(200, 1500)], 16, 4, 1, 64, seed=34)
    args, ref = (b.q.cuda(), b.cache(), b.tables()), b.attention(0.125)
    lib = slnr.lib()
    assert lib.slnr_set_wait_limit(ctypes.c_int64(100)) == 0
    try:
        with pytest.raises(slnr.SlnrError) as e:
            slnr.paged_attention(*args, validate=True)
        assert e.value.status == 7, str(e.value)
        assert slnr.device_flags() & 16
    finally:
        assert lib.slnr_set_wait_limit(ctypes.c_int64(0)) == 0
    b.check(slnr.paged_attention(*args, validate=True), ref)
    assert slnr.device_flags() == 0


def test_malformed_tables_are_reported(slnr):
    """Validate mode: a page outside the cache, too many keys, positions that do not add up, picked pages out of order."""
    b = P.Batch([(2, 100), (1, 30)], 16, 2, 1, 64, seed=35)
    q, cache = b.q.cuda(), b.cache()

    def refused(picked=None, **kw):
        with pytest.raises(slnr.SlnrError) as e:
            if picked is None:
                slnr.paged_attention(q, cache, b.tables(**kw), validate=True)
            else:
                slnr.selected_attention(q, cache, b.tables(**kw), picked, validate=True)
        assert e.value.status == 3, str(e.value)

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in (-1, b.npages):
        table = b.table.clone()
        table[1, 1] = bad
        refused(table=table.cuda())
    refused(k_len=i32([100, 113]))
    refused(k_len=i32([100, -1]))
    refused(q_pos=i32([0, 1, 2]))
    refused(q_pos=i32([1, 2, 3]))
    refused(q_pos=i32([0, 4, 3]))
    refused(req=i32([0, 1, 1]))
    refused(max_q=1)
    refused(picked=i32([[[3, 2]], [[0, 1]], [[0, 1]]]))
    refused(picked=i32([[[1, 1]], [[0, 1]], [[0, 1]]]))
    refused(picked=i32([[[0, 99]], [[0, 1]], [[0, 1]]]))


def test_wrapper_refusals(slnr):
    b = P.Batch([(2, 40)], 16, 4, 2, 64, seed=36)
    q, cache, tables = b.q.cuda(), b.cache(), b.tables()
    for bad in (b.q, q.half(), q.float(), q[:1], q[:, :, :32], q.transpose(1, 2), q[:, :3]):
        with pytest.raises((ValueError, slnr.SlnrError)):
            slnr.paged_attention(bad, cache, tables)
    with pytest.raises(ValueError):
        slnr.paged_attention(q, cache, tables, out=torch.empty_like(q).half())
    with pytest.raises(ValueError):
        slnr.paged_attention(q, cache, tables, lse=torch.empty((2, 4), device="cuda", dtype=torch.float64))
    with pytest.raises(ValueError):
        slnr.selected_attention(q, cache, tables, torch.zeros((2, 2, 3), device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError):
        slnr.selected_attention(q, cache, tables, torch.zeros((2, 2, 0), device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        slnr.page_select(q, cache, tables, 4)  # no summaries
    with pytest.raises(ValueError):
        slnr.page_append(cache, tables, b.k[0], b.v[0])  # no slots
    with pytest.raises(ValueError):
        b.tables(q_pos=b.q_pos.long().cuda())
    with pytest.raises(ValueError):
        b.tables(table=b.table.cuda().t())
    with pytest.raises(slnr.SlnrError) as e:
        slnr.paged_attention(q, cache, b.tables(max_k=49))
    assert e.value.status == 2
    with pytest.raises(ValueError):
        slnr.PagedCache(k=b.kd, v=b.vd.transpose(1, 3))


def test_no_room_for_keys(slnr):
    """A table without columns: no request has a key."""
    b = P.Batch([(3, 0), (1, 0)], 16, 4, 2, 64, seed=37)
    for q in (1, 100):
        t = b.tables(table=torch.empty((2, 0), dtype=torch.int32, device="cuda"), max_q=max(3, q), max_k=0)
        out, lse = slnr.paged_attention(b.q.cuda(), b.cache(), t)
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("lens", [[(1, 700), (2, 5)], [(100, 300)]])
def test_without_lse(slnr, lens):
    """The C entry point with no place for lse."""
    import ctypes
    from paper_2205_11622_gb300 import slnr_opts, slnr_rows
    b = P.Batch(lens, 16, 4, 2, 64, seed=38)
    cache, tables, q, lib, r = b.cache(), b.tables(), b.q.cuda(), slnr.lib(), ctypes.byref
    out, ref = torch.zeros_like(q), b.attention(0.125)
    o, need = slnr_opts(), ctypes.c_size_t()
    assert lib.slnr_paged_attention_workspace(r(cache._c), r(tables._c), 4, r(o), r(need)) == 0
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    o.workspace, o.workspace_bytes, o.stream = ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream
    rows = slnr_rows(q.data_ptr(), q.stride(0), q.stride(1))
    assert lib.slnr_paged_attention(r(rows), 4, r(cache._c), r(tables._c), 0.125, out.data_ptr(), None, r(o)) == 0
    b.check((out, ref[1].float()), ref)
    o.workspace_bytes = need.value - 256
    assert lib.slnr_paged_attention(r(rows), 4, r(cache._c), r(tables._c), 0.125, out.data_ptr(), None, r(o)) == 4
