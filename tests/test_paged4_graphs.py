"""Calls over a 4-bit cache and over whole pages on other streams, in graphs, from threads, and whose waits give up (GPU)."""
import ctypes
import threading

import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402
from _paged4 import i32  # noqa: E402

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


# the row kernel with items that shares cut, one of 32 rows, the tensor-core kernel
KINDS = [[(1, 9000), (1, 33)], [(8, 3000)], [(90, 700), (1, 50)]]


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("lens", KINDS)
def test_a_larger_call_after_the_capture(slnr, lens, own):
    """What a captured call writes beside its outputs is not memory that others were given since."""
    b = P.Batch4(slnr, lens, 16, 4, 1, 64, seed=60)
    larger = P.Batch4(slnr, [(1, 3000)] * 40 + [(300, 900)], 16, 8, 2, 128, seed=61)
    side, q, ref = torch.cuda.Stream(), torch.zeros_like(b.q).cuda(), b.attention(0.125)
    ws = dict(workspace=slnr.Workspace()) if own else {}
    cache, tables = b.cache(), b.tables()
    args = (larger.q.cuda(), larger.cache(), larger.tables())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        slnr.paged_attention(q, cache, tables, **ws)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = slnr.paged_attention(q, cache, tables, **ws)
        slnr.paged_attention(*args, **ws)
        q.copy_(b.q)
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in [1 << k for k in range(9, 26)] * 2]
        for _ in range(3):
            graph.replay()
    side.synchronize()
    b.check(got, ref)
    assert all((x == 7).all() for x in others)


def test_graphs_of_one_stream_replayed_on_two(slnr):
    batches = [P.Batch4(slnr, [(1, 9000), (1, 4000 + 70 * i)], 16, 8, 2, 64, seed=62 + i) for i in range(2)]
    side = torch.cuda.Stream()
    made = []
    for b in batches:
        q, cache, tables = b.q.cuda(), b.cache(), b.tables()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            slnr.paged_attention(q, cache, tables)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                made.append((graph, slnr.paged_attention(q, cache, tables), q, cache, tables))
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(50):
        for (graph, *_), s in zip(made, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for b, (_, got, *_) in zip(batches, made):
        b.check(got, b.attention(0.125))


def test_threads_that_share_a_stream(slnr):
    batches = [P.Batch4(slnr, lens, 16, 4, 2, 64, seed=70 + i) for i, lens in
               enumerate([[(100, 700)], [(1, 9000)], [(300, 310), (2, 50)], [(8, 2000)]])]
    on_gpu = [(b.q.cuda(), b.cache(), b.tables()) for b in batches]
    torch.cuda.synchronize()
    got = [[] for _ in batches]

    def work(i):
        for _ in range(20):
            got[i].append(slnr.paged_attention(*on_gpu[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(batches))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for b, results in zip(batches, got):
        ref = b.attention(0.125)
        assert len(results) == 20
        for r in results:
            b.check(r, ref)


def test_a_step_in_a_graph(slnr):
    """Fork, copy, append, attention, compaction and the free list, captured once and replayed on other contents."""
    page, H, D, width, npages, R = 16, 2, 64, 6, 60, 3
    g = torch.Generator().manual_seed(5)
    c4 = slnr.PagedCache4.empty(npages, page, H, D)
    table = torch.randperm(40, generator=g)[:R * width].reshape(R, width).to(torch.int32).cuda()
    lens, parent, one = i32([40, 5, 64]), i32([2, 0, 0, 1]), i32([1] * 4)
    kv = torch.randn((npages, page, 2, H, D), generator=g).to(BF16).cuda()
    every = torch.arange(npages, dtype=torch.int32, device="cuda")[:, None]
    i = torch.arange(npages * page, dtype=torch.int32, device="cuda")
    whole = slnr.PageTables(table=every, q_pos=i32([*range(0, npages * page + 1, page)]), k_len=torch.full_like(i[:npages], page),
                            req=i // page, slots=i, max_q=page, max_k=page)
    new = torch.randn((4, 2, H, D), generator=g).to(BF16).cuda()
    q = torch.randn((4, 2 * H, D), generator=g).to(BF16).cuda()

    def step():
        slnr.page_append(c4, whole, kv[:, :, 0].reshape(-1, H, D), kv[:, :, 1].reshape(-1, H, D))
        free, _ = slnr.page_free(table, lens, npages, page)
        t2, l2, src, dst, _ = slnr.page_fork(table, lens, parent, free, page)
        slnr.page_copy(c4, src, dst)
        free2, _ = slnr.page_free(t2, l2, npages, page)
        t, _ = slnr.page_tables(one, l2, t2, free2, page, 4, max_q=1)
        slnr.page_append(c4, t, new[:, 0], new[:, 1])
        before = slnr.paged_attention(q, c4, t)
        t3, src, dst, ids, used = slnr.page_compact(t2, t.k_len, npages, page)
        slnr.page_copy(c4, src, dst)
        after = slnr.paged_attention(q, c4, slnr.PageTables(table=t3, q_pos=t.q_pos, k_len=t.k_len, req=t.req, slots=None, max_q=1,
                                                            max_k=width * page))
        return before, after, t3, used

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            before, after, t3, used = step()
    results = []
    for lengths, parents in (([40, 5, 64], [2, 0, 0, 1]), ([1, 79, 33], [1, 1, 1, 2]), ([16, 0, 95], [0, 2, 2, 1])):
        lens.copy_(i32(lengths))
        parent.copy_(i32(parents))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])  # the same keys in the same order
        pages = [-(-(lengths[p] + 1) // page) for p in parents]
        assert int(t3.max()) < used.item() <= sum(pages) and (t3 >= 0).sum(1).tolist() == pages
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(want[0][0], before[0]) and torch.equal(want[2], t3)
        results.append(before[0].clone())
        # child n sees its parent's keys and its own
        held = [P.held(x.cpu()) for x in (kv[:, :, 0], kv[:, :, 1], new[:, 0], new[:, 1])]
        for n, p in enumerate(parents):
            j = torch.arange(lengths[p])
            at = table.cpu()[p, j // page].long(), j % page
            k, v = (torch.cat([held[e][at], held[2 + e][n:n + 1]]) for e in range(2))
            for h in range(2 * H):
                w = torch.softmax(k[:, h // 2] @ q[n, h].cpu().double() * D ** -0.5, 0)
                err = (before[0][n, h].cpu().double() - w @ v[:, h // 2]).abs()
                assert (err <= 2.5 * 2.0 ** -8 * (w @ v[:, h // 2].abs()) + 2.0 ** -30).all()
    assert not torch.equal(results[0], results[1])


def test_calls_on_a_stream_that_is_given(slnr):
    """Inputs that are dropped while the call is pending there are not given to others before."""
    b = P.Batch4(slnr, [(1, 9000), (1, 700)], 16, 4, 2, 64, seed=8)
    ref, side = b.attention(0.125), torch.cuda.Stream()
    busy = torch.randn((6000, 6000), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(6):
            busy = busy @ busy
    got = slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), stream=side)
    lens, table = i32([40, 3]), torch.arange(8, dtype=torch.int32, device="cuda").reshape(2, 4)
    free = slnr.page_free(table, lens, 10, 16, drop=i32([1]), stream=side)
    values = slnr.page_values(b.cache(), torch.arange(3, dtype=torch.int32, device="cuda"), stream=side)
    junk = [torch.full((n,), 1, dtype=torch.int32, device="cuda") for n in [1 << k for k in range(2, 20)] * 3]
    side.synchronize()
    b.check(got, ref)
    assert free[0].tolist() == [3, 4, 5, 6, 7, 8, 9, -1, -1, -1] and free[1].item() == 7 and lens.tolist() == [40, 0]
    want = slnr.page_values(b.cache())
    assert all(torch.equal(x.view(torch.int16), y[:3].view(torch.int16)) for x, y in zip(values, want))
    del junk


@pytest.mark.parametrize("lens,heads", [([(1, 9000), (1, 700)], (4, 2)), ([(6, 4000)], (4, 1)), ([(1, 20000)] * 6, (2, 2)),
                                        ([(200, 1500)], (4, 2)), ([(100, 1500), (20, 20)], (4, 2)),
                                        ([(90, 90), (300, 700)], (4, 2))])
def test_rows_whose_waits_gave_up(slnr, lens, heads):
    """NaN or right, never what the output's memory held; limits from none to more than a step takes.  Where a warp has one or
    two units its copies may have landed before it looks: then nothing gives up, whatever the limit."""
    b = P.Batch4(slnr, lens, 16, *heads, 64, seed=90)
    ref = b.attention(0.125)
    out, lse = torch.empty_like(b.q, device="cuda"), torch.empty(b.q.shape[:2], device="cuda")
    args = (b.q.cuda(), b.cache(), b.tables())
    lib = slnr.lib()
    gave_up, others = 0, torch.empty(400 << 20, dtype=torch.uint8, device="cuda")
    for limit in (1, 100, 1000, 3000, 10000, 30000, 100000, 0):
        out.fill_(7)
        lse.fill_(7)
        others.zero_()  # the cache comes from memory, not from L2
        assert lib.slnr_set_wait_limit(ctypes.c_int64(limit)) == 0
        try:
            slnr.paged_attention(*args, out=out, lse=lse)
            flags = slnr.device_flags()
            try:
                b.check(slnr.paged_attention(*args, validate=True), ref, f"limit {limit}, validated")
            except slnr.SlnrError as e:
                assert "SLNR_ERR_TIMEOUT" in str(e) and limit
        finally:
            assert lib.slnr_set_wait_limit(ctypes.c_int64(0)) == 0
        bad = torch.isnan(lse).cpu()
        assert torch.equal(torch.isnan(out).all(-1).cpu(), bad) and torch.equal(torch.isnan(out).any(-1).cpu(), bad)
        assert not bad.any() or flags & 16, limit
        gave_up += int(bad.sum())
        good = ~bad
        b.check((out.cpu()[good], lse.cpu()[good]), tuple(x[good] for x in ref), f"limit {limit}")
    assert (gave_up > 0 or max(n for n, _ in lens) < 10 and lens[0][1] < 20000) and not bad.any() and flags == 0


@pytest.mark.parametrize("lens", [[(1, 9000), (1, 3)], [(8, 3000)], [(90, 700), (1, 50)], [(300, 2000)]])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_no_wait_runs_out_unseen(slnr, lens, D):
    """Right results alone do not show a wait that gave up where nothing depended on it: it takes two seconds."""
    b = P.Batch4(slnr, lens, 16, 4, 1, D, seed=83)
    args = (b.q.cuda(), b.cache(), b.tables())
    slnr.paged_attention(*args)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    start.record()
    for _ in range(3):
        slnr.paged_attention(*args)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 500


def test_no_flag_on_memory_that_held_others(slnr):
    for lens in ([(1, 40)], [(0, 5), (1, 700)], [(1, 9000), (8, 3)], [(100, 300)]):
        b, ws = P.Batch4(slnr, lens, 16, 4, 1, 64, seed=80), slnr.Workspace()
        ws.get(64 << 20).fill_(255)
        slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), workspace=ws)
        assert slnr.device_flags() == 0 and slnr.device_flags(ws) == 0
    none = P.Batch4(slnr, [(0, 50), (0, 0)], 16, 4, 1, 64, seed=81)
    out, lse = slnr.paged_attention(none.q.cuda(), none.cache(), none.tables(), validate=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_validation(slnr):
    """Malformed tables, slots and lists are errors in validate mode."""
    b = P.Batch4(slnr, [(1, 40), (3, 9)], 16, 4, 2, 64, seed=82)
    q, c, x = b.q.cuda(), b.cache(), torch.zeros((4, 2, 64), dtype=BF16, device="cuda")
    bad_table = b.table.clone()
    bad_table[0, 1] = b.npages
    slots = i32([0, 1, 2, 3])
    for call in (lambda: slnr.paged_attention(q, c, b.tables(table=bad_table.cuda()), validate=True),
                 lambda: slnr.paged_attention(q, c, b.tables(k_len=i32([400, 9])), validate=True),
                 lambda: slnr.page_append(c, b.tables(slots=i32([0, 1, -1, 3])), x, x, validate=True),
                 lambda: slnr.page_append(c, b.tables(slots=i32([0, 1, b.npages * 16, 3])), x, x, validate=True),
                 lambda: slnr.page_values(c, i32([0, b.npages]), validate=True),
                 lambda: slnr.page_copy(c, i32([0, b.npages]), i32([1, 2]), validate=True),
                 lambda: slnr.page_copy(c, i32([0]), i32([b.npages]), validate=True),
                 lambda: slnr.page_fork(b.table.cuda(), i32([40, 9]), i32([0, 2]), i32([]), 16, validate=True),
                 lambda: slnr.page_fork(b.table.cuda(), i32([-1, 9]), i32([0]), i32([]), 16, validate=True),
                 lambda: slnr.page_free(b.table.cuda(), i32([40, 9]), b.npages, 16, drop=i32([2]), validate=True),
                 lambda: slnr.page_compact(bad_table.cuda(), i32([40, 9]), b.npages, 16, validate=True)):
        with pytest.raises(slnr.SlnrError, match="SLNR_ERR_INDEX"):
            call()
    slnr.page_append(c, b.tables(slots=slots), x, x, validate=True)
    slnr.page_values(c, i32([0, -1]), validate=True)
    slnr.page_copy(c, i32([0, -1]), i32([1, 2]), validate=True)
    slnr.page_fork(b.table.cuda(), i32([40, 9]), i32([0, -1, 1]), i32([]), 16, validate=True)
