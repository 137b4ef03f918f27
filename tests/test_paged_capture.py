"""Captured calls of attention over a paged cache beside calls that the same stream makes later, and threads that share one (GPU)."""
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


def captured(slnr, b, stream, q, **kw):
    """(graph, outputs) of one call with the queries in q, captured on a stream that made it once before."""
    cache, tables = b.cache(), b.tables()
    with torch.cuda.stream(stream):
        slnr.paged_attention(q, cache, tables, **kw)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = slnr.paged_attention(q, cache, tables, **kw)
    return graph, got, (cache, tables)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("lens", [[(1, 9000)], [(90, 700)]])  # splits joined through the workspace; the tensor-core kernel
def test_a_larger_call_after_the_capture(slnr, lens, own):
    """What a captured call writes beside its outputs is not memory that others were given since."""
    b, larger = P.Batch(lens, 16, 4, 2, 64, seed=60), P.Batch([(1, 9000)] * 40 + [(300, 900)], 16, 4, 2, 64, seed=61)
    side, q, ref = torch.cuda.Stream(), torch.zeros_like(b.q).cuda(), b.attention(0.125)
    ws = dict(workspace=slnr.Workspace()) if own else {}
    torch.cuda.synchronize()
    graph, got, keep = captured(slnr, b, side, q, **ws)
    args = (larger.q.cuda(), larger.cache(), larger.tables())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        slnr.paged_attention(*args, **ws)
        q.copy_(b.q)
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in
                  [1 << k for k in range(9, 27)] * 2 + [3 << k for k in range(9, 24)]]
        for _ in range(3):
            graph.replay()
    side.synchronize()
    b.check(got, ref)
    assert all((x == 7).all() for x in others)


def test_graphs_of_one_stream_replayed_on_two(slnr):
    """Each captured call has what it writes to itself."""
    batches = [P.Batch([(1, 9000), (1, 4000 + 70 * i)], 16, 8, 2, 64, seed=62 + i) for i in range(2)]
    side = torch.cuda.Stream()
    qs = [b.q.cuda() for b in batches]
    torch.cuda.synchronize()
    made = [captured(slnr, b, side, q) for b, q in zip(batches, qs)]
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(50):
        for (graph, _, _), s in zip(made, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for b, (_, got, _) in zip(batches, made):
        b.check(got, b.attention(0.125))


def test_threads_that_share_a_stream(slnr):
    """Calls of several launches from several threads, all on the current stream and its workspace."""
    import threading
    batches = [P.Batch(lens, 16, 4, 2, 64, seed=70 + i) for i, lens in
               enumerate([[(100, 700)], [(1, 9000)], [(300, 310), (2, 50)], [(90, 2000)]])]
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


@pytest.mark.parametrize("lens", [[(1, 9000)], [(90, 700)]])
def test_a_captured_stream_that_is_given(slnr, lens):
    """The call's stream joins the capture of another that is current; a larger call on it later."""
    b, larger = P.Batch(lens, 16, 4, 2, 64, seed=66), P.Batch([(1, 9000)] * 40 + [(300, 900)], 16, 4, 2, 64, seed=67)
    main, side, q, ref = torch.cuda.Stream(), torch.cuda.Stream(), torch.zeros_like(b.q).cuda(), b.attention(0.125)
    cache, tables = b.cache(), b.tables()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    args = (larger.q.cuda(), larger.cache(), larger.tables())
    torch.cuda.synchronize()
    slnr.paged_attention(q, cache, tables, out=out, lse=lse, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        slnr.paged_attention(q, cache, tables, out=out, lse=lse, stream=side)
        main.wait_stream(side)
    slnr.paged_attention(*args, stream=side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in [1 << k for k in range(9, 27)] * 2]
    torch.cuda.synchronize()
    q.copy_(b.q)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    b.check((out, lse), ref)
    assert all((x == 7).all() for x in others)
