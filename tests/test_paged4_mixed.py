"""Many single tokens over long contexts beside a chunk of a prompt, over a cache in 4 bits (GPU)."""
import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slnr():
    import paper_2205_11622_gb300 as m
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    m.build()
    m.lib()
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,D,page,chunk", [((8, 2), 128, 16, (150, 1201)), ((4, 4), 64, 32, (9, 777)), ((12, 1), 96, 16, (300, 300))])
def test_single_tokens_beside_a_chunk(slnr, dtype, heads, D, page, chunk):
    g = torch.Generator().manual_seed(D)
    lens = [(1, int(n)) for n in torch.randint(200, 4000, (70,), generator=g)]
    lens[33] = chunk
    lens[34] = (0, 900)
    b = P.Batch4(slnr, lens, page, *heads, D, dtype, seed=D + page)
    ref = b.attention(D ** -0.5)
    b.check(slnr.paged_attention(b.q.cuda(), b.cache(), b.tables(), validate=True), ref)
    # the same tokens in two calls, each with the bounds of its own
    alone = [r for r, (n, _) in enumerate(lens) if n == 1]
    t = slnr.PageTables(table=b.table[alone].cuda(), q_pos=P.i32(list(range(len(alone) + 1))), k_len=b.k_len[alone].cuda(),
                        req=P.i32(list(range(len(alone)))), slots=None, max_q=1, max_k=b.max_k)
    at = b.q_pos[:-1][alone].long()
    out, lse = slnr.paged_attention(b.q[at].cuda(), b.cache(), t)
    every, every_lse = (x.clone() for x in ref[:2])
    every[at], every_lse[at] = out.double().cpu(), lse.double().cpu()
    b.check((every, every_lse), ref)
