"""The beam example's steps against attention over what each beam has seen so far, in 64 bits (GPU)."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")

import _paged4 as P  # noqa: E402

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def search():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2205_11622_gb300 as slnr
    slnr.build()
    import paged_beams
    return paged_beams.search


@pytest.mark.parametrize("bits,page,heads,width", [(4, 16, (8, 2), 128), (4, 32, (4, 4), 64), (16, 16, (8, 2), 128)])
def test_beams(search, bits, page, heads, width):
    prompts, beams, steps = (130, 37, 64), 4, 12
    pool, record = search(prompts, beams, steps, *heads, width, page, bits, every=5)
    of = (lambda x: P.held(x.cpu())) if bits == 4 else (lambda x: x.cpu().double())
    seen = [torch.empty((2, 0, heads[1], width), dtype=torch.float64) for _ in prompts]
    for new, q, k, v, out, parents in record:
        kv, at, q, out = torch.stack([of(k), of(v)]), 0, q.cpu().double(), out.cpu().double()
        for r, n in enumerate(new):
            seen[r] = torch.cat([seen[r], kv[:, at:at + n]], dim=1)
            total = seen[r].shape[1]
            hidden = torch.arange(total) > torch.arange(total - n, total)[:, None]
            for h in range(heads[0]):
                key, value = seen[r][:, :, h // (heads[0] // heads[1])]
                w = torch.softmax((q[at:at + n, h] @ key.T * width ** -0.5).masked_fill(hidden, -math.inf), -1)
                # two roundings to bf16 (2^-8 each) and half of one for the scores; small weights: see _paged4.py
                tol = 2.5 * 2.0 ** -8 * (w @ value.abs()) + total * 2.0 ** -37 * value.abs().max()
                assert ((out[at:at + n, h] - w @ value).abs() <= tol).all(), (r, h)
            at += n
        seen = [seen[p] for p in parents.tolist()]
    assert pool.lens.tolist() == [s.shape[1] for s in seen]
    used = pool.pack()
    held = torch.unique(pool.table[pool.table >= 0])
    assert held.tolist() == list(range(used.item()))
    # beams share what they have in common: fewer pages than they would have alone
    assert used.item() < sum(-(-s.shape[1] // page) for s in seen)
    free = pool.free(torch.arange(len(seen), dtype=torch.int32, device="cuda"))
    assert free.tolist() == list(range(pool.npages)) and pool.lens.tolist() == [0] * len(seen)
