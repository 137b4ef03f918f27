"""The serving example's steps against attention over each request's tokens so far, in 64 bits (GPU)."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

HEADS_Q, HEADS, WIDTH, PAGE = 8, 2, 128, 64


@pytest.fixture(scope="module")
def serve():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2205_11622_gb300 as slnr
    slnr.build()
    import paged_serving
    return paged_serving.serve


def check(record, prompts, pages_of=None):
    """Every step's output; pages_of: the pages that a token at a position may see (None: all)."""
    keys = [torch.empty((0, HEADS, WIDTH), dtype=torch.float64, device="cuda") for _ in prompts]
    values = [k.clone() for k in keys]
    for new, q, k, v, out in record:
        at = 0
        for r, n in enumerate(new):
            keys[r] = torch.cat([keys[r], k[at:at + n].double()])
            values[r] = torch.cat([values[r], v[at:at + n].double()])
            pos = torch.arange(len(keys[r]) - n, len(keys[r]), device="cuda")[:, None]
            seen = torch.arange(len(keys[r]), device="cuda") <= pos
            for h in range(HEADS_Q):
                g = h // (HEADS_Q // HEADS)
                s = (q[at:at + n, h].double() @ keys[r][:, g].T * WIDTH ** -0.5).masked_fill(~seen, -math.inf)
                w = torch.softmax(s, -1)
                want, mag = w @ values[r][:, g], w @ values[r][:, g].abs()
                # two roundings to bf16 (2^-8 each) and half of one for the scores: see _paged.py
                assert ((out[at:at + n, h].double() - want).abs() <= 2.5 * 2.0 ** -8 * mag).all(), (r, h)
            at += n


def test_all_pages(serve):
    prompts = (300, 37, 700)
    record = serve(prompts=prompts, chunk=256, steps=5, heads_q=HEADS_Q, heads=HEADS, width=WIDTH, page_size=PAGE)
    assert [r[0] for r in record] == [[256, 37, 256], [44, 0, 256], [0, 0, 188]] + [[1, 1, 1]] * 5
    check(record, prompts)


def test_enough_picked_pages_are_all_pages(serve):
    prompts = (130, 300)
    check(serve(prompts=prompts, chunk=100, steps=3, heads_q=HEADS_Q, heads=HEADS, width=WIDTH, page_size=PAGE, picked=5),
          prompts)


def test_few_picked_pages(serve):
    """Finite, and not what all pages give."""
    args = dict(prompts=(900,), chunk=300, steps=3, heads_q=HEADS_Q, heads=HEADS, width=WIDTH, page_size=PAGE)
    few, every = serve(picked=4, **args)[-1], serve(**args)[-1]
    assert torch.equal(few[1], every[1]) and torch.isfinite(few[4].float()).all()
    assert (few[4] != every[4]).any()
