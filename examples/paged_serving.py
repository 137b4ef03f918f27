"""Serving a few requests over a paged key/value cache: one attention layer.

Each step gives every request its next tokens (a chunk of its prompt while that is
read, then one token at a time): pages and slots from the lengths, the new keys and
values into the cache, and attention over all pages, or over the pages that the cheap
score picks.  Queries, keys and values are random projections of random tokens.

    python examples/paged_serving.py [--picked 4] [--steps 12]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2205_11622_gb300 as slnr  # noqa: E402


class Layer:
    """One attention layer's cache, shared by its requests."""

    def __init__(self, npages, page_size, heads_q, heads, width, max_keys, requests, dtype=torch.bfloat16, device="cuda"):
        shape = (npages, page_size, heads, width)
        self.cache = slnr.PagedCache(
            k=torch.zeros(shape, dtype=dtype, device=device), v=torch.zeros(shape, dtype=dtype, device=device),
            codes=torch.zeros((npages, heads, width), dtype=torch.int8, device=device),
            scales=torch.zeros((npages, heads), device=device))
        self.page_size = page_size
        self.table = torch.full((requests, -(-max_keys // page_size)), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(npages, dtype=torch.int32, device=device)
        self.lens = [0] * requests
        self.device = device

    def step(self, new, q, k, v, picked=0):
        """Attention of `new` tokens of each request (packed in q, k, v): over all pages, or `picked` of each token."""
        i32 = dict(dtype=torch.int32, device=self.device)
        taken = sum(-(-(o + n) // self.page_size) - -(-o // self.page_size) for o, n in zip(self.lens, new))
        # The bounds on new tokens and keys lay out the work: near the truth, and whole pages, so that the sizes of a call
        # change once a page.  A step that is captured for replay takes the most keys it will ever have.
        most = max(o + n for o, n in zip(self.lens, new))
        tables, _ = slnr.page_tables(torch.tensor(new, **i32), torch.tensor(self.lens, **i32), self.table, self.free,
                                     self.page_size, sum(new), max_q=max(new),
                                     max_k=-(-most // self.page_size) * self.page_size)
        self.free = self.free[taken:]
        self.lens = [o + n for o, n in zip(self.lens, new)]
        slnr.page_append(self.cache, tables, k, v)
        if picked:
            pages = slnr.page_select(q, self.cache, tables, picked)
            return slnr.selected_attention(q, self.cache, tables, pages)[0]
        return slnr.paged_attention(q, self.cache, tables)[0]


def serve(prompts=(300, 37, 1000), chunk=256, steps=12, heads_q=8, heads=2, width=128, page_size=64, picked=0, seed=0):
    """Reads the prompts in chunks, then takes `steps` tokens of each; returns what each step was given and gave."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    max_keys = max(prompts) + steps
    npages = sum(-(-(p + steps) // page_size) for p in prompts)
    layer = Layer(npages, page_size, heads_q, heads, width, max_keys, len(prompts))
    left, record = list(prompts), []
    while any(left) or steps:
        new = [min(chunk, n) for n in left] if any(left) else [1] * len(prompts)
        if not any(left):
            steps -= 1
        left = [max(0, n - chunk) for n in left]
        rnd = lambda h: torch.randn((sum(new), h, width), generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        q, k, v = rnd(heads_q), rnd(heads), rnd(heads)
        record.append((new, q, k, v, layer.step(new, q, k, v, picked)))
    return record


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--picked", type=int, default=0, help="pages picked for each token (0: attention over all pages)")
    p.add_argument("--steps", type=int, default=12, help="tokens after the prompts")
    a = p.parse_args()
    slnr.build()
    record = serve(picked=a.picked, steps=a.steps)
    torch.cuda.synchronize()
    for i, (new, _, _, _, out) in enumerate(record):
        print(f"step {i}: {new} new tokens, output {tuple(out.shape)}, root mean square {float(out.float().square().mean().sqrt()):.4f}")


if __name__ == "__main__":
    main()
