"""Several beams for each prompt over a paged key/value cache held in 4 bits: one attention layer.

Each prompt is read at once, then its beams go on from it: they share its full pages.  Every step takes one token of each
beam and keeps the beams that go on, some of them twice, in the place of others.  Pages that no beam holds any more are
taken again; now and then all pages are packed to the front of the cache, so that the rest of it could be given back.
Queries, keys and values are random, and so is the choice of beams.

    python examples/paged_beams.py [--beams 4] [--steps 24] [--bits 4]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2205_11622_gb300 as slnr  # noqa: E402


class Pool:
    """One attention layer's cache, and the block tables of the requests that share its pages."""

    def __init__(self, npages, page_size, heads, width, max_keys, requests, bits=4, dtype=torch.bfloat16, device="cuda"):
        if bits == 4:
            self.cache = slnr.PagedCache4.empty(npages, page_size, heads, width, device=device)
        else:
            shape = (npages, page_size, heads, width)
            self.cache = slnr.PagedCache(k=torch.zeros(shape, dtype=dtype, device=device),
                                         v=torch.zeros(shape, dtype=dtype, device=device))
        i32 = dict(dtype=torch.int32, device=device)
        self.npages, self.page_size = npages, page_size
        self.table = torch.full((requests, -(-max_keys // page_size)), -1, **i32)
        self.lens = torch.zeros(requests, **i32)
        self.most = 0  # keys of the longest request, on the host: the work of a step is laid out by it

    def free(self, drop=None):
        """The pages that no request holds, without the requests in drop."""
        return slnr.page_free(self.table, self.lens, self.npages, self.page_size, drop=drop)[0]

    def step(self, new, q, k, v):
        """Attention of `new` tokens of each request (packed in q, k, v)."""
        self.most += max(new)
        tables, _ = slnr.page_tables(torch.tensor(new, dtype=torch.int32, device=q.device), self.lens, self.table, self.free(),
                                     self.page_size, sum(new), max_q=max(new),
                                     max_k=-(-self.most // self.page_size) * self.page_size)
        self.lens = tables.k_len
        slnr.page_append(self.cache, tables, k, v)
        return slnr.paged_attention(q, self.cache, tables)[0]

    def go_on(self, parents):
        """Request i goes on from request parents[i]; the others are gone."""
        self.table, self.lens, src, dst, _ = slnr.page_fork(self.table, self.lens, parents, self.free(), self.page_size)
        slnr.page_copy(self.cache, src, dst)

    def pack(self):
        """All pages in use to the front; returns how many (on the GPU)."""
        self.table, src, dst, _, used = slnr.page_compact(self.table, self.lens, self.npages, self.page_size)
        slnr.page_copy(self.cache, src, dst)
        return used


def search(prompts=(130, 300), beams=4, steps=24, heads_q=8, heads=2, width=128, page_size=16, bits=4, every=10, seed=0):
    """Reads the prompts, then takes `steps` tokens of each beam; returns the pool and what each step was given and gave:
    (new tokens, q, k, v, output, what each request goes on from after it)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, max_keys = len(prompts) * beams, max(prompts) + steps
    npages = sum(-(-p // page_size) for p in prompts) + rows * (steps // page_size + 3)
    pool, record = Pool(npages, page_size, heads, width, max_keys, len(prompts), bits), []
    first = torch.arange(rows, device="cuda") // beams
    for n in range(steps + 1):
        new = [1] * rows if n else list(prompts)
        rnd = lambda h: torch.randn((sum(new), h, width), generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        q, k, v = rnd(heads_q), rnd(heads), rnd(heads)
        out = pool.step(new, q, k, v)
        chosen = torch.randint(0, beams, (rows,), generator=g, device="cuda")  # the beams that a search would have kept
        parents = (first * beams + chosen if n else first).to(torch.int32)
        pool.go_on(parents)
        if n % every == every - 1:
            pool.pack()
        record.append((new, q, k, v, out, parents))
    return pool, record


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--beams", type=int, default=4, help="beams of each prompt")
    p.add_argument("--steps", type=int, default=24, help="tokens after the prompts")
    p.add_argument("--bits", type=int, default=4, choices=(4, 16), help="of a cached value")
    a = p.parse_args()
    slnr.build()
    pool, record = search(beams=a.beams, steps=a.steps, bits=a.bits)
    used = pool.pack().item()
    size = sum(x.numel() * x.element_size() for x in ((pool.cache.data,) if a.bits == 4 else (pool.cache.k, pool.cache.v)))
    print(f"{len(record)} steps, {pool.table.shape[0]} beams of {pool.most} keys in {used} pages of {pool.npages} "
          f"({size * used / pool.npages / 1e6:.2f} MB)")
    for i, (new, _, _, _, out, _) in enumerate(record[:3] + record[-1:]):
        print(f"step {i if i < 3 else len(record) - 1}: {sum(new)} new tokens, output {tuple(out.shape)}, "
              f"root mean square {float(out.float().square().mean().sqrt()):.4f}")


if __name__ == "__main__":
    main()
