"""A cache in 4 bits: what it holds, in 64 bits, and batches to run attention on.

Held values are a whole number times a scale, exact in 64 bits, so what the calls are
given back of them has to be equal.  Attention's tolerance is that of _paged.py (the
weights are rounded once and the output once, u each, half a u for the scores) and, as
held values are often zero, so that a column's A = sum_j w_j |v_j| can be the share of a
few small weights, two terms beside it: an fp16 output below 2^-14 is rounded to a
multiple of 2^-24, off by 2^-25 at most; an fp16 weight below 2^-14 likewise, where the
row's largest is 2^12 at least, so each of n weights by 2^-37 of the row's sum at most.
"""
import numpy as np
import torch

import _paged as P

BLOCK, MOST = 16, 9216.0


def held(x):
    """What x [..., D] (bf16 or fp16, on the CPU) is held as, in 64 bits."""
    b = x.double().numpy().reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    with np.errstate(invalid="ignore"):
        most = np.abs(b).max(-1, keepdims=True)
        bad = ~np.isfinite(b).all(-1, keepdims=True)
        most = np.where(bad, 0, most)
        # the least of all scales with 7.5 s >= most
        s = SCALES[np.searchsorted(SCALES * 7.5, np.minimum(most, 7.5 * MOST))]
        c = np.minimum(np.floor(np.abs(np.where(bad, 0, b)) / np.where(s > 0, s, 1) + 0.5), 7)
        y = np.where(bad, np.nan, c * s * np.sign(np.where(bad, 0, b)))
    return torch.from_numpy(y.reshape(x.shape))


# bytes as fp16 numbers, up to the largest that is written
SCALES = (np.arange(226, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
assert SCALES[-1] == MOST


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def written(slnr, k, v, table, lens, npages, page, H, D, data=None):
    """A PagedCache4 of which the slots of requests of `lens` keys are appended from k, v [npages, page, H, D] (CPU), and
    all others hold NaN."""
    data = torch.full((npages, H, page // 16, 18 * D), 0xff, dtype=torch.uint8, device="cuda") if data is None else data
    cache = slnr.PagedCache4(data)
    slots = [int(table[r, j // page]) * page + j % page for r, n in enumerate(lens) for j in range(n)]
    at = torch.tensor(slots, dtype=torch.long)
    tables = slnr.PageTables(table=table.cuda(), q_pos=i32([0, *np.cumsum(lens)]), k_len=i32(list(lens)),
                             req=i32([r for r, n in enumerate(lens) for _ in range(n)]), slots=i32(slots),
                             max_q=max([*lens, 0]), max_k=max([*lens, 0]))
    slnr.page_append(cache, tables, k.reshape(-1, H, D)[at].cuda(), v.reshape(-1, H, D)[at].cuda(), validate=True)
    return cache


class Batch4(P.Batch):
    """P.Batch over a cache in 4 bits: its keys and values are what the cache holds."""

    def __init__(self, slnr, *args, heads_first=False, **kw):
        super().__init__(*args, **kw)
        lens = [max(n, 0) for _, n in self.lens]
        data = None
        if not heads_first:  # another order of the axes than the packed one, and room between pages
            data = torch.full((self.H, self.npages + 1, self.page // 16 + 1, 18 * self.D), 0xff, dtype=torch.uint8,
                              device="cuda")[:, 1:, 1:].transpose(0, 1)
        self.c4 = written(slnr, self.k, self.v, self.table, lens, self.npages, self.page, self.H, self.D, data)
        self.k, self.v = held(self.k), held(self.v)

    def cache(self):
        return self.c4

    def check(self, got, ref, what=""):
        out, lse = (x.double().cpu() for x in got)
        want, want_lse, mag = ref
        assert torch.isfinite(out).all(), f"{what}: {int((~torch.isfinite(out)).sum())} values are not finite"
        tol = 2.5 * P.U[self.dtype] * mag + max([n for _, n in self.lens]) * 2.0 ** -37 * torch.nan_to_num(self.v).abs().max()
        if self.dtype == torch.float16:
            tol = tol + 2.0 ** -25
        dead = torch.isinf(want_lse)
        tol[dead] = 0
        err = (out - want).abs()
        assert (err <= tol).all(), f"{what}: {float((err - tol).max()):.3e} over; at {int((err - tol).argmax())}"
        assert torch.equal(lse[dead], want_lse[dead]), f"{what}: rows without keys"
        assert ((lse - want_lse)[~dead].abs() <= P.LSE_TOL).all(), \
            f"{what}: lse {float((lse - want_lse)[~dead].abs().max()):.2e}"
