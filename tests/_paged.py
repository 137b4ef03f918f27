"""The paged-cache operators in 64 bits, and caches to run them on.

Caches hold NaN wherever no call may look: slots past a request's last key, and
pages that no request has.

Attention's tolerance, as a share of A = sum_j w_j |v_j| (w the softmax): the
weights are rounded to the cache's type once and the output once, u A each (u =
2^-8 in bf16, 2^-11 in fp16); half a u more covers the fp32 scores, whose sums of
D products are off by D 2^-24 sum |q k| at most, 6e-5 of a weight's logarithm for
the normal inputs here, and the exponentials (2^-22).  A log-sum-exp is off by
the scores' error and its own few roundings.
"""
import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LSE_TOL = 2e-4


class Batch:
    """Requests of (new tokens, keys), their tables and a cache, on the GPU."""

    def __init__(self, lens, page, Hq, H, D, dtype=torch.bfloat16, seed=0, heads_first=False, width=None, spare=3):
        g = self.g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.Hq, self.H, self.D, self.dtype = lens, page, Hq, H, D, dtype
        R = len(lens)
        need = [-(-k // page) for _, k in lens]
        self.npages = sum(need) + spare
        ids = torch.randperm(self.npages, generator=g).tolist()
        self.width = max(need + [1]) if width is None else width
        table = torch.full((R, self.width), -1, dtype=torch.int32)
        k = torch.full((self.npages, page, H, D), math.nan)
        v = k.clone()
        for r, (_, n) in enumerate(lens):
            for i in range(need[r]):
                table[r, i] = at = ids.pop()
                fill = min(page, n - i * page)
                k[at, :fill] = torch.randn((fill, H, D), generator=g)
                v[at, :fill] = torch.randn((fill, H, D), generator=g)
        self.table = table
        self.q_pos = torch.tensor([0, *np.cumsum([q for q, _ in lens])], dtype=torch.int32)
        self.k_len = torch.tensor([n for _, n in lens], dtype=torch.int32)
        self.T = int(self.q_pos[-1])
        self.req = torch.tensor([r for r, (q, _) in enumerate(lens) for _ in range(q)], dtype=torch.int32)
        self.pos = torch.tensor([n - q + i for q, n in lens for i in range(q)], dtype=torch.int64)
        self.k, self.v = k.to(dtype), v.to(dtype)
        self.q = torch.randn((self.T, Hq, D), generator=g).to(dtype)
        self.max_q, self.max_k = max([q for q, _ in lens] + [0]), max([n for _, n in lens] + [0])
        if heads_first:
            self.kd = self.k.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            self.vd = self.v.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        else:
            self.kd, self.vd = self.k.cuda(), self.v.cuda()

    def tables(self, slots=None, **kw):
        import paper_2205_11622_gb300 as slnr
        a = dict(table=self.table.cuda(), q_pos=self.q_pos.cuda(), k_len=self.k_len.cuda(), req=self.req.cuda(),
                 slots=slots, max_q=self.max_q, max_k=self.max_k)
        return slnr.PageTables(**{**a, **kw})

    def cache(self, **kw):
        import paper_2205_11622_gb300 as slnr
        return slnr.PagedCache(k=self.kd, v=self.vd, **kw)

    def keys(self, r, h):
        """K and V of request r and head h in 64 bits, and each key's page of the request."""
        n = self.lens[r][1]
        j = torch.arange(n)
        at = self.table[r, j // self.page].long()
        return self.k[at, j % self.page, h].double(), self.v[at, j % self.page, h].double(), j // self.page

    def attention(self, scale, picked=None):
        """(out, lse, sum of softmax |v|) in 64 bits."""
        T, Hq, D, G = self.T, self.Hq, self.D, self.Hq // self.H
        out, mag = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
        lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
        for r, (n, k_len) in enumerate(self.lens):
            t0 = int(self.q_pos[r])
            for h in range(self.H):
                k, v, page = self.keys(r, h)
                for t in range(t0, t0 + n):
                    seen = torch.arange(k_len) <= self.pos[t]
                    if picked is not None:
                        seen &= torch.isin(page, picked[t, h].long())
                    if not seen.any():
                        continue
                    for g in range(h * G, (h + 1) * G):
                        s = k[seen] @ self.q[t, g].double() * scale
                        w = torch.softmax(s, 0)
                        out[t, g], mag[t, g] = w @ v[seen], w @ v[seen].abs()
                        lse[t, g] = torch.logsumexp(s, 0)
        return out, lse, mag

    def check(self, got, ref, what=""):
        out, lse = (x.double().cpu() for x in got)
        want, want_lse, mag = ref
        assert torch.isfinite(out).all(), f"{what}: {int((~torch.isfinite(out)).sum())} values are not finite"
        err = (out - want).abs()
        tol = 2.5 * U[self.dtype] * mag
        assert (err <= tol).all(), f"{what}: {float((err - tol).max()):.3e} over; at {int((err - tol).argmax())}"
        dead = torch.isinf(want_lse)
        assert torch.equal(lse[dead], want_lse[dead]), f"{what}: rows without keys"
        assert ((lse - want_lse)[~dead].abs() <= LSE_TOL).all(), f"{what}: lse {float((lse - want_lse)[~dead].abs().max()):.2e}"


def picks(b, n, seed=0, share=0.7):
    """Pages [T, H, n] picked at random for each token and head, ascending, -1 in random places; some rows empty."""
    g = torch.Generator().manual_seed(seed)
    out = torch.full((b.T, b.H, n), -1, dtype=torch.int32)
    for t in range(b.T):
        have = max(0, int(b.pos[t])) // b.page + 1
        for h in range(b.H):
            m = min(n, have, int(torch.randint(0, n + 1, (1,), generator=g)))
            pages = torch.randperm(have, generator=g)[:m].sort().values
            at = torch.randperm(n, generator=g)[:m].sort().values
            out[t, h, at] = pages.to(torch.int32)
    return out
