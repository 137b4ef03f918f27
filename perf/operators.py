"""The operators of one serving step over a paged key/value cache, and what their speed is measured on.

Each step of a program that serves requests takes a few new tokens of each request: it gives them pages and slots
(page_tables), writes their keys and values there (page_append), picks the pages that each token looks at (page_select),
and computes attention over all pages (paged_attention) or the picked ones (selected_attention).  A request has one new
token when it answers and a chunk of them when it is read in.  Keys and values are normal with a few larger columns,
queries likewise; pages lie in the cache in a shuffled order.  Head counts and widths are generic ones and those of the
repository's inner dimensions.
"""
import functools
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HEADS = ((8, 8), (16, 4), (32, 8), (16, 1), (64, 8), (12, 4), (32, 32))
FIRST, LAST = 1, 2  # pages that page_select always takes: the first one, the token's own and the one before it


def listed():
    gqa = dict(Hq=32, H=8, D=128, type="bf16", heads_first=False)
    return [
        # One new token for each of 64 requests: the smallest call, latency alone.
        dict(name="tables_decode_64", op="tables", R=64, q_lo=1, q_hi=1, k_lo=100, k_hi=8000, page=16),
        # 512 requests read in at once: 260k slots.
        dict(name="tables_chunks_512", op="tables", R=512, q_lo=256, q_hi=1024, k_lo=300, k_hi=16000, page=16),
        # One token each: a few pages become full.
        dict(name="append_decode_64", op="append", R=64, q_lo=1, q_hi=1, k_lo=128, k_hi=4096, page=64, **gqa),
        # 16 prompts, 31k tokens: two streams through memory.
        dict(name="append_chunks_16", op="append", R=16, q_lo=1501, q_hi=2600, k_lo=1501, k_hi=5000, page=64, **gqa),
        # Pages picked for one token of each of 32 long requests: reads the summaries.
        dict(name="select_decode_32", op="select", R=32, q_lo=1, q_hi=1, k_lo=4001, k_hi=32003, page=64, topk=32, **gqa),
        # Pages picked for a chunk of 2048 tokens of one long request.
        dict(name="select_chunk_2k", op="select", R=1, q_lo=2048, q_hi=2048, k_lo=32768, k_hi=32768, page=64, topk=16, **gqa),
        # One token of one request: split over the keys, latency counts.
        dict(name="attention_decode_1", op="attention", R=1, q_lo=1, q_hi=1, k_lo=4095, k_hi=4095, page=16, **gqa),
        # The ordinary answering step: 64 ragged requests, the cache is read once.
        dict(name="attention_decode_64", op="attention", R=64, q_lo=1, q_hi=1, k_lo=1001, k_hi=32003, page=16, **gqa),
        # A long prompt's chunk: the largest call.
        dict(name="attention_chunk_4k", op="attention", R=1, q_lo=4096, q_hi=4096, k_lo=16384, k_hi=16384, page=64, **gqa),
        # Chunks and single tokens in one batch, the other type and layout, narrower heads, odd lengths.
        dict(name="attention_mixed_16", op="attention", R=16, q_lo=1, q_hi=513, k_lo=701, k_hi=8191, page=16, Hq=16, H=4,
             D=64, type="fp16", heads_first=True),
        # One token each over 32 picked pages.
        dict(name="selected_decode_32", op="selected", R=32, q_lo=1, q_hi=1, k_lo=4001, k_hi=32003, page=64, topk=32, **gqa),
        # A chunk, 16 picked pages a token and head: neighbours pick alike, not the same.
        dict(name="selected_chunk_2k", op="selected", R=1, q_lo=2048, q_hi=2048, k_lo=32768, k_hi=32768, page=64, topk=16,
             **gqa),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "append", "select", "select", "attention", "attention", "attention", "selected", "selected"))
    largest = [c for c in listed() if c["op"] == op]
    most = {k: max(work(c)[k] for c in largest) for k in ("bytes", "flops")}
    room = max(_padded(c) for c in largest)
    while True:
        single = rng.random() < (0.3 if op in ("tables", "append") else 0.5)
        R = _log_int(rng, 1, 512 if op == "tables" else 64)
        q_lo = 1 if single else _log_int(rng, 1, 1000)
        q_hi = 1 if single else _log_int(rng, q_lo, 4096)
        k_lo = _log_int(rng, max(q_lo, 100), 32768)
        k_hi = _log_int(rng, max(k_lo, q_hi), 32768)
        case = dict(op=op, R=R, q_lo=q_lo, q_hi=q_hi, k_lo=k_lo, k_hi=k_hi, page=rng.choice((16, 32, 64, 128)))
        if op != "tables":
            case["Hq"], case["H"] = rng.choice(HEADS)
            case.update(D=rng.choice((128, 128, 64, 64, 32, 80, 96)), type=rng.choice(("bf16", "bf16", "fp16")),
                        heads_first=rng.random() < 0.3)
        if op in ("select", "selected"):
            case["page"] = rng.choice((32, 64, 128))
            case["topk"] = rng.choice((4, 8, 16, 31, 32))
        w = work(case)
        if all(w[k] <= most[k] for k in most) and _padded(case) <= room:
            return case


# ---- lengths -----------------------------------------------------------------------------

def _spread(lo, hi, n):
    return [round(lo * (hi / lo) ** (i / max(1, n - 1))) for i in range(n)]


def _lengths(case):
    """(new tokens, keys with them) of each request: spread from the least to the most, paired in a fixed shuffled order."""
    R = case["R"]
    q, k = _spread(case["q_lo"], case["q_hi"], R), _spread(case["k_lo"], case["k_hi"], R)
    random.Random(R).shuffle(q)
    return [(a, max(a, b)) for a, b in zip(q, k)]


def _padded(case):
    """Values of the largest tensor of the plain form, whose requests are padded to the longest."""
    lens = _lengths(case)
    q, k = max(a for a, _ in lens), max(b for _, b in lens)
    R, H, D = case["R"], case.get("H", 1), case.get("D", 1)
    keys = R * k * H * D
    if case["op"] == "attention":
        return max(R * q * case["Hq"] * k, keys)
    if case["op"] == "selected":
        return sum(a for a, _ in lens) * H * case["topk"] * case["page"] * D
    if case["op"] == "select":
        return R * q * H * -(-k // case["page"])
    return keys


# ---- inputs ------------------------------------------------------------------------------

def _normal(g, *shape, type):
    """Normal values, every 32nd column four times as large."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=type)
    x[..., ::32] *= 4
    return x


def _cache(g, case, npages, empty=False):
    """K or V as [page, slot, head, column]; with heads_first a page holds its heads one after another."""
    s, H, D, type = case["page"], case["H"], case["D"], TYPES[case["type"]]
    shape = (npages, H, s, D) if case["heads_first"] else (npages, s, H, D)
    x = _normal(g, *shape, type=type)
    return x.transpose(1, 2) if case["heads_first"] else x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lens = _lengths(case)
    random.Random(seed).shuffle(lens)
    op, s, R = case["op"], case["page"], case["R"]
    i32 = dict(dtype=torch.int32, device="cuda")
    new_len = torch.tensor([a for a, _ in lens], **i32)
    k_len = torch.tensor([b for _, b in lens], **i32)
    T, max_q, max_k = sum(a for a, _ in lens), max(a for a, _ in lens), max(b for _, b in lens)
    # block tables over shuffled pages, a few of them not in use
    need, width = (k_len + s - 1) // s, -(-max_k // s)
    used = sum(-(-b // s) for _, b in lens)
    npages = used + 7
    ids = torch.randperm(npages, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(width, **i32)
    first = torch.cumsum(need, 0) - need
    at = (first[:, None] + col).clamp_(max=npages - 1)
    table = torch.where(col < need[:, None], ids[at], -1)
    q_pos = torch.zeros(R + 1, **i32)
    q_pos[1:] = torch.cumsum(new_len, 0)
    req = torch.repeat_interleave(torch.arange(R, **i32), new_len, output_size=T)
    where = (k_len - new_len - q_pos[:-1])[req] + torch.arange(T, **i32)  # position of each token in its request
    slots = table[req, where // s] * s + where % s
    st = dict(op=op, R=R, T=T, max_q=max_q, max_k=max_k, page=s, table=table, q_pos=q_pos, k_len=k_len, req=req,
              slots=slots)
    if op == "tables":
        old = k_len - new_len
        held = (old + s - 1) // s
        st.update(new_len=new_len, old_len=old, free=ids[torch.randperm(npages, generator=g, device="cuda")],
                  table=torch.where(col < held[:, None], table, -1))
        return st
    Hq, H, D, type = case["Hq"], case["H"], case["D"], TYPES[case["type"]]
    st.update(H=H, D=D, type=type, scale=D ** -0.5)
    if op in ("append", "select"):
        st["codes"] = torch.randn((npages, H, D), generator=g, device="cuda").mul_(40).clamp_(-127, 127).to(torch.int8)
        st["scales"] = torch.rand((npages, H), generator=g, device="cuda").mul_(0.01).add_(0.002)
    if op == "select":
        st.update(topk=case["topk"])
    if op != "select":
        st.update(k=_cache(g, case, npages), v=_cache(g, case, npages))
    if op == "append":
        st.update(filled=sum(b // s - (b - a) // s for a, b in lens))
        st.update(k_new=_normal(g, T, H, D, type=type), v_new=_normal(g, T, H, D, type=type),
                  values=torch.empty((npages, H, D), dtype=type, device="cuda"))
    else:
        st["q"] = _normal(g, T, Hq, D, type=type)
    if op == "selected":
        st["pages"] = _picks(g, st, case["topk"], width)
    if own:
        import paper_2205_11622_gb300 as slnr
        st["tables"] = slnr.PageTables(table=table, q_pos=q_pos, k_len=k_len, req=req, slots=slots, max_q=max_q, max_k=max_k)
        if op == "select":
            st["cache"] = slnr.PagedCache(codes=st["codes"], scales=st["scales"], page_size=s)
        else:
            st["cache"] = slnr.PagedCache(k=st["k"], v=st["v"], codes=st.get("codes"), scales=st.get("scales"))
    return st


def _picks(g, st, topk, width):
    """Pages for each token and head: always the first and its own; the others by scores that drift along the tokens."""
    T, H = st["T"], st["H"]
    own_page = (_position(st) // st["page"])[:, None, None]
    rnd = lambda *n: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    score = rnd(st["R"], H, width)[st["req"]] + 0.3 * rnd(T // 32 + 1, H, width)[torch.arange(T, device="cuda") // 32]
    score += 0.2 * rnd(T, H, width)
    page = torch.arange(width, device="cuda")
    score = torch.where((page == 0) | (page == own_page), 9.0, score)
    score = torch.where(page > own_page, -1.0, score)
    top = torch.topk(score, min(topk, width), dim=-1)
    pages = torch.where(top.values > 0, top.indices, width).sort(dim=-1).values
    out = torch.full((T, H, topk), -1, dtype=torch.int32, device="cuda")
    out[..., :pages.shape[-1]] = torch.where(pages < width, pages, -1)
    return out


# ---- one pass ----------------------------------------------------------------------------

def run(st):
    return _own(st) if own else PLAIN[st["op"]](st)


def _own(st):
    import paper_2205_11622_gb300 as slnr
    op = st["op"]
    if op == "tables":
        t, used = slnr.page_tables(st["new_len"], st["old_len"], st["table"], st["free"], st["page"], st["T"])
        return {"table": t.table, "q_pos": t.q_pos, "k_len": t.k_len, "req": t.req, "slots": t.slots, "used": used}
    cache, tables = st["cache"], st["tables"]
    if op == "append":
        slnr.page_append(cache, tables, st["k_new"], st["v_new"])
        return _appended(st)
    if op == "select":
        return slnr.page_select(st["q"], cache, tables, st["topk"], first=FIRST, last=LAST)
    if op == "attention":
        out, lse = slnr.paged_attention(st["q"], cache, tables, scale=st["scale"])
    else:
        out, lse = slnr.selected_attention(st["q"], cache, tables, st["pages"], scale=st["scale"])
    return {"out": out, "lse": lse}


def _appended(st):
    # the summaries as the values that they stand for, rounded to the cache's type
    values = torch.mul(st["codes"], st["scales"].unsqueeze(-1), out=st["values"])
    return {"k": st["k"], "v": st["v"], "scales": st["scales"], "values": values}


def _position(st):
    return (st["k_len"] - st["q_pos"][1:])[st["req"]] + torch.arange(st["T"], dtype=torch.int32, device="cuda")


def _plain_tables(st):
    s, T, table, R = st["page"], st["T"], st["table"], st["R"]
    new, old = st["new_len"], st["old_len"]
    k_len = old + new
    q_pos = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    q_pos[1:] = torch.cumsum(new, 0)
    held, need = (old + s - 1) // s, (k_len + s - 1) // s
    first = torch.cumsum(need - held, 0) - (need - held)
    col = torch.arange(table.shape[1], dtype=torch.int32, device="cuda")
    taken = (col >= held[:, None]) & (col < need[:, None])
    at = (first - held)[:, None] + col
    table.copy_(torch.where(taken, st["free"][torch.where(taken, at, 0)], table))
    t = torch.arange(T, dtype=torch.int32, device="cuda")
    req = (torch.searchsorted(q_pos, t, right=True) - 1).to(torch.int32)
    p = (old - q_pos[:-1])[req] + t
    slots = table[req, p // s] * s + p % s
    return {"table": table, "q_pos": q_pos, "k_len": k_len, "req": req, "slots": slots,
            "used": (need - held).sum(dtype=torch.int32).reshape(1)}


def _plain_append(st):
    s, k, v = st["page"], st["k"], st["v"]
    page, off = st["slots"] // s, st["slots"] % s
    k[page, off] = st["k_new"]
    v[page, off] = st["v_new"]
    # the pages that became full: as many as there were, without asking the GPU
    page = page[torch.argsort((off != s - 1).to(torch.int8), stable=True)[:st["filled"]]]
    mean = k[page].sum(dim=1, dtype=torch.float32) / s
    scale = mean.abs().amax(dim=-1) / 127
    code = torch.where(scale[..., None] > 0, torch.round(mean / scale[..., None]), 0).clamp(-127, 127)
    st["codes"][page] = code.to(torch.int8)
    st["scales"][page] = scale
    return _appended(st)


def _rows(st):
    """Token of each place of the padded batch [R, max_q] (any token where there is none)."""
    at = st["q_pos"][:-1, None] + torch.arange(st["max_q"], dtype=torch.int32, device="cuda")
    return at.clamp(max=st["T"] - 1)


def _packed(st, x):
    """The padded batch's rows x [R, max_q, ...] in the tokens' order."""
    return x[st["req"], torch.arange(st["T"], device="cuda") - st["q_pos"][st["req"]]]


def _group_sum(q, H):
    """Sum of the query rows of each key head's group [T, H, D], in the heads' order: it is coded, so its rounding counts."""
    T, Hq, D = q.shape
    return functools.reduce(torch.add, q.float().reshape(T, H, Hq // H, D).unbind(2))


def _plain_select(st):
    s, H, topk, table = st["page"], st["H"], st["topk"], st["table"]
    u = _group_sum(st["q"], H)
    most = u.abs().amax(dim=-1, keepdim=True)
    code = torch.where(most > 0, torch.round(u * (127 / most)), 0)
    pages = table.clamp(min=0)
    # whole numbers below 2^24: exact in 32 bits in any order
    dot = torch.matmul(code[_rows(st)].transpose(1, 2), st["codes"][pages].float().permute(0, 2, 3, 1))
    score = dot * st["scales"][pages].transpose(1, 2)[:, :, None]
    own_page = (_position(st) // s)[_rows(st)][:, None, :, None]
    page = torch.arange(table.shape[1], dtype=torch.int32, device="cuda")
    score = torch.where((page < FIRST) | (page > own_page - LAST), math.inf, score)
    score = torch.where(page > own_page, -math.inf, score)
    score, page = torch.sort(score, dim=-1, descending=True, stable=True)
    n = min(topk, table.shape[1])
    page = torch.where(score[..., :n] > -math.inf, page[..., :n], table.shape[1]).sort(dim=-1).values
    page = torch.where(page < table.shape[1], page, -1).to(torch.int32)
    out = torch.full((st["T"], H, topk), -1, dtype=torch.int32, device="cuda")
    out[..., :n] = _packed(st, page.transpose(1, 2))
    return out


def _softmax_product(s, seen, v):
    """(softmax(s) . v, log of the sum of exponentials) over the seen columns; zeros and -inf for rows that see none."""
    s = torch.where(seen, s, -math.inf)
    most = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(most > -math.inf, most, 0))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1)
    return o, (most + torch.log(total)).squeeze(-1)


def _plain_attention(st):
    q, H, D, R = st["q"], st["H"], st["D"], st["R"]
    T, Hq, _ = q.shape
    G, max_q = Hq // H, st["max_q"]
    pages = st["table"].clamp(min=0)
    q = q.float().reshape(T, H, G, D)[_rows(st)].permute(0, 2, 3, 1, 4).reshape(R, H, G * max_q, D)
    k = st["k"][pages].reshape(R, -1, H, D).transpose(1, 2).float()
    v = st["v"][pages].reshape(R, -1, H, D).transpose(1, 2).float()
    p = _position(st)[_rows(st)]
    seen = (torch.arange(k.shape[2], device="cuda") <= p[..., None])[:, None, None]
    s = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).reshape(R, H, G, max_q, -1)
    o, lse = _softmax_product(s, seen, v[:, :, None])
    out = _packed(st, o.permute(0, 3, 1, 2, 4)).reshape(T, Hq, D)
    return {"out": out.to(st["type"]), "lse": _packed(st, lse.permute(0, 3, 1, 2)).reshape(T, Hq)}


def _plain_selected(st):
    q, H, D, s, pages = st["q"], st["H"], st["D"], st["page"], st["pages"]
    T, Hq, _ = q.shape
    at = st["table"][st["req"].long()[:, None, None], pages.clamp(min=0)]
    head, slot = torch.arange(H, device="cuda")[:, None, None], torch.arange(s, device="cuda")
    k = st["k"][at[..., None], slot, head].float().reshape(T, H, -1, D)
    v = st["v"][at[..., None], slot, head].float().reshape(T, H, -1, D)
    seen = (pages[..., None] >= 0) & (pages[..., None] * s + slot <= _position(st)[:, None, None, None])
    x = torch.matmul(q.float().reshape(T, H, Hq // H, D), k.transpose(2, 3)).mul_(st["scale"])
    o, lse = _softmax_product(x, seen.reshape(T, H, 1, -1), v)
    return {"out": o.reshape(T, Hq, D).to(st["type"]), "lse": lse.reshape(T, Hq)}


PLAIN = dict(tables=_plain_tables, append=_plain_append, select=_plain_select, attention=_plain_attention,
             selected=_plain_selected)


# ---- what a pass cannot do without ---------------------------------------------------------

def _tri(n):
    return n * (n + 1) // 2


def _picked(p, case):
    """Keys that a token at position p sees in its picked pages, its own page among them."""
    s = case["page"]
    return (min(case["topk"], p // s + 1) - 1) * s + p % s + 1


def work(case):
    lens, op, s = _lengths(case), case["op"], case["page"]
    T = sum(a for a, _ in lens)
    if op == "tables":
        new = sum(-(-b // s) - -(-(b - a) // s) for a, b in lens)
        return {"bytes": 16 * case["R"] + 8 * new + 8 * T, "flops": T}
    H, D = case["H"], case["D"]
    key = 2 * H * D  # bytes of one token's keys (or values)
    if op == "append":
        full = sum(b // s - (b - a) // s for a, b in lens)
        older = sum((b - a) % s for a, b in lens if b // s > (b - a) // s)
        return {"bytes": 4 * T * (key + 1) + older * key + full * H * (D + 4), "flops": full * s * H * D}
    Hq = case["Hq"]
    if op == "select":
        pages = sum(-(-b // s) for _, b in lens)
        pairs = sum(_page_sum(b, s) - _page_sum(b - a, s) for a, b in lens)
        return {"bytes": 2 * T * Hq * D + pages * H * (D + 4) + 4 * T * H * case["topk"], "flops": 2 * pairs * H * D}
    io = 4 * T * Hq * D + 4 * T * Hq
    if op == "attention":
        pairs = sum(_tri(b) - _tri(b - a) for a, b in lens)
        return {"bytes": io + 2 * key * sum(b for _, b in lens), "flops": 4 * D * Hq * pairs}
    seen = [[_picked(p, case) for p in range(b - a, b)] for a, b in lens]
    keys = sum(min(b, sum(x)) for x, (_, b) in zip(seen, lens))
    return {"bytes": io + 2 * key * keys + 4 * T * H * case["topk"], "flops": 4 * D * Hq * sum(map(sum, seen))}


def _page_sum(n, s):
    """Pages up to its own, summed over the positions below n."""
    return s * _tri(n // s) + n % s * (n // s + 1)


# ---- the definitions in 64 bits -------------------------------------------------------------

def exact(case, seed):
    op = case["op"]
    if op in ("tables", "select"):  # whole numbers
        return None
    st = prepare(case, seed)
    if op == "append":
        return _exact_append(st)
    ends, lens = st["q_pos"].tolist(), st["k_len"].tolist()
    q, H, D, s = st["q"], st["H"], st["D"], st["page"]
    T, Hq, _ = q.shape
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        lo, hi = ends[r], ends[r + 1]
        j = torch.arange(n, device="cuda")
        page = st["table"][r, j // s].long()
        for a in range(lo, hi, 1024):  # a thousand tokens at a time
            b = min(hi, a + 1024)
            p = torch.arange(n - hi + a, n - hi + b, device="cuda")[:, None]
            for h in range(Hq):
                g = h // (Hq // H)
                k, v = st["k"][page, j % s, g].double(), st["v"][page, j % s, g].double()
                seen = j <= p
                if op == "selected":
                    picked = torch.zeros((b - a, st["table"].shape[1] + 1), dtype=torch.bool, device="cuda")
                    picked.scatter_(1, st["pages"][a:b, g].long() % picked.shape[1], True)  # -1: the spare column
                    seen = seen & picked[:, j // s]
                x = (q[a:b, h].double() @ k.T * st["scale"]).masked_fill(~seen, -math.inf)
                lse[a:b, h] = torch.logsumexp(x, dim=-1)
                out[a:b, h] = torch.softmax(x, dim=-1) @ v
    return {"out": out, "lse": lse}


def _exact_append(st):
    s, slots = st["page"], st["slots"].long()
    k, v, scales = st["k"].clone(), st["v"].clone(), st["scales"].double()
    values = st["codes"].double() * scales[..., None]
    k[slots // s, slots % s], v[slots // s, slots % s] = st["k_new"], st["v_new"]
    full = slots[slots % s == s - 1] // s
    mean = k[full].double().mean(dim=1)
    scales[full] = mean.abs().amax(dim=-1) / 127
    values[full] = torch.round(mean / scales[full][..., None]) * scales[full][..., None]
    return {"k": k, "v": v, "scales": scales, "values": values}
