"""The operators around a paged key/value cache that is kept for long, and what their speed is measured on.

A program that serves many requests holds their keys and values in 4 bits to hold more of them: each step's new ones are
coded as they are appended (page_append on a PagedCache4), attention reads the codes (paged_attention), and page_values gives
the values that pages stand for.  Between steps it moves whole pages: page_fork lets requests go on from others, sharing
their full pages (several answers to a prompt, beams that are reordered), page_free lists the pages that no request holds
any more, and page_compact packs the pages in use to the front of the cache; page_copy moves what the last two ask for.
Keys and values are normal with a few larger columns, queries likewise; pages lie in the cache in a shuffled order.  Head
counts and widths are generic ones and those of the repository's inner dimensions.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HEADS = ((8, 8), (16, 4), (32, 8), (16, 1), (64, 8), (12, 4), (32, 32))
BLOCK = 16        # columns that share a scale
MOST = 9216.0     # the largest scale


def listed():
    gqa = dict(Hq=32, H=8, D=128, type="bf16")
    return [
        # One new token for each of 64 requests, coded into the cache: latency.
        dict(name="append4_decode_64", op="append", R=64, q_lo=1, q_hi=1, k_lo=128, k_hi=4096, page=64, **gqa),
        # 16 prompts, 31k tokens coded at once: streams through memory.
        dict(name="append4_chunks_16", op="append", R=16, q_lo=1501, q_hi=2600, k_lo=1501, k_hi=5000, page=64, **gqa),
        # One token of one request: split over the keys, latency counts.
        dict(name="attention4_decode_1", op="attention", R=1, q_lo=1, q_hi=1, k_lo=4095, k_hi=4095, page=16, **gqa),
        # The ordinary answering step: 64 ragged requests, the cache is read once.
        dict(name="attention4_decode_64", op="attention", R=64, q_lo=1, q_hi=1, k_lo=1001, k_hi=32003, page=16, **gqa),
        # A long prompt's chunk: the largest call.
        dict(name="attention4_chunk_4k", op="attention", R=1, q_lo=4096, q_hi=4096, k_lo=16384, k_hi=16384, page=64, **gqa),
        # Chunks and single tokens in one batch, the other type, narrower heads, odd lengths.
        dict(name="attention4_mixed_16", op="attention", R=16, q_lo=1, q_hi=513, k_lo=701, k_hi=8191, page=16, Hq=16, H=4,
             D=64, type="fp16"),
        # 32 beams reordered: some go on twice, some not at all; the last pages of the second ones are copied.
        dict(name="fork_beams_32", op="fork", R=32, n=32, k_lo=300, k_hi=4000, page=16, H=8, D=128, bits=16, type="bf16"),
        # 512 answers to 128 prompts that have just been read in.
        dict(name="fork_answers_512", op="fork", R=128, n=512, k_lo=500, k_hi=16000, page=64, H=2, D=128, bits=16, type="bf16"),
        # Three of 64 requests have ended.
        dict(name="free_3_of_64", op="free", R=64, n=3, k_lo=100, k_hi=8000, page=16),
        # 37 of 512 have, of a cache of 150k pages.
        dict(name="free_37_of_512", op="free", R=512, n=37, k_lo=300, k_hi=16000, page=16),
        # 8 requests spread over a small cache of 4 bits: latency, and the cache's values.
        dict(name="compact4_8", op="compact", R=8, k_lo=100, k_hi=2000, page=16, H=8, D=128, bits=4, type="bf16"),
        # 64 requests spread over half as many pages again: a third of their pages move.
        dict(name="compact_64", op="compact", R=64, k_lo=500, k_hi=4000, page=64, H=8, D=128, bits=16, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "attention", "fork", "free", "compact"))
    largest = [c for c in listed() if c["op"] == op]
    most = {k: max(work(c)[k] for c in largest) for k in ("bytes", "flops")}
    room = max(_padded(c) for c in largest)
    while True:
        case = dict(op=op, page=rng.choice((16, 32, 64, 128)))
        if op in ("append", "attention"):
            single = rng.random() < (0.3 if op == "append" else 0.5)
            q_lo = 1 if single else _log_int(rng, 1, 1000)
            q_hi = 1 if single else _log_int(rng, q_lo, 4096)
            k_lo = _log_int(rng, max(q_lo, 100), 32768)
            case.update(R=_log_int(rng, 1, 64), q_lo=q_lo, q_hi=q_hi, k_lo=k_lo, k_hi=_log_int(rng, max(k_lo, q_hi), 32768))
            case["Hq"], case["H"] = rng.choice(HEADS)
        else:
            case.update(R=_log_int(rng, 1, 512), k_lo=_log_int(rng, 20, 8000))
            case["k_hi"] = _log_int(rng, case["k_lo"], 16000)
            if op == "fork":
                case["n"] = _log_int(rng, 1, 512)
            elif op == "free":
                case["n"] = _log_int(rng, 1, case["R"])
            if op != "free":
                case.update(H=rng.choice((1, 2, 4, 8, 12)), bits=rng.choice((4, 16)))
        if op != "free":
            case.update(D=rng.choice((128, 128, 64, 64, 32, 96)), type=rng.choice(("bf16", "bf16", "fp16")))
        w = work(case)
        if all(w[k] <= most[k] for k in most) and _padded(case) <= room:
            return case


# ---- lengths -----------------------------------------------------------------------------

def _spread(lo, hi, n):
    return [round(lo * (hi / lo) ** (i / max(1, n - 1))) for i in range(n)]


def _lengths(case):
    """(new tokens, keys with them) of each request: spread from the least to the most, paired in a fixed shuffled order."""
    R = case["R"]
    q, k = _spread(case.get("q_lo", 1), case.get("q_hi", 1), R), _spread(case["k_lo"], case["k_hi"], R)
    random.Random(R).shuffle(q)
    return [(a, max(a, b)) for a, b in zip(q, k)]


def _padded(case):
    """Values of the largest tensor of the plain form, whose requests are padded to the longest."""
    lens = _lengths(case)
    q, k = max(a for a, _ in lens), max(b for _, b in lens)
    R, H, D = case["R"], case.get("H", 1), case.get("D", 1)
    if case["op"] == "attention":
        return max(R * q * case["Hq"] * k, R * k * H * D)
    if case["op"] == "append":
        return R * k * H * D
    return 2 * sum(b for _, b in lens) * H * D


# ---- the 4-bit form ----------------------------------------------------------------------

def _coded(x):
    """(codes int8, scales float32) of x [..., D]: blocks of 16 columns, whole numbers from -7 to 7 times a scale of four
    significant bits, the least that is a 7.5th of the block's largest value."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    least = x.abs().amax(dim=-1).double() / 7.5  # 64 bits: a least scale next to one of four bits is that one
    e = torch.frexp(least)[1].clamp(min=-13)     # multiples of 2^-17 below 2^-14
    s = torch.ldexp(torch.ceil(torch.ldexp(least, 4 - e) - 1e-6), e - 4).clamp(max=MOST).float()
    c = torch.floor(x.abs() / s.clamp(min=2.0 ** -17)[..., None] + 0.5).clamp(max=7)
    return (c * x.sign()).to(torch.int8).flatten(-2), s


def _values(codes, scales):
    return (codes.unflatten(-1, (-1, BLOCK)).float() * scales[..., None]).flatten(-2)


# ---- inputs ------------------------------------------------------------------------------

def _normal(g, *shape, type):
    """Normal values, every 32nd column four times as large."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=type)
    x[..., ::32] *= 4
    return x


def _table(g, case, need, npages):
    """Block tables over shuffled pages, and the pages that no request has, in a shuffled order."""
    ids = torch.randperm(npages, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(max(need), dtype=torch.int32, device="cuda")
    n = torch.tensor(need, dtype=torch.int32, device="cuda")
    at = ((torch.cumsum(n, 0) - n)[:, None] + col).clamp_(max=npages - 1)
    return torch.where(col < n[:, None], ids[at], -1), ids[sum(need):].contiguous()


def _held(st, k, v):
    """The cache of pages k, v [page, slot, head, column]: those tensors, or their 4-bit form."""
    if st["bits"] == 16:
        if own:
            import paper_2205_11622_gb300 as slnr
            st["cache"] = slnr.PagedCache(k=k, v=v)
        st.update(k=k, v=v)
    elif own:
        import paper_2205_11622_gb300 as slnr
        npages, s, H, D = k.shape
        st["cache"] = slnr.PagedCache4.empty(npages, s, H, D)
        i = torch.arange(npages * s, dtype=torch.int32, device="cuda")
        pages = i[:npages, None]
        whole = slnr.PageTables(table=pages, q_pos=i.new_tensor([*range(0, npages * s + 1, s)]),
                                k_len=torch.full_like(i[:npages], s), req=i // s, slots=i, max_q=s, max_k=s)
        slnr.page_append(st["cache"], whole, k.reshape(-1, H, D), v.reshape(-1, H, D))
    else:
        for name, x in (("k", k), ("v", v)):
            st[name], st[name + "_scales"] = _coded(x)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    lens, op, s, R = _lengths(case), case["op"], case["page"], case["R"]
    rng.shuffle(lens)
    i32 = dict(dtype=torch.int32, device="cuda")
    st = dict(op=op, page=s, R=R, bits=case.get("bits", 4))
    if op not in ("append", "attention"):
        return _prepare_pages(case, st, g, rng, [b for _, b in lens], i32)
    type, Hq, H, D = TYPES[case["type"]], case["Hq"], case["H"], case["D"]
    new_len, k_len = torch.tensor([a for a, _ in lens], **i32), torch.tensor([b for _, b in lens], **i32)
    T, max_q, max_k = sum(a for a, _ in lens), max(a for a, _ in lens), max(b for _, b in lens)
    need = [-(-b // s) for _, b in lens]
    npages = sum(need) + 7  # a few of them not in use
    table, _ = _table(g, case, need, npages)
    q_pos = torch.zeros(R + 1, **i32)
    q_pos[1:] = torch.cumsum(new_len, 0)
    req = torch.repeat_interleave(torch.arange(R, **i32), new_len, output_size=T)
    where = (k_len - new_len - q_pos[:-1])[req] + torch.arange(T, **i32)  # position of each token in its request
    slots = table[req, where // s] * s + where % s
    st.update(T=T, H=H, D=D, type=type, max_q=max_q, table=table, q_pos=q_pos, k_len=k_len, req=req, slots=slots,
              scale=D ** -0.5)
    _held(st, _normal(g, npages, s, H, D, type=type), _normal(g, npages, s, H, D, type=type))
    if op == "append":
        # the pages that the new tokens go to, each once
        st["touched"] = torch.cat([table[r, (b - a) // s:need[r]] for r, (a, b) in enumerate(lens)])
        st.update(k_new=_normal(g, T, H, D, type=type), v_new=_normal(g, T, H, D, type=type))
    else:
        st["q"] = _normal(g, T, Hq, D, type=type)
    if own:
        import paper_2205_11622_gb300 as slnr
        st["tables"] = slnr.PageTables(table=table, q_pos=q_pos, k_len=k_len, req=req, slots=slots, max_q=max_q, max_k=max_k)
    return st


def _prepare_pages(case, st, g, rng, lens, i32):
    op, s, R = case["op"], case["page"], case["R"]
    need = [-(-b // s) for b in lens]
    used = sum(need)
    npages = used + case["n"] + 7 if op == "fork" else used + used // 2 + 7
    table, free = _table(g, case, need, npages)
    for r in range(1, R, 4):  # every fourth request goes on from the one before it: they share the first half of a prompt
        n = min(lens[r - 1], lens[r]) // s // 2
        table[r, :n] = table[r - 1, :n]
    st.update(table=table, lens=torch.tensor(lens, **i32), npages=npages)
    if op == "free":
        st["drop"] = torch.tensor(rng.sample(range(R), case["n"]), **i32)
        return st
    if op == "fork":
        parent = [rng.randrange(R) for _ in range(case["n"])]
        st.update(parent=torch.tensor(parent, **i32), free=free)
        # how many last pages are copied, which the program knows from its lengths
        st["moved"] = sum(lens[p] % s != 0 and p in parent[:i] for i, p in enumerate(parent))
    else:
        held = torch.unique(table[table >= 0])
        st["moved"] = int((held >= held.numel()).sum())
    st["type"] = type = TYPES[case["type"]]
    shape = (npages, s, case["H"], case["D"])
    _held(st, _normal(g, *shape, type=type), _normal(g, *shape, type=type))
    return st


# ---- one pass ----------------------------------------------------------------------------

def run(st):
    return _own(st) if own else PLAIN[st["op"]](st)


def _own(st):
    import paper_2205_11622_gb300 as slnr
    op = st["op"]
    if op == "append":
        slnr.page_append(st["cache"], st["tables"], st["k_new"], st["v_new"])
        k, v = slnr.page_values(st["cache"], st["touched"], dtype=st["type"])
        return {"k": k, "v": v}
    if op == "attention":
        out, lse = slnr.paged_attention(st["q"], st["cache"], st["tables"], scale=st["scale"])
        return {"out": out, "lse": lse}
    if op == "free":
        free, count = slnr.page_free(st["table"], st["lens"], st["npages"], st["page"], drop=st["drop"])
        return {"free": free, "count": count, "lens": st["lens"]}
    if op == "fork":
        table, lens, src, dst, used = slnr.page_fork(st["table"], st["lens"], st["parent"], st["free"], st["page"])
        got = {"table": table, "lens": lens, "src": src, "dst": dst, "used": used}
    else:
        table, src, dst, ids, used = slnr.page_compact(st["table"], st["lens"], st["npages"], st["page"])
        got = {"table": table, "src": src, "dst": dst, "ids": ids, "used": used}
    slnr.page_copy(st["cache"], src, dst)
    if st["bits"] == 4:
        got["k"], got["v"] = slnr.page_values(st["cache"], dtype=st["type"])
        return got
    return {**got, "k": st["k"], "v": st["v"]}


def _plain_append(st):
    s = st["page"]
    page, off = st["slots"] // s, st["slots"] % s
    out = {}
    for name in ("k", "v"):
        st[name][page, off], st[name + "_scales"][page, off] = _coded(st[name + "_new"])
        out[name] = _values(st[name][st["touched"]], st[name + "_scales"][st["touched"]]).to(st["type"])
    return out


def _position(st):
    return (st["k_len"] - st["q_pos"][1:])[st["req"]] + torch.arange(st["T"], dtype=torch.int32, device="cuda")


def _rows(st):
    """Token of each place of the padded batch [R, max_q] (any token where there is none)."""
    at = st["q_pos"][:-1, None] + torch.arange(st["max_q"], dtype=torch.int32, device="cuda")
    return at.clamp(max=st["T"] - 1)


def _packed(st, x):
    """The padded batch's rows x [R, max_q, ...] in the tokens' order."""
    return x[st["req"], torch.arange(st["T"], device="cuda") - st["q_pos"][st["req"]]]


def _plain_attention(st):
    q, H, D, R = st["q"], st["H"], st["D"], st["R"]
    T, Hq, _ = q.shape
    G, max_q = Hq // H, st["max_q"]
    pages = st["table"].clamp(min=0)
    q = q.float().reshape(T, H, G, D)[_rows(st)].permute(0, 2, 3, 1, 4).reshape(R, H, G * max_q, D)
    k, v = (_values(st[n][pages], st[n + "_scales"][pages]).reshape(R, -1, H, D).transpose(1, 2) for n in ("k", "v"))
    p = _position(st)[_rows(st)]
    seen = (torch.arange(k.shape[2], device="cuda") <= p[..., None])[:, None, None]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).reshape(R, H, G, max_q, -1)
    x = torch.where(seen, x, -math.inf)
    most = x.amax(dim=-1, keepdim=True)
    x = torch.exp(x - torch.where(most > -math.inf, most, 0))
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x, v[:, :, None]) / torch.where(total > 0, total, 1)
    lse = (most + torch.log(total)).squeeze(-1)
    out = _packed(st, o.permute(0, 3, 1, 2, 4)).reshape(T, Hq, D)
    return {"out": out.to(st["type"]), "lse": _packed(st, lse.permute(0, 3, 1, 2)).reshape(T, Hq)}


def _moved(st, got):
    """The copies of `got`, and the cache after them."""
    n = st["moved"]
    order = torch.argsort((got["src"] < 0).to(torch.int8), stable=True)[:n]
    src, dst = got["src"][order], got["dst"][order]
    for name in ("k", "v") if st["bits"] == 16 else ("k", "v", "k_scales", "v_scales"):
        st[name][dst] = st[name][src]
    if st["bits"] == 16:
        return {**got, "k": st["k"], "v": st["v"]}
    return {**got, **{n: _values(st[n], st[n + "_scales"]).to(st["type"]) for n in ("k", "v")}}


def _plain_fork(st):
    s, table, parent, free = st["page"], st["table"], st["parent"].long(), st["free"]
    n, width = parent.numel(), table.shape[1]
    i = torch.arange(n, device="cuda")
    col = torch.arange(width, device="cuda")
    lens = st["lens"][parent]
    need = (lens + s - 1) // s
    rows = torch.where(col < need[:, None], table[parent], -1)
    first = torch.full((st["R"],), n, device="cuda").scatter_reduce_(0, parent, i, "amin")
    copied = (first[parent] != i) & (lens % s != 0)
    rank = torch.cumsum(copied, 0) - 1
    last = (need.long() - 1).clamp(min=0)
    src = torch.where(copied, rows[i, last], -1)
    dst = torch.where(copied, free[rank.clamp(min=0)], -1)
    rows[i, last] = torch.where(copied, dst, rows[i, last])
    return _moved(st, {"table": rows, "lens": lens, "src": src, "dst": dst,
                       "used": copied.sum(dtype=torch.int32).reshape(1)})


def _in_use(st):
    """One where a request holds the page."""
    table, n = st["table"], st["npages"]
    col = torch.arange(table.shape[1], device="cuda")
    held = col < ((st["lens"] + st["page"] - 1) // st["page"])[:, None]
    mark = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    mark[torch.where(held, table, n).flatten().long()] = 1
    return mark[:n]


def _listed_first(mark, size):
    """The places of the ones of `mark` in ascending order, in the first of `size` entries; -1 behind them."""
    at = torch.argsort(1 - mark, stable=True).to(torch.int32)[:size]
    return torch.where(torch.arange(size, device="cuda") < mark.sum(), at, -1)


def _plain_free(st):
    st["lens"][st["drop"].long()] = 0
    free = 1 - _in_use(st)
    return {"free": _listed_first(free, st["npages"]), "count": free.sum(dtype=torch.int32).reshape(1), "lens": st["lens"]}


def _plain_compact(st):
    mark, n = _in_use(st), st["npages"]
    used = mark.sum(dtype=torch.int32)
    page = torch.arange(n, dtype=torch.int32, device="cuda")
    src = _listed_first(mark * (page >= used), n // 2)
    dst = _listed_first((1 - mark) * (page < used), n // 2)
    ids = torch.full((n + 1,), -1, dtype=torch.int32, device="cuda")
    ids[:n] = torch.where((mark == 1) & (page < used), page, -1)
    ids[torch.where(src >= 0, src, n).long()] = dst
    col = torch.arange(st["table"].shape[1], device="cuda")
    held = col < ((st["lens"] + st["page"] - 1) // st["page"])[:, None]
    table = torch.where(held, ids[st["table"].clamp(min=0).long()], -1)
    return _moved(st, {"table": table, "src": src, "dst": dst, "ids": ids[:n], "used": used.reshape(1)})


PLAIN = dict(append=_plain_append, attention=_plain_attention, fork=_plain_fork, free=_plain_free, compact=_plain_compact)


# ---- what a pass cannot do without ---------------------------------------------------------

def _tri(n):
    return n * (n + 1) // 2


def work(case):
    lens, op, s = _lengths(case), case["op"], case["page"]
    H, D = case.get("H", 0), case.get("D", 0)
    code = 9 * H * D // 16  # bytes of one token's coded keys (or values)
    T, K = sum(a for a, _ in lens), sum(b for _, b in lens)
    if op == "append":
        touched = sum(-(-b // s) - (b - a) // s for a, b in lens) * s
        return {"bytes": 4 * T * H * D + 4 * T + 2 * T * code + touched * (2 * code + 4 * H * D), "flops": 4 * T * H * D}
    if op == "attention":
        Hq = case["Hq"]
        pairs = sum(_tri(b) - _tri(b - a) for a, b in lens)
        return {"bytes": 4 * T * Hq * D + 4 * T * Hq + 2 * code * K, "flops": 4 * D * Hq * pairs}
    entries = sum(-(-b // s) for _, b in lens)
    width = max(-(-b // s) for _, b in lens)
    if op == "free":
        return {"bytes": 4 * entries + 6 * entries + 8 * case["R"], "flops": entries}
    page = s * (2 * code if case["bits"] == 4 else 4 * H * D)
    if op == "fork":
        n = case["n"]
        npages, rows = entries + n + 7, 4 * n * (entries // case["R"] + width + 4)
        copies = max(n - case["R"], n // 4)  # about as many children are not a parent's first
    else:
        npages, rows = entries + entries // 2 + 7, 4 * entries + 4 * case["R"] * width + 8 * (entries + entries // 2)
        copies = entries // 3
    values = npages * s * (2 * code + 4 * H * D) if case["bits"] == 4 else 0
    return {"bytes": rows + 2 * copies * page + values, "flops": copies * s * H * D}


# ---- the definitions in 64 bits -------------------------------------------------------------

def _exact_values(x):
    """The values that x [..., D] stands for in 4 bits."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    least = x.abs().amax(dim=-1) / torch.full((), 7.5, dtype=torch.float64, device="cuda")
    step = torch.exp2(torch.floor(torch.log2(least.clamp(min=2.0 ** -14))) - 3)
    s = torch.ceil(least / step) * step
    s = s.clamp(max=MOST)[..., None]
    c = torch.floor(x.abs() / torch.where(s > 0, s, 1) + 0.5).clamp(max=7)
    return (c * s * x.sign()).flatten(-2)


def exact(case, seed):
    if case["op"] not in ("append", "attention"):  # whole numbers, and values that are moved
        return None
    st = prepare(case, seed)
    s, slots = st["page"], st["slots"].long()
    if case["op"] == "append":
        out = {}
        for name in ("k", "v"):
            x = st[name].double() * st[name + "_scales"].double().repeat_interleave(BLOCK, dim=-1)
            x[slots // s, slots % s] = _exact_values(st[name + "_new"])
            out[name] = x[st["touched"].long()]
        return out
    ends, lens = st["q_pos"].tolist(), st["k_len"].tolist()
    q, H, D = st["q"], st["H"], st["D"]
    T, Hq, _ = q.shape
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        lo, hi = ends[r], ends[r + 1]
        j = torch.arange(n, device="cuda")
        page = st["table"][r, j // s].long()
        held = [st[m][page, j % s].double() * st[m + "_scales"][page, j % s].double().repeat_interleave(BLOCK, dim=-1)
                for m in ("k", "v")]
        for a in range(lo, hi, 1024):  # a thousand tokens at a time
            b = min(hi, a + 1024)
            seen = j <= torch.arange(n - hi + a, n - hi + b, device="cuda")[:, None]
            for h in range(Hq):
                k, v = (x[:, h // (Hq // H)] for x in held)
                x = (q[a:b, h].double() @ k.T * st["scale"]).masked_fill(~seen, -math.inf)
                lse[a:b, h] = torch.logsumexp(x, dim=-1)
                out[a:b, h] = torch.softmax(x, dim=-1) @ v
    return {"out": out, "lse": lse}
