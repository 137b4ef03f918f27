"""Attention over a paged key/value cache (include/slnr.h): block tables, the
cache's writes, pages picked by a cheap score, and attention over all pages or
the picked ones; a cache held in 4 bits; and whole pages between the steps of a
program: forks of requests, copies, free pages, compaction.

Like the expressions' wrappers these only marshal torch CUDA tensors into the
C structures of the ABI; every step runs in the library's CUDA kernels.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass, field
from typing import Optional

import torch

from . import (SlnrError, _buffer, _capturing, _default_ws, _last_ws, _lock_of_others, _new_workspace, _query, _stream_ptr,
               last_error, lib, slnr_cache, slnr_cache4, slnr_opts, slnr_pages, slnr_rows)

_TYPES = {torch.bfloat16: 0, torch.float16: 1}


_byref = ctypes.byref
# without the objects that the public accessors make, where this torch has these (a call takes some 10 us)
_device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream_now = getattr(torch._C, "_cuda_getCurrentRawStream", lambda _: _stream_ptr(None))


def _ints(x, name, shape, device):
    """x's address, after its checks: an int32 CUDA tensor of that shape, contiguous."""
    if x.dtype != torch.int32 or x.device != device or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor on {device}")
    if x.shape != shape:
        raise ValueError(f"{name} has shape {tuple(x.shape)}, not {shape}")
    return x.data_ptr()


def _table(t):
    """(rows, columns, stride between rows) of a block table, after its checks."""
    if not t.is_cuda or t.dtype != torch.int32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("table must be a 2-D int32 CUDA tensor with packed rows")
    R, width = t.shape
    return R, width, t.stride(0) if R > 1 else width


@dataclass(frozen=True, eq=False)
class PageTables:
    """The requests of a step: their block tables, lengths, and each new token's request and slot (int32 CUDA tensors).

    table [R, width] (rows may be a slice of wider ones), q_pos [R + 1], k_len [R] (keys with the new tokens), req [T],
    slots [T] (page_append only).  max_q and max_k bound the new tokens and the keys of a request on the host.  The work
    is laid out by them: a result depends on them by its rounding alone, its time in earnest.  One token over 4095 keys (32/8 heads of 128)
    takes 17 us of the GPU with max_k = 4095, 25 with 16384, 33 with 32768 and 52 with 131072; 64 single tokens over 581k
    keys 421 with max_q = 1 and 658 with max_q = 64 (as chunks), page_select for them 52 and 263; over a PagedCache4 127 with
    max_q = 1, 306 with 8 and 543 with 9 or more (as chunks).  A captured call keeps its bounds for every replay.  The tensors are held and read by each call that takes the tables.
    """
    table: torch.Tensor
    q_pos: torch.Tensor
    k_len: torch.Tensor
    req: torch.Tensor
    slots: Optional[torch.Tensor]
    max_q: int
    max_k: int
    ntok: int = field(init=False)
    _c: slnr_pages = field(init=False, repr=False)
    _sizes: tuple = field(init=False, repr=False)

    def __post_init__(self):
        R, width, stride = _table(self.table)
        T, dev = self.req.shape[0], self.table.device
        self.__dict__["_c"] = slnr_pages(
            R, T, self.max_q, self.max_k, width, 0, stride, _ints(self.q_pos, "q_pos", (R + 1,), dev),
            _ints(self.k_len, "k_len", (R,), dev), self.table.data_ptr(), _ints(self.req, "req", (T,), dev),
            None if self.slots is None else _ints(self.slots, "slots", (T,), dev))
        self.__dict__["ntok"], self.__dict__["_sizes"] = T, (R, T, self.max_q, self.max_k, width)

    def _tensors(self):
        """What a call that takes the tables may read: held on the stream that it is given."""
        return self.table, self.q_pos, self.k_len, self.req, self.slots

    @classmethod
    def _of(cls, c, **fields):
        """Tables whose arrays a call of this module made: nothing to check."""
        self = object.__new__(cls)
        self.__dict__.update(fields, _c=c, ntok=c.ntok, _sizes=(c.nreq, c.ntok, c.max_q, c.max_k, c.width))
        return self


@dataclass(frozen=True, eq=False)
class PagedCache:
    """Keys and values [pages, slots of a page, heads, width], bf16 or fp16 CUDA tensors of any strides that are
    multiples of 8 values with a packed last axis (k.transpose(1, 2) of a cache that holds a page's heads one after
    another), and the pages' summaries: codes int8 [pages, heads, width], scales fp32 [pages, heads].

    Without a summary page_append writes none and page_select cannot be called; page_select needs no keys (page_size
    then says how many slots a page has).  The tensors are held, and read and written by the calls that take the cache.
    """
    k: Optional[torch.Tensor] = None
    v: Optional[torch.Tensor] = None
    codes: Optional[torch.Tensor] = None
    scales: Optional[torch.Tensor] = None
    page_size: Optional[int] = None
    device: torch.device = field(init=False, repr=False)
    _c: slnr_cache = field(init=False, repr=False)
    _sizes: tuple = field(init=False, repr=False)

    def __post_init__(self):
        k, v, codes, scales = self.k, self.v, self.codes, self.scales
        if (k is None) != (v is None) or (codes is None) != (scales is None) or (k is None and codes is None):
            raise ValueError("a cache has k and v, codes and scales, or all four")
        c = slnr_cache()
        if k is not None:
            if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in _TYPES:
                raise ValueError("k and v must be bf16 or fp16, of one shape [pages, slots, heads, width]")
            if not k.is_cuda or k.device != v.device:
                raise ValueError("k and v must be CUDA tensors on one device")
            if k.shape[3] > 1 and (k.stride(3) != 1 or v.stride(3) != 1):
                raise ValueError("the last axis of k and v must be packed")
            if self.page_size not in (None, k.shape[1]):
                raise ValueError(f"page_size is {self.page_size}, but k has {k.shape[1]} slots a page")
            object.__setattr__(self, "page_size", k.shape[1])
            c.dtype = _TYPES[k.dtype]
            c.k_stride[:], c.v_stride[:] = k.stride()[:3], v.stride()[:3]
            c.k, c.v = k.data_ptr(), v.data_ptr()
        elif self.page_size is None:
            raise ValueError("a cache without keys needs page_size")
        if codes is not None:
            if not (codes.is_cuda and codes.dtype == torch.int8 and codes.dim() == 3 and codes.is_contiguous()):
                raise ValueError("codes must be a contiguous int8 CUDA tensor [pages, heads, width]")
            if not (scales.dtype == torch.float32 and scales.shape == codes.shape[:2] and scales.is_contiguous()
                    and scales.device == codes.device):
                raise ValueError("scales must be a contiguous float32 tensor [pages, heads] beside codes")
            if k is not None and (codes.shape != (k.shape[0], *k.shape[2:]) or codes.device != k.device):
                raise ValueError("codes must be [pages, heads, width] of k, on its device")
            c.codes, c.scales = codes.data_ptr(), scales.data_ptr()
        c.npages, c.nheads, c.head_dim = codes.shape if k is None else (k.shape[0], *k.shape[2:])
        c.page_size = self.page_size
        object.__setattr__(self, "device", (codes if k is None else k).device)
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "_sizes", (c.npages, c.page_size, c.nheads, c.head_dim, c.dtype))


@dataclass(frozen=True, eq=False)
class PagedCache4:
    """Keys and values in 4 bits: data uint8 [pages, heads, page size / 16, 18 width], a CUDA tensor whose last two axes are
    packed and whose strides are multiples of 16.  Width is 32, 64, 96 or 128; 9/16 byte a value.

    page_append codes what it writes (blocks of 16 columns share a scale: include/slnr.h), paged_attention reads the codes,
    page_values gives the values; what the bytes mean is the library's own.  Queries, keys and values may be bf16 or fp16,
    whichever wrote the cache.  The tensor is held, and read and written by the calls that take the cache."""
    data: torch.Tensor
    page_size: int = field(init=False)
    device: torch.device = field(init=False, repr=False)
    _c: slnr_cache4 = field(init=False, repr=False)
    _sizes: tuple = field(init=False, repr=False)

    def __post_init__(self):
        x = self.data
        if x.dim() != 4 or x.dtype != torch.uint8 or not x.is_cuda or x.shape[3] not in (576, 1152, 1728, 2304):
            raise ValueError("data must be a uint8 CUDA tensor [pages, heads, page size / 16, 18 width], width 32, 64, 96 or 128")
        if x.stride(3) != 1 or (x.shape[2] > 1 and x.stride(2) != x.shape[3]):
            raise ValueError("the last two axes of data must be packed")
        npages, heads, slabs, row = x.shape
        # an axis of one entry is never stepped along
        c = slnr_cache4(npages, 16 * slabs, heads, row // 18, x.stride(0) if npages > 1 else 0,
                        x.stride(1) if heads > 1 else 0, x.data_ptr())
        self.__dict__.update(page_size=16 * slabs, device=x.device, _c=c, _sizes=(npages, 16 * slabs, heads, row // 18))

    @classmethod
    def empty(cls, npages, page_size, heads, width, device="cuda"):
        """A cache of that many pages, slots of a page, heads and columns; its memory holds anything."""
        if page_size < 16 or page_size % 16:
            raise ValueError(f"page_size is {page_size}, not a multiple of 16")
        if width not in (32, 64, 96, 128):
            raise ValueError(f"width is {width}, not 32, 64, 96 or 128")
        return cls(torch.empty((npages, heads, page_size // 16, 18 * width), dtype=torch.uint8, device=device))


def _same_device(cache, tables, name):
    if tables.table.device != cache.device:
        raise ValueError(f"{name}: the tables are on {tables.table.device}, the cache is on {cache.device}")


def _rows(x, name, cache, heads, ntok, dtype=None):
    """slnr_rows of x [tokens, heads, width]: any strides that are multiples of 8 values, packed last axis."""
    shape, strides, dt = x.shape, x.stride(), x.dtype
    width = cache._c.head_dim
    if len(shape) != 3 or shape[0] != ntok or shape[2] != width or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} has shape {tuple(shape)}, not ({ntok}, {heads or 'heads'}, {width})")
    if x.device != cache.device or dt not in _TYPES or (dtype is not None and dt != dtype):
        raise ValueError(f"{name} must be {dtype or 'a bf16 or fp16 tensor'} on {cache.device}")
    if strides[2] != 1 and width > 1:
        raise ValueError(f"the last axis of {name} must be packed")
    return slnr_rows(x.data_ptr(), strides[0] if ntok > 1 else 0, strides[1] if shape[1] > 1 else 0)


def _empty(shape, dtype, device, stream):
    """An output: of the stream that it is written on, so that its memory is not given to others before."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _checked(out, name, shape, dtype, device):
    if out.shape != shape or out.dtype != dtype or out.device != device or not out.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {device}")
    return out


def _call(name, args, index, need, validate, workspace, stream, tensors):
    """Call entry point `name` on device `index` with `need` bytes of workspace (0: none)."""
    if index != _device_now():
        raise ValueError(f"{name}: the tensors are on cuda:{index}, the current device is {_device_now()}")
    if stream is None:
        s = _stream_now(index)
    else:
        s = stream.cuda_stream
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    if validate and need < 256:
        need = 256
    if need:
        capturing = torch.cuda.is_current_stream_capturing() if stream is None else _capturing(s)
        if workspace is None:
            workspace = (None if capturing else _default_ws.get((index, s))) or _new_workspace(index, s, capturing)
        # a call's launches follow one another on the stream: no other thread's come between them
        with getattr(workspace, "lock", _lock_of_others):
            buf = getattr(workspace, "buf", None)
            if capturing or buf is None or buf.numel() < need:
                buf, _ = _buffer(workspace, need, stream, capturing, lambda w, n: (w.get(n), None))
            _last_ws[0] = buf
            o = slnr_opts(0, 0, 1 if validate else 0, 0, s, buf.data_ptr(), buf.numel())
            status = getattr(lib(), name)(*args, _byref(o))
    else:
        status = getattr(lib(), name)(*args, _byref(slnr_opts(0, 0, 0, 0, s, None, 0)))
    if status != 0:
        raise SlnrError(status, name, last_error())


def page_tables(new_len, old_len, table, free_pages, page_size, ntok, max_q=None, max_k=None, validate=False,
                workspace=None, stream=None):
    """Block tables and slot maps from request lengths (slnr_page_tables): returns (PageTables, pages taken [1]).

    new_len, old_len [R]: new tokens, and keys already in the cache; free_pages: the pages to take from, in order; ntok
    = sum of new_len.  table [R, width] is written in place.  max_q and max_k go to the PageTables; the defaults, ntok and
    what a row of the table holds, are right for any lengths and wide for most (PageTables says what that costs): pass
    max_q=1 where each request has one new token at most, and the longest request's keys as max_k where they are known.
    Where free pages run out the entries and slots of -1 are kept silently (validate refuses them)."""
    R, width, stride = _table(table)
    dev, n = table.device, free_pages.shape[0]
    ints = _empty(2 * R + 2 + 2 * ntok, torch.int32, dev, stream)
    q_pos, k_len, used, req, slots = ints.split_with_sizes((R + 1, R, 1, ntok, ntok))
    at = ints.data_ptr()
    at_k, at_req = at + 4 * (R + 1), at + 4 * (2 * R + 2)
    at_slots = at_req + 4 * ntok
    _call("slnr_page_tables",
          (R, _ints(new_len, "new_len", (R,), dev), _ints(old_len, "old_len", (R,), dev), table.data_ptr(), stride, width,
           _ints(free_pages, "free_pages", (n,), dev), n, page_size, ntok, at, at_k, at_req, at_slots, at_req - 4),
          dev.index, 0, validate, workspace, stream, (new_len, old_len, table, free_pages))
    max_q, max_k = ntok if max_q is None else max_q, width * page_size if max_k is None else max_k
    c = slnr_pages(R, ntok, max_q, max_k, width, 0, stride, at, at_k, table.data_ptr(), at_req, at_slots)
    return PageTables._of(c, table=table, q_pos=q_pos, k_len=k_len, req=req, slots=slots, max_q=max_q, max_k=max_k), used


def page_append(cache: PagedCache | PagedCache4, tables: PageTables, k, v, validate=False, workspace=None, stream=None):
    """New keys and values [T, heads, width] to their slots, and the summaries of the pages that became full
    (slnr_page_append); the cache's tensors are written in place.  A PagedCache4 gets their codes (slnr_page_append4)."""
    if type(cache) is PagedCache4:
        return _append4(cache, tables, k, v, validate, workspace, stream)
    if cache.k is None or tables.slots is None:
        raise ValueError("page_append needs a cache with keys, and tables with slots")
    _same_device(cache, tables, "page_append")
    T, H, dt = tables.ntok, cache._c.nheads, cache.k.dtype
    args = (_byref(cache._c), _byref(tables._c), _byref(_rows(k, "k", cache, H, T, dt)),
            _byref(_rows(v, "v", cache, H, T, dt)))
    _call("slnr_page_append", args, cache.device.index, 0, validate and T > 0, workspace, stream,
          (cache.k, cache.v, cache.codes, cache.scales, k, v, *tables._tensors()))


def _append4(cache, tables, k, v, validate, workspace, stream):
    if tables.slots is None:
        raise ValueError("page_append needs tables with slots")
    _same_device(cache, tables, "page_append")
    T, H, dt = tables.ntok, cache._c.nheads, k.dtype
    args = (_byref(cache._c), _byref(tables._c), _byref(_rows(k, "k", cache, H, T)), _byref(_rows(v, "v", cache, H, T, dt)),
            _TYPES[dt])
    _call("slnr_page_append4", args, cache.device.index, 0, validate and T > 0, workspace, stream,
          (cache.data, k, v, *tables._tensors()))


def page_values(cache: PagedCache4, pages=None, dtype=torch.bfloat16, out=None, validate=False, workspace=None, stream=None):
    """The values that pages of a cache in 4 bits stand for (slnr_page_values4): (k, v), each [pages, slots, heads, width]
    of that type.  pages: int32 page numbers, of which those that are no pages give zeros (None: all).  out: (k, v)."""
    if type(cache) is not PagedCache4:
        raise ValueError("page_values needs a PagedCache4")
    if dtype not in _TYPES:
        raise ValueError("dtype must be bf16 or fp16")
    c, dev = cache._c, cache.device
    n = c.npages if pages is None else pages.shape[0] if pages.dim() == 1 else -1
    at = None if pages is None else _ints(pages, "pages", (n,), dev)
    shape = (n, c.page_size, c.nheads, c.head_dim)
    if out is None:
        k, v = _empty(shape, dtype, dev, stream), _empty(shape, dtype, dev, stream)
    else:
        k, v = (_checked(x, name, shape, dtype, dev) for x, name in zip(out, ("out k", "out v"), strict=True))
    _call("slnr_page_values4", (_byref(c), at, n, k.data_ptr(), v.data_ptr(), _TYPES[dtype]), dev.index, 0,
          validate and n > 0, workspace, stream, (cache.data, pages, k, v))
    return k, v


def page_select(q, cache: PagedCache, tables: PageTables, npicked, first=1, last=2, out=None, validate=False,
                workspace=None, stream=None):
    """Pages for each new token and key head by the cheap score (slnr_page_select): int32 [T, heads, npicked], ascending,
    -1 behind.  The first `first` pages and the last `last` are always among them."""
    if type(cache) is PagedCache4 or cache.codes is None:
        raise ValueError("page_select needs a cache with summaries")
    _same_device(cache, tables, "page_select")
    c, T = cache._c, tables.ntok
    if cache.k is None and q.dtype in _TYPES:
        c = slnr_cache.from_buffer_copy(c)
        c.dtype = _TYPES[q.dtype]
    rows = _rows(q, "q", cache, None, T, None if cache.k is None else cache.k.dtype)
    shape = (T, c.nheads, npicked)
    out = _empty(shape, torch.int32, cache.device, stream) if out is None else \
        _checked(out, "out", shape, torch.int32, cache.device)
    args = (_byref(rows), q.shape[1], _byref(c), _byref(tables._c), out.data_ptr(), npicked, first, last)
    _call("slnr_page_select", args, cache.device.index, 0, validate and T > 0, workspace, stream,
          (q, cache.codes, cache.scales, out, *tables._tensors()))
    return out


@functools.lru_cache(maxsize=4096)
def _attention_bytes(cache, pages, heads_q, npicked):
    """Workspace of an attention call: a function of the sizes alone."""
    c = slnr_cache(*cache)
    p = slnr_pages(*pages, 0, pages[-1])
    o = slnr_opts()
    args = (_byref(c), _byref(p), heads_q)
    if npicked:
        return _query("slnr_selected_attention_workspace", *args, npicked, _byref(o))
    return _query("slnr_paged_attention_workspace", *args, _byref(o))


@functools.lru_cache(maxsize=4096)
def _attention4_bytes(cache, pages, heads_q):
    """The same over a cache in 4 bits."""
    return _query("slnr_paged_attention4_workspace", _byref(slnr_cache4(*cache)), _byref(slnr_pages(*pages, 0, pages[-1])),
                  heads_q, _byref(slnr_opts()))


def _attention4(q, cache, tables, scale, out, lse, validate, workspace, stream):
    _same_device(cache, tables, "paged_attention")
    c, T, dtype, device = cache._c, tables.ntok, q.dtype, cache.device
    rows = _rows(q, "q", cache, None, T)
    shape = q.shape
    out = _empty(shape, dtype, device, stream) if out is None else _checked(out, "out", shape, dtype, device)
    lse = _empty(shape[:2], torch.float32, device, stream) if lse is None else \
        _checked(lse, "lse", shape[:2], torch.float32, device)
    need = _attention4_bytes(cache._sizes, tables._sizes, shape[1]) if T else 0
    args = (_byref(rows), shape[1], _byref(c), _byref(tables._c), _TYPES[dtype],
            c.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), lse.data_ptr())
    _call("slnr_paged_attention4", args, device.index, need, validate and T > 0, workspace, stream,
          (q, cache.data, out, lse, *tables._tensors()))
    return out, lse


def _attention(name, q, cache, tables, picked, npicked, scale, out, lse, validate, workspace, stream):
    if cache.k is None:
        raise ValueError(f"{name} needs a cache with keys")
    _same_device(cache, tables, name)
    c, p, T = cache._c, tables._c, tables.ntok
    dtype, device = q.dtype, cache.device
    rows = _rows(q, "q", cache, None, T, cache.k.dtype)
    shape = q.shape
    heads_q = shape[1]
    out = _empty(shape, dtype, device, stream) if out is None else _checked(out, "out", shape, dtype, device)
    lse = _empty(shape[:2], torch.float32, device, stream) if lse is None else \
        _checked(lse, "lse", shape[:2], torch.float32, device)
    # without tokens nothing is launched, and no flag word is written
    need = _attention_bytes(cache._sizes, tables._sizes, heads_q, npicked) if T else 0
    scale = c.head_dim ** -0.5 if scale is None else scale
    if npicked:
        args = (_byref(rows), heads_q, _byref(c), _byref(p), picked.data_ptr(), npicked, scale, out.data_ptr(),
                lse.data_ptr())
    else:
        args = (_byref(rows), heads_q, _byref(c), _byref(p), scale, out.data_ptr(), lse.data_ptr())
    _call(name, args, device.index, need, validate and T > 0, workspace, stream,
          (q, cache.k, cache.v, picked, out, lse, *tables._tensors()))
    return out, lse


def paged_attention(q, cache: PagedCache | PagedCache4, tables: PageTables, scale=None, out=None, lse=None, validate=False,
                    workspace=None, stream=None):
    """Causal attention of the new tokens q [T, query heads, width] over all pages of their requests
    (slnr_paged_attention): returns (out [T, query heads, width], lse fp32 [T, query heads]).  scale: width ** -0.5.
    Over a PagedCache4 (slnr_paged_attention4) q may be bf16 or fp16; out has its type."""
    if type(cache) is PagedCache4:
        return _attention4(q, cache, tables, scale, out, lse, validate, workspace, stream)
    return _attention("slnr_paged_attention", q, cache, tables, None, 0, scale, out, lse, validate, workspace, stream)


def selected_attention(q, cache: PagedCache, tables: PageTables, picked, scale=None, out=None, lse=None, validate=False,
                       workspace=None, stream=None):
    """paged_attention over the pages picked [T, heads, n] for each token and key head only (slnr_selected_attention)."""
    if type(cache) is PagedCache4:
        raise ValueError("selected_attention needs a 16-bit cache")
    n = picked.shape[-1] if picked.dim() == 3 else 0
    if n < 1:
        raise ValueError("picked must be [tokens, heads, pages], with one page at least")
    _ints(picked, "picked", (tables.ntok, cache._c.nheads, n), cache.device)
    return _attention("slnr_selected_attention", q, cache, tables, picked, n, scale, out, lse, validate, workspace, stream)


# ---- whole pages between the steps -----------------------------------------------------------

def _held_by(table, lens, page_size):
    """(arguments of the tables, device): the checks that page_fork, page_free and page_compact share."""
    R, width, stride = _table(table)
    if page_size < 1:
        raise ValueError(f"page_size is {page_size}")
    return R, width, stride, _ints(lens, "lens", (R,), table.device), table.device


def page_copy(cache: PagedCache | PagedCache4, src, dst, source=None, validate=False, workspace=None, stream=None):
    """Pages src[i] to pages dst[i] (int32 [n]): keys, values and summaries, or codes (slnr_page_copy, slnr_page_copy4).
    Entries of -1 are skipped.  No page may be in dst twice, nor in src and dst of one cache.  source: the cache that they
    are copied from (None: cache itself), of the same kind, page size, heads and width."""
    source = cache if source is None else source
    if type(source) is not type(cache):
        raise ValueError("cache and source must be of one kind")
    dev, n = cache.device, src.shape[0] if src.dim() == 1 else -1
    if source.device != dev:
        raise ValueError(f"page_copy: the source is on {source.device}, the cache is on {dev}")
    args = (_byref(cache._c), _byref(source._c), _ints(src, "src", (n,), dev), _ints(dst, "dst", (n,), dev), n)
    if type(cache) is PagedCache4:
        name, tensors = "slnr_page_copy4", (cache.data, source.data, src, dst)
    else:
        name = "slnr_page_copy"
        tensors = (cache.k, cache.v, cache.codes, cache.scales, source.k, source.v, source.codes, source.scales, src, dst)
    _call(name, args, dev.index, 0, validate and n > 0, workspace, stream, tensors)


def page_fork(table, lens, parent, free_pages, page_size, validate=False, workspace=None, stream=None):
    """Requests that go on from others (slnr_page_fork): child i from request parent[i] of table [R, width] and lens [R].

    Returns (table [n, width], lens [n], src [n], dst [n], pages needed [1]) of the children; the old table and lengths are
    not changed.  Full pages are shared; a last page that is not full stays with a parent's first child, and for the others
    page_copy(cache, src, dst) has to copy it, in every cache that the tables are of.  Some hundred children take 10 us of
    the GPU; of thousands with a parent each the time grows with their number squared (4096: 81 us, 65536: 43 ms)."""
    R, width, stride, at_lens, dev = _held_by(table, lens, page_size)
    n, nfree = parent.shape[0] if parent.dim() == 1 else -1, free_pages.shape[0]
    at_parent, at_free = _ints(parent, "parent", (n,), dev), _ints(free_pages, "free_pages", (nfree,), dev)
    cells = n * width
    ints = _empty(cells + 3 * n + 1, torch.int32, dev, stream)
    out, out_lens, src, dst, used = ints.split_with_sizes((cells, n, n, n, 1))
    at, row = ints.data_ptr(), 4 * n
    at_out = at + 4 * cells
    _call("slnr_page_fork", (R, at_lens, table.data_ptr(), stride, width, page_size, at_parent, n, at_free, nfree, at,
                             at_out, at_out + row, at_out + 2 * row, at_out + 3 * row),
          dev.index, 0, validate, workspace, stream, (table, lens, parent, free_pages))
    return out.view(n, width), out_lens, src, dst, used


def page_free(table, lens, npages, page_size, drop=None, validate=False, workspace=None, stream=None):
    """The pages that no request of table [R, width] and lens [R] holds (slnr_page_free): (free_pages [npages], ascending, -1
    behind them; how many [1]).  First lens is set to 0, in place, for the requests in drop (int32)."""
    R, width, stride, at_lens, dev = _held_by(table, lens, page_size)
    ndrop = 0 if drop is None else drop.shape[0] if drop.dim() == 1 else -1
    at_drop = None if drop is None else _ints(drop, "drop", (ndrop,), dev)
    if npages < 0:
        raise ValueError(f"npages is {npages}")
    ints = _empty(npages + 1, torch.int32, dev, stream)
    free_pages, count = ints.split_with_sizes((npages, 1))
    at = ints.data_ptr()
    _call("slnr_page_free", (R, at_lens, table.data_ptr(), stride, width, page_size, at_drop, ndrop, npages, at,
                             at + 4 * npages), dev.index, 0, validate, workspace, stream, (table, lens, drop))
    return free_pages, count


def page_compact(table, lens, npages, page_size, validate=False, workspace=None, stream=None):
    """The pages that requests hold to the front of a cache of npages (slnr_page_compact): (table [R, width] with the new
    numbers, src and dst [npages // 2], new number of each page [npages] or -1, pages in use [1]).  page_copy(cache, src,
    dst) has to make the copies in every cache that the tables are of; the old table is not changed."""
    R, width, stride, at_lens, dev = _held_by(table, lens, page_size)
    if npages < 0:
        raise ValueError(f"npages is {npages}")
    half = npages // 2
    cells = R * width
    ints = _empty(cells + 2 * half + npages + 1, torch.int32, dev, stream)
    out, src, dst, ids, used = ints.split_with_sizes((cells, half, half, npages, 1))
    at = ints.data_ptr()
    at_src = at + 4 * cells
    _call("slnr_page_compact", (R, at_lens, table.data_ptr(), stride, width, page_size, npages, at, at_src,
                                at_src + 4 * half, at_src + 8 * half, at_src + 8 * half + 4 * npages),
          dev.index, 0, validate, workspace, stream, (table, lens))
    return out.view(R, width), src, dst, ids, used
