"""Attention over a paged key/value cache (include/slnr.h): block tables, the
cache's writes, pages picked by a cheap score, and attention over all pages or
the picked ones.

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
               last_error, lib, slnr_cache, slnr_opts, slnr_pages, slnr_rows)

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
    is laid out by them: a result does not depend on them, its time does.  One token over 4095 keys (32/8 heads of 128)
    takes 17 us of the GPU with max_k = 4095, 25 with 16384, 33 with 32768 and 52 with 131072; 64 single tokens over 581k
    keys 421 with max_q = 1 and 658 with max_q = 64 (as chunks), page_select for them 52 and 263.  A captured call keeps
    its bounds for every replay.  The tensors are held and read by each call that takes the tables.
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
    max_q=1 where each request has one new token at most, and the longest request's keys as max_k where they are known."""
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


def page_append(cache: PagedCache, tables: PageTables, k, v, validate=False, workspace=None, stream=None):
    """New keys and values [T, heads, width] to their slots, and the summaries of the pages that became full
    (slnr_page_append); the cache's tensors are written in place."""
    if cache.k is None or tables.slots is None:
        raise ValueError("page_append needs a cache with keys, and tables with slots")
    _same_device(cache, tables, "page_append")
    T, H, dt = tables.ntok, cache._c.nheads, cache.k.dtype
    args = (_byref(cache._c), _byref(tables._c), _byref(_rows(k, "k", cache, H, T, dt)),
            _byref(_rows(v, "v", cache, H, T, dt)))
    _call("slnr_page_append", args, cache.device.index, 0, validate and T > 0, workspace, stream,
          (cache.k, cache.v, cache.codes, cache.scales, k, v, *tables._tensors()))


def page_select(q, cache: PagedCache, tables: PageTables, npicked, first=1, last=2, out=None, validate=False,
                workspace=None, stream=None):
    """Pages for each new token and key head by the cheap score (slnr_page_select): int32 [T, heads, npicked], ascending,
    -1 behind.  The first `first` pages and the last `last` are always among them."""
    if cache.codes is None:
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


def paged_attention(q, cache: PagedCache, tables: PageTables, scale=None, out=None, lse=None, validate=False,
                    workspace=None, stream=None):
    """Causal attention of the new tokens q [T, query heads, width] over all pages of their requests
    (slnr_paged_attention): returns (out [T, query heads, width], lse fp32 [T, query heads]).  scale: width ** -0.5."""
    return _attention("slnr_paged_attention", q, cache, tables, None, 0, scale, out, lse, validate, workspace, stream)


def selected_attention(q, cache: PagedCache, tables: PageTables, picked, scale=None, out=None, lse=None, validate=False,
                       workspace=None, stream=None):
    """paged_attention over the pages picked [T, heads, n] for each token and key head only (slnr_selected_attention)."""
    n = picked.shape[-1] if picked.dim() == 3 else 0
    if n < 1:
        raise ValueError("picked must be [tokens, heads, pages], with one page at least")
    _ints(picked, "picked", (tables.ntok, cache._c.nheads, n), cache.device)
    return _attention("slnr_selected_attention", q, cache, tables, picked, n, scale, out, lse, validate, workspace, stream)
