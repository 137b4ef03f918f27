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

from . import (SlnrError, Workspace, _default_ws, _last_ws, _query, _stream_ptr, last_error, lib, slnr_cache, slnr_opts,
               slnr_pages, slnr_rows)

_TYPES = {torch.bfloat16: 0, torch.float16: 1}


def _ints(x, name, shape, device):
    """x's address, after its checks: an int32 CUDA tensor of that shape, contiguous."""
    if not (isinstance(x, torch.Tensor) and x.dtype == torch.int32 and x.device == device and x.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous int32 tensor on {device}")
    if tuple(x.shape) != shape:
        raise ValueError(f"{name} has shape {tuple(x.shape)}, not {shape}")
    return x.data_ptr()


@dataclass(frozen=True, eq=False)
class PageTables:
    """The requests of a step: their block tables, lengths, and each new token's request and slot (int32 CUDA tensors).

    table [R, width] (rows may be a slice of wider ones), q_pos [R + 1], k_len [R] (keys with the new tokens), req [T],
    slots [T] (page_append only).  max_q and max_k bound the new tokens and the keys of a request on the host; the work
    is laid out by them.  The tensors are held and read by each call that takes the tables.
    """
    table: torch.Tensor
    q_pos: torch.Tensor
    k_len: torch.Tensor
    req: torch.Tensor
    slots: Optional[torch.Tensor]
    max_q: int
    max_k: int
    _c: slnr_pages = field(init=False, repr=False)

    def __post_init__(self):
        t = self.table
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.int32 and t.dim() == 2
                and (t.shape[1] <= 1 or t.stride(1) == 1)):
            raise ValueError("table must be a 2-D int32 CUDA tensor with packed rows")
        R, width = t.shape
        T = self.req.shape[0]
        stride = t.stride(0) if R > 1 else width
        object.__setattr__(self, "_c", slnr_pages(
            R, T, self.max_q, self.max_k, width, 0, stride, _ints(self.q_pos, "q_pos", (R + 1,), t.device),
            _ints(self.k_len, "k_len", (R,), t.device), t.data_ptr(), _ints(self.req, "req", (T,), t.device),
            None if self.slots is None else _ints(self.slots, "slots", (T,), t.device)))

    @property
    def ntok(self) -> int:
        return self._c.ntok


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


def _rows(x, name, cache, heads, ntok, dtype=None):
    """slnr_rows of x [tokens, heads, width]: any strides that are multiples of 8 values, packed last axis."""
    c = cache._c
    if x.dim() != 3 or x.shape[0] != ntok or x.shape[2] != c.head_dim or (heads is not None and x.shape[1] != heads):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, not ({ntok}, {heads or 'heads'}, {c.head_dim})")
    if x.device != cache.device or x.dtype not in _TYPES or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"{name} must be {dtype or 'a bf16 or fp16 tensor'} on {cache.device}")
    if x.stride(2) != 1 and x.shape[2] > 1:
        raise ValueError(f"the last axis of {name} must be packed")
    return slnr_rows(x.data_ptr(), x.stride(0) if ntok > 1 else 0, x.stride(1) if x.shape[1] > 1 else 0)


def _empty(shape, dtype, device, stream):
    """An output: of the stream that it is written on, so that its memory is not given to others before."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _out(out, name, shape, dtype, device, stream):
    if out is None:
        return _empty(shape, dtype, device, stream)
    if tuple(out.shape) != shape or out.dtype != dtype or out.device != device or not out.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {device}")
    return out


def _call(name, args, device, need, validate, workspace, stream, tensors):
    """Call entry point `name` with `need` bytes of workspace (0: none)."""
    if device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: the tensors are on {device}, the current device is {torch.cuda.current_device()}")
    s = _stream_ptr(stream)
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    buf = None
    if validate and need < 256:
        need = 256
    if need:
        if workspace is None:
            workspace = _default_ws.get((device.index, s))
            if workspace is None:
                workspace = _default_ws.setdefault((device.index, s), Workspace(device=device))
        buf = getattr(workspace, "buf", None)
        if buf is None or buf.numel() < need:
            if stream is None:
                buf = workspace.get(need)
            else:
                with torch.cuda.stream(stream):
                    buf = workspace.get(need)
        _last_ws[0] = buf
    o = slnr_opts(0, 0, 1 if validate else 0, 0, s, None if buf is None else buf.data_ptr(),
                  0 if buf is None else buf.numel())
    status = getattr(lib(), name)(*args, ctypes.byref(o))
    if status != 0:
        raise SlnrError(status, name, last_error())


def page_tables(new_len, old_len, table, free_pages, page_size, ntok, max_q=None, max_k=None, validate=False,
                workspace=None, stream=None):
    """Block tables and slot maps from request lengths (slnr_page_tables): returns (PageTables, pages taken [1]).

    new_len, old_len [R]: new tokens, and keys already in the cache; free_pages: the pages to take from, in order; ntok
    = sum of new_len.  table [R, width] is written in place.  max_q and max_k go to the PageTables (defaults: ntok, and
    what a row of the table holds)."""
    dev = table.device
    if not (table.is_cuda and table.dtype == torch.int32 and table.dim() == 2
            and (table.shape[1] <= 1 or table.stride(1) == 1)):
        raise ValueError("table must be a 2-D int32 CUDA tensor with packed rows")
    R, width = table.shape
    ints = _empty(2 * R + 2 + 2 * ntok, torch.int32, dev, stream)
    q_pos, k_len, used = ints[:R + 1], ints[R + 1:2 * R + 1], ints[2 * R + 1:2 * R + 2]
    req, slots = ints[2 * R + 2:2 * R + 2 + ntok], ints[2 * R + 2 + ntok:]
    args = (R, _ints(new_len, "new_len", (R,), dev), _ints(old_len, "old_len", (R,), dev), table.data_ptr(),
            table.stride(0) if R > 1 else width, width, _ints(free_pages, "free_pages", tuple(free_pages.shape[:1]), dev),
            free_pages.shape[0], page_size, ntok, q_pos.data_ptr(), k_len.data_ptr(), req.data_ptr(), slots.data_ptr(),
            used.data_ptr())
    _call("slnr_page_tables", args, dev, 0, validate, workspace, stream, (new_len, old_len, table, free_pages))
    return PageTables(table, q_pos, k_len, req, slots, ntok if max_q is None else max_q,
                      width * page_size if max_k is None else max_k), used


def page_append(cache: PagedCache, tables: PageTables, k, v, validate=False, workspace=None, stream=None):
    """New keys and values [T, heads, width] to their slots, and the summaries of the pages that became full
    (slnr_page_append); the cache's tensors are written in place."""
    if cache.k is None or tables.slots is None:
        raise ValueError("page_append needs a cache with keys, and tables with slots")
    T, H, dt = tables.ntok, cache._c.nheads, cache.k.dtype
    args = (ctypes.byref(cache._c), ctypes.byref(tables._c), ctypes.byref(_rows(k, "k", cache, H, T, dt)),
            ctypes.byref(_rows(v, "v", cache, H, T, dt)))
    _call("slnr_page_append", args, cache.device, 0, validate, workspace, stream,
          (cache.k, cache.v, cache.codes, cache.scales, tables.slots, tables.req, tables.q_pos, k, v))


def page_select(q, cache: PagedCache, tables: PageTables, npicked, first=1, last=2, out=None, validate=False,
                workspace=None, stream=None):
    """Pages for each new token and key head by the cheap score (slnr_page_select): int32 [T, heads, npicked], ascending,
    -1 behind.  The first `first` pages and the last `last` are always among them."""
    if cache.codes is None:
        raise ValueError("page_select needs a cache with summaries")
    c, T = cache._c, tables.ntok
    if cache.k is None and q.dtype in _TYPES:
        c = slnr_cache.from_buffer_copy(c)
        c.dtype = _TYPES[q.dtype]
    rows = _rows(q, "q", cache, None, T, None if cache.k is None else cache.k.dtype)
    out = _out(out, "out", (T, c.nheads, npicked), torch.int32, cache.device, stream)
    args = (ctypes.byref(rows), q.shape[1], ctypes.byref(c), ctypes.byref(tables._c), out.data_ptr(), npicked, first, last)
    _call("slnr_page_select", args, cache.device, 0, validate, workspace, stream,
          (q, cache.codes, cache.scales, tables.table, tables.q_pos, tables.k_len, tables.req, out))
    return out


@functools.lru_cache(maxsize=4096)
def _attention_bytes(npages, page_size, heads, width, dtype, nreq, ntok, max_q, max_k, columns, heads_q, npicked):
    """Workspace of an attention call: a function of the sizes alone."""
    c = slnr_cache(npages, page_size, heads, width, dtype)
    p = slnr_pages(nreq, ntok, max_q, max_k, columns, 0, columns)
    o = slnr_opts()
    args = (ctypes.byref(c), ctypes.byref(p), heads_q)
    if npicked:
        return _query("slnr_selected_attention_workspace", *args, npicked, ctypes.byref(o))
    return _query("slnr_paged_attention_workspace", *args, ctypes.byref(o))


def _attention(name, q, cache, tables, picked, npicked, scale, out, lse, validate, workspace, stream):
    if cache.k is None:
        raise ValueError(f"{name} needs a cache with keys")
    c, p, T = cache._c, tables._c, tables.ntok
    rows = _rows(q, "q", cache, None, T, cache.k.dtype)
    heads_q = q.shape[1]
    shape = (T, heads_q, c.head_dim)
    need = _attention_bytes(c.npages, c.page_size, c.nheads, c.head_dim, c.dtype, p.nreq, T, p.max_q, p.max_k, p.width,
                            heads_q, npicked)
    out = _out(out, "out", shape, q.dtype, cache.device, stream)
    lse = _out(lse, "lse", shape[:2], torch.float32, cache.device, stream)
    scale = c.head_dim ** -0.5 if scale is None else scale
    head = (ctypes.byref(rows), heads_q, ctypes.byref(c), ctypes.byref(p))
    tail = (scale, out.data_ptr(), lse.data_ptr())
    mid = (picked.data_ptr(), npicked) if npicked else ()
    _call(name, (*head, *mid, *tail), cache.device, need, validate, workspace, stream,
          (q, cache.k, cache.v, tables.table, tables.q_pos, tables.k_len, tables.req, picked, out, lse))
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
