// C entry points of the paged cache (declared in include/slnr.h): argument
// checks, workspace layout and launches.
#include <cmath>
#include <utility>

#include "cache4.cuh"
#include "call.h"
#include "launch.h"
#include "page_sets.cuh"
#include "paged.cuh"
#include "paged4.cuh"

using namespace slnr;

namespace {

constexpr int kMaxWidth = 128;
constexpr int kMaxKeys = 0x7fff0000;  // whole pages of a request, and steps past its last key, stay below 2^31

slnr_status check_paged_opts(const slnr_opts* o) {
  if (!o) return fail(SLNR_ERR_NULL, "opts is NULL");
  if (o->reserved != 0) return fail(SLNR_ERR_UNSUPPORTED, "opts.reserved must be 0");
  return SLNR_OK;
}

slnr_status check_strides(const char* what, const int64_t* s, int n) {
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || s[i] % 8 != 0)
      return fail(SLNR_ERR_UNSUPPORTED, "%s: stride %lld must be a multiple of 8 values", what, (long long)s[i]);
  return SLNR_OK;
}

// need: the call reads or writes keys and values; else their pointers and strides are not looked at.
slnr_status check_cache(const slnr_cache* c, bool keys, bool summary, bool pointers) {
  if (!c) return fail(SLNR_ERR_NULL, "cache is NULL");
  if (c->reserved != 0) return fail(SLNR_ERR_UNSUPPORTED, "cache.reserved must be 0");
  if (c->npages < 0 || c->page_size <= 0 || c->nheads <= 0 || c->head_dim <= 0)
    return fail(SLNR_ERR_SHAPE, "cache of %d pages of %d slots, %d heads, width %d", (int)c->npages, (int)c->page_size,
                (int)c->nheads, (int)c->head_dim);
  if ((int64_t)c->npages * c->page_size >= (int64_t(1) << 31))
    return fail(SLNR_ERR_UNSUPPORTED, "the cache must have fewer than 2^31 slots");
  if (c->head_dim % 8 != 0 || c->head_dim > kMaxWidth)
    return fail(SLNR_ERR_UNSUPPORTED, "head_dim = %d: must be a multiple of 8 in [8, %d]", (int)c->head_dim, kMaxWidth);
  if (c->nheads > 65535) return fail(SLNR_ERR_UNSUPPORTED, "nheads = %d: at most 65535", (int)c->nheads);
  if (c->dtype != SLNR_BF16 && c->dtype != SLNR_FP16)
    return fail(SLNR_ERR_UNSUPPORTED, "unknown type %d", (int)c->dtype);
  if (keys) {
    SLNR_CHECK(check_strides("cache.k", c->k_stride, 3));
    SLNR_CHECK(check_strides("cache.v", c->v_stride, 3));
    if (pointers && c->npages > 0) {
      if (!c->k || !c->v) return fail(SLNR_ERR_NULL, "cache.k or cache.v is NULL");
      if (!aligned16(c->k) || !aligned16(c->v))
        return fail(SLNR_ERR_UNSUPPORTED, "cache.k and cache.v must be 16-byte aligned");
    }
  }
  if (summary && c->npages > 0 && pointers) {
    if (!c->codes || !c->scales) return fail(SLNR_ERR_NULL, "cache.codes or cache.scales is NULL");
    if (!aligned16(c->codes)) return fail(SLNR_ERR_UNSUPPORTED, "cache.codes must be 16-byte aligned");
  }
  return SLNR_OK;
}

slnr_status check_pages(const slnr_pages* p, const slnr_cache* c, bool pointers, bool req, bool slots) {
  if (!p) return fail(SLNR_ERR_NULL, "pages is NULL");
  if (p->reserved != 0) return fail(SLNR_ERR_UNSUPPORTED, "pages.reserved must be 0");
  if (p->max_k > 0 && ceil_div(p->max_k, c->page_size) * c->page_size > kMaxKeys)
    return fail(SLNR_ERR_UNSUPPORTED, "max_k = %d: at most %d in whole pages", (int)p->max_k, kMaxKeys);
  if (p->nreq < 0 || p->ntok < 0 || p->max_q < 0 || p->max_k < 0 || p->width < 0 || p->table_stride < p->width)
    return fail(SLNR_ERR_SHAPE, "negative size in pages, or rows of table that overlap");
  if ((int64_t)p->max_k > (int64_t)p->width * c->page_size)
    return fail(SLNR_ERR_SHAPE, "max_k = %d, but a row of table holds %lld keys", (int)p->max_k,
                (long long)p->width * c->page_size);
  if (p->ntok > 0 && (p->nreq == 0 || p->max_q == 0)) return fail(SLNR_ERR_SHAPE, "tokens without a request");
  if (pointers && p->ntok > 0) {
    if (!p->q_pos || !p->k_len || (p->width > 0 && !p->table)) return fail(SLNR_ERR_NULL, "an array of pages is NULL");
    if (req && !p->req) return fail(SLNR_ERR_NULL, "pages.req is NULL");
    if (slots && !p->slots) return fail(SLNR_ERR_NULL, "pages.slots is NULL");
  }
  return SLNR_OK;
}

slnr_status check_rows(const char* what, const slnr_rows* r, bool any) {
  if (!r) return fail(SLNR_ERR_NULL, "%s is NULL", what);
  const int64_t s[2] = {r->stride_tok, r->stride_head};
  SLNR_CHECK(check_strides(what, s, 2));
  if (any && !r->p) return fail(SLNR_ERR_NULL, "%s is NULL", what);
  if (!aligned16(r->p)) return fail(SLNR_ERR_UNSUPPORTED, "%s must be 16-byte aligned", what);
  return SLNR_OK;
}

slnr_status check_heads(const slnr_cache* c, int32_t nheads_q) {
  if (nheads_q <= 0 || nheads_q % c->nheads != 0)
    return fail(SLNR_ERR_SHAPE, "%d query heads over %d key heads", (int)nheads_q, (int)c->nheads);
  return SLNR_OK;
}

PagesView view(const slnr_pages& p) {
  return PagesView{p.nreq, p.ntok, p.width, p.max_q, p.max_k, p.table_stride, p.q_pos, p.k_len, p.table, p.req, p.slots};
}

CacheView view(const slnr_cache& c) {
  CacheView v{c.k, c.v, {}, {}, c.npages, c.nheads, c.head_dim, divisor(c.page_size), c.codes, c.scales};
  for (int i = 0; i < 3; ++i) {
    v.ks[i] = c.k_stride[i];
    v.vs[i] = c.v_stride[i];
  }
  return v;
}

RowsView view(const slnr_rows& r) { return RowsView{r.p, r.stride_tok, r.stride_head}; }

// Validate mode: the device check, and its flag word.
template <typename Launch>
slnr_status validated(const slnr_opts* o, Launch launch) {
  if (!o->validate) return SLNR_OK;
  SLNR_CHECK(check_ws(o, sizeof(WsHeader)));
  cudaStream_t s = (cudaStream_t)o->stream;
  WsHeader* hdr = (WsHeader*)o->workspace;
  SLNR_CUDA(cudaMemsetAsync(hdr, 0, sizeof(WsHeader), s));
  SLNR_CUDA(launch(hdr, s));
  int flag = 0;
  SLNR_CUDA(cudaMemcpyAsync(&flag, &hdr->error, sizeof(int), cudaMemcpyDeviceToHost, s));
  SLNR_CUDA(cudaStreamSynchronize(s));
  if (flag != 0) return fail(SLNR_ERR_INDEX, "malformed lengths, tables or slots (flags 0x%x)", flag);
  return SLNR_OK;
}

slnr_status check_type(int32_t dtype) {
  if (dtype != SLNR_BF16 && dtype != SLNR_FP16) return fail(SLNR_ERR_UNSUPPORTED, "unknown type %d", (int)dtype);
  return SLNR_OK;
}

// The sizes of a cache in 4 bits, for the checks that want no more.
slnr_cache sizes(const slnr_cache4& c) {
  slnr_cache s{};
  s.npages = c.npages;
  s.page_size = c.page_size;
  s.nheads = c.nheads;
  s.head_dim = c.head_dim;
  return s;
}

slnr_status check_cache4(const slnr_cache4* c, bool pointers) {
  if (!c) return fail(SLNR_ERR_NULL, "cache is NULL");
  const slnr_cache s = sizes(*c);
  SLNR_CHECK(check_cache(&s, false, false, false));
  if (c->head_dim % 32 != 0)
    return fail(SLNR_ERR_UNSUPPORTED, "head_dim = %d: 32, 64, 96 or 128 in 4 bits", (int)c->head_dim);
  if (c->page_size % kSlab != 0)
    return fail(SLNR_ERR_UNSUPPORTED, "page_size = %d: a multiple of %d in 4 bits", (int)c->page_size, kSlab);
  if (c->page_stride < 0 || c->page_stride % 16 != 0 || c->head_stride < 0 || c->head_stride % 16 != 0)
    return fail(SLNR_ERR_UNSUPPORTED, "cache strides %lld and %lld must be multiples of 16 bytes",
                (long long)c->page_stride, (long long)c->head_stride);
  if (pointers && c->npages > 0) {
    if (!c->data) return fail(SLNR_ERR_NULL, "cache.data is NULL");
    if (!aligned16(c->data)) return fail(SLNR_ERR_UNSUPPORTED, "cache.data must be 16-byte aligned");
  }
  return SLNR_OK;
}

Cache4View view(const slnr_cache4& c) {
  return Cache4View{(uint8_t*)c.data, c.page_stride, c.head_stride, c.npages, c.nheads, c.head_dim, divisor(c.page_size)};
}

// What slnr_page_fork, _free and _compact are given of the requests.
slnr_status check_tables(int32_t nreq, const int32_t* lens, const int32_t* table, int64_t table_stride, int32_t width,
                         int32_t page_size, const slnr_opts* opts) {
  SLNR_CHECK(check_paged_opts(opts));
  if (nreq < 0 || width < 0 || table_stride < width)
    return fail(SLNR_ERR_SHAPE, "negative size, or rows of table that overlap");
  if (page_size <= 0) return fail(SLNR_ERR_SHAPE, "page_size = %d must be positive", (int)page_size);
  if (nreq > 0 && (!lens || (width > 0 && !table))) return fail(SLNR_ERR_NULL, "lens or table is NULL");
  return SLNR_OK;
}

slnr_status check_set(int32_t npages) {
  if (npages < 0) return fail(SLNR_ERR_SHAPE, "npages = %d", (int)npages);
  if (npages > kMaxSetPages)
    return fail(SLNR_ERR_UNSUPPORTED, "npages = %d: at most %d", (int)npages, kMaxSetPages);
  return SLNR_OK;
}

slnr_status check_copy(const int32_t* src, const int32_t* dst, int32_t n, const slnr_opts* opts) {
  SLNR_CHECK(check_paged_opts(opts));
  if (n < 0) return fail(SLNR_ERR_SHAPE, "n = %d", (int)n);
  if (n > 0 && (!src || !dst)) return fail(SLNR_ERR_NULL, "src or dst is NULL");
  return SLNR_OK;
}

// Adds a tensor of outer x inner rows of `row` bytes a page.  False: too many units for an int.
bool add_part(CopyParts& c, const void* from, void* to, const int64_t (&f)[3], const int64_t (&t)[3], int64_t outer,
              int64_t inner, int64_t row, int unit) {
  const int64_t pieces = outer * inner * (row / unit);
  if (pieces > INT32_MAX - kCopyItem) return false;
  CopyPart& a = c.part[c.n++];
  a = CopyPart{(const char*)from, (char*)to, f[0], t[0], f[1], t[1], f[2], t[2], divisor((int)inner),
               divisor((int)(row / unit)), unit, (int)pieces, c.items};
  const int64_t items = c.items + (pieces + kCopyItem - 1) / kCopyItem;
  c.items = (int)items;
  return items <= INT32_MAX;
}

slnr_status copy_pages(const CopyParts& c, const int32_t* src, const int32_t* dst, int32_t n, int32_t from_pages,
                       int32_t to_pages, const slnr_opts* opts) {
  cudaStream_t s = (cudaStream_t)opts->stream;
  const TablesView none{0, 0, 0, divisor(1), nullptr, nullptr};
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_set(none, 0, src, n, from_pages, dst, to_pages, hdr, st);
  }));
  SLNR_LAUNCH("page_copy", launch_page_copy(c, src, dst, n, from_pages, to_pages, s));
  timing_end(s);
  return SLNR_OK;
}

constexpr int64_t kSms = 152;          // of one block of the tensor-core kernel, two of the row kernel's
constexpr int64_t kMaxBlocks = 16384;  // splits stop here
constexpr int64_t kMaxCluster = 16;
constexpr int64_t kManyKeys = 1 << 19;

// Whether picked pages go to the tensor-core kernel: steps of 128 keys are whole
// pages or parts of one.
bool whole_steps(int page) { return page >= kChunkKeys ? page % kChunkKeys == 0 : page >= 16 && kChunkKeys % page == 0; }

// Row tiles and key splits of an attention call: by the bounds alone, never by
// device data.  Calls with a request of more than 64 rows go to the tensor-core
// kernel (256 rows a block), the others to the row kernel; with picked pages its
// blocks take the rows of one token.  From 33 to 64 rows the tensor-core kernel
// also takes calls of many keys over all requests and key heads (us, key heads of
// 128, 64 rows, row kernel and tensor-core kernel): 64 requests of 4096 keys, 8
// heads, 408 and 294; 8 of 8192, 108 and 95; 32 of 1024, 58 and 57; but 1 of 32768
// 57 and 69, 1 of 4096 28 and 32, where its longer way through a step shows.  With
// 32 rows it has no such call (276 and 288).  A call whose bounds are wider than its
// requests is taken by the bounds: single tokens with max_q = 64 as chunks, 658 us
// where max_q = 1 takes 421, and few keys with a wide max_k in few splits, one
// request of 4095 keys 17 us with max_k = 4095, 33 with 32768.
AttnPlan attn_plan(const slnr_cache& c, const slnr_pages& p, int32_t nheads_q, int32_t npicked) {
  AttnPlan a{};
  const int64_t G = nheads_q / c.nheads, requests = p.nreq < p.ntok ? p.nreq : p.ntok;
  a.nsplit = 1;
  const bool many = p.max_q * G > 32 && npicked == 0 && (int64_t)p.nreq * c.nheads * p.max_k >= kManyKeys;
  if ((p.max_q * G > 64 || many) && (npicked == 0 || whole_steps(c.page_size))) {
    a.tile = kChunkRows;
    const int64_t tiles = p.ntok * G / a.tile + requests;
    a.ntiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
    if (npicked > 0) {
      const int64_t most = kChunkRows % G == 0 ? kChunkRows / G : (kChunkRows - 1) / G + 2;  // tokens of a tile
      const int64_t pages = ceil_div(p.max_k > 0 ? p.max_k : 1, c.page_size);
      a.words = (int)ceil_div(most < kChunkRows ? most : kChunkRows, 32);
      a.cap = (int)(pages < most * npicked ? pages : most * npicked);
    }
    return a;
  }
  const int64_t rows = npicked > 0 ? G : p.max_q * G;
  a.tile = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  const int64_t tiles = npicked > 0 ? p.ntok * ceil_div(G, a.tile) : p.nreq;
  const int64_t keys = npicked > 0 ? (int64_t)npicked * c.page_size : p.max_k;
  const int64_t blocks = tiles * c.nheads;
  int64_t chunk = keys;
  if (blocks > 0) {
    const int64_t want = 2 * kSms / blocks;
    chunk = ceil_div(keys, want > 1 ? want : 1);
    if (chunk < 128) chunk = 128;
    if (npicked == 0 && chunk > 2048) chunk = 2048;  // requests of other lengths beside the longest
    const int64_t least = ceil_div(keys * blocks, kMaxBlocks);
    if (chunk < least) chunk = least;
  }
  // Where all splits run at once and there are few of them, they are the blocks
  // of a cluster (a power of two): no second launch.  A larger call would keep
  // the blocks of short requests waiting for those of long ones.
  if (chunk < keys) {
    int64_t n = 2;
    while (n < kMaxCluster && n * chunk < keys) n *= 2;
    if (blocks * n <= 2 * kSms && keys <= n * (chunk > 512 ? chunk : 512)) {
      chunk = ceil_div(keys, n);
      a.cluster = true;
      a.nsplit = (int)n;
    }
  }
  chunk = ceil_div(chunk > 0 ? chunk : 1, kAttnKeys) * kAttnKeys;
  a.ntiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
  a.chunk = (int)chunk;
  if (!a.cluster) a.nsplit = keys > 0 ? (int)ceil_div(keys, chunk) : 1;
  return a;
}

// Workspace of an attention call after the header: partial rows, and the pages
// that row tiles picked.
struct AttnLayout {
  size_t part, ml, tiles, before, shares, pages, pickers, npages, total;
};
AttnLayout attn_layout(const slnr_cache& c, const slnr_pages& p, int32_t nheads_q, const AttnPlan& a) {
  AttnLayout l;
  size_t cur = sizeof(WsHeader);
  const auto take = [&cur](size_t bytes) {
    const size_t at = align256(cur);
    cur = at + bytes;
    return at;
  };
  const bool tc = a.tile == kChunkRows;
  const size_t rows = tc ? (size_t)2 * kChunkBlocks * kChunkRows
                         : a.nsplit > 1 && !a.cluster ? (size_t)p.ntok * nheads_q * a.nsplit : 0;
  const size_t items = tc ? (size_t)a.ntiles * c.nheads : 0, lists = a.cap > 0 ? items : 0;
  l.part = take(rows * c.head_dim * sizeof(float));
  l.ml = take(rows * sizeof(float2));
  l.tiles = take(tc ? (size_t)a.ntiles * 2 * sizeof(int4) : 0);
  l.before = take(items * sizeof(int64_t));
  l.shares = take(tc ? (kChunkBlocks + 2) * sizeof(int2) : 0);
  l.pages = take(lists * a.cap * sizeof(int32_t));
  l.pickers = take(lists * a.cap * a.words * sizeof(uint32_t));
  l.npages = take(lists * sizeof(int32_t));
  l.total = align256(cur);
  return l;
}

void place(AttnPlan& a, const AttnLayout& l, char* ws) {
  a.part = (float*)(ws + l.part);
  a.part_ml = (float2*)(ws + l.ml);
  a.tiles = (int4*)(ws + l.tiles);
  a.before = (int64_t*)(ws + l.before);
  a.shares = (int2*)(ws + l.shares);
  a.pages = (int32_t*)(ws + l.pages);
  a.pickers = (uint32_t*)(ws + l.pickers);
  a.npages = (int32_t*)(ws + l.npages);
}

slnr_status attention_workspace(const slnr_cache* cache, const slnr_pages* pages, int32_t nheads_q, int32_t npicked,
                                const slnr_opts* opts, size_t* bytes) {
  if (!bytes) return fail(SLNR_ERR_NULL, "bytes is NULL");
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache(cache, true, false, false));
  SLNR_CHECK(check_pages(pages, cache, false, true, false));
  SLNR_CHECK(check_heads(cache, nheads_q));
  *bytes = attn_layout(*cache, *pages, nheads_q, attn_plan(*cache, *pages, nheads_q, npicked)).total;
  return SLNR_OK;
}

slnr_status attention(const slnr_rows* q, int32_t nheads_q, const slnr_cache* cache, const slnr_pages* pages,
                      const int32_t* picked, int32_t npicked, float scale, void* out, float* lse,
                      const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache(cache, true, false, true));
  SLNR_CHECK(check_pages(pages, cache, true, true, false));
  SLNR_CHECK(check_heads(cache, nheads_q));
  SLNR_CHECK(check_rows("q", q, pages->ntok > 0));
  if (!std::isfinite(scale)) return fail(SLNR_ERR_SHAPE, "scale must be finite");
  if (pages->ntok == 0) return SLNR_OK;
  if (!out) return fail(SLNR_ERR_NULL, "out is NULL");
  if (!aligned16(out)) return fail(SLNR_ERR_UNSUPPORTED, "out must be 16-byte aligned");
  AttnArgs a{view(*pages), view(*cache), view(*q), divisor(nheads_q / cache->nheads), scale, out, lse, picked, npicked,
             attn_plan(*cache, *pages, nheads_q, npicked)};
  // Blocks of a launch and rows of a request are counted in ints: row tiles (times key heads on the tensor cores, where
  // they are items), splits (a grid's third axis).  Rows with splits to join are few: see attn_plan.
  const bool tc = a.plan.tile == kChunkRows;
  if (a.plan.nsplit > 65535 || a.plan.ntiles == INT32_MAX ||
      (tc && (int64_t)a.plan.ntiles * cache->nheads > kMaxKeys) ||
      (int64_t)pages->max_q * a.group.d >= (int64_t(1) << 31) || (int64_t)npicked * cache->page_size > kMaxKeys)
    return fail(SLNR_ERR_UNSUPPORTED, "too many rows or keys for one call");
  const AttnLayout l = attn_layout(*cache, *pages, nheads_q, a.plan);
  SLNR_CHECK(check_ws(opts, l.total));
  char* ws = (char*)opts->workspace;
  place(a.plan, l, ws);
  cudaStream_t s = (cudaStream_t)opts->stream;
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_pages(a.p, a.c.npages, a.c.page, false, picked, npicked, a.c.nheads, hdr, st);
  }));
  if (tc) {
    SLNR_LAUNCH("paged_plan", launch_paged_plan(a, (WsHeader*)ws, s));
    SLNR_LAUNCH("paged_chunk", launch_paged_chunk(a, cache->dtype, (WsHeader*)ws, s));
    SLNR_LAUNCH("paged_join", launch_paged_join(a, cache->dtype, s));
  } else {
    SLNR_LAUNCH("paged_rows", launch_paged_rows(a, cache->dtype, (WsHeader*)ws, s));
  }
  if (a.plan.nsplit > 1 && !a.plan.cluster) SLNR_LAUNCH("paged_combine", launch_paged_combine(a, cache->dtype, s));
  timing_end(s);
  if (tc && opts->validate) {
    int flag = 0;
    SLNR_CUDA(cudaMemcpyAsync(&flag, &((WsHeader*)ws)->error, sizeof(int), cudaMemcpyDeviceToHost, s));
    SLNR_CUDA(cudaStreamSynchronize(s));
    if (flag != 0) return fail(SLNR_ERR_TIMEOUT, "a bounded device-side wait gave up (flags 0x%x)", flag);
  }
  return SLNR_OK;
}

// Attention over a cache in 4 bits: calls whose bound max_q allows more than 32 query rows
// of a key head go to the tensor-core kernel, the others to the row kernel, which has
// registers for no more.  Up to there it is the faster one, whatever the number of requests
// and keys (us a call by the row kernel and by the other, 32/8 heads of 128; 4, 16 and 32 rows
// of each request: 1 request of 4096 keys 15, 17, 24 and 34-35; 1 of 32768 25, 27, 39 and 61-64;
// 64 of 9000 125, 184, 290 and 517-520; 256 of 600 57, 93, 160 and 196-197).
AttnPlan attn4_chunk_plan(const slnr_pages& p, int64_t group) {
  AttnPlan a{};
  const int64_t requests = p.nreq < p.ntok ? p.nreq : p.ntok, tiles = p.ntok * group / kChunkRows + requests;
  a.nsplit = 1;
  a.tile = kChunkRows;
  a.ntiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
  return a;
}

bool rows4(const slnr_pages& p, int64_t group) { return p.max_q * group <= 32; }

// Of the row kernel: rows of an item, blocks, units of a block's share at least, and
// its workspace after the header.  A unit is 32 keys, of which a block's four warps take
// one each; long requests are cut into fewer shares, as each is one more part to join (us
// of the GPU with 4, 8, 12 units: 500 keys of 8 heads 8.8, 9.5, 12.7; 4095 of 8 11.9,
// 10.9, 13.5; 32768 of one head, 16 rows, 32.2, 22.7, 19.7).
struct Rows4Layout {
  int tile, rows, nblocks, least;
  size_t shares, part, ml, total;
};
Rows4Layout rows4_layout(const slnr_cache& c, const slnr_pages& p, int64_t group) {
  Rows4Layout l;
  l.rows = (int)(p.max_q * group);
  l.tile = l.rows <= 8 ? 8 : l.rows <= 16 ? 16 : 32;
  l.nblocks = paged4_blocks(c.head_dim, l.tile, l.rows);
  l.least = p.max_k <= 2048 ? 4 : p.max_k <= 16384 ? 8 : 16;
  l.shares = align256(sizeof(WsHeader));
  l.part = align256(l.shares + (l.nblocks + 1) * sizeof(int4));
  l.ml = align256(l.part + (size_t)2 * l.nblocks * l.tile * c.head_dim * sizeof(float));
  l.total = align256(l.ml + (size_t)2 * l.nblocks * l.tile * sizeof(float2));
  return l;
}

slnr_status attention4(const slnr_rows* q, int32_t nheads_q, const slnr_cache4* cache, const slnr_pages* pages,
                       int32_t dtype, float scale, void* out, float* lse, const slnr_opts* opts) {
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache4(cache, true));
  SLNR_CHECK(check_type(dtype));
  const slnr_cache shape = sizes(*cache);
  SLNR_CHECK(check_pages(pages, &shape, true, true, false));
  SLNR_CHECK(check_heads(&shape, nheads_q));
  SLNR_CHECK(check_rows("q", q, pages->ntok > 0));
  if (!std::isfinite(scale)) return fail(SLNR_ERR_SHAPE, "scale must be finite");
  if (pages->ntok == 0) return SLNR_OK;
  if (!out) return fail(SLNR_ERR_NULL, "out is NULL");
  if (!aligned16(out)) return fail(SLNR_ERR_UNSUPPORTED, "out must be 16-byte aligned");
  const Divisor group = divisor(nheads_q / cache->nheads);
  const Cache4View c4 = view(*cache);
  const PagesView p = view(*pages);
  cudaStream_t s = (cudaStream_t)opts->stream;
  char* ws = (char*)opts->workspace;
  WsHeader* hdr = (WsHeader*)ws;
  const auto check = [&](WsHeader* h, cudaStream_t st) {
    return launch_validate_pages(p, c4.npages, c4.slots, false, nullptr, 0, 0, h, st);
  };
  if (rows4(*pages, group.d)) {
    const Rows4Layout l = rows4_layout(shape, *pages, group.d);
    SLNR_CHECK(check_ws(opts, l.total));
    SLNR_CHECK(validated(opts, check));
    const Attn4Args a{p, c4, view(*q), group, scale, out, lse, l.tile, l.rows, l.nblocks, l.least, (int4*)(ws + l.shares),
                      (float*)(ws + l.part), (float2*)(ws + l.ml)};
    SLNR_LAUNCH("paged4_rows", launch_paged4_rows(a, dtype, s));
    SLNR_LAUNCH("paged4_join", launch_paged4_join(a, dtype, hdr, s));
  } else {
    AttnArgs a{p, view(shape), view(*q), group, scale, out, lse, nullptr, 0, attn4_chunk_plan(*pages, group.d), c4};
    if (a.plan.ntiles == INT32_MAX || (int64_t)a.plan.ntiles * cache->nheads > kMaxKeys ||
        (int64_t)pages->max_q * group.d >= (int64_t(1) << 31))
      return fail(SLNR_ERR_UNSUPPORTED, "too many rows or keys for one call");
    const AttnLayout l = attn_layout(shape, *pages, nheads_q, a.plan);
    SLNR_CHECK(check_ws(opts, l.total));
    place(a.plan, l, ws);
    SLNR_CHECK(validated(opts, check));
    SLNR_LAUNCH("paged_plan", launch_paged_plan(a, hdr, s));
    SLNR_LAUNCH("paged4_chunk", launch_paged_chunk(a, dtype, hdr, s));
    SLNR_LAUNCH("paged_join", launch_paged_join(a, dtype, s));
  }
  timing_end(s);
  if (opts->validate) {
    int flag = 0;
    SLNR_CUDA(cudaMemcpyAsync(&flag, &hdr->error, sizeof(int), cudaMemcpyDeviceToHost, s));
    SLNR_CUDA(cudaStreamSynchronize(s));
    if (flag != 0) return fail(SLNR_ERR_TIMEOUT, "a bounded device-side wait gave up (flags 0x%x)", flag);
  }
  return SLNR_OK;
}

}  // namespace

extern "C" {

slnr_status slnr_page_tables(int32_t nreq, const int32_t* new_len, const int32_t* old_len, int32_t* table,
                             int64_t table_stride, int32_t width, const int32_t* free_pages, int32_t nfree,
                             int32_t page_size, int32_t ntok, int32_t* q_pos, int32_t* k_len, int32_t* req,
                             int32_t* slots, int32_t* used, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  if (nreq < 0 || ntok < 0 || width < 0 || nfree < 0 || table_stride < width)
    return fail(SLNR_ERR_SHAPE, "negative size, or rows of table that overlap");
  if (page_size <= 0) return fail(SLNR_ERR_SHAPE, "page_size = %d must be positive", (int)page_size);
  if (!q_pos || !used) return fail(SLNR_ERR_NULL, "q_pos or used is NULL");
  if (nreq > 0 && (!new_len || !old_len || !k_len || (width > 0 && !table)))
    return fail(SLNR_ERR_NULL, "an array of the requests is NULL");
  if (ntok > 0 && (!req || !slots)) return fail(SLNR_ERR_NULL, "req or slots is NULL");
  if (nfree > 0 && !free_pages) return fail(SLNR_ERR_NULL, "free_pages is NULL");
  cudaStream_t s = (cudaStream_t)opts->stream;
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_lengths(nreq, new_len, old_len, table, table_stride, width, nfree, page_size, ntok, hdr, st);
  }));
  SLNR_LAUNCH("page_tables", launch_page_tables(nreq, new_len, old_len, table, table_stride, width, free_pages, nfree,
                                               page_size, ntok, q_pos, k_len, req, slots, used, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_page_append(const slnr_cache* cache, const slnr_pages* pages, const slnr_rows* k, const slnr_rows* v,
                             const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache(cache, true, cache && cache->codes, true));
  SLNR_CHECK(check_pages(pages, cache, true, true, true));
  SLNR_CHECK(check_rows("k", k, pages->ntok > 0));
  SLNR_CHECK(check_rows("v", v, pages->ntok > 0));
  if (pages->ntok == 0) return SLNR_OK;
  if (pages->ntok > kMaxKeys)  // a block's loops step past its last token
    return fail(SLNR_ERR_UNSUPPORTED, "ntok = %d: at most %d", (int)pages->ntok, kMaxKeys);
  cudaStream_t s = (cudaStream_t)opts->stream;
  const PagesView p = view(*pages);
  const CacheView c = view(*cache);
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_pages(p, c.npages, c.page, true, nullptr, 0, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_append", launch_page_append(p, c, view(*k), view(*v), cache->dtype, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_page_select(const slnr_rows* q, int32_t nheads_q, const slnr_cache* cache, const slnr_pages* pages,
                             int32_t* picked, int32_t npicked, int32_t first, int32_t last, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache(cache, false, true, true));
  SLNR_CHECK(check_pages(pages, cache, true, true, false));
  SLNR_CHECK(check_heads(cache, nheads_q));
  SLNR_CHECK(check_rows("q", q, pages->ntok > 0));
  if (first < 0 || last < 1 || npicked < 1 || (int64_t)first + last > npicked)
    return fail(SLNR_ERR_SHAPE, "first = %d, last = %d of %d pages", (int)first, (int)last, (int)npicked);
  if (npicked > kAttnMaxPicked) return fail(SLNR_ERR_UNSUPPORTED, "npicked = %d: at most %d", (int)npicked, kAttnMaxPicked);
  if (select_tokens(pages->max_k > 0 ? (pages->max_k - 1) / cache->page_size + 1 : 1) == 0)
    return fail(SLNR_ERR_UNSUPPORTED, "max_k = %d keys are too many pages of %d", (int)pages->max_k,
                (int)cache->page_size);
  if (pages->ntok == 0) return SLNR_OK;
  if (!picked) return fail(SLNR_ERR_NULL, "picked is NULL");
  cudaStream_t s = (cudaStream_t)opts->stream;
  const PagesView p = view(*pages);
  const CacheView c = view(*cache);
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_pages(p, c.npages, c.page, false, nullptr, 0, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_select", launch_page_select(p, c, view(*q), cache->dtype, nheads_q, picked, npicked, first, last, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_paged_attention_workspace(const slnr_cache* cache, const slnr_pages* pages, int32_t nheads_q,
                                           const slnr_opts* opts, size_t* bytes) {
  return attention_workspace(cache, pages, nheads_q, 0, opts, bytes);
}

slnr_status slnr_selected_attention_workspace(const slnr_cache* cache, const slnr_pages* pages, int32_t nheads_q,
                                              int32_t npicked, const slnr_opts* opts, size_t* bytes) {
  if (npicked < 1) return fail(SLNR_ERR_SHAPE, "npicked = %d must be positive", (int)npicked);
  return attention_workspace(cache, pages, nheads_q, npicked, opts, bytes);
}

slnr_status slnr_paged_attention(const slnr_rows* q, int32_t nheads_q, const slnr_cache* cache, const slnr_pages* pages,
                                 float scale, void* out, float* lse, const slnr_opts* opts) {
  return attention(q, nheads_q, cache, pages, nullptr, 0, scale, out, lse, opts);
}

slnr_status slnr_selected_attention(const slnr_rows* q, int32_t nheads_q, const slnr_cache* cache,
                                    const slnr_pages* pages, const int32_t* picked, int32_t npicked, float scale,
                                    void* out, float* lse, const slnr_opts* opts) {
  if (npicked < 1) return fail(SLNR_ERR_SHAPE, "npicked = %d must be positive", (int)npicked);
  if (npicked > kAttnMaxPicked) return fail(SLNR_ERR_UNSUPPORTED, "npicked = %d: at most %d", (int)npicked, kAttnMaxPicked);
  if (!picked) return fail(SLNR_ERR_NULL, "picked is NULL");
  return attention(q, nheads_q, cache, pages, picked, npicked, scale, out, lse, opts);
}

slnr_status slnr_page_append4(const slnr_cache4* cache, const slnr_pages* pages, const slnr_rows* k, const slnr_rows* v,
                              int32_t dtype, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache4(cache, true));
  SLNR_CHECK(check_type(dtype));
  const slnr_cache shape = sizes(*cache);
  SLNR_CHECK(check_pages(pages, &shape, true, true, true));
  SLNR_CHECK(check_rows("k", k, pages->ntok > 0));
  SLNR_CHECK(check_rows("v", v, pages->ntok > 0));
  if (pages->ntok == 0) return SLNR_OK;
  cudaStream_t s = (cudaStream_t)opts->stream;
  const PagesView p = view(*pages);
  const Cache4View c = view(*cache);
  if (((int64_t)p.ntok + 7) / 8 * c.nheads * (c.width / 32) > INT32_MAX)  // warps
    return fail(SLNR_ERR_UNSUPPORTED, "too many tokens and heads for one call");
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_pages(p, c.npages, c.slots, true, nullptr, 0, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_append4", launch_page_append4(p, c, view(*k), view(*v), dtype, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_page_values4(const slnr_cache4* cache, const int32_t* ids, int32_t n, void* k, void* v, int32_t dtype,
                              const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache4(cache, true));
  SLNR_CHECK(check_type(dtype));
  if (n < 0 || (!ids && n > cache->npages)) return fail(SLNR_ERR_SHAPE, "n = %d pages", (int)n);
  if (n == 0) return SLNR_OK;
  if (!k || !v) return fail(SLNR_ERR_NULL, "k or v is NULL");
  if (!aligned16(k) || !aligned16(v)) return fail(SLNR_ERR_UNSUPPORTED, "k and v must be 16-byte aligned");
  const int64_t page = (int64_t)cache->page_size * cache->nheads * (cache->head_dim / kBlockCols);
  if (page > kMaxKeys || n * (page / 256 + 1) > INT32_MAX)  // 16 columns a thread, 256 threads a block
    return fail(SLNR_ERR_UNSUPPORTED, "too many values for one call");
  cudaStream_t s = (cudaStream_t)opts->stream;
  const TablesView none{0, 0, 0, divisor(1), nullptr, nullptr};
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_set(none, 0, ids, n, cache->npages, nullptr, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_values4", launch_page_values4(view(*cache), ids, n, k, v, dtype, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_paged_attention4_workspace(const slnr_cache4* cache, const slnr_pages* pages, int32_t nheads_q,
                                            const slnr_opts* opts, size_t* bytes) {
  if (!bytes) return fail(SLNR_ERR_NULL, "bytes is NULL");
  SLNR_CHECK(check_paged_opts(opts));
  SLNR_CHECK(check_cache4(cache, false));
  const slnr_cache shape = sizes(*cache);
  SLNR_CHECK(check_pages(pages, &shape, false, true, false));
  SLNR_CHECK(check_heads(&shape, nheads_q));
  const int64_t group = nheads_q / cache->nheads;
  *bytes = rows4(*pages, group) ? rows4_layout(shape, *pages, group).total
                                : attn_layout(shape, *pages, nheads_q, attn4_chunk_plan(*pages, group)).total;
  return SLNR_OK;
}

slnr_status slnr_paged_attention4(const slnr_rows* q, int32_t nheads_q, const slnr_cache4* cache, const slnr_pages* pages,
                                  int32_t dtype, float scale, void* out, float* lse, const slnr_opts* opts) {
  timing_begin();
  return attention4(q, nheads_q, cache, pages, dtype, scale, out, lse, opts);
}

slnr_status slnr_page_copy(const slnr_cache* to, const slnr_cache* from, const int32_t* src, const int32_t* dst,
                           int32_t n, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_copy(src, dst, n, opts));
  for (const slnr_cache* c : {to, from}) {
    const bool keys = c && c->k;
    SLNR_CHECK(check_cache(c, keys, c && c->codes, true));
    if (!keys && !c->codes && c->npages > 0) return fail(SLNR_ERR_NULL, "a cache without keys and summaries");
  }
  if (to->page_size != from->page_size || to->nheads != from->nheads || to->head_dim != from->head_dim ||
      to->dtype != from->dtype)
    return fail(SLNR_ERR_SHAPE, "caches of other pages, heads, widths or types");
  if (to->npages > 0 && from->npages > 0 && !to->k != !from->k)
    return fail(SLNR_ERR_NULL, "one of the caches has no keys");
  if (n == 0 || to->npages == 0 || from->npages == 0) return SLNR_OK;
  CopyParts c{};
  const int64_t slots = from->page_size, heads = from->nheads, width = from->head_dim;
  const auto bytes = [](const int64_t (&s)[3], int64_t (&b)[3]) {
    for (int i = 0; i < 3; ++i) b[i] = 2 * s[i];
  };
  bool fits = true;
  if (from->k) {
    // heads outside where a page of the destination holds them one after another
    for (int i = 0; i < 2; ++i) {
      int64_t f[3], t[3];
      bytes(i ? from->v_stride : from->k_stride, f);
      bytes(i ? to->v_stride : to->k_stride, t);
      const bool heads_first = t[2] > t[1];
      if (heads_first) {
        std::swap(f[1], f[2]);
        std::swap(t[1], t[2]);
      }
      fits = fits && add_part(c, i ? from->v : from->k, i ? to->v : to->k, f, t, heads_first ? heads : slots,
                              heads_first ? slots : heads, 2 * width, 16);
    }
  }
  if (from->codes && to->codes) {
    const int64_t code[3] = {heads * width, 0, 0}, scale[3] = {heads * 4, 0, 0};
    fits = fits && add_part(c, from->codes, to->codes, code, code, 1, 1, heads * width, 8);
    fits = fits && add_part(c, from->scales, to->scales, scale, scale, 1, 1, heads * 4, 4);
  }
  if (!fits) return fail(SLNR_ERR_UNSUPPORTED, "too large a page for one call");
  return copy_pages(c, src, dst, n, from->npages, to->npages, opts);
}

slnr_status slnr_page_copy4(const slnr_cache4* to, const slnr_cache4* from, const int32_t* src, const int32_t* dst,
                            int32_t n, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_copy(src, dst, n, opts));
  SLNR_CHECK(check_cache4(to, true));
  SLNR_CHECK(check_cache4(from, true));
  if (to->page_size != from->page_size || to->nheads != from->nheads || to->head_dim != from->head_dim)
    return fail(SLNR_ERR_SHAPE, "caches of other pages, heads or widths");
  if (n == 0 || to->npages == 0 || from->npages == 0) return SLNR_OK;
  CopyParts c{};
  const int64_t f[3] = {from->page_stride, 0, from->head_stride}, t[3] = {to->page_stride, 0, to->head_stride};
  if (!add_part(c, from->data, to->data, f, t, 1, from->nheads, (int64_t)from->page_size / kSlab * slab_bytes(from->head_dim),
                16))
    return fail(SLNR_ERR_UNSUPPORTED, "too large a page for one call");
  return copy_pages(c, src, dst, n, from->npages, to->npages, opts);
}

slnr_status slnr_page_fork(int32_t nreq, const int32_t* lens, const int32_t* table, int64_t table_stride, int32_t width,
                           int32_t page_size, const int32_t* parent, int32_t n, const int32_t* free_pages, int32_t nfree,
                           int32_t* out_table, int32_t* out_lens, int32_t* src, int32_t* dst, int32_t* used,
                           const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_tables(nreq, lens, table, table_stride, width, page_size, opts));
  if (n < 0 || nfree < 0) return fail(SLNR_ERR_SHAPE, "n = %d, nfree = %d", (int)n, (int)nfree);
  if (n > kMaxForks) return fail(SLNR_ERR_UNSUPPORTED, "n = %d: at most %d", (int)n, kMaxForks);
  if (!used) return fail(SLNR_ERR_NULL, "used is NULL");
  if (n > 0 && (!parent || (width > 0 && !out_table) || !out_lens || !src || !dst))
    return fail(SLNR_ERR_NULL, "an array of the children is NULL");
  if (nfree > 0 && !free_pages) return fail(SLNR_ERR_NULL, "free_pages is NULL");
  if (width > 0 && n > 0 && out_table == table) return fail(SLNR_ERR_UNSUPPORTED, "out_table is table");
  cudaStream_t s = (cudaStream_t)opts->stream;
  const TablesView t{nreq, width, table_stride, divisor(page_size), table, lens};
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_set(t, INT32_MAX, parent, n, nreq, nullptr, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_fork",
              launch_page_fork(t, parent, n, free_pages, nfree, out_table, out_lens, src, dst, used, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_page_free(int32_t nreq, int32_t* lens, const int32_t* table, int64_t table_stride, int32_t width,
                           int32_t page_size, const int32_t* drop, int32_t ndrop, int32_t npages, int32_t* free_pages,
                           int32_t* count, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_tables(nreq, lens, table, table_stride, width, page_size, opts));
  SLNR_CHECK(check_set(npages));
  if (ndrop < 0) return fail(SLNR_ERR_SHAPE, "ndrop = %d", (int)ndrop);
  if (!count || (npages > 0 && !free_pages)) return fail(SLNR_ERR_NULL, "free_pages or count is NULL");
  if (ndrop > 0 && !drop) return fail(SLNR_ERR_NULL, "drop is NULL");
  cudaStream_t s = (cudaStream_t)opts->stream;
  const TablesView t{nreq, width, table_stride, divisor(page_size), table, lens};
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_set(t, npages, drop, ndrop, nreq, nullptr, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_free", launch_page_free(t, lens, drop, ndrop, npages, free_pages, count, s));
  timing_end(s);
  return SLNR_OK;
}

slnr_status slnr_page_compact(int32_t nreq, const int32_t* lens, const int32_t* table, int64_t table_stride,
                              int32_t width, int32_t page_size, int32_t npages, int32_t* out_table, int32_t* src,
                              int32_t* dst, int32_t* ids, int32_t* used, const slnr_opts* opts) {
  timing_begin();
  SLNR_CHECK(check_tables(nreq, lens, table, table_stride, width, page_size, opts));
  SLNR_CHECK(check_set(npages));
  if (!used || (npages > 0 && !ids) || (npages > 1 && (!src || !dst)) || (nreq > 0 && width > 0 && !out_table))
    return fail(SLNR_ERR_NULL, "an output is NULL");
  if (nreq > 0 && width > 0 && out_table == table) return fail(SLNR_ERR_UNSUPPORTED, "out_table is table");
  cudaStream_t s = (cudaStream_t)opts->stream;
  const TablesView t{nreq, width, table_stride, divisor(page_size), table, lens};
  SLNR_CHECK(validated(opts, [&](WsHeader* hdr, cudaStream_t st) {
    return launch_validate_set(t, npages, nullptr, 0, 0, nullptr, 0, hdr, st);
  }));
  SLNR_LAUNCH("page_compact", launch_page_compact(t, npages, out_table, src, dst, ids, used, s));
  timing_end(s);
  return SLNR_OK;
}

}  // extern "C"
