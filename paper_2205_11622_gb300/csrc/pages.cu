// Block tables, slot maps and the cache's writes: the parts of a step over a
// paged cache that come before its attention.
#include "launch.h"
#include "paged_tile.cuh"

namespace slnr {
namespace {

// ---------------------------------------------------------------------------
// Block tables and slot maps from request lengths.
//
// With P_r = sum of the pages that requests before r take, request r's page n
// (held_r <= n < needed_r) is free[P_r + n - held_r].  A page that a request
// takes starts at one of its new tokens, so the thread of that token writes the
// table's entry, and no thread needs another's.  Every block scans the lengths
// of all requests (1024 at a time, a few hundred bytes to a few KB out of L2)
// and writes the tokens of its own range: one launch, nothing to wait for.
// Lengths that no cache holds (sums past 2^31) give slots of -1 where they are
// looked up, and no access outside the arrays.
// Bound by the latency of its dependent reads: 64 requests of one token 6 us,
// 512 requests of 284k tokens 7 us, caches cold.
constexpr int kTablesThreads = 1024;
constexpr int kTablesTokens = 2048;  // tokens of a block

__device__ __forceinline__ int clamped_div_up(int n, Divisor d) { return n > 0 ? d.div(n - 1) + 1 : 0; }

__global__ void __launch_bounds__(kTablesThreads)
k_page_tables(int nreq, const int32_t* __restrict__ new_len, const int32_t* __restrict__ old_len,
              int32_t* table, int64_t table_stride, int width, const int32_t* __restrict__ free_pages, int nfree,
              Divisor page, int ntok, int32_t* q_pos, int32_t* k_len, int32_t* req, int32_t* slots, int32_t* used) {
  __shared__ int s_tok[kTablesThreads], s_pg[kTablesThreads], s_old[kTablesThreads];
  __shared__ int s_warp[2][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * kTablesTokens;
  const int t1 = step_end(t0, kTablesTokens, ntok);
  int tok_base = 0, pg_base = 0;
  for (int r0 = 0; r0 < nreq; r0 = step_end(r0, kTablesThreads, nreq)) {
    const unsigned r = item(r0, tid);
    const bool on = inside(r0, tid, nreq);
    const int n = on ? max(new_len[r], 0) : 0, old = on ? max(old_len[r], 0) : 0;
    const int end = n > INT32_MAX - old ? INT32_MAX : old + n;
    const int take = clamped_div_up(end, page) - clamped_div_up(old, page);
    // inclusive sums of new tokens and taken pages over the block
    int a = n, b = take;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a2 = __shfl_up_sync(0xffffffffu, a, o), b2 = __shfl_up_sync(0xffffffffu, b, o);
      if (lane >= o) { a += a2; b += b2; }
    }
    __syncthreads();  // the previous step's readers are done
    if (lane == 31) { s_warp[0][warp] = a; s_warp[1][warp] = b; }
    __syncthreads();
    if (warp == 0) {
      int wa = s_warp[0][lane], wb = s_warp[1][lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int a2 = __shfl_up_sync(0xffffffffu, wa, o), b2 = __shfl_up_sync(0xffffffffu, wb, o);
        if (lane >= o) { wa += a2; wb += b2; }
      }
      s_warp[0][lane] = wa;
      s_warp[1][lane] = wb;
    }
    __syncthreads();
    if (warp > 0) { a += s_warp[0][warp - 1]; b += s_warp[1][warp - 1]; }
    const int tok_end = tok_base + s_warp[0][31], pg_end = pg_base + s_warp[1][31];
    s_tok[tid] = tok_base + a - n;  // first token of request r
    s_pg[tid] = pg_base + b - take;
    s_old[tid] = old;
    if (blockIdx.x == 0 && on) {
      q_pos[r] = tok_base + a - n;
      k_len[r] = end;
    }
    __syncthreads();
    const int lo = max(t0, tok_base), here = max(min(t1, tok_end), lo) - lo;
    for (int j = tid; j < here; j += kTablesThreads) {
      const int t = lo + j;
      // the last request of this step that starts at or before t (the ones after it that start there too are empty)
      int i = 0;
#pragma unroll
      for (int w = kTablesThreads / 2; w > 0; w >>= 1)
        if (s_tok[i + w] <= t) i += w;
      const int o = s_old[i], p = (int)((unsigned)o + (unsigned)t - (unsigned)s_tok[i]);
      int id = -1, off = 0;
      if (p >= o && inside(r0, i, nreq)) {
        const int held = clamped_div_up(o, page), n_page = page.div(p);
        off = p - n_page * page.d;
        if (n_page < held) {
          if (n_page < width) id = table[(r0 + i) * table_stride + n_page];
        } else {
          const int f = (int)((unsigned)s_pg[i] + (unsigned)(n_page - held));
          if ((unsigned)f < (unsigned)nfree && n_page < width) id = free_pages[f];
          if (off == 0 && n_page < width) table[(r0 + i) * table_stride + n_page] = id;
        }
      }
      req[t] = r0 + i;
      slots[t] = id < 0 ? -1 : id * page.d + off;
    }
    tok_base = tok_end;
    pg_base = pg_end;
  }
  // tokens that no request has
  const int rest = max(t0, tok_base);
  for (int j = tid; j < t1 - rest; j += kTablesThreads) {
    req[rest + j] = -1;
    slots[rest + j] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    q_pos[nreq] = tok_base;
    used[0] = pg_base;
  }
}

// ---------------------------------------------------------------------------
// Appending: K and V rows to their slots, and the summary of each page that a
// token fills.
//
// A block takes the new tokens that go to one page of one request (found from
// the lengths alone) and one key head: a thread a 16-byte piece of every
// ROWS-th row, K and V, kDeep rows in flight.  If the last of them fills the
// page, the block sums the keys while it has them, with the older ones out of
// the cache: no key is read twice, and no block reads what another writes.
// Bound by memory: 31k tokens, 8 heads of 128 (264 MB in and out) 47 us, 5.6
// TB/s.  Blocks that only copied, with the summaries in blocks of their own,
// read the keys twice and took 13 us more; 2 rows in flight 3 us more, 8 rows 17.
constexpr int kAppendThreads = 256;
constexpr int kDeep = 4;

template <typename T>
__device__ __forceinline__ float2 to_float2(uint32_t x);
template <>
__device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 to_float2<__half>(uint32_t x) {
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

// Pages that the new tokens of a request go to.
__device__ __forceinline__ int pages_touched(int old, int n, Divisor page) {
  return n > 0 ? page.div(max(old, 0) + n - 1) - page.div(max(old, 0)) + 1 : 0;
}

template <typename T>
__global__ void __launch_bounds__(kAppendThreads, 4)
k_page_append(PagesView p, CacheView c, RowsView kn, RowsView vn, Divisor pieces) {
  __shared__ float s_sum[kAppendThreads][9];  // a thread's 8 columns
  const int tid = threadIdx.x, lane = tid & 31, h = blockIdx.y;
  // request and which of its pages: at most one new token each, or parts counted request after request
  int r = blockIdx.x, nth = 0;
  if (p.max_q > 1)
    find_part(
        p.nreq, blockIdx.x,
        [&](int i) {
          const int q = __ldg(p.q_pos + i + 1) - __ldg(p.q_pos + i);
          return pages_touched(__ldg(p.k_len + i) - q, q, c.page);
        },
        r, nth);
  if (r < 0) return;
  const int s = c.page.d, q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
  if (qn <= 0) return;
  const int old = max(__ldg(p.k_len + r) - qn, 0);
  // tokens [t0, t1) at positions from `at` on, slots [at % s, ..) of their page
  const int page0 = c.page.div(old) + nth, at = max(old, page0 * s);
  const int t0 = q0 + at - old, t1 = q0 + min(qn, (page0 + 1) * s - old);
  const int col = tid % pieces.d, row0 = tid / pieces.d, rows = kAppendThreads / pieces.d;
  const bool on = row0 < rows;  // pieces that do not divide the block leave some threads out
  const int last = __ldg(p.slots + t1 - 1);
  const int last_page = last >= 0 ? page_of(last, c) : 0;
  const bool fills = c.codes && last >= 0 && last_page < c.npages && last - last_page * s == s - 1;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  auto add = [&](const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 y = to_float2<T>(w[e]);
      sum[2 * e] += y.x;
      sum[2 * e + 1] += y.y;
    }
  };
  const T* src_k = (const T*)kn.p + (int64_t)h * kn.head + col * 8;
  const T* src_v = (const T*)vn.p + (int64_t)h * vn.head + col * 8;
  T* dst_k = (T*)c.k + h * c.ks[2] + col * 8;
  T* dst_v = (T*)c.v + h * c.vs[2] + col * 8;
  if (on) {
    for (int t = t0 + row0; t < t1; t += rows * kDeep) {
      uint4 x[kDeep], y[kDeep];
      int slot[kDeep];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        const int u = t + d * rows;
        slot[d] = u < t1 ? __ldg(p.slots + u) : -1;
        x[d] = y[d] = make_uint4(0, 0, 0, 0);
        if (u < t1) {
          x[d] = __ldg(reinterpret_cast<const uint4*>(src_k + u * kn.tok));
          y[d] = __ldg(reinterpret_cast<const uint4*>(src_v + u * vn.tok));
        }
      }
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        if (fills) add(x[d]);
        const int pg = slot[d] >= 0 ? page_of(slot[d], c) : c.npages, off = slot[d] - pg * s;
        if (pg < c.npages) {
          *reinterpret_cast<uint4*>(dst_k + pg * c.ks[0] + off * c.ks[1]) = x[d];
          *reinterpret_cast<uint4*>(dst_v + pg * c.vs[0] + off * c.vs[1]) = y[d];
        }
      }
    }
  }
  if (!fills) return;
  if (on) {  // the page's older keys
    for (int j = row0; j < s - (t1 - t0); j += rows * kDeep) {
      uint4 x[kDeep];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        x[d] = make_uint4(0, 0, 0, 0);
        if (j + d * rows < s - (t1 - t0))
          x[d] = *reinterpret_cast<const uint4*>(dst_k + last_page * c.ks[0] + (j + d * rows) * c.ks[1]);
      }
#pragma unroll
      for (int d = 0; d < kDeep; ++d) add(x[d]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_sum[tid][e] = sum[e];
  __syncthreads();
  // warp 0: columns 4 lane .. 4 lane + 3, in the threads' order
  if (tid >= 32) return;
  float m[4] = {0.f, 0.f, 0.f, 0.f}, most = 0.f;
  const bool mine = 4 * lane < c.width;
  if (mine) {
    for (int i = 0; i < rows; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] += s_sum[i * pieces.d + lane / 2][4 * (lane & 1) + e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = __fdiv_rn(m[e], (float)s);
    most = fmaxf(most, fabsf(m[e]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  const float scale = __fdiv_rn(most, 127.f);
  const int64_t to = (int64_t)last_page * c.nheads + h;
  if (mine) {
    char4 code = make_char4(0, 0, 0, 0);
    if (scale > 0.f) {
      code.x = (signed char)min(max(__float2int_rn(__fdiv_rn(m[0], scale)), -127), 127);
      code.y = (signed char)min(max(__float2int_rn(__fdiv_rn(m[1], scale)), -127), 127);
      code.z = (signed char)min(max(__float2int_rn(__fdiv_rn(m[2], scale)), -127), 127);
      code.w = (signed char)min(max(__float2int_rn(__fdiv_rn(m[3], scale)), -127), 127);
    }
    *reinterpret_cast<char4*>(c.codes + to * c.width + 4 * lane) = code;
  }
  if (lane == 0) c.scales[to] = scale;
}

// ---------------------------------------------------------------------------
// Validate mode

__global__ void k_validate_lengths(int nreq, const int32_t* new_len, const int32_t* old_len, const int32_t* table,
                                   int64_t table_stride, int width, int nfree, Divisor page, int ntok, WsHeader* hdr) {
  __shared__ long long s_tok, s_pg;
  if (threadIdx.x == 0) s_tok = s_pg = 0;
  __syncthreads();
  int bad = 0;
  for (int64_t r = threadIdx.x; r < nreq; r += blockDim.x) {
    const long long n = new_len[r], o = old_len[r];
    if (n < 0 || o < 0 || n + o > (long long)width * page.d || n + o >= (1ll << 31)) {
      bad |= kErrPos;
      continue;
    }
    const int held = clamped_div_up((int)o, page);
    atomicAdd((unsigned long long*)&s_tok, (unsigned long long)n);
    atomicAdd((unsigned long long*)&s_pg, (unsigned long long)(clamped_div_up((int)(o + n), page) - held));
    if (held > 0 && o % page.d != 0 && table[r * table_stride + held - 1] < 0) bad |= kErrCrdRange;
  }
  if (bad) atomicOr(&hdr->error, bad);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (s_tok != ntok) atomicOr(&hdr->error, kErrPos);
    if (s_pg > nfree) atomicOr(&hdr->error, kErrOverflow);
  }
}

__global__ void k_validate_pages(PagesView p, int npages, Divisor page, bool slots, const int32_t* picked, int npicked,
                                 int nheads, WsHeader* hdr) {
  const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  int bad = 0;
  if (id == 0 && (p.q_pos[0] != 0 || p.q_pos[p.nreq] != p.ntok)) bad |= kErrPos;
  for (int64_t r = id; r < p.nreq; r += step) {
    const long long n = (long long)p.q_pos[r + 1] - p.q_pos[r], k = p.k_len[r];
    if (n < 0 || n > p.max_q || k < (slots ? n : 0) || k > p.max_k || k > (long long)p.width * page.d) bad |= kErrPos;
    else
      for (int i = 0; i < clamped_div_up((int)k, page); ++i)
        if ((unsigned)p.table[r * p.table_stride + i] >= (unsigned)npages) bad |= kErrCrdRange;
  }
  for (int64_t t = id; t < p.ntok; t += step) {
    if (p.req) {
      const int r = p.req[t];
      if ((unsigned)r >= (unsigned)p.nreq || t < p.q_pos[r] || t >= p.q_pos[r + 1]) bad |= kErrCrdRange;
    }
    if (slots && (p.slots[t] < 0 || page.div(p.slots[t]) >= npages)) bad |= kErrCrdRange;
    if (picked)
      for (int64_t h = 0; h < nheads; ++h) {
        const int32_t* row = picked + (t * nheads + h) * npicked;
        int before = -1;
        for (int i = 0; i < npicked; ++i) {
          if (row[i] < 0) continue;
          if (row[i] >= p.width) bad |= kErrCrdRange;
          if (row[i] <= before) bad |= kErrCrdOrder;
          before = row[i];
        }
      }
  }
  if (bad) atomicOr(&hdr->error, bad);
}

}  // namespace

cudaError_t launch_page_tables(int nreq, const int32_t* new_len, const int32_t* old_len, int32_t* table,
                               int64_t table_stride, int width, const int32_t* free_pages, int nfree, int page_size,
                               int ntok, int32_t* q_pos, int32_t* k_len, int32_t* req, int32_t* slots, int32_t* used,
                               cudaStream_t s) {
  const int grid = ntok > 0 ? pieces(ntok, kTablesTokens) : 1;
  k_page_tables<<<SLNR_COUNTED(grid), kTablesThreads, 0, s>>>(nreq, new_len, old_len, table, table_stride, width,
                                                             free_pages, nfree, divisor(page_size), ntok, q_pos, k_len,
                                                             req, slots, used);
  return cudaGetLastError();
}

cudaError_t launch_page_append(const PagesView& p, const CacheView& c, const RowsView& k, const RowsView& v, int dtype,
                               cudaStream_t s) {
  if (p.ntok == 0) return cudaSuccess;
  const int64_t pages = p.max_q > 1 ? p.ntok / c.page.d + 2 * (int64_t)(p.nreq < p.ntok ? p.nreq : p.ntok) : p.nreq;
  if (pages >= (int64_t(1) << 31)) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)pages, (unsigned)c.nheads);
  auto kernel = dtype == SLNR_FP16 ? k_page_append<__half> : k_page_append<__nv_bfloat16>;
  kernel<<<(SLNR_COUNTED(grid)), kAppendThreads, 0, s>>>(p, c, k, v, divisor(c.width / 8));
  return cudaGetLastError();
}

cudaError_t launch_validate_lengths(int nreq, const int32_t* new_len, const int32_t* old_len, const int32_t* table,
                                    int64_t table_stride, int width, int nfree, int page_size, int ntok, WsHeader* hdr,
                                    cudaStream_t s) {
  k_validate_lengths<<<SLNR_COUNTED(1), 1024, 0, s>>>(nreq, new_len, old_len, table, table_stride, width, nfree,
                                                     divisor(page_size), ntok, hdr);
  return cudaGetLastError();
}

cudaError_t launch_validate_pages(const PagesView& p, int npages, Divisor page, bool slots, const int32_t* picked,
                                  int npicked, int nheads, WsHeader* hdr, cudaStream_t s) {
  k_validate_pages<<<SLNR_COUNTED(304), 256, 0, s>>>(p, npages, page, slots, picked, npicked, nheads, hdr);
  return cudaGetLastError();
}

}  // namespace slnr
