// Block tables, slot maps and the cache's writes: the parts of a step over a
// paged cache that come before its attention.
#include "launch.h"
#include "paged.cuh"

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
// Bound by the latency of its dependent reads.
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
  for (int r0 = 0; r0 < nreq; r0 += kTablesThreads) {
    const int r = r0 + tid;
    const bool on = r < nreq;
    const int n = on ? max(new_len[r], 0) : 0, old = on ? max(old_len[r], 0) : 0;
    const int take = clamped_div_up(old + n, page) - clamped_div_up(old, page);
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
      k_len[r] = old + n;
    }
    __syncthreads();
    const int lo = max(t0, tok_base), hi = min(t1, tok_end);
    for (int t = lo + tid; t < hi; t += kTablesThreads) {
      // the last request of this step that starts at or before t (the ones after it that start there too are empty)
      int i = 0;
#pragma unroll
      for (int w = kTablesThreads / 2; w > 0; w >>= 1)
        if (s_tok[i + w] <= t) i += w;
      const int o = s_old[i], p = o + (t - s_tok[i]);
      const int held = clamped_div_up(o, page), n_page = page.div(p), off = p - n_page * page.d;
      int id = -1;
      if (n_page < held) {
        if (n_page < width) id = table[(r0 + i) * table_stride + n_page];
      } else {
        const int f = s_pg[i] + (n_page - held);
        if (f < nfree && n_page < width) id = free_pages[f];
        if (off == 0 && n_page < width) table[(r0 + i) * table_stride + n_page] = id;
      }
      req[t] = r0 + i;
      slots[t] = id < 0 ? -1 : id * page.d + off;
    }
    tok_base = tok_end;
    pg_base = pg_end;
  }
  // tokens that no request has
  for (int t = max(t0, tok_base) + tid; t < t1; t += kTablesThreads) {
    req[t] = -1;
    slots[t] = -1;
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
// The last blocks copy: a thread takes one 16-byte piece of a row for
// kCopyTokens tokens, K and V, so 2 kCopyTokens loads are in flight and the
// divisions that find the piece are made once.  The others look at 32 tokens
// and one head each; for a token in a page's last slot the block's warps sum
// that head's keys over the page.  Rows of this call are read from the call's own
// input, so no block reads what another writes.  Bound by memory.
constexpr int kCopyThreads = 256;
constexpr int kCopyTokens = 4;

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__global__ void __launch_bounds__(kCopyThreads)
k_page_append(PagesView p, CacheView c, RowsView kn, RowsView vn, int sum_blocks, Divisor of_token, Divisor of_head) {
  if ((int)blockIdx.x >= sum_blocks) {
    const int lin = (blockIdx.x - sum_blocks) * kCopyThreads + threadIdx.x;
    const int group = of_token.div(lin), piece = lin - group * of_token.d;
    const int h = of_head.div(piece), col = (piece - h * of_head.d) * 8;
    const int t0 = group * kCopyTokens;
    if (t0 >= p.ntok) return;
    int slot[kCopyTokens];
    uint4 a[kCopyTokens], b[kCopyTokens];
#pragma unroll
    for (int i = 0; i < kCopyTokens; ++i) {
      slot[i] = inside(t0, i, p.ntok) ? __ldg(p.slots + t0 + i) : -1;
      if (slot[i] >= 0 && page_of(slot[i], c) >= c.npages) slot[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < kCopyTokens; ++i)
      if (slot[i] >= 0) {
        a[i] = __ldg(reinterpret_cast<const uint4*>((const T*)kn.p + (int64_t)(t0 + i) * kn.tok + h * kn.head + col));
        b[i] = __ldg(reinterpret_cast<const uint4*>((const T*)vn.p + (int64_t)(t0 + i) * vn.tok + h * vn.head + col));
      }
#pragma unroll
    for (int i = 0; i < kCopyTokens; ++i)
      if (slot[i] >= 0) {
        const int pg = page_of(slot[i], c), off = slot[i] - pg * c.page.d;
        *reinterpret_cast<uint4*>((T*)c.k + pg * c.ks[0] + off * c.ks[1] + h * c.ks[2] + col) = a[i];
        *reinterpret_cast<uint4*>((T*)c.v + pg * c.vs[0] + off * c.vs[1] + h * c.vs[2] + col) = b[i];
      }
    return;
  }
  // one head of 32 tokens; the block's warps share the keys of each filled page
  __shared__ float2 s_sum[kCopyThreads / 32][2][32];
  constexpr int WARPS = kCopyThreads / 32, DEEP = 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t w = blockIdx.x;
  const int h = (int)(w % c.nheads);
  const int64_t first = w / c.nheads * 32;
  int slot = -1;
  if (first + lane < p.ntok) slot = __ldg(p.slots + first + lane);
  bool fills = slot >= 0;
  if (fills) {
    const int pg = page_of(slot, c);
    fills = pg < c.npages && slot - pg * c.page.d == c.page.d - 1;
  }
  unsigned todo = __ballot_sync(0xffffffffu, fills);  // the same in all warps
  while (todo) {
    const int i = __ffs(todo) - 1;
    todo &= todo - 1;
    const int pg = page_of(__shfl_sync(0xffffffffu, slot, i), c);
    const int t = (int)first + i, r = __ldg(p.req + t);
    // slot j of the page: a token of this call from j0 on, an older key before
    const int s = c.page.d, fresh = min(t - __ldg(p.q_pos + r) + 1, s), j0 = s - fresh;
    const T* src_old = (const T*)c.k + pg * c.ks[0] + h * c.ks[2];
    const T* src_new = (const T*)kn.p + (int64_t)(t - (s - 1)) * kn.tok + h * kn.head;
    // lane: columns 2 lane and 2 lane + 64, in pairs; warp: every eighth key, DEEP of them in flight
    const int col = 2 * lane;
    float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
    for (int jb = warp; jb < s; jb += WARPS * DEEP) {
      uint32_t x[DEEP][2];
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        const int j = jb + d * WARPS;
        const T* row = j < j0 ? src_old + j * c.ks[1] : src_new + (int64_t)j * kn.tok;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          x[d][e] = j < s && col + 64 * e < c.width ? *reinterpret_cast<const uint32_t*>(row + col + 64 * e) : 0u;
      }
#pragma unroll
      for (int d = 0; d < DEEP; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          alignas(4) T y[2];
          *reinterpret_cast<uint32_t*>(y) = x[d][e];
          sum[e].x += to_float(y[0]);
          sum[e].y += to_float(y[1]);
        }
    }
    s_sum[warp][0][lane] = sum[0];
    s_sum[warp][1][lane] = sum[1];
    __syncthreads();
    if (warp == 0) {
      float most = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        for (int k = 1; k < WARPS; ++k) {
          const float2 y = s_sum[k][e][lane];
          sum[e].x += y.x;
          sum[e].y += y.y;
        }
        sum[e].x = __fdiv_rn(sum[e].x, (float)s);
        sum[e].y = __fdiv_rn(sum[e].y, (float)s);
        most = fmaxf(most, fmaxf(fabsf(sum[e].x), fabsf(sum[e].y)));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      const float scale = __fdiv_rn(most, 127.f);
      int8_t* code = c.codes + ((int64_t)pg * c.nheads + h) * c.width;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (col + 64 * e < c.width) {
          char2 x = make_char2(0, 0);
          if (scale > 0.f) {
            x.x = (signed char)min(max(__float2int_rn(__fdiv_rn(sum[e].x, scale)), -127), 127);
            x.y = (signed char)min(max(__float2int_rn(__fdiv_rn(sum[e].y, scale)), -127), 127);
          }
          *reinterpret_cast<char2*>(code + col + 64 * e) = x;
        }
      if (lane == 0) c.scales[(int64_t)pg * c.nheads + h] = scale;
    }
    __syncthreads();  // s_sum is read before the next page's sums are written
  }
}

// ---------------------------------------------------------------------------
// Validate mode

__global__ void k_validate_lengths(int nreq, const int32_t* new_len, const int32_t* old_len, const int32_t* table,
                                   int64_t table_stride, int width, int nfree, Divisor page, int ntok, WsHeader* hdr) {
  __shared__ long long s_tok, s_pg;
  if (threadIdx.x == 0) s_tok = s_pg = 0;
  __syncthreads();
  int bad = 0;
  for (int r = threadIdx.x; r < nreq; r += blockDim.x) {
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
    if (n < 0 || n > p.max_q || k < 0 || k > p.max_k || k > (long long)p.width * page.d) bad |= kErrPos;
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
  const int per_row = c.width / 8;
  const int64_t copy_blocks = ceil_div(ceil_div(p.ntok, kCopyTokens) * c.nheads * per_row, kCopyThreads);
  const int64_t sum_blocks = c.codes ? ceil_div(p.ntok, 32) * c.nheads : 0;
  const unsigned grid = (unsigned)(copy_blocks + sum_blocks);
  auto kernel = dtype == SLNR_FP16 ? k_page_append<__half> : k_page_append<__nv_bfloat16>;
  kernel<<<SLNR_COUNTED(grid), kCopyThreads, 0, s>>>(p, c, k, v, (int)sum_blocks,
                                                     divisor(c.nheads * per_row), divisor(per_row));
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
