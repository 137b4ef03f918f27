// Attention of new tokens over a paged cache, rows of a few tokens at a time:
// the kernel of single tokens, of short chunks and of selected pages.
//
//   o = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q.k_j - m),  m = max_j scale q.k_j
//
// over the keys j that the row sees.  One pass over the keys: m, the sum and o
// are held in fp32 registers and rescaled when m grows.  The weights are rounded
// to the cache's type for the product with V (their sum is not): the error of
// one rounding of the output.  fp16 rounds by a share of a weight down to 2^-14
// only and to nothing below 2^-25, so there m - 14 takes m's place: weights of up
// to 2^14, and what is lost of n small ones is n 2^-39 of the largest at most.
//
// A block takes one key head and a request's rows (the query rows of that head's
// group, token after token; 16 WM at most), or with picked pages a token's, and
// streams its keys through shared memory, 64 at a time, by asynchronous 16-byte copies; each thread finds one key's row
// of K or V by its page, three steps ahead, and all read the rows' offsets from
// shared memory.  Few rows are split over their keys: up to 16 splits are the
// blocks of a cluster, which join their results through each other's shared
// memory; more go through the workspace and k_paged_combine.  WM warps share the rows; the 4 / WM warps of one
// row set take a part of each 64 keys and join their sums at the end, so
// every key is read from shared memory by WM warps only.
//
// Single tokens are bound by memory: 64 requests of 1001 to 32003 keys (2.4 GB),
// 32 query and 8 key heads of 128, bf16, 407 us, 5.8 TB/s.  With each thread
// finding every row that it copies by itself 568.  One request of 4095 keys: 13
// us on the GPU, latency, in 16 splits a head joined in a cluster.  Products run
// on mma.sync: 16 rows are an eighth of a tcgen05 tile, and its way through
// tensor memory takes longer than these products do.
#include "launch.h"
#include "mma16.cuh"
#include "paged_tile.cuh"

namespace slnr {
namespace {

constexpr int kThreads = 128;
constexpr int kStages = 3;
constexpr int kOffsets = kStages + 1;  // steps whose rows' offsets are held

template <int W>
constexpr int stage_bytes() { return 2 * kAttnKeys * W * 2; }
template <int W>
constexpr size_t smem_bytes() { return (size_t)kStages * stage_bytes<W>(); }

// What weights are taken against, from their scores' maximum (in powers of two): no
// weight is above 2^14 in fp16, however large the maximum (rounded up).
template <typename T>
__device__ __forceinline__ float reference(float m);
template <>
__device__ __forceinline__ float reference<__nv_bfloat16>(float m) { return m; }
template <>
__device__ __forceinline__ float reference<__half>(float m) { return __fsub_ru(m, 14.f); }

template <bool SEL>
struct Smem {
  int64_t row[kOffsets][2][kAttnKeys];       // bytes from the head's first row of K and V to each key's; -1: zeros
  int key_at[SEL ? kOffsets : 1][kAttnKeys]; // selected: the keys' positions
  int2 pick[SEL ? kAttnMaxPicked : 1];       // selected: {page of the cache, page of the request}
  float2 ml[4][16];                          // a warp's (reference, sum) of each row
  float2 joined[64];                         // the same of the block's rows
  int count;
};

// The other blocks of a cluster.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t address_in(uint32_t local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ float2 load2_far(uint32_t at) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float4 load4_far(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}

// Eight columns of a finished row.
template <typename T>
__device__ __forceinline__ void store_row(const AttnArgs& a, int64_t at, int col, const float (&v)[8], float lse2) {
  if (col < a.c.width) {
    uint4 y;
    y.x = Half2<T>::pack(v[0], v[1]);
    y.y = Half2<T>::pack(v[2], v[3]);
    y.z = Half2<T>::pack(v[4], v[5]);
    y.w = Half2<T>::pack(v[6], v[7]);
    *reinterpret_cast<uint4*>((T*)a.out + at * a.c.width + col) = y;
  }
  if (col == 0 && a.lse) a.lse[at] = lse2 * 0.6931471805599453f;
}

template <typename T, int W, int WM, bool SEL, bool CLUSTER>
__global__ void __launch_bounds__(kThreads)
k_paged_rows(AttnArgs a, WsHeader* hdr) {
  constexpr int WK = 4 / WM, KW = kAttnKeys / WK, PIECES = W / 8, ROWS = kThreads / PIECES;
  extern __shared__ __align__(128) unsigned char tiles[];
  __shared__ Smem<SEL> sm;
  const PagesView& p = a.p;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % WM, wk = warp / WM;
  const int G = a.group.d, h = blockIdx.y, tile = 16 * WM;

  if (!CLUSTER) let_next_start();  // k_paged_combine
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) hdr->error = 0;  // no wait here can give up
  // the block's rows: [x0, x0 + n) of request r and head h
  int r, x0, q0, qn;
  if (SEL) {
    const int per = tiles_of(G, tile), t = blockIdx.x / per;
    r = __ldg(p.req + t);
    if (r < 0) return;
    q0 = __ldg(p.q_pos + r);
    x0 = (t - q0) * G + (blockIdx.x - t * per) * tile;
  } else {
    r = blockIdx.x;  // its rows fit a tile
    x0 = 0;
    q0 = __ldg(p.q_pos + r);
  }
  qn = __ldg(p.q_pos + r + 1) - q0;
  if (!SEL && qn == 0) return;
  const int n = SEL ? min(tile, G - x0 % G) : min(tile, qn * G - x0);
  const int shift = __ldg(p.k_len + r) - qn;  // position of the request's first new token
  const int p_first = shift + a.group.div(x0), p_last = shift + a.group.div(x0 + n - 1);

  // its keys: [u0, u1) of the request's keys, or of the picked pages' slots
  const int32_t* table = p.table + r * p.table_stride;
  int end;
  if (SEL) {
    const int32_t* row = a.picked + ((int64_t)(q0 + x0 / G) * c.nheads + h) * a.npicked;
    if (tid == 0) sm.count = 0;
    __syncthreads();
    int most = 0;
    for (int i = tid; i < a.npicked; i += kThreads) {
      const int pg = __ldg(row + i);
      const bool ok = pg >= 0 && pg < p.width && pg <= c.page.div(max(p_last, 0));
      sm.pick[i] = make_int2(ok ? __ldg(table + pg) : -1, ok ? pg : -1);
      if (ok) most = i + 1;
    }
    if (most > 0) atomicMax(&sm.count, most);
    __syncthreads();
    end = sm.count * c.page.d;
  } else {
    end = max(p_last + 1, 0);
  }
  const int u0 = blockIdx.z * a.plan.chunk;
  if (!SEL && !CLUSTER && u0 > 0 && u0 >= end) return;
  const int u1 = max(min(end, u0 + a.plan.chunk), u0);
  const int steps = (u1 - u0 + kAttnKeys - 1) / kAttnKeys;

  // Rows' offsets: threads 0-63 find the 64 keys of a step for K, the others for
  // V.  The block table is read a step before its entry is needed.
  const int key = tid & (kAttnKeys - 1);
  int id = -1;
  auto find = [&](int step) {
    const int u = u0 + step * kAttnKeys + key;
    id = -1;
    if (!SEL && u < u1) {
      const int i = c.page.div(u);
      if (i < p.width) id = __ldg(table + i);
    }
  };
  auto place = [&](int step) {
    const int u = u0 + step * kAttnKeys + key, i = c.page.div(u), off = u - i * c.page.d;
    bool on = u < u1;
    if (SEL) {
      int at = INT32_MAX;
      id = -1;
      if (on) {
        const int2 pk = sm.pick[i];
        id = pk.x;
        on = pk.y >= 0 && pk.y * c.page.d + off <= p_last;  // slots past the token hold anything
        if (on) at = pk.y * c.page.d + off;
      }
      if (tid < kAttnKeys) sm.key_at[step % kOffsets][key] = at;
    }
    on = on && (unsigned)id < (unsigned)c.npages;
    const int64_t* st = tid < kAttnKeys ? c.ks : c.vs;
    sm.row[step % kOffsets][tid / kAttnKeys][key] = on ? 2 * (id * st[0] + off * st[1]) : -1;
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    find(s);
    place(s);
  }
  find(kStages);

  // query fragments: rows lane / 4 and + 8 of the warp's 16
  uint32_t qf[W / 16][4];
  int pos[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int x = wm * 16 + lane / 4 + 8 * i;
    const bool on = x < n;
    const int tok = on ? a.group.div(x0 + x) : 0, g = on ? x0 + x - tok * G : 0;
    pos[i] = on ? shift + tok : -1;
    const T* row = (const T*)a.q.p + (int64_t)(q0 + tok) * a.q.tok + (int64_t)(h * G + g) * a.q.head;
#pragma unroll
    for (int kk = 0; kk < W / 16; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = kk * 16 + e * 8 + (lane & 3) * 2;
        qf[kk][i + 2 * e] = on && col < c.width ? __ldg(reinterpret_cast<const uint32_t*>(row + col)) : 0u;
      }
  }

  // copies: a thread's 16-byte piece of ROWS-th rows, at the same swizzle in all of them
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(tiles);
  const int piece = tid % PIECES, row0 = tid / PIECES;
  const bool col_on = piece * 8 < c.width;
  const char* src_k = (const char*)c.k + 2 * (c.ks[2] * h + (col_on ? piece * 8 : 0));
  const char* src_v = (const char*)c.v + 2 * (c.vs[2] * h + (col_on ? piece * 8 : 0));
  auto load = [&](int step) {
    if (step < steps) {
      const uint32_t dst = base + (step % kStages) * stage_bytes<W>() + tile_offset<W>(row0, piece);
      const int64_t* rows = sm.row[step % kOffsets][0] + row0;
#pragma unroll
      for (int k = 0; k < kAttnKeys / ROWS; ++k) {
        const int64_t ok = rows[k * ROWS], ov = rows[kAttnKeys + k * ROWS];
        copy16(dst + k * ROWS * W * 2, src_k + (ok >= 0 ? ok : 0), col_on && ok >= 0);
        copy16(dst + (kAttnKeys + k * ROWS) * W * 2, src_v + (ov >= 0 ? ov : 0), col_on && ov >= 0);
      }
    }
    copy_commit();
  };

  float o[W / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < W / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  const float sl2 = a.scale * 1.4426950408889634f;

  __syncthreads();
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) load(s);
  for (int step = 0; step < steps; ++step) {
    copy_wait<kStages - 2>();
    __syncthreads();
    load(step + kStages - 1);
    place(step + kStages);
    find(step + kStages + 1);
    const uint32_t ks = base + (step % kStages) * stage_bytes<W>(), vs = ks + kAttnKeys * W * 2;
    const int kb = wk * KW;  // the warp's keys of the step
    const int ub = u0 + step * kAttnKeys + kb;

    float s[KW / 8][4];
#pragma unroll
    for (int j = 0; j < KW / 8; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
    for (int kk = 0; kk < W / 16; ++kk) {
      if (kk * 16 < c.width) {
#pragma unroll
        for (int j = 0; j < KW / 16; ++j) {
          uint32_t b[4];
          ldmatrix4(b, ks + tile_offset<W>(kb + j * 16 + (lane >> 4) * 8 + (lane & 7), 2 * kk + ((lane >> 3) & 1)));
          Half2<T>::mma(s[2 * j], qf[kk], b[0], b[1]);
          Half2<T>::mma(s[2 * j + 1], qf[kk], b[2], b[3]);
        }
      }
    }
    // scores in units of log 2; -inf where the row does not see the key
    const bool masked = SEL || ub + KW - 1 > p_first;
#pragma unroll
    for (int j = 0; j < KW / 8; ++j) {
      int at[2];
      if (SEL) {
        const int2 k2 = *reinterpret_cast<const int2*>(&sm.key_at[step % kOffsets][kb + j * 8 + (lane & 3) * 2]);
        at[0] = k2.x;
        at[1] = k2.y;
      } else {
        at[0] = ub + j * 8 + (lane & 3) * 2;
        at[1] = at[0] + 1;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[j][e] = __fmul_rn(s[j][e], sl2);  // one value here and below, so that no weight passes its reference
        if (masked && at[e & 1] > pos[e >> 1]) s[j][e] = -INFINITY;
      }
    }
    float scale_o[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float mx = m[i];
#pragma unroll
      for (int j = 0; j < KW / 8; ++j) mx = fmaxf(mx, fmaxf(s[j][2 * i], s[j][2 * i + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float b = mx == -INFINITY ? 0.f : reference<T>(mx);  // no key seen yet: every weight is 2^-inf
      scale_o[i] = exp2_fast(reference<T>(m[i]) - b);
      m[i] = mx;
      l[i] *= scale_o[i];
#pragma unroll
      for (int j = 0; j < KW / 8; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[j][2 * i + e] = exp2_fast(__fsub_rn(s[j][2 * i + e], b));
          l[i] += s[j][2 * i + e];
        }
    }
    if (__any_sync(0xffffffffu, scale_o[0] != 1.f || scale_o[1] != 1.f)) {
#pragma unroll
      for (int i = 0; i < W / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= scale_o[e >> 1];
    }
#pragma unroll
    for (int j = 0; j < KW / 16; ++j) {
      const uint32_t w[4] = {Half2<T>::pack(s[2 * j][0], s[2 * j][1]), Half2<T>::pack(s[2 * j][2], s[2 * j][3]),
                             Half2<T>::pack(s[2 * j + 1][0], s[2 * j + 1][1]),
                             Half2<T>::pack(s[2 * j + 1][2], s[2 * j + 1][3])};
#pragma unroll
      for (int i = 0; i < W / 16; ++i) {
        if (i * 16 < c.width) {
          uint32_t b[4];
          ldmatrix4_trans(b, vs + tile_offset<W>(kb + j * 16 + (lane & 15), 2 * i + (lane >> 4)));
          Half2<T>::mma(o[2 * i], w, b[0], b[1]);
          Half2<T>::mma(o[2 * i + 1], w, b[2], b[3]);
        }
      }
    }
  }
  copy_wait<0>();
  __syncthreads();

  // the warps' sums to shared memory (row r of a warp at r * (W + 4)), joined there
  float* rows = reinterpret_cast<float*>(tiles);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    const int row = lane / 4 + 8 * i;
    if ((lane & 3) == 0) sm.ml[warp][row] = make_float2(reference<T>(m[i]), l[i]);
#pragma unroll
    for (int j = 0; j < W / 8; ++j)
      *reinterpret_cast<float2*>(rows + (warp * 16 + row) * (W + 4) + j * 8 + (lane & 3) * 2) =
          make_float2(o[j][2 * i], o[j][2 * i + 1]);
  }
  __syncthreads();

  // a group of PIECES lanes a row, 8 columns a lane
  const int splits = SEL ? a.plan.nsplit : (end > 0 ? (end - 1) / a.plan.chunk + 1 : 1);
  const int64_t hq = (int64_t)c.nheads * G;
  const int col = piece * 8;
  for (int x = row0; x < n; x += ROWS) {
    float mx = -INFINITY, sum = 0.f, acc[8];
#pragma unroll
    for (int k = 0; k < WK; ++k) mx = fmaxf(mx, sm.ml[k * WM + x / 16][x % 16].x);
    const float b = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int k = 0; k < WK; ++k) {
      const int w = k * WM + x / 16;
      const float2 ml = sm.ml[w][x % 16];
      const float f = exp2_fast(ml.x - b);
      sum += f * ml.y;
      const float4* y = reinterpret_cast<const float4*>(rows + (w * 16 + x % 16) * (W + 4) + col);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 z = y[e];
        acc[4 * e] += f * z.x;
        acc[4 * e + 1] += f * z.y;
        acc[4 * e + 2] += f * z.z;
        acc[4 * e + 3] += f * z.w;
      }
    }
    const float inv = __fdividef(1.f, sum);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = sum == 0.f ? 0.f : acc[e] * inv;  // no key: zeros
    const int tok = a.group.div(x0 + x), g = x0 + x - tok * G;
    const int64_t at = (q0 + tok) * hq + h * G + g;
    if (CLUSTER) {  // for the other blocks, where the first warp's row was
      float4* y = reinterpret_cast<float4*>(rows + x * (W + 4) + col);
      y[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      y[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (col == 0) sm.joined[x] = make_float2(mx, sum);
    } else if (splits == 1) {
      store_row<T>(a, at, col, acc, mx + __log2f(sum));  // no key: -inf
    } else {
      const int64_t slot = at * a.plan.nsplit + blockIdx.z;
      if (col < c.width) {
        float4* y = reinterpret_cast<float4*>(a.plan.part + slot * c.width + col);
        y[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        y[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
      }
      if (col == 0) a.plan.part_ml[slot] = make_float2(mx, sum);
    }
  }
  if (CLUSTER) {
    // the splits of a row are the blocks of the cluster: each joins a share of the rows, in the splits' order
    cluster_sync();
    const int size = gridDim.z, rank = (int)cluster_rank();
    const uint32_t ml_at = (uint32_t)__cvta_generic_to_shared(sm.joined);
    for (int x = rank + row0 * size; x < n; x += ROWS * size) {
      float mx = -INFINITY, sum = 0.f, acc[8];
      for (int k = 0; k < size; ++k) mx = fmaxf(mx, load2_far(address_in(ml_at + 8 * x, k)).x);
      const float b = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll 4
      for (int k = 0; k < size; ++k) {
        const float2 ml = load2_far(address_in(ml_at + 8 * x, k));
        const float f = exp2_fast(ml.x - b) * ml.y;
        const uint32_t y = address_in(base + (x * (W + 4) + col) * 4, k);
        const float4 z0 = load4_far(y), z1 = load4_far(y + 16);
        sum += f;
        acc[0] += f * z0.x;
        acc[1] += f * z0.y;
        acc[2] += f * z0.z;
        acc[3] += f * z0.w;
        acc[4] += f * z1.x;
        acc[5] += f * z1.y;
        acc[6] += f * z1.z;
        acc[7] += f * z1.w;
      }
      const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= inv;
      const int tok = a.group.div(x0 + x), g = x0 + x - tok * G;
      store_row<T>(a, (q0 + tok) * hq + h * G + g, col, acc, mx + __log2f(sum));
    }
    cluster_sync();  // a block's shared memory stays until the others have read it
  }
}

// Rows of several splits: o = sum_s 2^(m_s - m) l_s o_s / sum_s 2^(m_s - m) l_s.  A
// block a row, every fourth split a warp: a long cache of few heads has hundreds
// of splits, whose loads would follow one another in one warp: 32768 keys of one
// key head of 128 and 16 query heads, 256 splits, 65 us a call with a warp a row,
// 23 so.  Each warp adds its splits in their order, the warps' sums are added in
// theirs.
template <typename T>
__global__ void __launch_bounds__(128)
k_paged_combine(AttnArgs a) {
  __shared__ float4 sums[4][32];
  __shared__ float weights[4];
  wait_for_previous();
  const PagesView& p = a.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = a.group.d;
  const int64_t hq = (int64_t)a.c.nheads * G, at = blockIdx.x;
  const int t = (int)(at / hq), g = (int)(at % hq) % G;
  const int r = __ldg(p.req + t);
  if (r < 0) return;
  int splits = a.plan.nsplit;
  if (!a.picked) {
    const int q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
    const int end = __ldg(p.k_len + r) - qn + (min(a.plan.tile, qn * G) - 1) / G + 1;
    splits = end > 0 ? (end - 1) / a.plan.chunk + 1 : 1;
  }
  if (splits == 1) return;
  const float2* ml = a.plan.part_ml + at * a.plan.nsplit;
  float m = -INFINITY;
  for (int s = lane; s < splits; s += 32) m = fmaxf(m, ml[s].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float b = m == -INFINITY ? 0.f : m;
  const int col = 4 * lane;
  const float* part = a.plan.part + at * a.plan.nsplit * a.c.width + col;
  float sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = warp; s < splits; s += 4) {
    const float f = exp2_fast(ml[s].x - b) * ml[s].y;
    sum += f;
    if (col < a.c.width) {
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)s * a.c.width);
      acc.x += f * x.x;
      acc.y += f * x.y;
      acc.z += f * x.z;
      acc.w += f * x.w;
    }
  }
  sums[warp][lane] = acc;
  if (lane == 0) weights[warp] = sum;
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    const float4 x = sums[w][lane];
    sum += weights[w];
    acc.x += x.x;
    acc.y += x.y;
    acc.z += x.z;
    acc.w += x.w;
  }
  const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);  // the parts of a row without keys are zeros
  if (col < a.c.width) {
    uint2 y;
    y.x = Half2<T>::pack(acc.x * inv, acc.y * inv);
    y.y = Half2<T>::pack(acc.z * inv, acc.w * inv);
    *reinterpret_cast<uint2*>((T*)a.out + at * a.c.width + col) = y;
  }
  if (lane == 0 && a.lse) a.lse[at] = (m + __log2f(sum)) * 0.6931471805599453f;
}

template <typename T, int W, int WM, bool SEL, bool CLUSTER>
cudaError_t launch_rows(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  auto kernel = k_paged_rows<T, W, WM, SEL, CLUSTER>;
  static_assert(4 * 16 * (W + 4) * 4 <= (int)smem_bytes<W>(), "the joined rows fit in the stages");
  static OncePerDevice once;
  cudaError_t e = once([&] {
    cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<W>());
    if (r == cudaSuccess && CLUSTER) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return r;
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.plan.ntiles, (unsigned)a.c.nheads, (unsigned)a.plan.nsplit);
  if (CLUSTER) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = grid.z;
    cfg.gridDim = SLNR_COUNTED(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<W>();
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, hdr);
  }
  kernel<<<(SLNR_COUNTED(grid)), kThreads, smem_bytes<W>(), s>>>(a, hdr);
  return cudaGetLastError();
}

template <typename T, int W, int WM>
cudaError_t launch_rows_m(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  if (a.picked)
    return a.plan.cluster ? launch_rows<T, W, WM, true, true>(a, hdr, s) : launch_rows<T, W, WM, true, false>(a, hdr, s);
  return a.plan.cluster ? launch_rows<T, W, WM, false, true>(a, hdr, s) : launch_rows<T, W, WM, false, false>(a, hdr, s);
}

template <typename T, int W>
cudaError_t launch_rows_w(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  switch (a.plan.tile) {
    case 16: return launch_rows_m<T, W, 1>(a, hdr, s);
    case 32: return launch_rows_m<T, W, 2>(a, hdr, s);
    default: return launch_rows_m<T, W, 4>(a, hdr, s);
  }
}

template <typename T>
cudaError_t launch_rows_t(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  return a.c.width <= 64 ? launch_rows_w<T, 64>(a, hdr, s) : launch_rows_w<T, 128>(a, hdr, s);
}

}  // namespace

cudaError_t launch_paged_rows(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s) {
  return dtype == SLNR_FP16 ? launch_rows_t<__half>(a, hdr, s) : launch_rows_t<__nv_bfloat16>(a, hdr, s);
}

cudaError_t launch_paged_combine(const AttnArgs& a, int dtype, cudaStream_t s) {
  const unsigned grid = (unsigned)((int64_t)a.p.ntok * a.c.nheads * a.group.d);
  auto kernel = dtype == SLNR_FP16 ? k_paged_combine<__half> : k_paged_combine<__nv_bfloat16>;
  return launch_next(kernel, SLNR_COUNTED(dim3(grid)), dim3(128), 0, s, a);
}

}  // namespace slnr
