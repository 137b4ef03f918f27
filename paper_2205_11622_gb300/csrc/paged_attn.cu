// Attention of new tokens over a paged cache, rows of a few tokens at a time:
// the kernel of single tokens, of short chunks and of selected pages.
//
//   o = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q.k_j - m),  m = max_j scale q.k_j
//
// over the keys j that the row sees.  One pass over the keys: m, the sum and o
// are held in fp32 registers and rescaled when m grows.  The weights are rounded
// to the cache's type for the product with V (their sum is not): the error of
// one rounding of the output.
//
// A block takes one key head and up to 16 WM rows (the query rows of that
// head's group, token after token) and streams its keys through shared memory,
// 64 at a time, by asynchronous 16-byte copies that find each key's page in a
// window of the block table.  WM warps share the rows; the 4 / WM warps of one
// row set take a part of each 64 keys and join their sums at the end, so
// every key is read from shared memory by WM warps only.
#include "launch.h"
#include "mma16.cuh"
#include "paged_tile.cuh"

namespace slnr {
namespace {

constexpr int kThreads = 128;
constexpr int kWindow = 256;  // entries of the block table held in shared memory
constexpr int kStages = 3;

template <int W>
constexpr int stage_bytes() { return 2 * kAttnKeys * W * 2; }
template <int W>
constexpr size_t smem_bytes() { return (size_t)kStages * stage_bytes<W>(); }

struct Smem {
  int2 window[kAttnMaxPicked > kWindow ? kAttnMaxPicked : kWindow];  // {page of the cache, page of the request}
  int key_at[kStages][kAttnKeys];                                     // selected: the keys' positions
  float2 ml[4][16];                                                   // a warp's (maximum, sum) of each row
  int r, x0, count;
};

template <typename T, int W, int WM, bool SEL>
__global__ void __launch_bounds__(kThreads)
k_paged_rows(AttnArgs a) {
  constexpr int WK = 4 / WM, KW = kAttnKeys / WK, PIECES = W / 8;
  extern __shared__ __align__(128) unsigned char tiles[];
  __shared__ Smem sm;
  const PagesView& p = a.p;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % WM, wk = warp / WM;
  const int G = a.group.d, h = blockIdx.y, tile = 16 * WM;

  // the block's rows: [x0, x0 + n) of request r and head h
  int r, x0, q0, qn;
  if (SEL) {
    const int per = tiles_of(G, tile), t = blockIdx.x / per;
    r = __ldg(p.req + t);
    if (r < 0) return;
    q0 = __ldg(p.q_pos + r);
    x0 = (t - q0) * G + (blockIdx.x - t * per) * tile;
  } else {
    find_tile(p, G, tile, blockIdx.x, r, x0);
    if (r < 0) return;
    q0 = __ldg(p.q_pos + r);
  }
  qn = __ldg(p.q_pos + r + 1) - q0;
  const int n = SEL ? min(tile, G - x0 % G) : min(tile, qn * G - x0);
  const int shift = __ldg(p.k_len + r) - qn;  // position of the request's first new token
  const int p_first = shift + a.group.div(x0), p_last = shift + a.group.div(x0 + n - 1);

  // its keys: [u0, u1) of the request's keys, or of the picked pages' slots
  int end;
  if (SEL) {
    const int32_t* row = a.picked + ((int64_t)(q0 + x0 / G) * c.nheads + h) * a.npicked;
    if (tid == 0) sm.count = 0;
    __syncthreads();
    int most = 0;
    for (int i = tid; i < a.npicked; i += kThreads) {
      const int pg = __ldg(row + i);
      const bool ok = pg >= 0 && pg < p.width && pg <= c.page.div(max(p_last, 0));
      sm.window[i] = make_int2(ok ? __ldg(p.table + r * p.table_stride + pg) : -1, ok ? pg : -1);
      if (ok) most = i + 1;
    }
    if (most > 0) atomicMax(&sm.count, most);
    __syncthreads();
    end = sm.count * c.page.d;
  } else {
    end = max(p_last + 1, 0);
  }
  const int u0 = blockIdx.z * a.plan.chunk;
  if (!SEL && u0 > 0 && u0 >= end) return;
  const int u1 = max(min(end, u0 + a.plan.chunk), u0);
  const int steps = (u1 - u0 + kAttnKeys - 1) / kAttnKeys;

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

  const uint32_t base = (uint32_t)__cvta_generic_to_shared(tiles);
  int w0 = 0, w1 = 0;  // dense: entries of the block table in the window
  auto load = [&](int step) {
    if (step < steps) {
      const int ub = u0 + step * kAttnKeys, ue = min(ub + kAttnKeys, u1);
      if (!SEL) {
        const int need = c.page.div(ue - 1) + 1;
        if (need > w1) {  // the same for all threads
          __syncthreads();
          w0 = c.page.div(ub);
          w1 = min(w0 + kWindow, p.width);
          for (int i = tid; i < w1 - w0; i += kThreads)
            sm.window[i].x = __ldg(p.table + r * p.table_stride + w0 + i);
          __syncthreads();
        }
      }
      const uint32_t ks = base + (step % kStages) * stage_bytes<W>(), vs = ks + kAttnKeys * W * 2;
#pragma unroll
      for (int i = 0; i < kAttnKeys * PIECES / kThreads; ++i) {
        const int row = i * (kThreads / PIECES) + tid / PIECES, piece = tid % PIECES;
        const int u = ub + row;
        bool on = u < ue;
        int idx = 0, off = 0, id = -1;
        if (on) {
          idx = c.page.div(u);
          off = u - idx * c.page.d;
          const int2 w = sm.window[idx - w0];
          id = w.x;
          on = (unsigned)id < (unsigned)c.npages;
          if (SEL) {
            on = on && w.y >= 0 && w.y * c.page.d + off <= p_last;  // slots past the token hold anything
            if (piece == 0) sm.key_at[step % kStages][row] = on ? w.y * c.page.d + off : INT32_MAX;
          }
        } else if (SEL && piece == 0) {
          sm.key_at[step % kStages][row] = INT32_MAX;
        }
        on = on && piece * 8 < c.width;
        const int64_t pg = on ? id : 0;
        const int o = on ? off : 0, col = on ? piece * 8 : 0;
        copy16(ks + tile_offset<W>(row, piece), (const T*)c.k + pg * c.ks[0] + o * c.ks[1] + h * c.ks[2] + col, on);
        copy16(vs + tile_offset<W>(row, piece), (const T*)c.v + pg * c.vs[0] + o * c.vs[1] + h * c.vs[2] + col, on);
      }
    }
    copy_commit();
  };

  float o[W / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < W / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  const float sl2 = a.scale * 1.4426950408889634f;

#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) load(s);
  for (int step = 0; step < steps; ++step) {
    copy_wait<kStages - 2>();
    __syncthreads();
    load(step + kStages - 1);
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
      int key[2];
      if (SEL) {
        const int2 k2 = *reinterpret_cast<const int2*>(&sm.key_at[step % kStages][kb + j * 8 + (lane & 3) * 2]);
        key[0] = k2.x;
        key[1] = k2.y;
      } else {
        key[0] = ub + j * 8 + (lane & 3) * 2;
        key[1] = key[0] + 1;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[j][e] *= sl2;
        if (masked && key[e & 1] > pos[e >> 1]) s[j][e] = -INFINITY;
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
      const float b = mx == -INFINITY ? 0.f : mx;  // no key seen yet: every weight is 2^-inf
      scale_o[i] = exp2_fast(m[i] - b);
      m[i] = mx;
      l[i] *= scale_o[i];
#pragma unroll
      for (int j = 0; j < KW / 8; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[j][2 * i + e] = exp2_fast(s[j][2 * i + e] - b);
          l[i] += s[j][2 * i + e];
        }
    }
#pragma unroll
    for (int i = 0; i < W / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] *= scale_o[e >> 1];
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
    if ((lane & 3) == 0) sm.ml[warp][row] = make_float2(m[i], l[i]);
#pragma unroll
    for (int j = 0; j < W / 8; ++j)
      *reinterpret_cast<float2*>(rows + (warp * 16 + row) * (W + 4) + j * 8 + (lane & 3) * 2) =
          make_float2(o[j][2 * i], o[j][2 * i + 1]);
  }
  __syncthreads();

  // a group of PIECES lanes a row, 8 columns a lane
  const int splits = SEL ? a.plan.nsplit : (end > 0 ? (end - 1) / a.plan.chunk + 1 : 1);
  const int64_t hq = (int64_t)c.nheads * G;
  for (int x = tid / PIECES; x < n; x += kThreads / PIECES) {
    const int col = (tid % PIECES) * 8;
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
    const float lse2 = mx + __log2f(sum);  // no key: -inf
    const int tok = a.group.div(x0 + x), g = x0 + x - tok * G;
    const int64_t at = (q0 + tok) * hq + h * G + g;
    if (splits == 1) {
      if (col < c.width) {
        uint4 y;
        y.x = Half2<T>::pack(acc[0], acc[1]);
        y.y = Half2<T>::pack(acc[2], acc[3]);
        y.z = Half2<T>::pack(acc[4], acc[5]);
        y.w = Half2<T>::pack(acc[6], acc[7]);
        *reinterpret_cast<uint4*>((T*)a.out + at * c.width + col) = y;
      }
      if (col == 0 && a.lse) a.lse[at] = lse2 * 0.6931471805599453f;
    } else {
      const int64_t slot = at * a.plan.nsplit + blockIdx.z;
      if (col < c.width) {
        float4* y = reinterpret_cast<float4*>(a.plan.part + slot * c.width + col);
        y[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        y[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
      }
      if (col == 0) a.plan.part_lse[slot] = lse2;
    }
  }
}

// Rows of several splits: o = sum_s 2^(lse_s - m) o_s / sum_s 2^(lse_s - m), in
// the splits' order.  A warp a row.
template <typename T>
__global__ void __launch_bounds__(128)
k_paged_combine(AttnArgs a) {
  const PagesView& p = a.p;
  const int lane = threadIdx.x & 31, G = a.group.d;
  const int64_t hq = (int64_t)a.c.nheads * G, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (at >= p.ntok * hq) return;
  const int t = (int)(at / hq), g = (int)(at % hq) % G;
  const int r = __ldg(p.req + t);
  if (r < 0) return;
  int splits = a.plan.nsplit;
  if (!a.picked) {
    const int q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
    const int x = (t - q0) * G + g, last = min((x / a.plan.tile + 1) * a.plan.tile, qn * G) - 1;
    const int end = __ldg(p.k_len + r) - qn + last / G + 1;
    splits = end > 0 ? (end - 1) / a.plan.chunk + 1 : 1;
  }
  if (splits == 1) return;
  const float* lse = a.plan.part_lse + at * a.plan.nsplit;
  float m = -INFINITY;
  for (int s = lane; s < splits; s += 32) m = fmaxf(m, lse[s]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float b = m == -INFINITY ? 0.f : m;
  const int col = 4 * lane;
  const float* part = a.plan.part + at * a.plan.nsplit * a.c.width + col;
  float sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float f = exp2_fast(lse[s] - b);
    sum += f;
    if (col < a.c.width) {
      const float4 x = *reinterpret_cast<const float4*>(part + (int64_t)s * a.c.width);
      acc.x += f * x.x;
      acc.y += f * x.y;
      acc.z += f * x.z;
      acc.w += f * x.w;
    }
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

template <typename T, int W, int WM, bool SEL>
cudaError_t launch_rows(const AttnArgs& a, cudaStream_t s) {
  auto kernel = k_paged_rows<T, W, WM, SEL>;
  static_assert(4 * 16 * (W + 4) * 4 <= (int)smem_bytes<W>(), "the joined rows fit in the stages");
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<W>());
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.plan.ntiles, (unsigned)a.c.nheads, (unsigned)a.plan.nsplit);
  kernel<<<(SLNR_COUNTED(grid)), kThreads, smem_bytes<W>(), s>>>(a);
  return cudaGetLastError();
}

template <typename T, int W>
cudaError_t launch_rows_w(const AttnArgs& a, cudaStream_t s) {
  const bool sel = a.picked != nullptr;
  switch (a.plan.tile) {
    case 16: return sel ? launch_rows<T, W, 1, true>(a, s) : launch_rows<T, W, 1, false>(a, s);
    case 32: return sel ? launch_rows<T, W, 2, true>(a, s) : launch_rows<T, W, 2, false>(a, s);
    default: return sel ? launch_rows<T, W, 4, true>(a, s) : launch_rows<T, W, 4, false>(a, s);
  }
}

template <typename T>
cudaError_t launch_rows_t(const AttnArgs& a, cudaStream_t s) {
  return a.c.width <= 64 ? launch_rows_w<T, 64>(a, s) : launch_rows_w<T, 128>(a, s);
}

}  // namespace

cudaError_t launch_paged_rows(const AttnArgs& a, int dtype, cudaStream_t s) {
  return dtype == SLNR_FP16 ? launch_rows_t<__half>(a, s) : launch_rows_t<__nv_bfloat16>(a, s);
}

cudaError_t launch_paged_combine(const AttnArgs& a, int dtype, cudaStream_t s) {
  const int64_t rows = (int64_t)a.p.ntok * a.c.nheads * a.group.d;
  const unsigned grid = (unsigned)ceil_div(rows, 4);
  auto kernel = dtype == SLNR_FP16 ? k_paged_combine<__half> : k_paged_combine<__nv_bfloat16>;
  kernel<<<SLNR_COUNTED(grid), 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace slnr
