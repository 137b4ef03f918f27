// Attention of chunks of new tokens over a paged cache, on the tcgen05 tensor
// cores.
//
// A block takes 256 rows (two tiles of 128: the query rows of one key head's
// group, token after token) and streams their keys, 128 at a time.  Tensor
// memory holds both tiles' scores S (128 x 128 fp32) and outputs O; the weights
// P, rounded to the cache's type, are written over the scores that they come
// from and are the A operand of the product with V.
//   8 softmax warps: one row of a tile a thread; scores out of tensor memory,
//       maximum, weights and their sum, weights back.  O is rescaled only where
//       a row's maximum grew by more than 2^8 since the last time: until then
//       its weights are taken against the older maximum, at most 256 each, and
//       the sum is in the same units, so the quotient is the same;
//   1 MMA warp:  for each 128 keys and tile: O += P V, then the next S = Q K^T;
//   3 load warps: Q once, then K and V into a ring of buffers of 128 keys by
//       asynchronous 16-byte copies, each key's row by its page (any page size
//       and stride), zeros past the last key.
// While one tile's warps are at its weights, the tensor cores work on the
// other's.  Keys in 128-byte swizzled rows serve both products: K as the
// K-major operand of Q K^T, V as the MN-major one of P V.
#include <type_traits>

#include "launch.h"
#include "mma16.cuh"
#include "paged_tile.cuh"
#include "tcgen05.cuh"

namespace slnr {
namespace {

constexpr int kRows = 128;              // of a tile
constexpr int kSoftWarps = 8;
constexpr int kMmaWarp = kSoftWarps;
constexpr int kLoadWarps = 3;
constexpr int kLoaders = 32 * kLoadWarps;
constexpr int kThreads = 32 * (kSoftWarps + 1 + kLoadWarps);
constexpr int kBlock = kRows * 128;     // 128 rows of 64 values, swizzled
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 256;   // S and P of tile t at 128 t, O at kColO + 128 t
constexpr float kGrow = 8.f;            // growth of a maximum, in powers of two, that O is rescaled for

template <int W>
constexpr int tile_bytes() { return kBlock * (W / 64); }
template <int W>
constexpr int buffers() { return W == 128 ? 5 : 8; }
template <int W>
constexpr size_t smem_bytes() { return (size_t)(2 + buffers<W>()) * tile_bytes<W>() + 1024; }
static_assert(smem_bytes<128>() + 512 <= (size_t)227 * 1024, "shared memory of a block");

struct Barriers {
  uint64_t q_full, s_full[2], p_full[2], o_full, full[8], empty[8], drained;
  uint32_t tmem;
  int failed;
};

// Waits for the phase of that parity; false (and *failed set) after `limit` cycles or once another wait gave up.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* failed, long long limit) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!tc::mbar_try_wait(bar, parity)) {
    if (*failed) return false;
    if (clock64() - t0 > limit) {
      *failed = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* failed, long long limit) {
  return __all_sync(0xffffffffu, wait(bar, parity, failed, limit));
}

// Byte of 16-byte piece `piece` of a row inside a swizzled tile of 128 rows.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  return (uint32_t)((piece >> 3) * kBlock + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

template <typename T, int W>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_chunk(AttnArgs a, WsHeader* hdr, long long limit) {
  constexpr int PIECES = W / 8, NB = buffers<W>();
  extern __shared__ unsigned char smem_raw[];
  __shared__ Barriers bars;
  const PagesView& p = a.p;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.group.d, h = blockIdx.x;

  int r, x0;
  find_tile(p, G, kChunkRows, gridDim.y - 1 - blockIdx.y, r, x0);  // the last tiles see the most keys: first
  if (r < 0) return;
  const int q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
  const int n = min(kChunkRows, qn * G - x0), tiles = n > kRows ? 2 : 1;
  const int shift = __ldg(p.k_len + r) - qn;
  const int end = max(shift + a.group.div(x0 + n - 1) + 1, 0);
  const int u0 = blockIdx.z * a.plan.chunk;
  if (u0 > 0 && u0 >= end) return;
  const int u1 = max(min(end, u0 + a.plan.chunk), u0);
  const int steps = (u1 - u0 + kChunkKeys - 1) / kChunkKeys;

  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  auto q_tile = [&](int t) { return base + t * tile_bytes<W>(); };
  auto buffer = [&](int b) { return base + (2 + b) * tile_bytes<W>(); };
  if (tid == 0) {
    tc::mbar_init(&bars.q_full, kLoaders);
    tc::mbar_init(&bars.o_full, 1);
    tc::mbar_init(&bars.drained, 1);
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(&bars.s_full[t], 1);
      tc::mbar_init(&bars.p_full[t], kRows);
    }
    for (int b = 0; b < NB; ++b) {
      tc::mbar_init(&bars.full[b], kLoaders);
      tc::mbar_init(&bars.empty[b], 1);
    }
    bars.failed = 0;
    tc::fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tc::tmem_alloc(&bars.tmem, kTmemCols);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::tc_fence_after_sync();
  const uint32_t tmem = bars.tmem;
  volatile int* failed = &bars.failed;

  if (warp > kMmaWarp) {
    // ---- loads ----
    const int lt = tid - 32 * (kMmaWarp + 1), piece = lt % PIECES;
    const bool col_on = piece * 8 < c.width;
    for (int x = lt / PIECES; x < 2 * kRows; x += kLoaders / PIECES) {
      const bool on = x < n && col_on;
      const int tok = on ? a.group.div(x0 + x) : 0, g = on ? x0 + x - tok * G : 0;
      copy16(q_tile(x / kRows) + piece_at(x % kRows, piece),
             (const T*)a.q.p + (int64_t)(q0 + tok) * a.q.tok + (int64_t)(h * G + g) * a.q.head + (on ? piece * 8 : 0), on);
    }
    copy_commit();
    // ring step i: K of keys i / 2 (i even) or V; a step's copies are waited for two steps later
    const int total = 2 * steps;
    const int32_t* table = p.table + r * p.table_stride;
    for (int i = 0; i < total + 2; ++i) {
      if (i < total) {
        const int b = i % NB;
        if (!wait_warp(&bars.empty[b], ((i / NB) & 1) ^ 1, failed, limit)) break;
        const uint32_t dst = buffer(b);
        const int ub = u0 + (i >> 1) * kChunkKeys;
        const char* src = (const char*)((i & 1) ? c.v : c.k);
        const int64_t* st = (i & 1) ? c.vs : c.ks;
        const int64_t s0 = st[0] * 2, s1 = st[1] * 2;
        src += st[2] * 2 * h + (col_on ? piece * 16 : 0);
        constexpr int STEP = kLoaders / PIECES, BATCH = 8;
        for (int row0 = lt / PIECES; row0 < kChunkKeys; row0 += STEP * BATCH) {
          int id[BATCH], off[BATCH];
#pragma unroll
          for (int k = 0; k < BATCH; ++k) {
            const int u = ub + row0 + k * STEP;
            id[k] = -1;
            off[k] = 0;
            if (row0 + k * STEP < kChunkKeys && u < u1) {
              const int idx = c.page.div(u);
              off[k] = u - idx * c.page.d;
              if (idx < p.width) id[k] = __ldg(table + idx);
            }
          }
#pragma unroll
          for (int k = 0; k < BATCH; ++k) {
            const int row = row0 + k * STEP;
            if (row < kChunkKeys) {
              const bool on = col_on && (unsigned)id[k] < (unsigned)c.npages;
              copy16(dst + piece_at(row, piece), src + (on ? id[k] * s0 + off[k] * s1 : 0), on);
            }
          }
        }
      }
      copy_commit();
      if (i >= 1) {
        copy_wait<2>();
        tc::fence_proxy_async_smem();
        if (i == 1) tc::mbar_arrive(&bars.q_full);
        if (i >= 2) tc::mbar_arrive(&bars.full[(i - 2) % NB]);
      }
    }
    copy_wait<0>();
  } else if (warp == kMmaWarp) {
    // ---- products ----
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
    const uint32_t id_s = tc::idesc_f16(type, kRows, kChunkKeys, false);
    const int no = (c.width + 15) & ~15;  // columns of O
    const uint32_t id_o = tc::idesc_f16(type, kRows, no, true);
    const int ksteps = (c.width + 15) / 16;
    auto scores = [&](int t, int b) {
      if (lane == 0) {
        for (int k = 0; k < ksteps; ++k) {
          const uint32_t at = (k >> 2) * kBlock + (k & 3) * 32;
          tc::mma_f16(tmem + kColS + t * 128, tc::desc_k_sw128(q_tile(t) + at), tc::desc_k_sw128(buffer(b) + at), id_s, k > 0);
        }
        tc::mma_commit(&bars.s_full[t]);
      }
    };
    auto output = [&](int t, int b, bool first) {
      if (lane == 0)
        for (int k = 0; k < kChunkKeys / 16; ++k)
          tc::mma_f16_ta(tmem + kColO + t * 128, tmem + kColS + t * 128 + 8 * k,
                         tc::desc_mn_sw128(buffer(b) + k * 2048, kBlock), id_o, !first || k > 0);
    };
    auto release = [&](int b) {
      if (lane == 0) tc::mma_commit(&bars.empty[b]);
    };
    bool ok = steps > 0 && wait_warp(&bars.q_full, 0, failed, limit) && wait_warp(&bars.full[0], 0, failed, limit);
    if (ok) {
      tc::tc_fence_after_sync();
      for (int t = 0; t < tiles; ++t) scores(t, 0);
      release(0);
    }
    for (int j = 0; ok && j < steps; ++j) {
      const int iv = 2 * j + 1, ik = 2 * j + 2;  // ring steps of V and of the next K
      ok = wait_warp(&bars.full[iv % NB], (iv / NB) & 1, failed, limit);
      if (ok && j + 1 < steps) ok = wait_warp(&bars.full[ik % NB], (ik / NB) & 1, failed, limit);
      for (int t = 0; ok && t < tiles; ++t) {
        ok = wait_warp(&bars.p_full[t], j & 1, failed, limit);
        if (!ok) break;
        tc::tc_fence_after_sync();
        output(t, iv % NB, j == 0);
        if (t == tiles - 1) release(iv % NB);
        if (j + 1 < steps) {
          scores(t, ik % NB);
          if (t == tiles - 1) release(ik % NB);
        }
      }
    }
    if (ok && lane == 0) tc::mma_commit(&bars.o_full);
  } else if ((warp >> 2) < tiles) {
    // ---- softmax: thread = row ----
    const int t = warp >> 2, x = t * kRows + (warp & 3) * 32 + lane;
    const bool row_on = x < n;
    const int tok = row_on ? a.group.div(x0 + x) : 0, g = row_on ? x0 + x - tok * G : 0;
    const int pos = row_on ? shift + tok : -1;
    const int pos_min = shift + a.group.div(x0 + t * kRows);  // of the tile's rows
    const bool tail = n - t * kRows < kRows;                  // rows that are none: their scores are dropped
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t col_s = tmem + lanes + kColS + t * 128, col_o = tmem + lanes + kColO + t * 128;
    // scores are kept raw and take their factor inside the exponential; one that is not positive goes to them first
    const bool raw = a.scale > 0.f;
    const float factor = a.scale * 1.4426950408889634f, sl2 = raw ? factor : 1.f;
    float m = -INFINITY, l = 0.f;  // maximum of the scores that weights are taken against, sum of weights
    bool ok = true;
    for (int j = 0; j < steps; ++j) {
      ok = wait_warp(&bars.s_full[t], j & 1, failed, limit);
      if (!ok) break;
      tc::tc_fence_after_sync();
      uint32_t s[128];
#pragma unroll
      for (int k = 0; k < 4; ++k) tc::tmem_ld32_start(col_s + 32 * k, s + 32 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k) tc::tmem_ld_done(s + 32 * k);
      if (!raw) {
#pragma unroll
        for (int k = 0; k < 128; ++k) s[k] = __float_as_uint(__uint_as_float(s[k]) * factor);
      }
      const int key0 = u0 + j * kChunkKeys;
      if (tail || key0 + kChunkKeys - 1 > pos_min) {
        const int seen = pos - key0;  // keys 0 .. seen of these 128
#pragma unroll
        for (int k = 0; k < 128; ++k)
          if (k > seen) s[k] = 0xff800000u;
      }
      float mx[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) mx[k] = __uint_as_float(s[k]);
#pragma unroll
      for (int k = 4; k < 128; ++k) mx[k & 3] = fmaxf(mx[k & 3], __uint_as_float(s[k]));
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      // the first keys that a row sees set m; later m moves only where it has to
      const bool grow = (top - m) * sl2 > kGrow;  // m = -inf: true for any seen key
      if (__any_sync(0xffffffffu, grow)) {
        const float f = grow ? exp2_fast((m - top) * sl2) : 1.f;
        if (grow) {
          l *= f;
          m = top;
        }
        if (j > 0) {
#pragma unroll
          for (int k = 0; k < W / 16; ++k) {
            float o[16];
            uint32_t y[16];
            tc::tmem_ld16(col_o + 16 * k, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(o[e] * f);
            tc::tmem_st16(col_o + 16 * k, y);
          }
        }
      }
      const float b = m == -INFINITY ? 0.f : m * sl2;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float w0 = exp2_fast(fmaf(__uint_as_float(s[32 * k + 2 * e]), sl2, -b));
          const float w1 = exp2_fast(fmaf(__uint_as_float(s[32 * k + 2 * e + 1]), sl2, -b));
          sum[(2 * e) & 3] += w0;
          sum[(2 * e + 1) & 3] += w1;
          w[e] = Half2<T>::pack(w0, w1);
        }
        tc::tmem_st16(col_s + 16 * k, w);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      tc::tmem_st_done();
      tc::tc_fence_before_sync();
      tc::mbar_arrive(&bars.p_full[t]);
    }
    if (ok && steps > 0) ok = wait_warp(&bars.o_full, 0, failed, limit);
    if (ok) {
      tc::tc_fence_after_sync();
      const int splits = end > 0 ? (end - 1) / a.plan.chunk + 1 : 1;
      const int64_t at = (q0 + tok) * ((int64_t)c.nheads * G) + h * G + g;
      const int64_t slot = at * a.plan.nsplit + blockIdx.z;
      const float inv = __fdividef(1.f, l);
      const float lse2 = l == 0.f ? -INFINITY : m * sl2 + __log2f(l);
#pragma unroll
      for (int k = 0; k < W / 32; ++k) {
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
        if (steps > 0) tc::tmem_ld32(col_o + 32 * k, o);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = l == 0.f ? 0.f : o[e] * inv;  // no key: zeros
        if (!row_on) continue;
        if (splits == 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (32 * k + 8 * e < c.width) {
              uint4 y;
              y.x = Half2<T>::pack(o[8 * e], o[8 * e + 1]);
              y.y = Half2<T>::pack(o[8 * e + 2], o[8 * e + 3]);
              y.z = Half2<T>::pack(o[8 * e + 4], o[8 * e + 5]);
              y.w = Half2<T>::pack(o[8 * e + 6], o[8 * e + 7]);
              *reinterpret_cast<uint4*>((T*)a.out + at * c.width + 32 * k + 8 * e) = y;
            }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (32 * k + 4 * e < c.width)
              *reinterpret_cast<float4*>(a.plan.part + slot * c.width + 32 * k + 4 * e) =
                  make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      }
      if (row_on) {
        if (splits != 1) a.plan.part_lse[slot] = lse2;
        else if (a.lse) a.lse[at] = lse2 * 0.6931471805599453f;
      }
    }
  }

  __syncwarp();
  tc::tc_fence_before_sync();
  __syncthreads();
  if (*failed) {
    if (warp == kMmaWarp && lane == 0) {  // the products that were issued end before the tensor memory is freed
      tc::mma_commit(&bars.drained);
      const long long t0 = clock64();
      while (!tc::mbar_try_wait(&bars.drained, 0))
        if (clock64() - t0 > kWaitCycles) break;
    }
    if (tid == 0) atomicOr(&hdr->error, kErrTimeout);
  }
  __syncthreads();
  tc::tc_fence_after_sync();
  if (warp == kMmaWarp) tc::tmem_dealloc(tmem, kTmemCols);
}

template <typename T, int W>
cudaError_t launch(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  auto kernel = k_paged_chunk<T, W>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<W>());
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.c.nheads, (unsigned)a.plan.ntiles, (unsigned)a.plan.nsplit);
  kernel<<<(SLNR_COUNTED(grid)), kThreads, smem_bytes<W>(), s>>>(a, hdr, wait_limit_cycles());
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_chunk(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s) {
  if (a.c.width <= 64) return dtype == SLNR_FP16 ? launch<__half, 64>(a, hdr, s) : launch<__nv_bfloat16, 64>(a, hdr, s);
  return dtype == SLNR_FP16 ? launch<__half, 128>(a, hdr, s) : launch<__nv_bfloat16, 128>(a, hdr, s);
}

}  // namespace slnr
