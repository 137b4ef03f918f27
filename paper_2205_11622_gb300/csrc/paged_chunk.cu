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
//   4 load warps: Q once, then K and V into a ring of buffers of 128 keys by
//       asynchronous 16-byte copies (any page size and stride), zeros past the
//       last key.  Each thread finds one key's row by its page, a step ahead,
//       and all read the rows' offsets from shared memory.
// Picked pages: a block streams every page that a token of its rows picked, in
// ascending order (k_paged_union lists them, with the tokens that picked each),
// and a row's weights are zero in pages that its token did not pick.  A page is
// read once for all tokens that share it, and never more pages are multiplied
// than the tokens picked in all.
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
constexpr int kLoadWarp = 8;            // warps 0-7: softmax
constexpr int kLoaders = 128;
constexpr int kMmaWarp = 12;            // 13-15 only complete its warpgroup
constexpr int kThreads = 512;
constexpr int kSoftRegs = 200, kOtherRegs = 56;  // of 128 a thread at launch
static_assert(2 * (kSoftRegs + kOtherRegs) <= 4 * 128, "register shares of the four warpgroups");
static_assert(kLoaders == kChunkKeys, "a load thread finds one key's row");
constexpr int kBlock = kRows * 128;     // 128 rows of 64 values, swizzled
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 256;   // S and P of tile t at 128 t, O at kColO + 128 t
constexpr float kGrow = 8.f;            // growth of a maximum, in powers of two, that O is rescaled for

template <int W>
constexpr int tile_bytes() { return kBlock * (W / 64); }
template <int W>
constexpr int buffers() { return W == 128 ? 4 : 8; }
template <int W>
constexpr size_t smem_bytes() { return (size_t)(2 + buffers<W>()) * tile_bytes<W>() + 1024; }
template <int W>
constexpr int lag() { return buffers<W>() - 2; }  // ring steps in flight before one is waited for

struct Barriers {
  uint64_t q_full, s_full[2], p_full[2], o_full, full[8], empty[8], drained;
  uint32_t tmem;
  int failed;
  int64_t row_k[2][kChunkKeys], row_v[2][kChunkKeys];  // bytes from the head's first row to each key's; -1: zeros
};

static_assert(smem_bytes<128>() + sizeof(Barriers) <= (size_t)227 * 1024, "shared memory of a block");

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

// Drops the scores of the keys that a row does not see: those past seen[g] of
// segment g, for `segs` (a power of two) equal segments.
template <int SEGS>
__device__ __forceinline__ void mask_equal(uint32_t (&s)[128], const int (&seen)[8]) {
#pragma unroll
  for (int k = 0; k < 128; ++k)
    if (k % (128 / SEGS) > seen[k / (128 / SEGS)]) s[k] = 0xff800000u;
}
__device__ __forceinline__ void mask_segments(uint32_t (&s)[128], const int (&seen)[8], int segs) {
  switch (segs) {
    case 1: return mask_equal<1>(s, seen);
    case 2: return mask_equal<2>(s, seen);
    case 4: return mask_equal<4>(s, seen);
    default: return mask_equal<8>(s, seen);
  }
}

// Register shares of the calling warpgroup.
template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// The pages that the tokens of a row tile picked for one head, and who picked
// each: bits set in shared memory for 1024 pages at a time, then the pages with
// any written in order.
constexpr int kUnionThreads = 256;
constexpr int kUnionPages = 1024;
constexpr int kMaxWords = 8;  // 256 tokens of one row each

__global__ void __launch_bounds__(kUnionThreads)
k_paged_union(AttnArgs a) {
  __shared__ uint32_t s_bits[kUnionPages * kMaxWords];
  __shared__ int s_count[kUnionThreads / 32 + 1];
  const PagesView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.x, words = a.plan.words;
  int r, x0;
  find_tile(p, a.group.d, kChunkRows, blockIdx.y, r, x0);
  const int64_t at = (int64_t)blockIdx.y * gridDim.x + h;
  if (r < 0) {
    if (tid == 0) a.plan.npages[at] = 0;
    return;
  }
  const int q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
  const int n = min(kChunkRows, qn * a.group.d - x0), shift = __ldg(p.k_len + r) - qn;
  const int t0 = a.group.div(x0), t1 = a.group.div(x0 + n - 1) + 1;
  const int last = shift + t1 - 1;
  const int npages = last < 0 ? 0 : min(a.c.page.div(last) + 1, p.width);
  int total = 0;
  for (int w0 = 0; w0 < npages; w0 += kUnionPages) {
    for (int i = tid; i < kUnionPages * words; i += kUnionThreads) s_bits[i] = 0;
    __syncthreads();
    for (int i = tid; i < (t1 - t0) * a.npicked; i += kUnionThreads) {
      const int t = i / a.npicked, pg = __ldg(a.picked + ((int64_t)(q0 + t0 + t) * a.c.nheads + h) * a.npicked + i % a.npicked);
      const int pos = shift + t0 + t;
      if (pg >= w0 && pg < w0 + kUnionPages && pg < npages && pos >= 0 && pg <= a.c.page.div(pos))
        atomicOr(&s_bits[(pg - w0) * words + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    // each warp lists 128 pages
    constexpr int SHARE = kUnionPages / (kUnionThreads / 32);
    uint32_t any[SHARE / 32];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < SHARE / 32; ++k) {
      const uint32_t* b = s_bits + (warp * SHARE + k * 32 + lane) * words;
      uint32_t x = 0;
      for (int w = 0; w < words; ++w) x |= b[w];
      any[k] = __ballot_sync(0xffffffffu, x != 0);
      mine += __popc(any[k]);
    }
    if (lane == 0) s_count[warp] = mine;
    __syncthreads();
    int e = total;
    for (int w = 0; w < kUnionThreads / 32; ++w) {
      if (w < warp) e += s_count[w];
      total += s_count[w];
    }
#pragma unroll
    for (int k = 0; k < SHARE / 32; ++k) {
      const int slot = e + __popc(any[k] & ((1u << lane) - 1)), local = warp * SHARE + k * 32 + lane;
      if (((any[k] >> lane) & 1) && slot < a.plan.cap) {
        a.plan.pages[at * a.plan.cap + slot] = w0 + local;
        for (int w = 0; w < words; ++w) a.plan.pickers[(at * a.plan.cap + slot) * words + w] = s_bits[local * words + w];
      }
      e += __popc(any[k]);
    }
    __syncthreads();
  }
  if (tid == 0) a.plan.npages[at] = min(total, a.plan.cap);
}

template <typename T, int W, bool SEL>
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
  const int row_tile = gridDim.y - 1 - blockIdx.y;  // the last tiles see the most keys: first
  find_tile(p, G, kChunkRows, row_tile, r, x0);
  if (r < 0) return;
  const int q0 = __ldg(p.q_pos + r), qn = __ldg(p.q_pos + r + 1) - q0;
  const int n = min(kChunkRows, qn * G - x0), tiles = n > kRows ? 2 : 1;
  const int shift = __ldg(p.k_len + r) - qn;
  // its keys: [u0, u1) of the request's keys, or of the slots of the listed pages
  const int last = shift + a.group.div(x0 + n - 1);  // position of the last row's token
  const int64_t list_at = ((int64_t)row_tile * gridDim.x + h) * a.plan.cap;
  int u0, u1, splits;
  if (SEL) {
    const int end = __ldg(a.plan.npages + (int64_t)row_tile * gridDim.x + h) * c.page.d;
    splits = a.plan.nsplit;
    const int share = ((end + kChunkKeys - 1) / kChunkKeys + splits - 1) / splits * kChunkKeys;
    u0 = min((int)blockIdx.z * share, end);
    u1 = min(u0 + share, end);
  } else {
    const int end = max(last + 1, 0);
    splits = end > 0 ? (end - 1) / a.plan.chunk + 1 : 1;
    u0 = blockIdx.z * a.plan.chunk;
    if (u0 > 0 && u0 >= end) return;
    u1 = max(min(end, u0 + a.plan.chunk), u0);
  }
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

  if (warp >= kLoadWarp) {
    regs_down<kOtherRegs>();
    if (warp < kMmaWarp) {
      // ---- loads ----
      constexpr int ROWS = kLoaders / PIECES;  // rows of a pass: a multiple of 8, so a thread's swizzle is fixed
      const int lt = tid - 32 * kLoadWarp, piece = lt % PIECES, row0 = lt / PIECES;
      const bool col_on = piece * 8 < c.width;
      const uint32_t at = piece_at(row0, piece);
      for (int x = row0; x < 2 * kRows; x += ROWS) {
        const bool on = x < n && col_on;
        const int tok = on ? a.group.div(x0 + x) : 0, g = on ? x0 + x - tok * G : 0;
        copy16(q_tile(x / kRows) + piece_at(x % kRows, piece),
               (const T*)a.q.p + (int64_t)(q0 + tok) * a.q.tok + (int64_t)(h * G + g) * a.q.head + (on ? piece * 8 : 0), on);
      }
      copy_commit();
      const int32_t* table = p.table + r * p.table_stride;
      const char* src_k = (const char*)c.k + 2 * (c.ks[2] * h + (col_on ? piece * 8 : 0));
      const char* src_v = (const char*)c.v + 2 * (c.vs[2] * h + (col_on ? piece * 8 : 0));
      int id = -1, off = 0, next = -1;  // next: the listed page of the key after
      auto listed = [&](int j) {
        const int u = u0 + j * kChunkKeys + lt;
        next = SEL && u < u1 ? __ldg(a.plan.pages + list_at + c.page.div(u)) : -1;
      };
      auto find = [&](int j) {  // page and slot of this thread's key of step j
        const int u = u0 + j * kChunkKeys + lt;
        id = -1;
        if (u < u1) {
          int i = c.page.div(u);
          off = u - i * c.page.d;
          if (SEL) i = next;
          if (i < p.width && (!SEL || i * c.page.d + off <= last)) id = __ldg(table + i);
        }
        if (SEL) listed(j + 1);
      };
      if (SEL) listed(0);
      find(0);
      // ring step i: K of keys i / 2 (i even) or V; its copies are waited for `lag` steps later
      const int total = 2 * steps;
      constexpr int LAG = lag<W>();
      bool ok = true;  // where a wait gave up the loop goes on without copies: its warps meet at a barrier
      for (int i = 0; i < total + LAG; ++i) {
        // hand over what has landed before waiting for room: the copies of step i - 1 stay in flight
        if (ok && i >= LAG - 1) {
          copy_wait<LAG - 1>();
          tc::fence_proxy_async_smem();
          tc::mbar_arrive(i == LAG - 1 ? &bars.q_full : &bars.full[(i - LAG) % NB]);
        }
        if (i < total) {
          const int j = i >> 1, b = i % NB;
          if (!(i & 1)) {
            const bool on = (unsigned)id < (unsigned)c.npages;
            bars.row_k[j & 1][lt] = on ? 2 * (id * c.ks[0] + off * c.ks[1]) : -1;
            bars.row_v[j & 1][lt] = on ? 2 * (id * c.vs[0] + off * c.vs[1]) : -1;
            find(j + 1);
            asm volatile("bar.sync 1, 128;" ::: "memory");
          }
          ok = ok && wait_warp(&bars.empty[b], ((i / NB) & 1) ^ 1, failed, limit);
          const uint32_t dst = buffer(b) + at;
          const char* src = (i & 1) ? src_v : src_k;
          const int64_t* rows = ((i & 1) ? bars.row_v[j & 1] : bars.row_k[j & 1]) + row0;
          if (ok) {
            constexpr int HALF = kChunkKeys / ROWS / 2;  // offsets are read ahead of the copies that wait for them
#pragma unroll
            for (int k0 = 0; k0 < 2 * HALF; k0 += HALF) {
              int64_t o[HALF];
#pragma unroll
              for (int k = 0; k < HALF; ++k) o[k] = rows[(k0 + k) * ROWS];
#pragma unroll
              for (int k = 0; k < HALF; ++k) {
                const bool on = col_on && o[k] >= 0;
                copy16(dst + (k0 + k) * ROWS * 128, src + (on ? o[k] : 0), on);
              }
            }
          }
        }
        copy_commit();
      }
      copy_wait<0>();
    } else if (warp == kMmaWarp) {
      // ---- products ----
      const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
      const uint32_t id_s = tc::idesc_f16(type, kRows, kChunkKeys, false);
      const int no = (c.width + 15) & ~15;  // columns of O
      const uint32_t id_o = tc::idesc_f16(type, kRows, no, true);
      const int ksteps = (c.width + 15) / 16;
      // descriptors differ from the first tile's, buffer's and step's by their address, in units of 16 bytes
      const uint64_t q_desc = tc::desc_k_sw128(q_tile(0)), k_desc = tc::desc_k_sw128(buffer(0));
      const uint64_t v_desc = tc::desc_mn_sw128(buffer(0), kBlock);
      constexpr uint64_t TILE = tile_bytes<W>() >> 4;
      auto scores = [&](int t, int b) {
        const uint64_t qd = q_desc + t * TILE, kd = k_desc + b * TILE;
        if (tc::elect_one()) {
#pragma unroll
          for (int k = 0; k < W / 16; ++k) {
            const uint64_t at = ((k >> 2) * kBlock + (k & 3) * 32) >> 4;
            if (k < ksteps) tc::mma_f16(tmem + kColS + t * 128, qd + at, kd + at, id_s, k > 0);
          }
          tc::mma_commit(&bars.s_full[t]);
        }
      };
      auto output = [&](int t, int b, bool first) {
        const uint64_t vd = v_desc + b * TILE;
        const uint32_t o = tmem + kColO + t * 128, w = tmem + kColS + t * 128;
        if (tc::elect_one()) {
#pragma unroll
          for (int k = 0; k < kChunkKeys / 16; ++k)
            tc::mma_f16_ta(o, w + 8 * k, vd + k * (2048 >> 4), id_o, !first || k > 0);
        }
      };
      auto release = [&](int b) {
        if (tc::elect_one()) tc::mma_commit(&bars.empty[b]);
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
      if (ok && tc::elect_one()) tc::mma_commit(&bars.o_full);
    }
  } else {
    regs_up<kSoftRegs>();
    if ((warp >> 2) < tiles) {
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
      // selected: the row's token in the tile, its page's bit and last slot seen in a listed page
      const int tl = tok - a.group.div(x0), segs = SEL ? (c.page.d < kChunkKeys ? kChunkKeys / c.page.d : 1) : 0;
      const uint32_t* pickers = a.plan.pickers + list_at * a.plan.words + (row_on ? tl >> 5 : 0);
      for (int j = 0; j < steps; ++j) {
        int seen_in[8];  // per segment of the step: keys 0 .. seen_in of it
        if (SEL) {
#pragma unroll
          for (int g2 = 0; g2 < 8; ++g2) {
            seen_in[g2] = -1;
            const int u = u0 + j * kChunkKeys + g2 * c.page.d;
            if (g2 < segs && u < u1 && row_on) {
              const int e = c.page.div(u);
              const int pg = __ldg(a.plan.pages + list_at + e);
              const bool on = (__ldg(pickers + (int64_t)e * a.plan.words) >> (tl & 31)) & 1;
              if (on) seen_in[g2] = pos - pg * c.page.d - (u - e * c.page.d);
            }
          }
        }
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
        if (SEL) {
          mask_segments(s, seen_in, segs);
        } else if (tail || key0 + kChunkKeys - 1 > pos_min) {
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
  }

  __syncwarp();
  tc::tc_fence_before_sync();
  __syncthreads();
  if (*failed) {
    if (warp == kMmaWarp && tc::elect_one()) {  // the products that were issued end before the tensor memory is freed
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

template <typename T, int W, bool SEL>
cudaError_t launch(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  auto kernel = k_paged_chunk<T, W, SEL>;
  static OncePerDevice once;
  cudaError_t e = once(
      [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<W>()); });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)a.c.nheads, (unsigned)a.plan.ntiles, (unsigned)a.plan.nsplit);
  kernel<<<(SLNR_COUNTED(grid)), kThreads, smem_bytes<W>(), s>>>(a, hdr, wait_limit_cycles());
  return cudaGetLastError();
}

template <typename T, bool SEL>
cudaError_t launch_w(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  return a.c.width <= 64 ? launch<T, 64, SEL>(a, hdr, s) : launch<T, 128, SEL>(a, hdr, s);
}

}  // namespace

cudaError_t launch_paged_union(const AttnArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.c.nheads, (unsigned)a.plan.ntiles);
  k_paged_union<<<(SLNR_COUNTED(grid)), kUnionThreads, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_paged_chunk(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s) {
  if (a.picked) return dtype == SLNR_FP16 ? launch_w<__half, true>(a, hdr, s) : launch_w<__nv_bfloat16, true>(a, hdr, s);
  return dtype == SLNR_FP16 ? launch_w<__half, false>(a, hdr, s) : launch_w<__nv_bfloat16, false>(a, hdr, s);
}

}  // namespace slnr
