// Attention of chunks of new tokens over a paged cache, on the tcgen05 tensor
// cores.
//
// An item is 256 rows (two tiles of 128: the query rows of one key head's group,
// token after token) with all their keys, 128 a step.  One block runs on each
// SM; the steps of all items, one after another, are cut into as many equal
// shares, so a block ends one item, takes some whole ones and begins another,
// and k_paged_join adds up the items that a cut went through.  (A block an item,
// the last wave of a 4096-token chunk left a fifth of the time unused.)  Tensor
// memory holds both tiles' scores S (128 x 128 fp32) and outputs O; the weights
// P, rounded to the cache's type, are written over the scores that they come
// from and are the A operand of the product with V.
//   8 softmax warps: one row of a tile a thread; scores out of tensor memory,
//       maximum, weights and their sum, weights back.  O is rescaled only where
//       a row's maximum grew by more than 2^8 since the last time: until then
//       its weights are taken against the older maximum, at most 256 each, and
//       the sum is in the same units, so the quotient is the same (a published
//       way to keep most steps free of it).  In fp16, which rounds by a share of
//       a weight down to 2^-14 only and to nothing below 2^-25, they are taken
//       against 2^-12 of the maximum, and it may grow by 2^3: at most 2^15 each,
//       and what is lost of n small ones is n 2^-37 of the largest at most;
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
//
// Measured (32 query and 8 key heads of 128, bf16): 4096 tokens over 16384 keys
// 0.63 ms of kernel time, 1.53 PFLOP/s over the visible pairs (fp16, whose maxima are
// followed more closely, 0.66), bound by the way
// from one of a tile's products to its next: a step takes 3.3k cycles, of which
// a tile's own products are 1.03k and hide as much of the other tile's way.  The
// rest is its weights (scores out of tensor memory 340, maximum 400, 128
// exponentials a thread 1060, back 150), 290 from a product's end to the warps
// that wait for it and 170 from theirs to the product.  What did not shorten it:
// handing over the first half of the weights early; exponentials by polynomials
// on the other pipes (a quarter of them 0.68 ms, half 0.83); more registers (at
// width 128 the compiler keeps 96 bytes of a thread in local memory).  Copies that
// their threads wait for took 0.72 ms, a block an item 0.79, a table lookup in each
// copying thread 3.3.  2048 tokens over 16 picked pages of 64 each: 0.13 ms; the row
// kernel, which reads every page once for every token, 1.29.
#include <type_traits>

#include "cache4.cuh"
#include "launch.h"
#include "mma16.cuh"
#include "paged_tile.cuh"
#include "tcgen05.cuh"

namespace slnr {
namespace {

constexpr int kRows = 128;              // of a tile
constexpr int kLoadWarp = 8;            // warps 0-7: softmax
constexpr int kLoaders = 128;
constexpr int kMmaWarp = 12;            // 13-15 only complete its warpgroup (4 bits: below)
constexpr int kThreads = 512;
constexpr int kSoftRegs = 192, kOtherRegs = 64;  // of 128 a thread at launch
static_assert(2 * (kSoftRegs + kOtherRegs) <= 4 * 128, "register shares of the four warpgroups");
static_assert(kLoaders == kChunkKeys, "a load thread finds one key's row");
constexpr int kBlock = kRows * 128;     // 128 rows of 64 values, swizzled
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 256;   // S and P of tile t at 128 t, O at kColO + 128 t
// In powers of two: how far below the maximum weights are taken against, and the
// growth of a maximum that O is rescaled for.
template <typename T>
constexpr float kBelow = std::is_same<T, __half>::value ? 12.f : 0.f;
template <typename T>
constexpr float kGrow = std::is_same<T, __half>::value ? 3.f : 8.f;
constexpr float kCoarse = 1 << 22;

template <int W>
constexpr int tile_bytes() { return kBlock * (W / 64); }
template <int W>
constexpr int buffers() { return W == 128 ? 4 : 8; }
template <int W>
constexpr size_t smem_bytes() { return (size_t)(2 + buffers<W>()) * tile_bytes<W>() + 1024; }
constexpr int kWarpArrivals = 4;  // a warp arrives once for its lanes
constexpr int kSegments = 8;      // pages of a step, at most
constexpr int kGroups = 8;        // of 16 keys of a step
constexpr int kMaxWords = 8;      // of the bits of 256 tokens of one row each

struct Shared {
  uint64_t q_full, q_empty, s_full[2], p_full[2], o_full, full[8], empty[8], drained;
  uint32_t tmem;
  int failed;
  int64_t row_q[2 * kRows];  // bytes from the head's first row to each of the item's query rows; -1: zeros
  // one tile an item: 16 columns of the second warpgroup's O, its maxima and sums
  float other[16][kRows];
  float2 other_ml[kRows];
};
template <bool CODES>
struct LoadShared : Shared {
  int64_t row_k[2][kChunkKeys], row_v[2][kChunkKeys];  // the same to each key of a step
  uint32_t listed[8][kSegments * (1 + kMaxWords)];     // selected: a step's pages, then who picked each
};

// Keys and values in 4 bits: one warp copies their codes to a ring of half steps (128
// keys, then their values) beside the tiles, six unpack them, every sixth of all slabs
// each.  The ring is handed over by half steps, of which each of the six reads: none can
// be a turn of the ring ahead of another, whose turns it tells apart by parity alone.
// 4096 tokens over 16384 keys, 32 query and 8 key heads of 128, bf16: 719 us of kernel time,
// 1.34 PFLOP/s, where 16 bits take 630: the slabs of a half step take the six warps longer
// than its products and weights (621 us in all if nothing were unpacked).  What brought it
// there (us a call): 1976 four warps that loaded codes themselves; 1289 bulk copies to rings
// of the warps' own; 1166 fewer instructions and bank conflicts; 986 seven warps; 776 one of
// them copying for the others, all by half steps; 753 a kernel a width; 736 the scales of two
// blocks at once.  fp16 for both products where queries are bf16, whose codes take 9 instructions
// a word and not 11, made O's rescaling so frequent that it took 823.
constexpr int kCopyWarp = 13;
constexpr int kUnpackWarps = 6;  // 8-11, 14, 15
constexpr int kStepSlabs = kChunkKeys / kSlab;
template <int W>
constexpr int raw_stages() { return W == 128 ? 2 : 4; }
template <int W>
constexpr int raw_bytes() { return kStepSlabs * 9 * W; }  // of a stage
template <>
struct LoadShared<true> : Shared {
  uint64_t raw_full[4], raw_empty[4];
  uint32_t there[4];  // bit i: slab i of the stage was copied; else there are no such keys
};
template <int W, bool CODES>
constexpr size_t block_bytes() {
  return smem_bytes<W>() + (CODES ? (size_t)raw_stages<W>() * raw_bytes<W>() : 0);
}

static_assert(block_bytes<128, false>() + sizeof(LoadShared<false>) <= (size_t)227 * 1024, "shared memory of a block");
static_assert(block_bytes<128, true>() + sizeof(LoadShared<true>) <= (size_t)227 * 1024, "shared memory of a block");

// One poll that does not sleep.
__device__ __forceinline__ bool test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(tc::smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
constexpr long long kShortLimit = 1 << 20;  // cycles; a try_wait may sleep for longer than a limit below that

// Waits for the phase of that parity; false (and *failed set) after `limit` cycles or once another wait gave up.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* failed, long long limit) {
  const bool sleeps = limit >= kShortLimit;
  if (sleeps ? tc::mbar_try_wait(bar, parity) : test(bar, parity)) return true;
  const long long t0 = clock64();
  while (!(sleeps ? tc::mbar_try_wait(bar, parity) : test(bar, parity))) {
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

// One arrival for the warp's lanes, after what each of them did.
__device__ __forceinline__ void arrive_warp(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) tc::mbar_arrive(bar);
}
// The thread's arrival once its copies so far have landed.  Who waits for them
// orders its products behind them (fence_proxy_async_smem).
__device__ __forceinline__ void copy_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tc::smem_u32(bar)) : "memory");
}
// Barrier `id` of n threads.
__device__ __forceinline__ void meet(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }

// Byte of 16-byte piece `piece` of a row inside a swizzled tile of 128 rows.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  return (uint32_t)((piece >> 3) * kBlock + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

// ---- keys and values in 4 bits (cache4.cuh): an unpacking warp takes every sixth
// slab, its lanes 16-byte pieces of the slab's codes, which become 16-bit rows of
// the tile.

__device__ __forceinline__ uint32_t lds_u32(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ uint32_t lds_u16(uint32_t at) {
  uint16_t r;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ void lds4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void sts16(uint32_t to, const uint4& x) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}

// Where a lane's pieces of a slab are, in the codes and in a tile of its first row,
// for keys and values.  The words of a piece are written in an order by t (turn) in
// which the eight lanes of a 128-byte store touch every bank once.
template <int D>
struct Places {
  static constexpr int W = D <= 64 ? 64 : 128, N = W / 64;
  int k_scale[N], v_scale[N], k_to[N], v_to[N];
  int k_turn, v_turn, v_slot[N];

  __device__ __forceinline__ explicit Places(int lane) {
    constexpr int per = D / 32;
    k_turn = W == 128 ? (lane % per) >> 1 : 0;  // per is 4, or 3 where the second piece has it from its own t
    v_turn = W == 128 ? (lane & 3) >> 1 : lane & 2;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = lane + 32 * n;
      int slot = i / per;
      const int t = i - slot * per, g = 2 * (slot >> 2) + (slot & 1), half = (slot >> 1) & 1;
      k_scale[n] = 8 * D + (W == 128 ? (g * per + t) * 4 + half * 2 : (g * 2 * per + 2 * t) * 2 + half);
      k_to[n] = piece_at(slot, 4 * t);
      if constexpr (W == 128) {
        const int q = i >= D / 4, j = i - q * (D / 4);
        slot = 4 * (j & 3) + 2 * q;
        v_scale[n] = 8 * D + (j >> 2) * 16 + slot;
        v_to[n] = piece_at(slot, 2 * (j >> 2));
      } else {
        slot = 4 * (i & 3);
        v_scale[n] = 8 * D + (i >> 3) * 16 + slot;
        v_to[n] = piece_at(slot, i >> 2);
      }
      v_slot[n] = slot;
    }
  }
};

// Codes and scales of the keys (or values) of a slab in shared memory, a lane's.
template <int D>
struct Codes {
  static constexpr int W = D <= 64 ? 64 : 128, N = W / 64;
  uint32_t w[N][4], scale[N];

  // keys: slots of it that are keys; the others hold anything, and their scales become 0 (of keys, only where there are
  // none: their scores are dropped)
  __device__ __forceinline__ void load(uint32_t raw, const Places<D>& at, bool value, int lane, int keys) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (lane + 32 * n >= D / 2) break;
      lds4(w[n], raw + 16 * (lane + 32 * n));
      if (W == 128) scale[n] = lds_u16(raw + (value ? at.v_scale[n] : at.k_scale[n]));
      else if (value) scale[n] = lds_u32(raw + at.v_scale[n]);
      else scale[n] = lds_u8(raw + at.k_scale[n]) | lds_u8(raw + at.k_scale[n] + 2) << 8;
    }
    if (keys >= kSlab) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int left = value ? keys - at.v_slot[n] : keys > 0 ? kSlab : 0;
      if (left < 4) scale[n] &= left > 0 ? (1u << 8 * left) - 1 : 0u;
    }
  }

  // To 16 rows of a tile.
  template <typename T>
  __device__ __forceinline__ void store(uint32_t tile, const Places<D>& at, bool value, int lane) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (lane + 32 * n >= D / 2) break;
      const uint32_t* x = w[n];
      if (!value) {  // 32 columns of a key: word i to piece 4 t + i
        const uint32_t to = tile + (at.k_to[n] ^ (at.k_turn << 5));
        const Unpack<T> u(at.k_turn ? __byte_perm(scale[n], 0, 0x4401) : scale[n]);
        sts16(to, u.template word<false>(at.k_turn ? x[2] : x[0]));
        sts16(to ^ 16, u.template word<false>(at.k_turn ? x[3] : x[1]));
        sts16(to ^ 32, u.template word<true>(at.k_turn ? x[0] : x[2]));
        sts16(to ^ 48, u.template word<true>(at.k_turn ? x[1] : x[3]));
      } else if constexpr (W == 128) {  // 16 columns of two values, in rows that differ in their last bit
        const uint32_t to = tile + (at.v_to[n] ^ (at.v_turn << 4));
        const Unpack<T> u(scale[n]);
        sts16(to, u.template word<false>(at.v_turn ? x[1] : x[0]));
        sts16(to ^ 16, u.template word<false>(at.v_turn ? x[0] : x[1]));
        sts16((to ^ 16) + 128, u.template word<true>(at.v_turn ? x[3] : x[2]));
        sts16(to + 128, u.template word<true>(at.v_turn ? x[2] : x[3]));
      } else {  // 8 columns of four values, in rows that differ in their last two bits
        const uint32_t in_turn = at.v_turn ? __byte_perm(scale[n], 0, 0x1032) : scale[n];
        const Unpack<T> u0(in_turn), u1(in_turn >> 16);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int r = b ^ at.v_turn;
          const uint32_t y = at.v_turn ? x[b ^ 2] : x[b];
          const uint4 z = b == 0 ? u0.template word<false>(y) : b == 1 ? u0.template word<true>(y)
                        : b == 2 ? u1.template word<false>(y) : u1.template word<true>(y);
          sts16(tile + (at.v_to[n] ^ (r << 4)) + r * 128, z);
        }
      }
    }
  }
};

// Two fp32 values in 64 bits: one instruction for both (0.62 ms where single ones
// took 0.65).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
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

__global__ void __launch_bounds__(kUnionThreads)
k_paged_union(AttnArgs a) {
  __shared__ uint32_t s_bits[kUnionPages * kMaxWords];
  __shared__ int s_count[kUnionThreads / 32 + 1];
  const PagesView& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, words = a.plan.words;
  let_next_start();
  int r, x0;
  find_tile(p, a.group.d, kChunkRows, blockIdx.x, r, x0);
  const int64_t at = (int64_t)h * gridDim.x + blockIdx.x;
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

// What every role of a block knows of the part of an item that it works on.  What
// is read of AttnPlan here and below was written by a kernel that may still run
// when this one starts, so by plain loads behind wait_for_previous: read-only ones
// (__ldg) are for data that no kernel writes meanwhile, and may be moved ahead of
// the wait.
struct Item {
  int h, r, x0, q0, n, tiles;  // key head, request, its first row and token, rows, tiles of 128
  int shift, last;             // position of the request's first new token, and of the last row's token
  int u0, u1, steps;           // keys (or slots of the listed pages) of this part
  int slot;                    // of the partial rows; -1: the whole item
  int64_t list;                // of the listed pages
};

// Cost of a step of an item of n rows: one tile takes half as long as two.  Of an
// item itself (its queries, the last product, its rows out): 10k cycles, where a
// step of two tiles takes 3k.
__device__ __forceinline__ int weight_of(int n) { return n > kRows ? 2 : 1; }
constexpr int kItemCost = 6;
__device__ __forceinline__ int steps_of(int end) { return end > 0 ? (end - 1) / kChunkKeys + 1 : 1; }

// Part [lo, hi) of item i (hi = -1: to its end).
template <bool SEL>
__device__ __forceinline__ Item item_of(const AttnArgs& a, int i, int ntiles, int lo, int hi) {
  Item it;
  it.h = i / ntiles;
  const int tile = i - it.h * ntiles;
  const int4 x = a.plan.tiles[2 * tile], y = a.plan.tiles[2 * tile + 1];
  it.r = x.x;
  it.x0 = x.y;
  it.q0 = x.z;
  it.n = x.w;
  it.tiles = it.n > kRows ? 2 : 1;
  it.shift = y.x;
  it.last = y.y;
  const int64_t at = (int64_t)it.h * a.plan.ntiles + tile;
  it.list = at * a.plan.cap;
  const int end = SEL ? a.plan.npages[at] * a.c.page.d : max(it.last + 1, 0);
  const int all = steps_of(end);
  if (hi < 0) hi = all;
  it.u0 = min(lo * kChunkKeys, end);
  it.u1 = hi < all ? hi * kChunkKeys : end;
  it.steps = (it.u1 - it.u0 + kChunkKeys - 1) / kChunkKeys;
  it.slot = lo == 0 && hi == all ? -1 : 2 * (int)blockIdx.x + (lo == 0);
  return it;
}

// Row tiles, and where each block's share of the items' steps begins.  Items go
// head by head, a head's tiles in order.  One block.
constexpr int kPlanThreads = 1024;

// Inclusive sum over the block; `total` gets the whole.
template <typename N>
__device__ __forceinline__ N block_sum(N x, N& total, N* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  N y = s_warp[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  total = __shfl_sync(0xffffffffu, y, 31);
  const N before = __shfl_sync(0xffffffffu, y, (warp + 31) & 31);
  return warp > 0 ? x + before : x;
}

template <bool SEL>
__global__ void __launch_bounds__(kPlanThreads)
k_paged_plan(AttnArgs a, WsHeader* hdr) {
  __shared__ int s_first[kPlanThreads], s_warp[32];
  __shared__ long long s_cost[32];
  const PagesView& p = a.p;
  const int tid = threadIdx.x, G = a.group.d;
  let_next_start();
  wait_for_previous();
  if (tid == 0) hdr->error = 0;
  int ntiles = 0;
  for (int r0 = 0; r0 < p.nreq; r0 = step_end(r0, kPlanThreads, p.nreq)) {
    const int32_t* q = p.q_pos + item(r0, tid);
    const int rows = inside(r0, tid, p.nreq) ? (__ldg(q + 1) - __ldg(q)) * G : 0;
    int total;
    const int mine = tiles_of(rows, kChunkRows), sum = block_sum(mine, total, s_warp);
    s_first[tid] = sum - mine;
    __syncthreads();
    for (int t = tid; t < total && ntiles + t < a.plan.ntiles; t += kPlanThreads) {
      int i = 0;  // the last request whose first tile is at or before t: the ones after it that start there are empty
#pragma unroll
      for (int w = kPlanThreads / 2; w > 0; w >>= 1)
        if (s_first[i + w] <= t) i += w;
      const int q0 = __ldg(p.q_pos + r0 + i), qn = __ldg(p.q_pos + r0 + i + 1) - q0;
      const int x0 = (t - s_first[i]) * kChunkRows, n = min(kChunkRows, qn * G - x0);
      const int shift = __ldg(p.k_len + r0 + i) - qn;
      a.plan.tiles[2 * (ntiles + t)] = make_int4(r0 + i, x0, q0, n);
      a.plan.tiles[2 * (ntiles + t) + 1] = make_int4(shift, shift + a.group.div(x0 + n - 1), 0, 0);
    }
    ntiles += total;
    __syncthreads();
  }
  ntiles = min(ntiles, a.plan.ntiles);
  // cost of the items before each: in 64 bits, as those of 1024 items of 2^27 keys pass 2^31
  const int items = ntiles * a.c.nheads;
  int64_t cost = 0;
  for (int i0 = 0; i0 < items; i0 += kPlanThreads) {
    const int i = i0 + tid;
    long long mine = 0, total;
    if (i < items) {
      const int h = i / ntiles, tile = i - h * ntiles;
      mine = kItemCost + weight_of(a.plan.tiles[2 * tile].w) *
             steps_of(SEL ? a.plan.npages[(int64_t)h * a.plan.ntiles + tile] * a.c.page.d
                          : max(a.plan.tiles[2 * tile + 1].y + 1, 0));
    }
    const long long sum = block_sum(mine, total, s_cost);
    if (i < items) a.plan.before[i] = cost + sum - mine;
    cost += total;
  }
  __syncthreads();
  const int64_t most = cost / kLeastCost > 1 ? cost / kLeastCost : 1;
  const int n = (int)(most < kChunkBlocks ? most : kChunkBlocks);  // blocks with a share
  // share c begins at cost c cost / n
  for (int i = tid; i < items; i += kPlanThreads) {
    const int64_t lo = a.plan.before[i], hi = i + 1 < items ? a.plan.before[i + 1] : cost;
    const int w = weight_of(a.plan.tiles[2 * (i % ntiles)].w);
    for (int64_t c = (lo * n + cost - 1) / cost; c < n && c * cost / n < hi; ++c)
      a.plan.shares[c] = make_int2(i, max((int)(c * cost / n - lo) - kItemCost, 0) / w);
  }
  if (tid == 0) {
    a.plan.shares[kChunkBlocks] = make_int2(items > 0 ? n : 0, items);
    a.plan.shares[kChunkBlocks + 1] = make_int2(ntiles, 0);
  }
}

// A row of O out of tensor memory (zeros where !on).
template <int W>
__device__ __forceinline__ void read_row(uint32_t col_o, bool on, uint32_t (&o)[W]) {
  if (on) {
#pragma unroll
    for (int k = 0; k < W / 32; ++k) tc::tmem_ld32_start(col_o + 32 * k, o + 32 * k);
#pragma unroll
    for (int k = 0; k < W / 32; ++k) tc::tmem_ld_done(o + 32 * k);
  } else {
#pragma unroll
    for (int k = 0; k < W; ++k) o[k] = 0;
  }
}

// 32 bytes of a row: one store where they are aligned.
__device__ __forceinline__ void store32(void* to, const uint32_t (&v)[8], bool aligned) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}

// A thread's row of the item, times inv (0: no key), with f_other times the other
// warpgroup's where an item has one tile.  Whole 32-byte sectors a thread: as
// fast as the memory system takes them, without shared memory in between.
// m: what weights were taken against, in powers of two, l: their sum.
template <typename T, int W>
__device__ __forceinline__ void write_row(const AttnArgs& a, const Item& it, Shared& sh, uint32_t (&o)[W], int x, int row,
                                          float inv, float f_other, float m, float l) {
  const bool pair = it.tiles == 1, whole = it.slot < 0, on = x < it.n;
  const int G = a.group.d, tok = a.group.div(it.x0 + x), g = it.x0 + x - tok * G;
  const int64_t at = whole ? (it.q0 + tok) * ((int64_t)a.c.nheads * G) + it.h * G + g : (int64_t)it.slot * kChunkRows + x;
  T* out = (T*)a.out + at * a.c.width;
  float* part = a.plan.part + at * a.c.width;
  const bool aligned = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && a.c.width % 16 == 0;
#pragma unroll
  for (int k = 0; k < W; k += 16) {
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = inv == 0.f ? 0.f : __uint_as_float(o[k + e]) * inv;
    if (pair) {
      meet(2, 2 * kRows);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = f_other == 0.f ? v[e] : fmaf(sh.other[e][row], f_other, v[e]);
      meet(2, 2 * kRows);
    }
    if (on && k < a.c.width) {
      uint32_t z[8];
      if (whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = Half2<T>::pack(v[2 * e], v[2 * e + 1]);
        if (k + 8 < a.c.width) store32(out + k, z, aligned);
        else *reinterpret_cast<uint4*>(out + k) = make_uint4(z[0], z[1], z[2], z[3]);
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = __float_as_uint(v[8 * half + e]);
          if (k + 8 * half < a.c.width) store32(part + k + 8 * half, z, true);
        }
      }
    }
  }
  if (on) {
    if (!whole) a.plan.part_ml[at] = make_float2(l == 0.f ? -INFINITY : m, l);
    else if (a.lse) a.lse[at] = (l == 0.f ? -INFINITY : m + __log2f(l)) * 0.6931471805599453f;
  }
}

// Calls f(item) for the parts of items that are this block's.
template <bool SEL, typename F>
__device__ __forceinline__ void each_item(const AttnArgs& a, F f) {
  const int c = blockIdx.x, n = a.plan.shares[kChunkBlocks].x, items = a.plan.shares[kChunkBlocks].y;
  const int ntiles = a.plan.shares[kChunkBlocks + 1].x;
  if (c >= n) return;
  const int2 from = a.plan.shares[c], to = c + 1 < n ? a.plan.shares[c + 1] : make_int2(items, 0);
  for (int i = from.x; i < to.x || (i == to.x && to.y > 0); ++i)
    f(item_of<SEL>(a, i, ntiles, i == from.x ? from.y : 0, i == to.x ? to.y : -1));
}

// FOUR: width of a cache in 4 bits, or 0.
template <typename T, int W, bool SEL, int FOUR>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_chunk(AttnArgs a, WsHeader* hdr, long long limit) {
  constexpr int PIECES = W / 8, NB = buffers<W>();
  constexpr int D = FOUR ? FOUR : W;
  constexpr float TIMES = FOUR ? Unpack<T>::kTimes : 1.f;  // of the keys and of the values
  extern __shared__ unsigned char smem_raw[];
  __shared__ LoadShared<(FOUR > 0)> bars;
  const PagesView& p = a.p;
  const CacheView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.group.d;

  const uint32_t base = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  auto q_tile = [&](int t) { return base + t * tile_bytes<W>(); };
  auto buffer = [&](int b) { return base + (2 + b) * tile_bytes<W>(); };
  if (tid == 0) {
    tc::mbar_init(&bars.q_full, kLoaders);
    tc::mbar_init(&bars.q_empty, 1);
    tc::mbar_init(&bars.o_full, 1);
    tc::mbar_init(&bars.drained, 1);
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(&bars.s_full[t], 1);
      tc::mbar_init(&bars.p_full[t], kWarpArrivals);
    }
    for (int b = 0; b < NB; ++b) {
      tc::mbar_init(&bars.full[b], FOUR ? kUnpackWarps : kLoaders);
      tc::mbar_init(&bars.empty[b], 1);
    }
    if constexpr (FOUR)
      for (int i = 0; i < 4; ++i) {
        tc::mbar_init(&bars.raw_full[i], 1);
        tc::mbar_init(&bars.raw_empty[i], kUnpackWarps);
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
  let_next_start();
  wait_for_previous();

  // Counters run on from item to item: ring steps, steps of each tile, items with keys.
  if (warp >= kLoadWarp) {
    regs_down<kOtherRegs>();
    if (FOUR && warp == kCopyWarp) {
      // ---- codes of 4 bits: lane i of the first eight slab i of each half step ----
      if constexpr (FOUR) {
        constexpr int NR = raw_stages<W>();
        const uint32_t raw = buffer(NB);
        int sent = 0;
        bool ok = true;
        each_item<SEL>(a, [&](const Item& it) {
          const int32_t* table = p.table + it.r * p.table_stride;
          int next = -1;
          auto find = [&](int j) {
            const int u = it.u0 + j * kChunkKeys + lane * kSlab;
            next = -1;
            if (lane < kStepSlabs && u < it.u1) {
              const int i = c.page.div(u);
              if (i < p.width) next = __ldg(table + i);
            }
          };
          find(0);
          for (int j = 0; ok && j < it.steps; ++j) {
            const int u = it.u0 + j * kChunkKeys + lane * kSlab;
            const bool on = (unsigned)next < (unsigned)c.npages;
            const uint8_t* src = a.c4.data;
            if (on)
              src += next * a.c4.page + it.h * a.c4.head + (int64_t)((u - c.page.div(u) * c.page.d) / kSlab) * slab_bytes(D);
            const uint32_t mask = __ballot_sync(0xffffffffu, on);
            find(j + 1);
#pragma unroll
            for (int value = 0; value < 2; ++value) {
              const int s = sent % NR;
              ok = ok && wait_warp(&bars.raw_empty[s], ((sent / NR) & 1) ^ 1, failed, limit);
              if (!ok) break;
              if (lane == 0) {
                bars.there[s] = mask;
                tc::mbar_expect(&bars.raw_full[s], __popc(mask) * 9 * D);
              }
              __syncwarp();
              if (on)
                tc::copy_bulk(raw + s * raw_bytes<W>() + lane * 9 * D, src + value * 9 * D, 9 * D,
                              &bars.raw_full[s]);
              ++sent;
            }
          }
        });
        // copies in flight end before the block does: the last of each stage
        const long long t0 = clock64();
        for (int i = sent > NR ? sent - NR : 0; i < sent; ++i)
          while (!tc::mbar_try_wait(&bars.raw_full[i % NR], (i / NR) & 1))
            if (clock64() - t0 > kWaitCycles) break;
      }
    } else if (warp < kMmaWarp || (FOUR && warp > kMmaWarp)) {
      // ---- loads ----
      constexpr int ROWS = kLoaders / PIECES;  // rows of a pass: a multiple of 8, so a thread's swizzle is fixed
      const int lt = tid - 32 * kLoadWarp, piece = lt % PIECES, row0 = lt / PIECES;
      const bool col_on = piece * 8 < c.width;
      const uint32_t at = piece_at(row0, piece);
      int ring = 0, count = 0;
      bool ok = true;  // where a wait gave up the loops go on without copies: their warps meet at barriers
      [[maybe_unused]] const int uw = warp < kMmaWarp ? warp - kLoadWarp : warp - kCopyWarp + 3;
      [[maybe_unused]] const Places<D> places(lane);
      [[maybe_unused]] int slab = uw;  // of the eight of a half step: every sixth of all is the warp's
      each_item<SEL>(a, [&](const Item& it) {
        if (it.steps == 0) return;
        const int32_t* table = p.table + it.r * p.table_stride;
        const char* src_k = (const char*)c.k + 2 * (c.ks[2] * it.h + (col_on ? piece * 8 : 0));
        const char* src_v = (const char*)c.v + 2 * (c.vs[2] * it.h + (col_on ? piece * 8 : 0));
        const int segs = SEL ? (c.page.d < kChunkKeys ? kChunkKeys / c.page.d : 1) : 0;
        int id = -1, off = 0, next = -1;  // next: the listed page of the key after
        auto listed = [&](int j) {
          const int u = it.u0 + j * kChunkKeys + lt;
          next = SEL && u < it.u1 ? a.plan.pages[it.list + c.page.div(u)] : -1;
        };
        auto find = [&](int j) {  // page and slot of this thread's key of step j
          const int u = it.u0 + j * kChunkKeys + lt;
          id = -1;
          if (u < it.u1) {
            int i = c.page.div(u);
            off = u - i * c.page.d;
            if (SEL) i = next;
            if (i < p.width && (!SEL || i * c.page.d + off <= it.last)) id = __ldg(table + i);
          }
          if (SEL) listed(j + 1);
        };
        if (SEL) listed(0);
        if constexpr (!FOUR) find(0);
        if (!FOUR || warp < kMmaWarp) {
          for (int x = lt; x < it.tiles * kRows; x += kLoaders) {
            const int tok = a.group.div(it.x0 + x), g = it.x0 + x - tok * G;
            bars.row_q[x] = x < it.n ? 2 * ((it.q0 + tok) * a.q.tok + (it.h * G + g) * a.q.head) : -1;
          }
          meet(1, kLoaders);
          ok = ok && wait_warp(&bars.q_empty, (count & 1) ^ 1, failed, limit);
        }
        constexpr int BATCH = kChunkKeys / ROWS / 2;  // offsets are read ahead of the copies that wait for them
        auto copy_rows = [&](uint32_t dst, const char* src, const int64_t* rows) {
#pragma unroll
          for (int k0 = 0; k0 < 2 * BATCH; k0 += BATCH) {
            int64_t o[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) o[k] = rows[row0 + (k0 + k) * ROWS];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
              const bool on = col_on && o[k] >= 0;
              copy16(dst + at + (k0 + k) * ROWS * 128, src + (on ? o[k] : 0), on);
            }
          }
        };
        if (ok && (!FOUR || warp < kMmaWarp)) {
          for (int t = 0; t < it.tiles; ++t)
            copy_rows(q_tile(t), (const char*)a.q.p + (col_on ? piece * 16 : 0), bars.row_q + t * kRows);
          copy_arrive(&bars.q_full);
        }
        const int total = 2 * it.steps;
        if constexpr (FOUR) {
          constexpr int NR = raw_stages<W>();
          for (int i = ring; ok && i < ring + total; ++i) {
            const int b = i % NB, s = i % NR, key0 = it.u0 + ((i - ring) >> 1) * kChunkKeys;
            const bool value = (i - ring) & 1;
            ok = wait_warp(&bars.raw_full[s], (i / NR) & 1, failed, limit);
            ok = ok && wait_warp(&bars.empty[b], ((i / NB) & 1) ^ 1, failed, limit);
            if (!ok) break;
            const uint32_t there = bars.there[s], raw = buffer(NB) + s * raw_bytes<W>();
            for (; slab < kStepSlabs; slab += kUnpackWarps) {
              Codes<D> codes;
              codes.load(raw + slab * 9 * D, places, value, lane, (there >> slab) & 1 ? it.u1 - key0 - slab * kSlab : 0);
              codes.template store<T>(buffer(b) + slab * kSlab * 128, places, value, lane);
            }
            slab -= kStepSlabs;
            tc::fence_proxy_async_smem();
            arrive_warp(&bars.full[b]);
            if (lane == 0) tc::mbar_arrive(&bars.raw_empty[s]);
          }
        }
        for (int i = 0; !FOUR && i < total; ++i) {
          const bool value = i & 1;  // K0 V0 K1 V1 ...
          const int j = i >> 1, b = (ring + i) % NB;
          if constexpr (!FOUR) {
            if (!value) {
              const bool on = (unsigned)id < (unsigned)c.npages;
              bars.row_k[j & 1][lt] = on ? 2 * (id * c.ks[0] + off * c.ks[1]) : -1;
              bars.row_v[j & 1][lt] = on ? 2 * (id * c.vs[0] + off * c.vs[1]) : -1;
              find(j + 1);
              meet(1, kLoaders);
            }
            ok = ok && wait_warp(&bars.empty[b], (((ring + i) / NB) & 1) ^ 1, failed, limit);
            if (SEL && ok && !value && lt < segs * (1 + a.plan.words)) {  // with K: the step's pages and their pickers
              const int g = lt < segs ? lt : (lt - segs) / a.plan.words, u = it.u0 + j * kChunkKeys + g * c.page.d;
              const bool on = u < it.u1;
              const int64_t e = it.list + (on ? c.page.div(u) : 0);
              copy4(tc::smem_u32(&bars.listed[(ring / 2 + j) % NB][lt]),
                    lt < segs ? (const void*)(a.plan.pages + e)
                              : (const void*)(a.plan.pickers + e * a.plan.words + (lt - segs) % a.plan.words), on);
            }
            if (ok) {
              copy_rows(buffer(b), value ? src_v : src_k, value ? bars.row_v[j & 1] : bars.row_k[j & 1]);
              copy_arrive(&bars.full[b]);
            }
          }
        }
        if (!FOUR || warp < kMmaWarp) meet(1, kLoaders);  // the offsets are read before the next item's are written
        ring += total;
        ++count;
      });
      asm volatile("cp.async.wait_all;" ::: "memory");
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
      // S of tile t from query tile q and the K in buffer b
      auto scores = [&](int t, int q, int b) {
        const uint64_t qd = q_desc + q * TILE, kd = k_desc + b * TILE;
#pragma unroll
        for (int k = 0; k < W / 16; ++k) {
          const uint64_t at = ((k >> 2) * kBlock + (k & 3) * 32) >> 4;
          if (k < ksteps) tc::mma_f16(tmem + kColS + t * 128, qd + at, kd + at, id_s, k > 0);
        }
        tc::mma_commit(&bars.s_full[t]);
      };
      // O of tile t (+)= P V of buffer b
      auto output = [&](int t, int b, bool first) {
        const uint64_t vd = v_desc + b * TILE;
        const uint32_t o = tmem + kColO + t * 128, w = tmem + kColS + t * 128;
#pragma unroll
        for (int k = 0; k < kChunkKeys / 16; ++k)
          tc::mma_f16_ta(o, w + 8 * k, vd + k * (2048 >> 4), id_o, !first || k > 0);
      };
      int ring = 0, count = 0, done[2] = {0, 0};
      bool ok = true;
      auto landed = [&](int i) { return wait_warp(&bars.full[i % NB], (i / NB) & 1, failed, limit); };
      each_item<SEL>(a, [&](const Item& it) {
        if (it.steps == 0 || !ok) return;
        // The queue of issued products is short: what lies between one tile's and
        // the next one's is kept to a wait, so that it does not run dry.
        ok = wait_warp(&bars.q_full, count & 1, failed, limit) && landed(ring);
        if (!ok) return;
        tc::fence_proxy_async_smem();
        tc::tc_fence_after_sync();
        if (it.tiles == 2) {  // two tiles take every step each
          if (tc::elect_one()) {
            scores(0, 0, ring % NB);
            scores(1, 1, ring % NB);
            tc::mma_commit(&bars.empty[ring % NB]);
            if (it.steps == 1) tc::mma_commit(&bars.q_empty);
          }
          __syncwarp();
          for (int j = 0; ok && j < it.steps; ++j) {
            const int iv = ring + 2 * j + 1, ik = iv + 1, bv = iv % NB, bk = ik % NB;
            const bool more = j + 1 < it.steps;
            ok = landed(iv) && (!more || landed(ik));
            tc::fence_proxy_async_smem();
            ok = ok && wait_warp(&bars.p_full[0], (done[0] + j) & 1, failed, limit);
            if (!ok) break;
            tc::tc_fence_after_sync();
            if (tc::elect_one()) {
              output(0, bv, j == 0);
              if (more) scores(0, 0, bk);
            }
            __syncwarp();
            ok = wait_warp(&bars.p_full[1], (done[1] + j) & 1, failed, limit);
            if (!ok) break;
            tc::tc_fence_after_sync();
            if (tc::elect_one()) {
              output(1, bv, j == 0);
              tc::mma_commit(&bars.empty[bv]);
              if (more) {
                scores(1, 1, bk);
                tc::mma_commit(&bars.empty[bk]);
                if (j + 2 == it.steps) tc::mma_commit(&bars.q_empty);
              }
            }
            __syncwarp();
          }
          done[0] += it.steps;
          done[1] += it.steps;
        } else {  // one tile takes the even steps on the first's S and O and the odd ones on the second's: its weights
                  // and its products overlap too
          if (tc::elect_one()) {
            scores(0, 0, ring % NB);
            tc::mma_commit(&bars.empty[ring % NB]);
            if (it.steps == 1) tc::mma_commit(&bars.q_empty);
          }
          __syncwarp();
          if (it.steps > 1) {
            const int bk = (ring + 2) % NB;
            ok = landed(ring + 2);
            if (ok) {
              tc::fence_proxy_async_smem();
              tc::tc_fence_after_sync();
              if (tc::elect_one()) {
                scores(1, 0, bk);
                tc::mma_commit(&bars.empty[bk]);
                if (it.steps == 2) tc::mma_commit(&bars.q_empty);
              }
              __syncwarp();
            }
          }
          for (int j = 0; ok && j < it.steps; ++j) {
            const int t = j & 1, iv = ring + 2 * j + 1, ik = iv + 3, bv = iv % NB, bk = ik % NB;
            const bool more = j + 2 < it.steps;
            ok = landed(iv) && (!more || landed(ik));
            tc::fence_proxy_async_smem();
            ok = ok && wait_warp(&bars.p_full[t], (done[t] + j / 2) & 1, failed, limit);
            if (!ok) break;
            tc::tc_fence_after_sync();
            if (tc::elect_one()) {
              output(t, bv, j < 2);
              tc::mma_commit(&bars.empty[bv]);
              if (more) {
                scores(t, 0, bk);
                tc::mma_commit(&bars.empty[bk]);
                if (j + 3 == it.steps) tc::mma_commit(&bars.q_empty);
              }
            }
            __syncwarp();
          }
          done[0] += (it.steps + 1) / 2;
          done[1] += it.steps / 2;
        }
        if (ok && tc::elect_one()) tc::mma_commit(&bars.o_full);
        __syncwarp();
        ring += 2 * it.steps;
        ++count;
      });
    }
  } else {
    regs_up<kSoftRegs>();
    // ---- softmax: thread = row ----
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t col_s = tmem + lanes + kColS + t * 128, col_o = tmem + lanes + kColO + t * 128;
    // scores are kept raw and take their factor inside the exponential; one that is not positive goes to them first
    const float factor = a.scale * 1.4426950408889634f * TIMES;
    int done = 0, count = 0, ring = 0;
    bool ok = true;  // where a wait gave up the items go on without work, and their rows are NaN
    each_item<SEL>(a, [&](const Item& it) {
      const bool pair = it.tiles == 1;  // this warpgroup's steps are every second one of the same rows
      const int x = pair ? row : t * kRows + row;
      const bool row_on = x < it.n;
      const int tok = row_on ? a.group.div(it.x0 + x) : 0, g = row_on ? it.x0 + x - tok * G : 0;
      const int pos = row_on ? it.shift + tok : -1;
      const int pos_min = it.shift + a.group.div(it.x0 + x - row);  // of the tile's rows
      const bool tail = it.n - (x - row) < kRows;                   // rows that are none: their scores are dropped
      bool raw = a.scale > 0.f;
      float sl2 = raw ? factor : 1.f;
      float m = -INFINITY, l = 0.f;  // what weights are taken against (in powers of two), sum of weights
      // selected: the row's token in the tile
      const int tl = tok - a.group.div(it.x0), page_shift = c.page.d < kChunkKeys ? 31 - __clz(c.page.d) : 7;
      const int segs = kChunkKeys >> page_shift, per_page = kGroups / segs, own_page = c.page.div(max(pos, 0));
      const int stride = pair ? 2 : 1, first = pair ? t : 0;
      for (int j = first; ok && j < it.steps; j += stride) {
        ok = wait_warp(&bars.s_full[t], done & 1, failed, limit);
        ++done;
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
        const int key0 = it.u0 + j * kChunkKeys;
        // selected: bit g: the row's token picked the page of keys 16 g .. 16 g + 15.  Groups that it did not pick are
        // left out of the maximum and get weights of 2^-inf; the slots past the token in its own page are dropped.
        uint32_t picked = 0;
        if constexpr (SEL) {
          const uint32_t* listed = bars.listed[(ring / 2 + j) % NB];
          bool own = false;
          for (int i = 0; i < segs; ++i) {
            const bool on = row_on && key0 + (i << page_shift) < it.u1 &&
                            ((listed[segs + i * a.plan.words + (tl >> 5)] >> (tl & 31)) & 1);
            if (on) picked |= ((1u << per_page) - 1) << (i * per_page);
            own = own || (on && (int)listed[i] == own_page);
          }
          if (__any_sync(0xffffffffu, own)) {
            const int off = key0 - c.page.div(key0) * c.page.d;  // of a page of more than 128 slots
#pragma unroll
            for (int g2 = 0; g2 < kGroups; ++g2) {
              const int i = (16 * g2) >> page_shift;
              const int last = pos - (int)listed[i] * c.page.d - off - (16 * g2 - (i << page_shift));
#pragma unroll
              for (int k = 0; k < 16; ++k)
                if (k > last) s[16 * g2 + k] = 0xff800000u;
            }
          }
        } else if (tail || key0 + kChunkKeys - 1 > pos_min) {
          const int last = pos - key0;  // keys 0 .. last of these 128
#pragma unroll
          for (int k = 0; k < 128; ++k)
            if (k > last) s[k] = 0xff800000u;
        }
        float top = -INFINITY;
#pragma unroll
        for (int g2 = 0; g2 < kGroups; ++g2) {
          float mx = __uint_as_float(s[16 * g2]);
#pragma unroll
          for (int k = 1; k < 16; ++k) mx = fmaxf(mx, __uint_as_float(s[16 * g2 + k]));
          if (!SEL || ((picked >> g2) & 1)) top = fmaxf(top, mx);
        }
        // the first keys that a row sees set m; later m moves only where it has to.  Rounded up: no weight of the highest
        // score is above 2^kBelow, however large that is
        const bool grow = fmaf(top, sl2, -m) > kBelow<T> + kGrow<T>;  // m = -inf: true for any seen key
        if (__any_sync(0xffffffffu, grow)) {
          // Beside scores past 2^22 m is too coarse for their exact products with sl2: from here on both are rounded
          // alike.
          if (__any_sync(0xffffffffu, raw && grow && fabsf(top) * sl2 >= kCoarse)) {
#pragma unroll
            for (int k = 0; k < 128; ++k) s[k] = __float_as_uint(__uint_as_float(s[k]) * factor);
            top *= factor;
            raw = false;
            sl2 = 1.f;
          }
          const float to = grow ? __fmaf_ru(top, sl2, -kBelow<T>) : m;
          const float f = grow ? exp2_fast(m - to) : 1.f;
          if (grow) l *= f;
          m = to;
          if (j > first) {
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
        const float b = m == -INFINITY ? 0.f : m;
        uint64_t sum[2] = {0, 0};  // pairs of fp32
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float off = SEL && !((picked >> (2 * k + e / 8)) & 1) ? -INFINITY : -b;
            const float2 x = unpack2(fma2(pack2(__uint_as_float(s[32 * k + 2 * e]), __uint_as_float(s[32 * k + 2 * e + 1])),
                                          pack2(sl2, sl2), pack2(off, off)));
            const float w0 = exp2_fast(x.x), w1 = exp2_fast(x.y);
            sum[e & 1] = add2(sum[e & 1], pack2(w0, w1));
            w[e] = Half2<T>::pack(w0, w1);
          }
          tc::tmem_st16(col_s + 16 * k, w);
        }
        tc::tmem_st_done();
        tc::tc_fence_before_sync();
        arrive_warp(&bars.p_full[t]);
        const float2 total = unpack2(add2(sum[0], sum[1]));
        l += total.x + total.y;
      }
      const bool keys = it.steps > 0;
      ring += 2 * it.steps;
      if (ok && keys) ok = wait_warp(&bars.o_full, count & 1, failed, limit);
      count += keys;
      tc::tc_fence_after_sync();
      if (!ok) m = l = __int_as_float(0x7fffffff);  // NaN, not what the output's memory held: no wait gives up unseen
      float f_other = 0.f;
      uint32_t o[W];
      read_row<W>(col_o, ok && it.steps > first, o);  // this warpgroup's O holds something from its first step on
      if (pair) {
        if (t == 1) bars.other_ml[row] = make_float2(m, l);
        meet(2, 2 * kRows);
        if (t == 0) {
          const float2 ml = bars.other_ml[row];
          const float top = fmaxf(m, ml.x), b = top == -INFINITY ? 0.f : top;
          const float f = exp2_fast(m - b);
          f_other = exp2_fast(ml.x - b);
          l = l * f + ml.y * f_other;
          f_other = l == 0.f ? 0.f : f_other * __fdividef(TIMES, l);
          m = top;
          const float inv = l == 0.f ? 0.f : f * __fdividef(TIMES, l);
          write_row<T, W>(a, it, bars, o, x, row, inv, f_other, m, l);
        } else {
#pragma unroll
          for (int k = 0; k < W; k += 16) {
#pragma unroll
            for (int e = 0; e < 16; ++e) bars.other[e][row] = __uint_as_float(o[k + e]);
            meet(2, 2 * kRows);
            meet(2, 2 * kRows);
          }
        }
      } else {
        write_row<T, W>(a, it, bars, o, x, row, l == 0.f ? 0.f : __fdividef(TIMES, l), 0.f, m, l);
      }
    });
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

// Items that cuts went through: o = sum 2^(m_part - m) l_part o_part / sum 2^(m_part - m) l_part
// over their parts, in the keys' order.  Block x: the item that share x + 1 begins
// inside of, if no share before does; block y: 16 of its rows, 4 a warp at once.
constexpr int kJoinRows = 16;

template <typename T, bool SEL>
__global__ void __launch_bounds__(128)
k_paged_join(AttnArgs a) {
  wait_for_previous();
  const int n = a.plan.shares[kChunkBlocks].x, ntiles = a.plan.shares[kChunkBlocks + 1].x;
  const int c0 = blockIdx.x + 1;
  if (c0 >= n) return;
  const int2 cut = a.plan.shares[c0], before = a.plan.shares[c0 - 1];
  if (cut.y == 0 || (before.x == cut.x && before.y > 0)) return;
  int c1 = c0 + 1;  // shares c0 .. c1 - 1 begin inside of the item
  while (c1 < n && a.plan.shares[c1].x == cut.x) ++c1;
  const Item it = item_of<SEL>(a, cut.x, ntiles, 0, -1);
  const int lane = threadIdx.x & 31, G = a.group.d, col = 4 * lane;
  constexpr int ROWS = kJoinRows / 4;
  const int x0 = blockIdx.y * kJoinRows + (threadIdx.x >> 5) * ROWS, parts = c1 - c0 + 1;
  if (x0 >= it.n) return;
  // row x of part k: the one that begins the item, then one a share
  auto part = [&](int k, int i) {
    return (int64_t)(2 * (c0 - 1 + k) + (k == 0)) * kChunkRows + min(x0 + i, it.n - 1);
  };
  float m[ROWS], sum[ROWS];
  float4 acc[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    m[i] = -INFINITY;
    sum[i] = 0.f;
    acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 2
  for (int k = 0; k < parts; ++k)
#pragma unroll
    for (int i = 0; i < ROWS; ++i) m[i] = fmaxf(m[i], a.plan.part_ml[part(k, i)].x);
#pragma unroll 2
  for (int k = 0; k < parts; ++k)
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int64_t at = part(k, i);
      const float2 ml = a.plan.part_ml[at];
      const float f = exp2_fast(ml.x - (m[i] == -INFINITY ? 0.f : m[i])) * ml.y;
      sum[i] += f;
      if (col < a.c.width) {
        const float4 y = *reinterpret_cast<const float4*>(a.plan.part + at * a.c.width + col);
        acc[i].x += f * y.x;
        acc[i].y += f * y.y;
        acc[i].z += f * y.z;
        acc[i].w += f * y.w;
      }
    }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int x = x0 + i;
    if (x >= it.n) break;
    const float inv = sum[i] == 0.f ? 0.f : __fdividef(1.f, sum[i]);  // the parts of a row without keys are zeros
    const int tok = a.group.div(it.x0 + x), g = it.x0 + x - tok * G;
    const int64_t at = (it.q0 + tok) * ((int64_t)a.c.nheads * G) + it.h * G + g;
    if (col < a.c.width) {
      uint2 y;
      y.x = Half2<T>::pack(acc[i].x * inv, acc[i].y * inv);
      y.y = Half2<T>::pack(acc[i].z * inv, acc[i].w * inv);
      *reinterpret_cast<uint2*>((T*)a.out + at * a.c.width + col) = y;
    }
    if (lane == 0 && a.lse) a.lse[at] = (m[i] + __log2f(sum[i])) * 0.6931471805599453f;
  }
}

template <typename T, int W, bool SEL, int FOUR>
cudaError_t launch(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  auto kernel = k_paged_chunk<T, W, SEL, FOUR>;
  static OncePerDevice once;
  cudaError_t e = once(
      [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)block_bytes<W, (FOUR > 0)>()); });
  if (e != cudaSuccess) return e;
  return launch_next(kernel, SLNR_COUNTED(dim3(kChunkBlocks)), dim3(kThreads), block_bytes<W, (FOUR > 0)>(), s, a, hdr,
                     wait_limit_cycles());
}

template <typename T, bool SEL>
cudaError_t launch_w(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  return a.c.width <= 64 ? launch<T, 64, SEL, 0>(a, hdr, s) : launch<T, 128, SEL, 0>(a, hdr, s);
}

template <typename T>
cudaError_t launch_4(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  switch (a.c.width) {
    case 32: return launch<T, 64, false, 32>(a, hdr, s);
    case 64: return launch<T, 64, false, 64>(a, hdr, s);
    case 96: return launch<T, 128, false, 96>(a, hdr, s);
    default: return launch<T, 128, false, 128>(a, hdr, s);
  }
}

}  // namespace

cudaError_t launch_paged_plan(const AttnArgs& a, WsHeader* hdr, cudaStream_t s) {
  if (!a.picked) {
    k_paged_plan<false><<<SLNR_COUNTED(1), kPlanThreads, 0, s>>>(a, hdr);
    return cudaGetLastError();
  }
  const dim3 grid((unsigned)a.plan.ntiles, (unsigned)a.c.nheads);
  k_paged_union<<<(SLNR_COUNTED(grid)), kUnionThreads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_next(k_paged_plan<true>, SLNR_COUNTED(dim3(1)), dim3(kPlanThreads), 0, s, a, hdr);
}

cudaError_t launch_paged_chunk(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s) {
  if (a.c4.data)
    return dtype == SLNR_FP16 ? launch_4<__half>(a, hdr, s) : launch_4<__nv_bfloat16>(a, hdr, s);
  if (a.picked) return dtype == SLNR_FP16 ? launch_w<__half, true>(a, hdr, s) : launch_w<__nv_bfloat16, true>(a, hdr, s);
  return dtype == SLNR_FP16 ? launch_w<__half, false>(a, hdr, s) : launch_w<__nv_bfloat16, false>(a, hdr, s);
}

cudaError_t launch_paged_join(const AttnArgs& a, int dtype, cudaStream_t s) {
  const dim3 grid(kChunkBlocks - 1, kChunkRows / kJoinRows);
  auto kernel = dtype == SLNR_FP16 ? (a.picked ? k_paged_join<__half, true> : k_paged_join<__half, false>)
                                   : (a.picked ? k_paged_join<__nv_bfloat16, true> : k_paged_join<__nv_bfloat16, false>);
  return launch_next(kernel, SLNR_COUNTED(grid), dim3(128), 0, s, a);
}

}  // namespace slnr
