// Attention of new tokens over a cache in 4 bits, rows of a few tokens at a time:
// the kernel of single tokens and of short chunks (32 query rows of a key head).
//
//   o = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q.k_j - m),  m = max_j scale q.k_j
//
// over the keys j that the row sees, in one pass.  At the rate of memory an SM takes 24
// bytes, 43 values of 9/16 of a byte, a cycle, and has 128 lanes for them: 3 instructions
// of a lane a value, and no more than one in two of them logical.  So:
//   - Keys are the rows of both products (S^T = K Q^T, O^T = V^T P^T), 16 at a time,
//     and the query rows their columns, 8 at a time: 8 query rows cost half of what
//     16 would.  P^T is turned from the one product's result into the other's
//     operand by the matrix transpose of a warp.
//   - A pair of codes becomes a pair of fp16 numbers by one logical instruction and one
//     multiplication and addition, with the scale (cache4.cuh).  Held values / 128 are
//     exact in fp16 whatever type wrote them; queries of bf16 are taken as fp16
//     times a power of two of their row, weights as fp16 against 2^-12 of the
//     maximum, which is followed when it grew by 2^3, so none passes 2^15, and what
//     is lost of n small ones is n 2^-37 of the largest at most.
//   - A slab of 16 slots lies as its lanes read it: 16-byte loads without bank
//     conflicts, no shuffles.
//   - Each warp has a ring of slabs of its own, filled by bulk copies that its own lanes
//     issue and wait for: no barrier of the block inside of an item.
//   - What a warp knows of its copies and the queries' fragments are in shared memory, a
//     kernel is for one width, and units that every row sees whole have code without masks:
//     with 128 registers the compiler else makes values again that it had.
//
// The units (32 keys) of all requests and key heads, one after another, are cut into
// equal shares, one a block; its warps take them in turn.  Items that a cut goes
// through are joined by k_paged4_join.
//
// 64 single tokens over 9000 keys each, 32 query and 8 key heads of 128, bf16 (663 MB):
// 119 us of kernel time, 5.6 TB/s, and a call of 125.  No unit is full: 281 instructions of a
// warp a slab, 2.2 a value, take 60 % of the issue slots, the logical and byte-permuting ones
// 56 % of their pipe's time, fp16 ones 40 %, products 27 %, memory 70 %.  Of the four warps that
// a scheduler has (registers allow no more) 1.3 are ready on average.  A warp's time is 21 % the
// fixed delay of the instruction before in its chain (load, unpack, product, exponential,
// transpose, product), 19 % another warp's turn, 17 % issuing, 16 % a pipe that another uses,
// 11 % dispatch, 7 % global memory.  What brought it here (us a call, 64 tokens over 1001
// to 32003 keys): 179 to begin with; 153 two values at a time in the softmax, whole units
// without masks, look-ups of 16 units at once, 16 warps an SM; 147 the copies' state in
// shared memory; 142 a kernel a width; 136 the scales of two keys side by side, halves of
// which the multiplications pick by themselves.  12 or 16 warps an SM, two or three stages, 16
// or 32 keys at once made no difference, nor did keys out of L2 alone (3 % less).  Of 17 to
// 32 rows a warp takes a slab at a time (64 requests of 8 tokens 290 us; two slabs, with
// registers spilled, 686; the tensor cores' kernel, as for 36 rows, 523).
#include <type_traits>

#include "cache4.cuh"
#include "launch.h"
#include "mma16.cuh"
#include "paged4.cuh"
#include "tcgen05.cuh"

namespace slnr {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 2;
constexpr int kUnit = 2 * kSlab;   // keys of a stage
constexpr int kBatch = 16;         // units whose pages a warp looks up at once
constexpr float kBelow = 12.f, kGrow = 3.f;

// What is copied in the place of slabs whose entry of the table is no page: zeros (a stage
// keeps the last item's keys where nothing is copied).  A mask that each unit looked at
// took 1.4 % longer.
__device__ __align__(128) uint8_t nothing[2 * slab_bytes(128)];

// Slabs, the item's queries (a warp's fragments), and the warps' sums of the rows of an item.
size_t smem_bytes(int width, int tile, int rows) {
  const int w = width <= 64 ? 64 : 128;
  return (size_t)kWarps * kStages * 2 * slab_bytes(width) + (size_t)tile * w * 2 + (size_t)kWarps * rows * (w + 4) * 4;
}

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

// Waits for the phase of that parity; false after `limit` cycles.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, long long limit) {
  const bool sleeps = limit >= kShortLimit;
  if (sleeps ? tc::mbar_try_wait(bar, parity) : test(bar, parity)) return true;
  const long long t0 = clock64();
  while (!(sleeps ? tc::mbar_try_wait(bar, parity) : test(bar, parity)))
    if (clock64() - t0 > limit) return false;
  return true;
}

__device__ __forceinline__ void lds4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void lds2(uint32_t& a, uint32_t& b, uint32_t at) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t lds1(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(at) : "memory");
  return r;
}
__device__ __forceinline__ uint32_t lds_half(uint32_t at) {
  uint16_t r;
  asm volatile("ld.shared.b16 %0, [%1];" : "=h"(r) : "r"(at) : "memory");
  return r;
}
// An 8 x 8 matrix of 16-bit values, a pair of a row's neighbours a lane, turned.
__device__ __forceinline__ uint32_t turned(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// Two fp32 values in 64 bits: one instruction for both.
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
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <typename T>
__device__ __forceinline__ float2 to_float2(uint32_t x);
template <>
__device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
// What a block knows of a request.
struct Request {
  int r, q0, qn, keys, units;  // its first token, tokens, keys, units of 32 keys (0: no tokens)
};
__device__ __forceinline__ int units_of(int qn, int keys) {
  return qn > 0 ? (keys > 0 ? (keys - 1) / kUnit + 1 : 1) : 0;
}
__device__ __forceinline__ Request request(const PagesView& p, int r) {
  Request q{r, 0, 0, 0, 0};
  if (r < p.nreq) {
    q.q0 = __ldg(p.q_pos + r);
    q.qn = __ldg(p.q_pos + r + 1) - q.q0;
    q.keys = max(__ldg(p.k_len + r), 0);
    q.units = units_of(q.qn, q.keys);
  }
  return q;
}

// Units (of one key head) of requests r0 .. r0 + 127, four neighbours a lane.  Every warp
// reads the lengths of all requests (4096 of one token and 100 keys 302 us of the GPU, 20000
// of 20 keys 494; 32 at a time 375 and 962).  A part of them a thread, joined by the block,
// took 270 and 262, but left the compiler with a slower loop for everyone (64 tokens over
// 9000 keys 121 -> 125).
struct Units {
  int n[4];
  __device__ __forceinline__ Units(const PagesView& p, int r0) {
    const unsigned r = item(r0, 4 * (threadIdx.x & 31));
    const int32_t *q = p.q_pos + r, *k = p.k_len + r;
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = r + i < (unsigned)p.nreq ? units_of(__ldg(q + i + 1) - __ldg(q + i), __ldg(k + i)) : 0;
  }
  __device__ __forceinline__ int64_t sum() const { return (int64_t)n[0] + n[1] + n[2] + n[3]; }
};
// The request that holds unit `at` of `heads` heads each, and the units of one head
// before it (a whole warp); first: of requests 0 .. 127.
__device__ __forceinline__ int find_unit(const PagesView& p, int heads, int64_t at, const Units& first, int64_t& before) {
  const int lane = threadIdx.x & 31;
  before = 0;
  for (int r0 = 0; r0 < p.nreq; r0 = step_end(r0, 128, p.nreq)) {
    const Units u = r0 == 0 ? first : Units(p, r0);
    int64_t sum = u.sum();
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, (before + sum) * heads > at);
    if (past) {
      const int from = __ffs(past) - 1;
      before += __shfl_sync(0xffffffffu, sum - u.sum(), from);
      int r = r0 + 4 * from;
      for (int i = 0; i < 3; ++i) {
        const int64_t next = before + __shfl_sync(0xffffffffu, i == 0 ? u.n[0] : i == 1 ? u.n[1] : u.n[2], from);
        if (next * heads > at) break;
        before = next;
        ++r;
      }
      return r;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return p.nreq;
}

// The part of an item that a block works on: units [u0, u1) of request q.r and head h.
struct Part {
  Request q;
  int h, u0, u1;
  int64_t left;  // units of the share behind it
};
__device__ __forceinline__ void clip(Part& s, int64_t left) {
  s.u1 = (int)(s.q.units - s.u0 < left ? s.q.units : s.u0 + left);
  s.left = left - (s.u1 - s.u0);
}
// The first request behind r (at most nreq) with new tokens, 32 at a look (a whole warp; nreq: none).
__device__ __forceinline__ int next_request(const PagesView& p, int r) {
  for (int r0 = step_end(r, 1, p.nreq); r0 < p.nreq; r0 = step_end(r0, 32, p.nreq)) {
    const int32_t* q = p.q_pos + item(r0, threadIdx.x & 31);
    const unsigned on = __ballot_sync(0xffffffffu, inside(r0, threadIdx.x & 31, p.nreq) && __ldg(q + 1) > __ldg(q));
    if (on) return r0 + __ffs(on) - 1;
  }
  return p.nreq;
}
// The next part (a whole warp); its left is below 0 where there is none.
__device__ __forceinline__ void advance(const Attn4Args& a, Part& s) {
  if (s.left <= 0) {
    s.left = -1;
    return;
  }
  if (++s.h == a.c.nheads) {
    s.h = 0;
    s.q = request(a.p, s.q.r + 1);
    if (s.q.units == 0) s.q = request(a.p, next_request(a.p, s.q.r));
    if (s.q.units == 0) {  // not met: the shares end with the last item
      s.left = -1;
      return;
    }
  }
  s.u0 = 0;
  clip(s, s.left);
}

// How far the copies of a warp are: its next unit, and the batch that it is sending.
// Here, as registers are short: looked at once a unit.
struct Ahead {
  Part part;
  int unit;
  uint32_t have;               // bit l: slab l has keys
  const uint8_t* src[2 * kBatch];  // of unit i of the batch, slab k: at 2 i + k
};
struct Shared {
  Ahead ahead[kWarps];
  Part part[kWarps];  // that the warp works on
  uint64_t full[kWarps][kStages];
  float2 ml[kWarps][32];  // a warp's (reference, sum) of each row
  int failed[kWarps];
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 4 : 2)
k_paged4_rows(const __grid_constant__ Attn4Args a, long long limit) {
  constexpr int W = D <= 64 ? 64 : 128;  // of the products
  constexpr int WORDS = W / 32;          // of a key, a lane: its columns are 8 WORDS t ..
  constexpr int MT = W / 16;
  constexpr int SL = NT == 4 ? 1 : 2;  // slabs that are multiplied together: 32 rows have no registers for more
  extern __shared__ __align__(128) unsigned char raw[];
  __shared__ Shared sh;
  const PagesView& p = a.p;
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  constexpr int slab = slab_bytes(D);
  const int G = a.group.d;
  let_next_start();

  // the block's share
  const Units first_units(p, 0);
  int64_t total = first_units.sum();
#pragma unroll 2
  for (int r0 = 128; r0 < p.nreq; r0 = step_end(r0, 128, p.nreq)) total += Units(p, r0).sum();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  total *= c.nheads;
  const int64_t most = (total + a.least - 1) / a.least;
  const int n = (int)(most < gridDim.x ? most : gridDim.x);
  if (blockIdx.x >= n) {
    if (blockIdx.x == 0 && tid == 0) a.shares[a.nblocks] = make_int4(0, 0, 0, 0);
    return;
  }
  const int64_t lo = total / n * blockIdx.x + total % n * blockIdx.x / n;
  const int64_t hi = total / n * (blockIdx.x + 1) + total % n * (blockIdx.x + 1) / n;
  Part s;
  {
    int64_t before;
    s.q = request(p, find_unit(p, c.nheads, lo, first_units, before));
    const int64_t in = lo - before * c.nheads;
    s.h = (int)(in / s.q.units);
    s.u0 = (int)(in - (int64_t)s.h * s.q.units);
    clip(s, hi - lo);
  }
  if (tid == 0) {
    a.shares[blockIdx.x] = make_int4(s.q.r, s.h, s.u0, 0);
    if (blockIdx.x == 0) a.shares[a.nblocks] = make_int4(n, 0, 0, 0);
  }

  uint64_t* full = sh.full[warp];
  if (lane < kStages) tc::mbar_init(full + lane, 1);
  tc::fence_mbar_init();
  __syncwarp();
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(raw) + warp * kStages * 2 * slab;
  const uint32_t queries = (uint32_t)__cvta_generic_to_shared(raw) + kWarps * kStages * 2 * slab + lane * 16;
  float* rows = reinterpret_cast<float*>(raw + kWarps * kStages * 2 * slab + 8 * NT * W * 2);

  // The copies run ahead of the work, a batch of up to 16 units of one part at a time.
  Ahead& ahead = sh.ahead[warp];
  const bool whole = c.slots.d % kUnit == 0;  // both slabs of a unit lie in one page, one after another
  int units = 0, done = 0, issued = 0;        // of the batch; of all
  auto look_up = [&] {
    Part cs = ahead.part;
    int cu = ahead.unit;
    while (cs.left >= 0 && cu >= cs.u1) {
      advance(a, cs);
      cu = cs.u0 + warp;
    }
    units = cs.left < 0 ? 0 : min((cs.u1 - cu - 1) / kWarps + 1, kBatch);
    done = 0;
    const int key = (cu + kWarps * (lane >> 1)) * kUnit + (lane & 1) * kSlab;
    int id = -1, at = 0;
    const bool keys = (lane >> 1) < units && key < cs.q.keys;
    if (keys) {
      const int i = c.slots.div(key);
      at = (int)((unsigned)(key - i * c.slots.d) / kSlab);
      if (i < p.width) id = __ldg(p.table + cs.q.r * p.table_stride + i);
    }
    const bool on = (unsigned)id < (unsigned)c.npages;
    const uint32_t have = __ballot_sync(0xffffffffu, keys);
    if (keys) ahead.src[lane] = on ? c.data + id * c.page + cs.h * c.head + (int64_t)at * slab : nothing;
    if (lane == 0) {
      ahead.part = cs;
      ahead.unit = cu + kWarps * units;
      ahead.have = have;
    }
    __syncwarp();
  };
  auto issue = [&](int stage) {
    if (done == units) look_up();
    if (units == 0) return;
    if ((lane >> 1) == done) {
      const uint32_t both = (ahead.have >> 2 * done) & 3;
      uint64_t* bar = full + stage;
      if ((lane & 1) == 0) tc::mbar_expect(bar, __popc(both) * slab);
      __syncwarp(3u << (2 * done));
      if ((both >> (lane & 1) & 1) && !(whole && lane & 1 && both == 3))
        tc::copy_bulk(ring + (stage * 2 + (lane & 1)) * slab, ahead.src[lane], whole && both == 3 ? 2 * slab : slab, bar);
    }
    ++done;
    ++issued;
  };
  if (lane == 0) {
    ahead.part = s;
    ahead.unit = s.u0 + warp;
    sh.part[warp] = s;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kStages; ++i) issue(i);

  int taken = 0, stage_i = 0;
  uint32_t phase = 0;
  bool ok = true;
  while (s.left >= 0) {
    const Request& q = s.q;
    const int n_rows = min(q.qn * G, a.rows);
    const int first = q.keys - q.qn;  // position of its first token (lengths below 0 are 0: all tokens see nothing)
    // query fragments to shared memory (registers are short), by the first warp; and what a row's scores are multiplied by:
    // log2 e scale, 128 of the held values, its power of two
    float f[NT][2], m[NT][2];
    uint64_t l[NT];  // a pair of fp32
    int pos[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int x = 8 * nt + g;
      const bool on = x < n_rows;
      const int tok = on ? a.group.div(x) : 0, gg = on ? x - tok * G : 0;
      const T* row = (const T*)a.q.p + (int64_t)(q.q0 + tok) * a.q.tok + (int64_t)(s.h * G + gg) * a.q.head + 8 * WORDS * t;
      uint4 raw_q[WORDS];
#pragma unroll
      for (int w = 0; w < WORDS; ++w)
        raw_q[w] = on && 8 * (WORDS * t + w) < D ? __ldg(reinterpret_cast<const uint4*>(row) + w) : make_uint4(0, 0, 0, 0);
      float factor = a.scale * 1.4426950408889634f;
      if constexpr (std::is_same<T, __half>::value) {
        factor *= 128.f;
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          const uint32_t e[4] = {raw_q[w].x, raw_q[w].y, raw_q[w].z, raw_q[w].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, max(e[i] & 0x7fffu, (e[i] >> 16) & 0x7fffu));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // the row times 2^(14 - e), e the exponent of its largest value, which is below 2^15 then: in two steps, as either
        // power alone may not be a number.  Zeros, infinities and NaN: times 1.
        const int ex = top == 0 || top >= 0x7f80u ? 14 : max((int)(top >> 7), 1) - 127;
        const float up = __uint_as_float((uint32_t)(127 + (14 - ex) / 2) << 23);
        const float up2 = __uint_as_float((uint32_t)(127 + (14 - ex) - (14 - ex) / 2) << 23);
        factor = factor * (128.f / up) / up2;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          uint32_t* e = &raw_q[w].x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 y = to_float2<__nv_bfloat16>(e[i]);
            e[i] = Half2<__half>::pack(y.x * up * up2, y.y * up * up2);
          }
        }
      }
      if (warp == 0)
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(queries + (nt * WORDS + w) * 512), "r"(raw_q[w].x),
                       "r"(raw_q[w].y), "r"(raw_q[w].z), "r"(raw_q[w].w)
                       : "memory");
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // of the columns that this lane has of the products
        f[nt][i] = __shfl_sync(0xffffffffu, factor, 4 * (2 * t + i));
        const int y = 8 * nt + 2 * t + i;
        pos[nt][i] = y < n_rows ? first + a.group.div(y) : INT32_MAX;
        m[nt][i] = -INFINITY;
      }
      l[nt] = 0;
    }
    __syncthreads();
    float o[MT][NT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) o[i][j][0] = o[i][j][1] = o[i][j][2] = o[i][j][3] = 0.f;

    // scores, weights and outputs of SL slabs; FULL: every key is there and seen by every row
    auto unit = [&](auto full_unit, int key0, uint32_t stage) {
      constexpr bool FULL = decltype(full_unit)::value;
      const int slabs = FULL ? SL : q.keys - key0 > kSlab ? 2 : q.keys > key0 ? 1 : 0;
      float x[SL][NT][4];
#pragma unroll
      for (int b = 0; b < SL; ++b) {
#pragma unroll
        for (int j = 0; j < NT; ++j) x[b][j][0] = x[b][j][1] = x[b][j][2] = x[b][j][3] = 0.f;
        if (!FULL && b >= slabs) continue;
        const uint32_t at = stage + b * slab;
        uint32_t w0[WORDS] = {}, w1[WORDS] = {}, sc = 0;
        if (8 * WORDS * t < D) {
          const uint32_t from = at + (4 * (g >> 1) + (g & 1)) * (D / 2) + 4 * WORDS * t;
          if constexpr (W == 128) {
            lds4(w0, from);
            lds4(w1, from + D);  // two slots on
            sc = lds1(at + 8 * D + (g * (D / 32) + t) * 4);
          } else {
            lds2(w0[0], w0[1], from);
            lds2(w1[0], w1[1], from + D);
            sc = lds_half(at + 8 * D + (g * (D / 16) + t) * 2);
          }
        }
        // scales of the two keys side by side: of the first block, and of the second
        const ScalePair sa = scale_pair(W == 128 ? (sc & 0x00ff00ffu) << 7 : scales_of(sc, 0, 1));
        const ScalePair sb = W == 128 ? scale_pair((sc >> 1) & 0x7f807f80u) : sa;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          const ScalePair& s2 = w < 2 ? sa : sb;
          uint32_t qf[NT][4];
#pragma unroll
          for (int j = 0; j < NT; ++j) lds4(qf[j], queries + (j * WORDS + w) * 512);
          uint32_t y0[4], y1[4];
          raw_pairs(w0[w], y0);
          raw_pairs(w1[w], y1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const __half2 o = as_half2(i & 1 ? s2.o256 : s2.o16), m2 = as_half2(s2.s);
            y0[i] = bits_of(__hfma2(as_half2(y0[i]), __low2half2(m2), __low2half2(o)));
            y1[i] = bits_of(__hfma2(as_half2(y1[i]), __high2half2(m2), __high2half2(o)));
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t key[4] = {y0[2 * k], y1[2 * k], y0[2 * k + 1], y1[2 * k + 1]};
#pragma unroll
            for (int j = 0; j < NT; ++j) Half2<__half>::mma(x[b][j], key, qf[j][2 * k], qf[j][2 * k + 1]);
          }
        }
      }
      // scores in units of log 2; -inf where the row does not see the key.  [i]: slab i / 2, key i % 2 of the lane's
      uint64_t y[NT][2 * SL];
      float top[NT][2];
      bool grow = false;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float2 z[2 * SL];
#pragma unroll
        for (int i = 0; i < 2 * SL; ++i) {
          y[j][i] = mul2(pack2(x[i >> 1][j][2 * (i & 1)], x[i >> 1][j][2 * (i & 1) + 1]), pack2(f[j][0], f[j][1]));
          z[i] = unpack2(y[j][i]);
          if constexpr (!FULL) {
            const int key = key0 + (i >> 1) * kSlab + 4 * (g >> 1) + (g & 1) + 2 * (i & 1);
            if (key > pos[j][0] || key >= q.keys) z[i].x = -INFINITY;
            if (key > pos[j][1] || key >= q.keys) z[i].y = -INFINITY;
            y[j][i] = pack2(z[i].x, z[i].y);
          }
        }
        top[j][0] = fmaxf(z[0].x, z[1].x);
        top[j][1] = fmaxf(z[0].y, z[1].y);
        if constexpr (SL == 2) {
          top[j][0] = fmaxf(top[j][0], fmaxf(z[2].x, z[3].x));
          top[j][1] = fmaxf(top[j][1], fmaxf(z[2].y, z[3].y));
        }
        grow = grow || top[j][0] - m[j][0] > kBelow + kGrow || top[j][1] - m[j][1] > kBelow + kGrow;
      }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float by[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float most = top[j][i];
#pragma unroll
            for (int d = 4; d < 32; d *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            by[i] = 1.f;
            if (most - m[j][i] > kBelow + kGrow) {  // rounded up: no weight passes 2^kBelow, however large the maximum
              const float to = __fsub_ru(most, kBelow);
              by[i] = exp2_fast(m[j][i] - to);
              m[j][i] = to;
            }
#pragma unroll
            for (int k = 0; k < MT; ++k) {
              o[k][j][i] *= by[i];
              o[k][j][2 + i] *= by[i];
            }
          }
          l[j] = mul2(l[j], pack2(by[0], by[1]));
        }
      }
      uint32_t w[SL][NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const uint64_t ref = pack2(m[j][0] == -INFINITY ? 0.f : -m[j][0], m[j][1] == -INFINITY ? 0.f : -m[j][1]);
#pragma unroll
        for (int i = 0; i < 2 * SL; ++i) {
          const float2 z = unpack2(add2(y[j][i], ref));
          const float w0 = exp2_fast(z.x), w1 = exp2_fast(z.y);
          l[j] = add2(l[j], pack2(w0, w1));
          w[i >> 1][j][i & 1] = turned(Half2<__half>::pack(w0, w1));
        }
      }
#pragma unroll
      for (int b = 0; b < SL; ++b) {
        if (!FULL && b >= slabs) break;
        const uint32_t at = stage + b * slab;
        uint32_t v0[W / 32] = {}, v1[W / 32] = {}, sc = 0;  // W = 128: two words a slot; 64: one
        if (W / 8 * g < D) {
          if constexpr (W == 128) {
            lds4(v0, at + 9 * D + lane * 16);
            lds4(v1, at + 13 * D + lane * 16);
            sc = lds1(at + 17 * D + g * 16 + 4 * t);
          } else {
            uint32_t v[4];
            lds4(v, at + 9 * D + lane * 16);
            v0[0] = v[0];
            v0[1] = v[1];
            v1[0] = v[2];
            v1[1] = v[3];
            sc = lds1(at + 17 * D + (g >> 1) * 16 + 4 * t);
          }
        }
        if constexpr (!FULL) {
          const int left = q.keys - key0 - b * kSlab - 4 * t;  // slots past the last key hold anything: scales of 0
          if (left < 4) sc &= left > 0 ? (1u << 8 * left) - 1 : 0u;
        }
        const ScalePair s0 = scale_pair(scales_of(sc, 0, 1)), s1 = scale_pair(scales_of(sc, 2, 3));
#pragma unroll
        for (int e = 0; e < W / 64; ++e) {
          // slots 4 t and 4 t + 1, 4 t + 2 and 4 t + 3: of each pair the even columns, the odd ones
          uint32_t r[4][4];
          const uint32_t a0 = v0[e], a1 = v0[e + W / 64], b0 = v1[e], b1 = v1[e + W / 64];
          raw_pairs(__byte_perm(a0, a1, 0x5410), r[0]);
          raw_pairs(__byte_perm(a0, a1, 0x7632), r[1]);
          raw_pairs(__byte_perm(b0, b1, 0x5410), r[2]);
          raw_pairs(__byte_perm(b0, b1, 0x7632), r[3]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t val[4] = {hfma2(r[0][i], s0.s, i & 1 ? s0.o256 : s0.o16),
                                     hfma2(r[1][i], s0.s, i & 1 ? s0.o256 : s0.o16),
                                     hfma2(r[2][i], s1.s, i & 1 ? s1.o256 : s1.o16),
                                     hfma2(r[3][i], s1.s, i & 1 ? s1.o256 : s1.o16)};
#pragma unroll
            for (int j = 0; j < NT; ++j) Half2<__half>::mma(o[4 * e + i][j], val, w[b][j][0], w[b][j][1]);
          }
        }
      }
    };
    for (int u = s.u0 + warp, end = s.u1; u < end; u += kWarps) {
      ok = ok && __all_sync(0xffffffffu, wait(full + stage_i, phase, limit));
      if (!ok) continue;  // no more copies are issued
      const int key0 = u * kUnit;
      const uint32_t stage = ring + stage_i * 2 * slab;
#pragma unroll
      for (int b = 0; b < 2; b += SL) {
        if (key0 + (b + SL) * kSlab - 1 <= first) unit(std::true_type(), key0 + b * kSlab, stage + b * slab);
        else unit(std::false_type(), key0 + b * kSlab, stage + b * slab);
      }
      __syncwarp();  // the stage has been read
      issue(stage_i);
      ++taken;
      if (++stage_i == kStages) {
        stage_i = 0;
        phase ^= 1;
      }
    }
    s = sh.part[warp];

    // the warps' sums, joined
    if (!ok) {  // NaN, not what the memory held: no wait gives up unseen
#pragma unroll
      for (int j = 0; j < NT; ++j) m[j][0] = m[j][1] = __int_as_float(0x7fffffff), l[j] = pack2(m[j][0], m[j][0]);
    }
    float* mine = rows + warp * a.rows * (W + 4);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = i ? unpack2(l[j]).y : unpack2(l[j]).x;
#pragma unroll
        for (int d = 4; d < 32; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int y = 8 * j + 2 * t + i;
        if (g == 0) sh.ml[warp][y] = make_float2(m[j][i], sum);
        if (y >= n_rows) continue;
        // columns 16 g .. (W = 128), 8 g ..
#pragma unroll
        for (int k = 0; k < MT; ++k)
          *reinterpret_cast<float2*>(mine + y * (W + 4) + MT * 2 * g + 2 * k) = make_float2(o[k][j][i], o[k][j][2 + i]);
      }
    __syncthreads();
    constexpr int PIECES = W / 8, ROWS = kThreads / PIECES;
    const int col = tid % PIECES * 8;
    const bool all = s.u0 == 0 && s.u1 == q.units;
    for (int y = tid / PIECES; y < n_rows; y += ROWS) {
      float mx = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float v = sh.ml[k][y].x;
        mx = v != v ? v : fmaxf(mx, v);
      }
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float2 ml = sh.ml[k][y];
        const float by = exp2_fast(ml.x - ref);
        sum += by * ml.y;
        const float4* z = reinterpret_cast<const float4*>(rows + (k * a.rows + y) * (W + 4) + col);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 v = z[e];
          acc[4 * e] += by * v.x;
          acc[4 * e + 1] += by * v.y;
          acc[4 * e + 2] += by * v.z;
          acc[4 * e + 3] += by * v.w;
        }
      }
      const float inv = sum == 0.f ? 0.f : __fdividef(128.f, sum);  // no key: zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = sum == 0.f ? 0.f : acc[e] * inv;
      if (col >= D) continue;
      if (all) {
        const int tok = a.group.div(y);
        const int64_t at = (int64_t)(q.q0 + tok) * c.nheads * G + s.h * G + y - tok * G;
        const uint4 z = make_uint4(Half2<T>::pack(acc[0], acc[1]), Half2<T>::pack(acc[2], acc[3]),
                                   Half2<T>::pack(acc[4], acc[5]), Half2<T>::pack(acc[6], acc[7]));
        *reinterpret_cast<uint4*>((T*)a.out + at * D + col) = z;
        if (col == 0 && a.lse) a.lse[at] = (mx + __log2f(sum)) * 0.6931471805599453f;
      } else {
        const int64_t at = (int64_t)(2 * blockIdx.x + (s.u0 == 0)) * (8 * NT) + y;
        float4* z = reinterpret_cast<float4*>(a.part + at * D + col);
        z[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        z[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        if (col == 0) a.part_ml[at] = make_float2(mx, sum);
      }
    }
    __syncthreads();
    advance(a, s);
    if (lane == 0) sh.part[warp] = s;
    __syncwarp();
  }
  if (lane == 0) sh.failed[warp] = !ok;
  // the copies in flight end before the block does
  if (!ok)
    for (; taken < issued; ++taken) wait(full + taken % kStages, taken / kStages & 1, kWaitCycles);
  __syncthreads();
  if (tid == 0) {
    int failed = 0;
    for (int k = 0; k < kWarps; ++k) failed |= sh.failed[k];
    if (failed) a.shares[blockIdx.x].w = 1;
  }
}

// Items that cuts went through: o = sum 2^(m_part - m) l_part o_part / sum 2^(m_part - m) l_part
// over their parts.  Block x: the item that share x + 1 begins inside of, if no share
// before does; block y: a row of it.  Each of the 4 warps adds every fourth part in
// their order, the warps' sums are added in theirs.
template <typename T>
__global__ void __launch_bounds__(128)
k_paged4_join(const __grid_constant__ Attn4Args a, WsHeader* hdr) {
  __shared__ float4 sums[4][32];
  __shared__ float weights[4];
  wait_for_previous();
  const int n = a.shares[a.nblocks].x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x == 0 && blockIdx.y == 0 && warp == 0) {
    int failed = 0;
    for (int i = lane; i < n; i += 32) failed |= a.shares[i].w;
    failed = __any_sync(0xffffffffu, failed);
    if (lane == 0) hdr->error = failed ? kErrTimeout : 0;
  }
  const int c0 = blockIdx.x + 1;
  if (c0 >= n) return;
  const int4 cut = a.shares[c0], before = a.shares[c0 - 1];
  if (cut.z == 0 || (before.x == cut.x && before.y == cut.y && before.z > 0)) return;
  const int G = a.group.d, D = a.c.width, y = blockIdx.y;
  const int q0 = __ldg(a.p.q_pos + cut.x), n_rows = (__ldg(a.p.q_pos + cut.x + 1) - q0) * G;
  if (y >= n_rows) return;
  int c1 = c0 + 1;  // shares c0 .. c1 - 1 begin inside of the item; 32 at a look
  for (uint32_t others = 0; others == 0;) {
    bool same = false;
    if (c1 + lane < n) {
      const int4 s = a.shares[c1 + lane];
      same = s.x == cut.x && s.y == cut.y && s.z != 0;
    }
    others = ~__ballot_sync(0xffffffffu, same);
    c1 += others ? __ffs(others) - 1 : 32;
  }
  const int parts = c1 - c0 + 1;
  auto part = [&](int k) { return (int64_t)(2 * (c0 - 1 + k) + (k == 0)) * a.tile + y; };
  float m = -INFINITY;
  bool nan = false;
  for (int k = lane; k < parts; k += 32) {
    const float v = a.part_ml[part(k)].x;
    nan = nan || v != v;
    m = fmaxf(m, v);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (__any_sync(0xffffffffu, nan)) m = __int_as_float(0x7fffffff);
  const float ref = m == -INFINITY ? 0.f : m;
  const int col = 4 * lane;
  float sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = warp; k < parts; k += 4) {
    const int64_t at = part(k);
    const float2 ml = a.part_ml[at];
    const float f = exp2_fast(ml.x - ref) * ml.y;
    sum += f;
    if (col < D) {
      const float4 x = *reinterpret_cast<const float4*>(a.part + at * D + col);
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
  const int tok = a.group.div(y);
  const int64_t at = (int64_t)(q0 + tok) * a.c.nheads * G + cut.y * G + y - tok * G;
  if (col < D) {
    uint2 z;
    z.x = Half2<T>::pack(acc.x * inv, acc.y * inv);
    z.y = Half2<T>::pack(acc.z * inv, acc.w * inv);
    *reinterpret_cast<uint2*>((T*)a.out + at * D + col) = z;
  }
  if (lane == 0 && a.lse) a.lse[at] = (m + __log2f(sum)) * 0.6931471805599453f;
}

template <typename T, int D, int NT>
cudaError_t launch_rows(const Attn4Args& a, cudaStream_t s) {
  auto kernel = k_paged4_rows<T, D, NT>;
  static OncePerDevice once;
  const cudaError_t e = once([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(D, 8 * NT, 8 * NT));
  });
  if (e != cudaSuccess) return e;
  kernel<<<SLNR_COUNTED((unsigned)a.nblocks), kThreads, smem_bytes(D, a.tile, a.rows), s>>>(a, wait_limit_cycles());
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_rows_d(const Attn4Args& a, cudaStream_t s) {
  switch (a.tile) {
    case 8: return launch_rows<T, D, 1>(a, s);
    case 16: return launch_rows<T, D, 2>(a, s);
    default: return launch_rows<T, D, 4>(a, s);
  }
}

template <typename T>
cudaError_t launch_rows_t(const Attn4Args& a, cudaStream_t s) {
  switch (a.c.width) {
    case 32: return launch_rows_d<T, 32>(a, s);
    case 64: return launch_rows_d<T, 64>(a, s);
    case 96: return launch_rows_d<T, 96>(a, s);
    default: return launch_rows_d<T, 128>(a, s);
  }
}

}  // namespace

int paged4_blocks(int width, int tile, int rows) {
  const int by_registers = tile == 8 ? 4 : 2;
  const int by_memory = (int)((size_t)228 * 1024 / (smem_bytes(width, tile, rows) + sizeof(Shared) + 1024));
  return 152 * (by_registers < by_memory ? by_registers : by_memory);
}

cudaError_t launch_paged4_rows(const Attn4Args& a, int dtype, cudaStream_t s) {
  return dtype == SLNR_FP16 ? launch_rows_t<__half>(a, s) : launch_rows_t<__nv_bfloat16>(a, s);
}

cudaError_t launch_paged4_join(const Attn4Args& a, int dtype, WsHeader* hdr, cudaStream_t s) {
  const dim3 grid((unsigned)a.nblocks, (unsigned)a.rows);
  auto kernel = dtype == SLNR_FP16 ? k_paged4_join<__half> : k_paged4_join<__nv_bfloat16>;
  return launch_next(kernel, SLNR_COUNTED(grid), dim3(128), 0, s, a, hdr);
}

}  // namespace slnr
