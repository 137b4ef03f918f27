// The writes of a cache in 4 bits, and the values that its pages stand for.
#include <type_traits>

#include "cache4.cuh"
#include "launch.h"
#include "mma16.cuh"

namespace slnr {
namespace {

constexpr int kThreads = 256;

// Scale byte of a block whose largest magnitude is `most`.  As a number of 2^-112 times
// its size a scale has the byte as its first bits (exponents of both end at 0, where
// both go on without their leading bit).  The factor is below 2^-112 / 7.5 by 2^-21 of
// it: a scale that is right to the last bit stays at or below itself, and the others lie
// 2^-13 of themselves from one at least (x has 11 significant bits at most, a scale 4).
constexpr float kUp = 5.192296858534828e33f;      // 2^112
constexpr float kPart = 2.5679053680430326e-35f;  // (1 - 2^-21) / 7.5 / 2^112
__device__ __forceinline__ uint32_t scale_of(float most) {
  const uint32_t b = min((__float_as_uint(most * kPart) + 0xfffffu) >> 20, 225u);
  return most <= 3.4028235e38f ? b : 0xffu;  // infinity and NaN
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 20) * kUp; }

__device__ __forceinline__ uint64_t mul2(float a, float b, float by) {  // two products in one instruction
  uint64_t x, y, r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
  asm("mov.b64 %0, {%1, %1};" : "=l"(y) : "f"(by));
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, float b) {
  uint64_t y, r;
  asm("mov.b64 %0, {%1, %1};" : "=l"(y) : "f"(b));
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(y));
  return r;
}

// Largest magnitude of a block's 16 values, as an fp32 number; NaN above all.  Magnitudes
// are in the order of their bits.
template <typename T>
__device__ __forceinline__ float largest(const uint32_t (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(x[i] & 0x7fff7fffu));
  const uint32_t one = max(m & 0xffffu, m >> 16);
  return std::is_same<T, __half>::value ? __half2float(__ushort_as_half((unsigned short)one)) : __uint_as_float(one << 16);
}

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

// Eight columns' n (code + 8), of pairs of an even column and the odd one after it, 16
// bits each, as a word: half_word of both halves.
__device__ __forceinline__ uint32_t word_of(const uint32_t (&pair)[4]) {
  return pair[0] * 64 + pair[1] * 4 + pair[3] * 1024 + (pair[2] & 0x00030003u) * 16384 + ((pair[2] >> 2) & 0x00030003u);
}
constexpr float kWhole = 12582920.f;  // 1.5 2^23 + 8: the last bits of a sum with it are the whole number + 8

// A pair within -most .. most.
template <typename T>
__device__ __forceinline__ uint32_t within(uint32_t x, uint32_t most);
template <>
__device__ __forceinline__ uint32_t within<__nv_bfloat16>(uint32_t x, uint32_t most) {
  asm("min.bf16x2 %0, %0, %1;\n\tmax.bf16x2 %0, %0, %2;" : "+r"(x) : "r"(most), "r"(most ^ 0x80008000u));
  return x;
}
template <>
__device__ __forceinline__ uint32_t within<__half>(uint32_t x, uint32_t most) {
  asm("min.f16x2 %0, %0, %1;\n\tmax.f16x2 %0, %0, %2;" : "+r"(x) : "r"(most), "r"(most ^ 0x80008000u));
  return x;
}

// The scale byte and the two words of a block.  x / s is taken with 2^-20 of it more, so
// that a quotient half way between two whole numbers, which is exact before that, goes
// away from zero; the others lie 2^-12 from one at least.  What is past 7 s has the code
// 7: it is made 7 s, a number of both types, two at a time (one in 16 largest values is
// 7.5 s itself).
template <typename T>
__device__ __forceinline__ uint32_t coded(const uint4& lo, const uint4& hi, uint2& words) {
  const uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const float most = largest<T>(x);
  const uint32_t byte = scale_of(most);
  const float s = scale_value(byte), inv = s > 0.f ? __fmul_ru(__fdividef(1.f, s), 1.000001f) : 0.f;
  const uint32_t limit = Half2<T>::pack(7.f * s, 7.f * s);
  uint32_t pair[2][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 y = to_float2<T>(within<T>(x[i], limit));
    const uint64_t z = add2(mul2(y.x, y.y, inv), kWhole);
    pair[i / 4][i & 3] = __byte_perm((uint32_t)z, (uint32_t)(z >> 32), 0x5410);
  }
  words = make_uint2(word_of(pair[0]), word_of(pair[1]));
  return byte;
}

// Which blocks of 16 columns a warp takes: of 8 rows (tokens, or slots of a page) that
// lie together four blocks of one head, or two where a row has no fours, of twice as many
// rows.  Codes of eight slots from a multiple of 8 on then fill whole 32-byte sectors.
struct Group {
  int blocks, rows;  // of a warp
  Divisor per_head, units;  // warps of a head's row, and of a row
};
Group group(int width, int heads) {
  const int blocks = width / kBlockCols, n = blocks % 4 == 0 ? 4 : 2;
  return {n, 32 / n, divisor(blocks / n), divisor(blocks / n * heads)};
}

// A thread a block of 16 columns of one token's key and value of one head.  Per value
// one instruction to make it fp32, one each for two values to take the quotient, the
// whole number and the pair, one and a half to place it.  32k tokens of 8 heads of 128
// (168 MB in and out) 33 us, 5.1 TB/s, two thirds of the issue slots.  52 with each value limited to 7
// in fp32 and a division; 38 with limits that only blocks with a value past 7 s took (one
// block in 16: most warps have one).
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_page_append4(PagesView p, Cache4View c, RowsView kn, RowsView vn, Group gr, int warps) {
  const int w = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (w >= warps) return;
  const Slab slab{c.width};
  const int set = gr.units.div(w), unit = w - set * gr.units.d, h = gr.per_head.div(unit);
  const int row = lane / gr.blocks, b = (unit - h * gr.per_head.d) * gr.blocks + lane - row * gr.blocks;
  const int t = step_end(set * gr.rows, row, p.ntok);
  if (t >= p.ntok) return;
  const int slot = __ldg(p.slots + t);
  const uint4* from_k = reinterpret_cast<const uint4*>((const T*)kn.p + t * kn.tok + h * kn.head + b * kBlockCols);
  const uint4* from_v = reinterpret_cast<const uint4*>((const T*)vn.p + t * vn.tok + h * vn.head + b * kBlockCols);
  const uint4 k0 = __ldg(from_k), k1 = __ldg(from_k + 1), v0 = __ldg(from_v), v1 = __ldg(from_v + 1);
  const int page = slot >= 0 ? c.slots.div(slot) : c.npages;
  if (page >= c.npages) return;
  const int off = slot - page * c.slots.d, in = off & (kSlab - 1);
  uint8_t* to = c.data + page * c.page + h * c.head + (int64_t)(off / kSlab) * slab_bytes(c.width);
  uint2 words;
  to[slab.k_scale(in, b)] = (uint8_t)coded<T>(k0, k1, words);
  *reinterpret_cast<uint2*>(to + slab.k_word(in, 2 * b)) = words;
  to[slab.v_scale(in, b)] = (uint8_t)coded<T>(v0, v1, words);
  if (c.width > 64) {
    *reinterpret_cast<uint2*>(to + slab.v_word(in, 2 * b)) = words;
  } else {
    *reinterpret_cast<uint32_t*>(to + slab.v_word(in, 2 * b)) = words.x;
    *reinterpret_cast<uint32_t*>(to + slab.v_word(in, 2 * b + 1)) = words.y;
  }
}

// A thread a block of 16 columns of one slot's key and value of one head.
template <typename T>
__device__ __forceinline__ void store_values(T* to, uint2 x, uint32_t byte, bool aligned) {
  const Unpack<T> u(byte);
  uint4 y[2] = {u.template word<false>(x.x), u.template word<false>(x.y)};
  uint32_t* e = &y[0].x;
  if (Unpack<T>::kTimes != 1.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = bits_of(__hmul2(as_half2(e[i]), __float2half2_rn(Unpack<T>::kTimes)));
  }
  if (aligned) {  // 32 bytes at once: a whole sector a lane (26 us for 32k slots where 16-byte stores took 33)
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(y[0].x), "r"(y[0].y), "r"(y[0].z),
                 "r"(y[0].w), "r"(y[1].x), "r"(y[1].y), "r"(y[1].z), "r"(y[1].w)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = y[0];
    reinterpret_cast<uint4*>(to)[1] = y[1];
  }
}
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_page_values4(Cache4View c, const int32_t* __restrict__ pages, T* k, T* v, Group gr, Divisor page_warps, int64_t warps) {
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (w >= warps) return;
  const int lane = threadIdx.x & 31, i = (int)(w / page_warps.d), in_page = (int)(w - (int64_t)i * page_warps.d);
  const int page = pages ? __ldg(pages + i) : i;
  const Slab slab{c.width};
  const int set = gr.units.div(in_page), unit = in_page - set * gr.units.d, h = gr.per_head.div(unit);
  const int sub = lane / gr.blocks, b = (unit - h * gr.per_head.d) * gr.blocks + lane - sub * gr.blocks;
  const int slot = set * gr.rows + sub;  // a page's slots are a multiple of a warp's
  uint2 kx = make_uint2(0, 0), vx = kx;
  uint32_t ks = 0, vs = 0;
  if ((unsigned)page < (unsigned)c.npages) {
    const int in = slot & (kSlab - 1);
    const uint8_t* from = c.data + page * c.page + h * c.head + (int64_t)(slot / kSlab) * slab_bytes(c.width);
    kx = *reinterpret_cast<const uint2*>(from + slab.k_word(in, 2 * b));
    ks = from[slab.k_scale(in, b)];
    if (c.width > 64) {
      vx = *reinterpret_cast<const uint2*>(from + slab.v_word(in, 2 * b));
    } else {
      vx.x = *reinterpret_cast<const uint32_t*>(from + slab.v_word(in, 2 * b));
      vx.y = *reinterpret_cast<const uint32_t*>(from + slab.v_word(in, 2 * b + 1));
    }
    vs = from[slab.v_scale(in, b)];
  }
  const int64_t at = (((int64_t)i * c.slots.d + slot) * c.nheads + h) * c.width + b * kBlockCols;
  store_values(k + at, kx, ks, (reinterpret_cast<uintptr_t>(k) & 31) == 0);
  store_values(v + at, vx, vs, (reinterpret_cast<uintptr_t>(v) & 31) == 0);
}

}  // namespace

cudaError_t launch_page_append4(const PagesView& p, const Cache4View& c, const RowsView& k, const RowsView& v, int dtype,
                                cudaStream_t s) {
  const Group gr = group(c.width, c.nheads);
  const int64_t warps = (int64_t)pieces(p.ntok, gr.rows) * gr.units.d;
  if (warps > INT32_MAX) return cudaErrorInvalidConfiguration;
  const unsigned grid = (unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32));
  auto kernel = dtype == SLNR_FP16 ? k_page_append4<__half> : k_page_append4<__nv_bfloat16>;
  kernel<<<SLNR_COUNTED(grid), kThreads, 0, s>>>(p, c, k, v, gr, (int)warps);
  return cudaGetLastError();
}

cudaError_t launch_page_values4(const Cache4View& c, const int32_t* pages, int n, void* k, void* v, int dtype,
                                cudaStream_t s) {
  const Group gr = group(c.width, c.nheads);
  const int page_warps = c.slots.d / gr.rows * gr.units.d;
  const int64_t warps = (int64_t)n * page_warps;
  const unsigned grid = (unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32));
  if (dtype == SLNR_FP16)
    k_page_values4<__half><<<SLNR_COUNTED(grid), kThreads, 0, s>>>(c, pages, (__half*)k, (__half*)v, gr, divisor(page_warps),
                                                                  warps);
  else
    k_page_values4<__nv_bfloat16><<<SLNR_COUNTED(grid), kThreads, 0, s>>>(c, pages, (__nv_bfloat16*)k, (__nv_bfloat16*)v, gr,
                                                                         divisor(page_warps), warps);
  return cudaGetLastError();
}

}  // namespace slnr
