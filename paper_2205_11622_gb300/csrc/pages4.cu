// The writes of a cache in 4 bits, and the values that its pages stand for.
#include "cache4.cuh"
#include "launch.h"
#include "mma16.cuh"

namespace slnr {
namespace {

constexpr int kThreads = 256;

// Scale byte of a block whose largest magnitude is `most` (the bits of an fp32
// number; of infinity and NaN alike).  t is below most / 7.5 by 2^-20 of it at
// most, so the byte below it is the right one or one or two short; 7.5 s is exact.
__device__ __forceinline__ uint32_t scale_of(float most) {
  if (!(most <= 3.4028235e38f)) return 0xff;
  const float t = __fmul_rd(fminf(most, 69120.f), 0.13333321f);
  uint32_t b = __half_as_ushort(__float2half_rd(t)) >> 7;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float s = __half2float(__ushort_as_half((unsigned short)(b << 7)));
    if (7.5f * s < fminf(most, 69120.f)) ++b;
  }
  return b;
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

// code + 8 of x.  inv is 1 / s and 2^-20 of it more: a quotient half way between two
// whole numbers, which is then away from zero, is exact before that, and the others
// lie 2^-12 from one at least (x has 11 significant bits at most, s 4).
__device__ __forceinline__ uint32_t code_of(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -7.f), 7.f);
  return (__float_as_uint(y + 12582920.f)) & 15u;  // 1.5 2^23 + 8: the sum's last bits are the whole number
}

// A thread a block of 16 columns of one token's key or value (blockIdx.y) of one head.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_page_append4(PagesView p, Cache4View c, RowsView kn, RowsView vn, Divisor blocks, Divisor units, int tokens) {
  const bool value = blockIdx.y;
  const RowsView src = value ? vn : kn;
  const Slab slab{c.width};
  const int n = tokens * units.d;
  for (int u = threadIdx.x; u < n; u += kThreads) {
    const int local = units.div(u), t = step_end(blockIdx.x * tokens, local, p.ntok);
    if (t >= p.ntok) return;
    const int unit = u - local * units.d, h = blocks.div(unit), b = unit - h * blocks.d;
    const int slot = __ldg(p.slots + t);
    const int page = slot >= 0 ? c.slots.div(slot) : c.npages;
    if (page >= c.npages) continue;
    const int off = slot - page * c.slots.d;
    const uint4* from = reinterpret_cast<const uint4*>((const T*)src.p + t * src.tok + h * src.head + b * kBlockCols);
    const uint4 lo = __ldg(from), hi = __ldg(from + 1);
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    float x[16], most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 y = to_float2<T>(w[i]);
      x[2 * i] = y.x;
      x[2 * i + 1] = y.y;
    }
    uint32_t bits = 0;  // magnitudes in the order of their bits: NaN above infinity above all numbers
#pragma unroll
    for (int i = 0; i < 16; ++i) bits = max(bits, __float_as_uint(x[i]) & 0x7fffffffu);
    most = __uint_as_float(bits);
    const uint32_t byte = scale_of(most);
    const float s = __half2float(__ushort_as_half((unsigned short)(byte << 7)));
    const float inv = s > 0.f ? __fmul_ru(__fdiv_rn(1.f, s), 1.000001f) : 0.f;  // NaN: 0, its codes say nothing
    uint32_t code[16], word[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) code[i] = code_of(x[i], inv);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t* e = code + 8 * i;
      word[i] = half_word(e[0], e[2], e[4], e[6]) | (half_word(e[1], e[3], e[5], e[7]) << 16);
    }
    const int in = off & (kSlab - 1);
    uint8_t* to = c.data + page * c.page + h * c.head + (int64_t)(off / kSlab) * slab_bytes(c.width);
    if (value) {
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<uint32_t*>(to + slab.v_word(in, 2 * b + i)) = word[i];
      to[slab.v_scale(in, b)] = (uint8_t)byte;
    } else {
      *reinterpret_cast<uint2*>(to + slab.k_word(in, 2 * b)) = make_uint2(word[0], word[1]);
      to[slab.k_scale(in, b)] = (uint8_t)byte;
    }
  }
}

// A thread a block of 16 columns of one slot's key or value (blockIdx.y) of one head;
// blockIdx.x: page and part of its slots.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_page_values4(Cache4View c, const int32_t* __restrict__ pages, T* k, T* v, Divisor blocks, Divisor heads, Divisor parts) {
  const bool value = blockIdx.y;
  const Slab slab{c.width};
  const int i = parts.div(blockIdx.x), page = pages ? __ldg(pages + i) : i;
  const int unit = (blockIdx.x - i * parts.d) * kThreads + threadIdx.x;  // [slot][head][block]
  const int row = blocks.div(unit), b = unit - row * blocks.d, slot = heads.div(row), h = row - slot * heads.d;
  if (slot >= c.slots.d) return;
  uint32_t x[2] = {0, 0}, byte = 0;
  if ((unsigned)page < (unsigned)c.npages) {
    const int in = slot & (kSlab - 1);
    const uint8_t* from = c.data + page * c.page + h * c.head + (int64_t)(slot / kSlab) * slab_bytes(c.width);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = *reinterpret_cast<const uint32_t*>(from + (value ? slab.v_word(in, 2 * b + e) : slab.k_word(in, 2 * b + e)));
    byte = from[value ? slab.v_scale(in, b) : slab.k_scale(in, b)];
  }
  const ScalePair sp = scale_pair(scale_twice(byte, 0));
  uint32_t y[8];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    uint32_t r[4];
    raw_pairs(x[e], r);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t z = hfma2(r[j], sp.s, j & 1 ? sp.o256 : sp.o16);  // of values / 128
      const float2 f = to_float2<__half>(z);
      y[4 * e + j] = Half2<T>::pack(f.x * 128.f, f.y * 128.f);
    }
  }
  T* to = (value ? v : k) + ((int64_t)i * c.slots.d * c.nheads + row) * c.width + b * kBlockCols;
  reinterpret_cast<uint4*>(to)[0] = make_uint4(y[0], y[1], y[2], y[3]);
  reinterpret_cast<uint4*>(to)[1] = make_uint4(y[4], y[5], y[6], y[7]);
}

}  // namespace

cudaError_t launch_page_append4(const PagesView& p, const Cache4View& c, const RowsView& k, const RowsView& v, int dtype,
                                cudaStream_t s) {
  const int blocks = c.width / kBlockCols, units = blocks * c.nheads;
  const int tokens = units >= kThreads ? 1 : kThreads / units;
  const dim3 grid((unsigned)pieces(p.ntok, tokens), 2);
  auto kernel = dtype == SLNR_FP16 ? k_page_append4<__half> : k_page_append4<__nv_bfloat16>;
  kernel<<<(SLNR_COUNTED(grid)), kThreads, 0, s>>>(p, c, k, v, divisor(blocks), divisor(units), tokens);
  return cudaGetLastError();
}

cudaError_t launch_page_values4(const Cache4View& c, const int32_t* pages, int n, void* k, void* v, int dtype,
                                cudaStream_t s) {
  const int blocks = c.width / kBlockCols;
  const int parts = pieces(c.slots.d * c.nheads * blocks, kThreads);
  const dim3 grid((unsigned)((int64_t)n * parts), 2);
  if (dtype == SLNR_FP16)
    k_page_values4<__half><<<(SLNR_COUNTED(grid)), kThreads, 0, s>>>(c, pages, (__half*)k, (__half*)v, divisor(blocks),
                                                                    divisor(c.nheads), divisor(parts));
  else
    k_page_values4<__nv_bfloat16><<<(SLNR_COUNTED(grid)), kThreads, 0, s>>>(
        c, pages, (__nv_bfloat16*)k, (__nv_bfloat16*)v, divisor(blocks), divisor(c.nheads), divisor(parts));
  return cudaGetLastError();
}

}  // namespace slnr
