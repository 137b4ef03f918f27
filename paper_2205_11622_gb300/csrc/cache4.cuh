// Keys and values held in 4 bits (slab4.h): their way back to 16 bits.
#pragma once

#include "mma16.cuh"
#include "paged.cuh"
#include "slab4.h"

namespace slnr {

#ifdef __CUDACC__
// x & MASK | bits.
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "n"(MASK), "r"(bits));
  return r;
}

// The four pairs of a word as fp16: (16 + n) / 128 (pairs 0 and 2) and (256 + n) / 128 (1 and 3).
__device__ __forceinline__ void raw_pairs(uint32_t x, uint32_t (&r)[4]) {
  const uint32_t y = __byte_perm(x, 0, 0x2301);
  r[0] = and_or<0x03c003c0u>(x, 0x30003000u);
  r[1] = and_or<0x003c003cu>(x, 0x40004000u);
  r[2] = and_or<0x03c003c0u>(y, 0x30003000u);
  r[3] = and_or<0x003c003cu>(y, 0x40004000u);
}

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t bits_of(const __half2& x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  return bits_of(__hfma2(as_half2(a), as_half2(b), as_half2(c)));
}

// Two scales as what (16 + n) / 128 and (256 + n) / 128 are multiplied by and added to
// for code s / 128.  All exact: s is a whole multiple of 2^-17, 264 s / 128 has 10
// significant bits and is below 2^15.  (264 s itself would pass fp16's largest number.)
struct ScalePair {
  uint32_t s, o16, o256;
};
__device__ __forceinline__ ScalePair scale_pair(uint32_t fp16x2) {
  const __half2 s = as_half2(fp16x2);
  return {fp16x2, bits_of(__hmul2(s, __float2half2_rn(-24.f / 128))), bits_of(__hmul2(s, __float2half2_rn(-264.f / 128)))};
}
// Byte `i` of x as the fp16 number that it stands for, twice.
__device__ __forceinline__ uint32_t scale_twice(uint32_t x, int i) {
  return __byte_perm(x, 0, 0x0404 | (i << 12) | (i << 4)) >> 1;
}
// Bytes `i` and `j` side by side, the first in the lower half.
__device__ __forceinline__ uint32_t scales_of(uint32_t x, int i, int j) {
  return __byte_perm(x, 0, 0x0404 | (j << 12) | (i << 4)) >> 1;
}
// Scales of two blocks (bytes 0 and 1 of x), ready for the words of both, whose values
// they make: bf16 holds every value, fp16 every 128th part.  A multiplication picks its
// half of the pair by itself.
template <typename T>
struct Unpack;
template <>
struct Unpack<__half> {
  static constexpr float kTimes = 128.f;  // what the unpacked values lack
  ScalePair p;
  __device__ __forceinline__ explicit Unpack(uint32_t x) : p(scale_pair(scales_of(x, 0, 1))) {}
  // 8 columns of block SECOND.
  template <bool SECOND>
  __device__ __forceinline__ uint4 word(uint32_t x) const {
    uint32_t r[4];
    raw_pairs(x, r);
    auto value = [&](uint32_t n, uint32_t off) {
      const __half2 s = as_half2(p.s), o = as_half2(off);
      return bits_of(SECOND ? __hfma2(as_half2(n), __high2half2(s), __high2half2(o))
                            : __hfma2(as_half2(n), __low2half2(s), __low2half2(o)));
    };
    return make_uint4(value(r[0], p.o16), value(r[1], p.o256), value(r[2], p.o16), value(r[3], p.o256));
  }
};
template <>
struct Unpack<__nv_bfloat16> {
  static constexpr float kTimes = 1.f;
  __nv_bfloat162 s, off;
  __device__ __forceinline__ explicit Unpack(uint32_t x) {
    const float2 f = __half22float2(as_half2(scales_of(x, 0, 1)));
    s = __floats2bfloat162_rn(f.x, f.y);
    off = __hmul2(s, __float2bfloat162_rn(-40.f));
  }
  template <bool SECOND>
  __device__ __forceinline__ uint4 word(uint32_t x) const {  // n as the fraction bits 5..2 of 32 + n
    const uint32_t y = __byte_perm(x, 0, 0x2301);
    auto value = [&](uint32_t n) {
      n = and_or<0x003c003cu>(n, 0x42004200u);
      const __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162*>(&n);
      const __nv_bfloat162 r = SECOND ? __hfma2(a, __high2bfloat162(s), __high2bfloat162(off))
                                      : __hfma2(a, __low2bfloat162(s), __low2bfloat162(off));
      return *reinterpret_cast<const uint32_t*>(&r);
    };
    return make_uint4(value(x >> 4), value(x), value(y >> 4), value(y));
  }
};
#endif

// pages4.cu
cudaError_t launch_page_append4(const PagesView& p, const Cache4View& c, const RowsView& k, const RowsView& v, int dtype,
                                cudaStream_t s);
cudaError_t launch_page_values4(const Cache4View& c, const int32_t* pages, int n, void* k, void* v, int dtype,
                                cudaStream_t s);

}  // namespace slnr
