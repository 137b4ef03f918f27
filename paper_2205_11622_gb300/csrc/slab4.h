// Keys and values held in 4 bits: the numbers and their places in a page.  Also
// compiled for the host.
//
// Blocks of 16 consecutive columns of one key (or value) of one head share a
// scale s, an unsigned number of 5 exponent and 3 fraction bits: the upper bits of
// an fp16 number below its sign, so a byte b is the fp16 number with the bits b << 7.
//   s = the smallest such number with 7.5 s >= max |x|, at most 9216;
//   code = x / s rounded to the nearest whole number, halves away from zero, in [-7, 7].
// So |x - code s| <= s / 2 up to |x| = 69120, above which x is held as 64512.  A
// block with a value that is not finite has the scale 0xff, an fp16 NaN.  For
// normal values the root mean square error is 8.5 % of theirs; with a largest code
// taken as the 7th instead of the 7.5th part, 9.3 %; 2-bit exponents and 1-bit
// fractions in the place of whole numbers (the 4-bit floats of the tensor cores,
// scales alike) 9.5 %.
//
// code s has 7 significant bits: exact in bf16 and fp16.  Codes are held as n =
// code + 8, placed so that one logical instruction makes a pair of fp16 numbers of
// them.  A 32-bit word holds 8 columns; its lower half the even ones, its upper
// half the odd ones, a half's four n at
//   n0: bits 9..6   n1: bits 5..2   n2: bits 1..0 and 15..14   n3: bits 13..10
// so that n0 and n1, and after a swap of a half's bytes n2 and n3, are fraction bits
// of 16 + n (exponent bits of 16) and 256 + n (of 256), or of the 128th part of these.
//
// A page of one head is a run of slabs of 16 slots, each 18 width bytes: codes of
// the keys (8 width bytes), their scales (width), codes of the values, their
// scales.  Inside of a slab the order is the one that a warp's lanes read (paged4_rows.cu):
// lane 4 c + t takes columns of all keys by t and of four values, slots 4 t .. 4 t
// + 3, by c, each in 16-byte pieces that lie beside its neighbours'.
#pragma once

#include <cstdint>

#include "range.h"

namespace slnr {

constexpr int kSlab = 16;      // slots
constexpr int kBlockCols = 16;  // columns that share a scale

SLNR_HD constexpr int slab_bytes(int width) { return 18 * width; }

// Byte offsets inside of a slab: of a word of 8 columns, and of a block's scale.
struct Slab {
  int width;
  SLNR_HD int k_word(int slot, int w) const { return slot * (width / 2) + 4 * w; }
  // keys' scales: those of the slots that a lane multiplies together, side by side
  SLNR_HD int k_scale(int slot, int block) const {
    const int g = 2 * (slot >> 2) + (slot & 1), half = (slot >> 1) & 1;
    return 8 * width + (width > 64 ? (g * (width / 32) + (block >> 1)) * 4 + half * 2 + (block & 1)
                                   : (g * (width / 16) + block) * 2 + half);
  }
  SLNR_HD int v_word(int slot, int w) const {
    const int t = slot >> 2, i = slot & 3;
    return 9 * width + (width > 64 ? (i >> 1) * 4 * width + ((w >> 1) * 4 + t) * 16 + (i & 1) * 8 + (w & 1) * 4
                                   : (w * 4 + t) * 16 + i * 4);
  }
  SLNR_HD int v_scale(int slot, int block) const { return 17 * width + block * 16 + slot; }
};

// The half of a word with n0 .. n3.
SLNR_HD uint32_t half_word(uint32_t n0, uint32_t n1, uint32_t n2, uint32_t n3) {
  return (n0 << 6) | (n1 << 2) | (n2 >> 2) | ((n2 & 3) << 14) | (n3 << 10);
}

}  // namespace slnr
