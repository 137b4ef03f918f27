"""Places of keys, values and scales in a slab of a 4-bit cache (csrc/slab4.h), on the CPU: the header as it is."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_11622_gb300", "csrc")

SOURCE = """
#include "slab4.h"
using namespace slnr;
extern "C" {
int bytes(int width) { return slab_bytes(width); }
int place(int width, int what, int slot, int at) {
  const Slab s{width};
  return what == 0 ? s.k_word(slot, at) : what == 1 ? s.k_scale(slot, at) : what == 2 ? s.v_word(slot, at) : s.v_scale(slot, at);
}
unsigned half(unsigned a, unsigned b, unsigned c, unsigned d) { return half_word(a, b, c, d); }
}
"""
WIDTHS = (32, 64, 96, 128)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("slab4")
    (d / "slab4.cpp").write_text(SOURCE)
    so = str(d / "slab4.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "slab4.cpp"),
                    "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("width", WIDTHS)
def test_every_byte_has_one_use(lib, width):
    used = [0] * lib.bytes(width)
    assert len(used) == 18 * width and len(used) % 16 == 0
    for slot in range(16):
        for what, n, size in ((0, width // 8, 4), (1, width // 16, 1), (2, width // 8, 4), (3, width // 16, 1)):
            for i in range(n):
                at = lib.place(width, what, slot, i)
                assert at % size == 0
                for b in range(size):
                    used[at + b] += 1
    assert used == [1] * len(used)


@pytest.mark.parametrize("width", WIDTHS)
def test_lanes_find_what_they_multiply(lib, width):
    """The addresses that lane 4 g + t reads (paged4_rows.cu), for both widths of its products."""
    wide = width > 64
    words = 4 if wide else 2
    for g in range(8):
        for t in range(4):
            if 8 * words * t < width:  # two keys, g's and two slots on
                for half in range(2):
                    slot = 4 * (g >> 1) + (g & 1) + 2 * half
                    for w in range(words):
                        assert lib.place(width, 0, slot, words * t + w) == \
                            (4 * (g >> 1) + (g & 1)) * (width // 2) + 4 * words * t + half * width + 4 * w
                        block = (words * t + w) // 2
                        at = 8 * width + ((g * (width // 32) + t) * 4 + 2 * half + w // 2 if wide else
                                          (g * (width // 16) + t) * 2 + half)
                        assert lib.place(width, 1, slot, block) == at
            if (width // 8 if not wide else 16) * g < width and (16 if wide else 8) * g < width:
                lane = 4 * g + t
                for i in range(4):
                    assert lib.place(width, 3, 4 * t + i, g if wide else g >> 1) == \
                        17 * width + (g if wide else g >> 1) * 16 + 4 * t + i
                    if wide:
                        for e in range(2):
                            assert lib.place(width, 2, 4 * t + i, 2 * g + e) == \
                                9 * width + (i >> 1) * 4 * width + lane * 16 + (i & 1) * 8 + 4 * e
                    else:
                        assert lib.place(width, 2, 4 * t + i, g) == 9 * width + lane * 16 + 4 * i


def test_bits_of_a_half(lib):
    """n0 and n1 as fraction bits of fp16 numbers 16 + n and 256 + n; n2 and n3 after the half's bytes are swapped."""
    for n in ((1, 2, 4, 8), (15, 0, 7, 9), (8, 8, 8, 8), (5, 10, 15, 3)):
        x = lib.half(*n)
        y = (x & 255) << 8 | x >> 8
        assert x < 1 << 16
        assert ((x >> 6) & 15, (x >> 2) & 15, (y >> 6) & 15, (y >> 2) & 15) == n
