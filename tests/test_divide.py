"""The kernels' division by a shared divisor (csrc/divide.h) over its whole range, on the CPU: the header as it is."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_11622_gb300", "csrc")
MOST = 2 ** 31 - 1

SOURCE = """
#include "divide.h"
// first n at which the quotient is wrong (-1: none): around every `step`-th multiple of d, and at the ends
extern "C" long long first_wrong(int d, long long step) {
  const slnr::Divisor v = slnr::divisor(d);
  for (long long k = 0; k <= 2147483647LL / d; k += step)
    for (long long n = k * d - 1; n <= k * d + 1; ++n)
      if (n >= 0 && n <= 2147483647LL && v.div((int)n) != n / d) return n;
  for (long long n = 2147483647LL; n > 2147483647LL - 4096 && n >= 0; --n)
    if (v.div((int)n) != n / d) return n;
  return -1;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("divide")
    (d / "divide.cpp").write_text(SOURCE)
    so = str(d / "divide.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "divide.cpp"),
                    "-o", so], check=True)
    l = ctypes.CDLL(so)
    l.first_wrong.restype = ctypes.c_longlong
    l.first_wrong.argtypes = [ctypes.c_int, ctypes.c_longlong]
    return l


@pytest.mark.parametrize("d", [*range(1, 130), 255, 256, 257, 1000, 4095, 65537, 2 ** 24 + 1, 2 ** 30 - 1, 2 ** 30,
                               2 ** 30 + 1, MOST - 1, MOST])
def test_quotients(lib, d):
    assert lib.first_wrong(d, max(1, MOST // d // 100000)) == -1
