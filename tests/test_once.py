"""What a launcher does once a device (csrc/once.h), on the CPU: the header as it is, with the current device faked."""
import ctypes
import os
import subprocess

import pytest

import paper_2205_11622_gb300 as slnr

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_11622_gb300", "csrc")

SOURCE = """
#include <cuda_runtime.h>
static int device = 0, runs = 0;
static cudaError_t found = cudaSuccess;
static cudaError_t fake_device(int* d) { *d = device; return found; }
#define cudaGetDevice fake_device  // by name: the process may have the CUDA runtime loaded
#include "once.h"
static slnr::OncePerDevice once;
// one call on device d, whose work ends with `status`; runs so far
extern "C" int call(int d, int status, int query, int* result) {
  device = d;
  found = (cudaError_t)query;
  *result = once([&] { ++runs; return (cudaError_t)status; });
  return runs;
}
"""


@pytest.fixture
def call(tmp_path):
    (tmp_path / "once.cpp").write_text(SOURCE)
    so = str(tmp_path / "once.so")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(slnr._build.nvcc_path()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-isystem", include,
                    str(tmp_path / "once.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)

    def one(device, status=0, query=0):
        result = ctypes.c_int(-1)
        return lib.call(device, status, query, ctypes.byref(result)), result.value
    return one


def test_once_a_device(call):
    assert [call(0), call(0), call(1), call(0), call(1), call(63)] == [(1, 0), (1, 0), (2, 0), (2, 0), (2, 0), (3, 0)]
    assert [call(64), call(64)] == [(4, 0), (5, 0)]  # past the ones that are kept: every time


def test_a_failure_is_not_kept(call):
    """A first call without room for the kernel; a later one has it."""
    assert call(2, status=2) == (1, 2)
    assert call(2, status=2) == (2, 2)
    assert call(2) == (3, 0)
    assert call(2, status=2) == (3, 0)


def test_no_device(call):
    assert call(0, query=100) == (0, 100)
    assert call(0) == (1, 0)
