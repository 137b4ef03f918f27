// Row tiles of an attention call: which rows of which request a block takes.
#pragma once

#include "paged.cuh"

namespace slnr {

// Row tiles of a request with n rows.
__device__ __forceinline__ int tiles_of(int rows, int tile) { return rows > 0 ? (rows - 1) / tile + 1 : 0; }

// Request and first row of flat row tile `b`; r = -1 past the last one.  A whole
// warp looks at 32 requests a step.
__device__ __forceinline__ void find_tile(const PagesView& p, int group, int tile, int b, int& r, int& x0) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int r0 = 0; r0 < p.nreq; r0 += 32) {
    int n = 0;
    if (r0 + lane < p.nreq) n = tiles_of((__ldg(p.q_pos + r0 + lane + 1) - __ldg(p.q_pos + r0 + lane)) * group, tile);
    int sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + sum > b);
    if (past) {
      const int i = __ffs(past) - 1;
      r = r0 + i;
      x0 = (b - before - __shfl_sync(0xffffffffu, sum - n, i)) * tile;
      return;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  r = -1;
  x0 = 0;
}

}  // namespace slnr
