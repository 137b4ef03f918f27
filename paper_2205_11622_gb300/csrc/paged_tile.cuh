// Row tiles of an attention call: which rows of which request a block takes.
#pragma once

#include "paged.cuh"

namespace slnr {

// Row tiles of a request with n rows.
__device__ __forceinline__ int tiles_of(int rows, int tile) { return rows > 0 ? (rows - 1) / tile + 1 : 0; }

// Which request's part number `b` is, where request r has parts(r) of them, and
// which of its parts; r = -1 past the last one.  A whole warp looks at 128
// requests a step, four a lane.
template <typename Parts>
__device__ __forceinline__ void find_part(int nreq, int b, Parts parts, int& r, int& nth) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int r0 = 0; r0 < nreq; r0 = step_end(r0, 128, nreq)) {
    int n[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = inside(r0, 4 * lane + i, nreq) ? parts(r0 + 4 * lane + i) : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += n[i];
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + sum > b);
    if (past) {
      const int from = __ffs(past) - 1;
      int at = b - before - (sum - mine), i = 0;  // the lane's own, where it is the one
      while (i < 3 && at >= n[i]) at -= n[i++];
      r = __shfl_sync(0xffffffffu, (int)item(r0, 4 * lane + i), from);
      nth = __shfl_sync(0xffffffffu, at, from);
      return;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  r = -1;
  nth = 0;
}

// Request and first row of flat row tile `b`.
__device__ __forceinline__ void find_tile(const PagesView& p, int group, int tile, int b, int& r, int& x0) {
  find_part(
      p.nreq, b, [&](int i) { return tiles_of((__ldg(p.q_pos + i + 1) - __ldg(p.q_pos + i)) * group, tile); }, r, x0);
  x0 *= tile;
}

}  // namespace slnr
