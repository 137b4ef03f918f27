// Attention over a cache in 4 bits: the arguments of the row kernel.
#pragma once

#include "cache4.cuh"

namespace slnr {

struct Attn4Args {
  PagesView p;
  Cache4View c;
  RowsView q;
  Divisor group;  // query heads of a key head
  float scale;
  void* out;      // [ntok][nheads_q][width], packed
  float* lse;     // [ntok][nheads_q] or NULL
  int tile;       // rows that a warp multiplies: 8, 16 or 32
  int rows;       // of an item, at most: max_q query heads of a key head
  int nblocks;    // blocks, of a share each
  int least;      // units of a share, at least
  int4* shares;   // [nblocks] {request, key head, unit that it begins at, a wait gave up}, then {shares, 0, 0, 0}
  float* part;    // [2 nblocks][tile][width] partial rows, each divided by its own sum, and
  float2* part_ml;  // {what their weights were taken against (a power of two), that sum}
};

// Blocks that run at once.
int paged4_blocks(int width, int tile, int rows);

// paged4_rows.cu, in this order; the second writes hdr's flag word
cudaError_t launch_paged4_rows(const Attn4Args& a, int dtype, cudaStream_t s);
cudaError_t launch_paged4_join(const Attn4Args& a, int dtype, WsHeader* hdr, cudaStream_t s);

}  // namespace slnr
