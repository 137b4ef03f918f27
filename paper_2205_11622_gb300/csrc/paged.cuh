// What the paged-cache kernels share: their views of the arguments, the
// division by the page size, and the launchers that the C entry points call.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "divide.h"
#include "once.h"

namespace slnr {

// The requests of a step (slnr_pages) as kernels take them.
struct PagesView {
  int nreq, ntok, width, max_q, max_k;
  int64_t table_stride;
  const int32_t *q_pos, *k_len, *table, *req, *slots;
};

// Rows of a tensor [token, head, column]; strides in values.
struct RowsView {
  const void* p;
  int64_t tok, head;
};

// The cache (slnr_cache); strides in values.
struct CacheView {
  void *k, *v;
  int64_t ks[3], vs[3];  // page, slot, head
  int npages, nheads, width;
  Divisor page;
  int8_t* codes;
  float* scales;
};

#ifdef __CUDACC__
// Page of a slot.
__device__ __forceinline__ int page_of(int slot, const CacheView& c) { return c.page.div(slot); }
#endif

// How the rows of an attention call go to blocks.
//
// The rows of a request and key head are its tokens' query rows of that head's
// group: row x is token x / G, query head g = x % G.  A block of the row kernel
// takes `tile` of them and at most `chunk` keys; the partial results of a row's
// `nsplit` chunks are combined in the chunks' order.
struct AttnPlan {
  int tile;     // rows a block takes
  int ntiles;   // bound of the row tiles of all requests
  int chunk;    // keys of one split, a multiple of the kernel's step
  int nsplit;   // splits of the longest request (1: the block writes the result)
  bool cluster; // the splits of a row are joined by the blocks of a cluster (row kernel, nsplit in 2 .. 16)
  // the tensor-core kernel's items (paged_chunk.cu): row tiles, cost of the items
  // before each, the item and step that each block's share begins at
  int4* tiles;      // [ntiles][2]
  int64_t* before;  // [ntiles * nheads]
  int2* shares;     // [kChunkBlocks], then {blocks with a share, items}, {row tiles, 0}
  // picked pages there: what the tokens of a tile's rows picked together, for each key head and row tile
  int32_t* pages;    // [nheads][ntiles][cap] pages of the request, ascending
  uint32_t* pickers; // [nheads][ntiles][cap][words] bit i: the tile's token i picked the page
  int32_t* npages;   // [nheads][ntiles]
  int cap, words;
  // partial rows, each divided by its own sum, and {what their weights were taken against (a power of two), that sum}:
  // [ntok * nheads_q][nsplit], or of the tensor-core kernel [2 kChunkBlocks][kChunkRows].  One number for the two, the
  // logarithm of the sum, would lose the sum beside large scores.
  float* part;      // [...][width]
  float2* part_ml;
};

constexpr int kAttnKeys = 64;       // keys of one step of the row kernel
constexpr int kChunkKeys = 128;     // and of the tensor-core kernel, whose blocks take
constexpr int kChunkRows = 256;     // that many rows; one block on each of 152 SMs,
constexpr int kChunkBlocks = 152;   // with a share of
constexpr int kLeastCost = 8;       // that much of their cost or more
constexpr int kAttnMaxPicked = 1024;  // pages picked for one row

struct AttnArgs {
  PagesView p;
  CacheView c;
  RowsView q;
  Divisor group;  // G
  float scale;
  void* out;      // [ntok][nheads_q][width], packed
  float* lse;     // [ntok][nheads_q] or NULL
  const int32_t* picked;  // selected attention: [ntok][nheads][npicked]
  int npicked;
  AttnPlan plan;
};

// Launches that follow one another in a call: the next grid may start once every
// block of the one before has called let_next_start (or ended), and waits in
// wait_for_previous until that one is done and its writes can be read.
#ifdef __CUDACC__
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
cudaError_t launch_next(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
#endif

// pages.cu
cudaError_t launch_page_tables(int nreq, const int32_t* new_len, const int32_t* old_len, int32_t* table,
                               int64_t table_stride, int width, const int32_t* free_pages, int nfree, int page_size,
                               int ntok, int32_t* q_pos, int32_t* k_len, int32_t* req, int32_t* slots, int32_t* used,
                               cudaStream_t s);
cudaError_t launch_page_append(const PagesView& p, const CacheView& c, const RowsView& k, const RowsView& v, int dtype,
                               cudaStream_t s);
cudaError_t launch_validate_lengths(int nreq, const int32_t* new_len, const int32_t* old_len, const int32_t* table,
                                    int64_t table_stride, int width, int nfree, int page_size, int ntok, WsHeader* hdr,
                                    cudaStream_t s);
cudaError_t launch_validate_pages(const PagesView& p, int npages, Divisor page, bool slots, const int32_t* picked,
                                  int npicked, int nheads, WsHeader* hdr, cudaStream_t s);

// page_select.cu
// Tokens whose scores over `pages` pages one block holds; 0: too many pages.
int select_tokens(int pages);
cudaError_t launch_page_select(const PagesView& p, const CacheView& c, const RowsView& q, int dtype, int nheads_q,
                               int32_t* picked, int npicked, int first, int last, cudaStream_t s);

// paged_chunk.cu (plan.tile == kChunkRows), in this order; the first zeroes hdr's
// flag word.  Picked pages: the page size divides 128 or is a multiple of it.
cudaError_t launch_paged_plan(const AttnArgs& a, WsHeader* hdr, cudaStream_t s);
cudaError_t launch_paged_chunk(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s);
cudaError_t launch_paged_join(const AttnArgs& a, int dtype, cudaStream_t s);

// paged_attn.cu (any other plan); the first zeroes hdr's flag word
cudaError_t launch_paged_rows(const AttnArgs& a, int dtype, WsHeader* hdr, cudaStream_t s);
cudaError_t launch_paged_combine(const AttnArgs& a, int dtype, cudaStream_t s);

}  // namespace slnr
