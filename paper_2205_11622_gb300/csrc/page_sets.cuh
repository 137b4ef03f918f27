// Whole pages between the steps: which ones requests hold, and their copies.
#pragma once

#include "paged.cuh"

namespace slnr {

// The block tables of all requests and their lengths.
struct TablesView {
  int nreq, width;
  int64_t stride;
  Divisor page;  // slots
  const int32_t* table;
  const int32_t* lens;
};

// One of the tensors that make up a page: outer x inner rows of `row` bytes, copied
// `unit` bytes a lane (16, 8 or 4); strides in bytes.
struct CopyPart {
  const char* from;
  char* to;
  int64_t from_page, to_page, from_outer, to_outer, from_inner, to_inner;
  Divisor inner, row;  // row: units
  int unit, pieces;    // pieces: units of a page
  int first;           // item of a page that its first piece is in
};
constexpr int kCopyParts = 4;
struct CopyParts {
  CopyPart part[kCopyParts];
  int n, items;  // items of a page
};
constexpr int kCopyLoads = 8;                 // in flight, a lane
constexpr int kCopyItem = 32 * kCopyLoads;    // units that a warp takes at once

constexpr int kSetBlocks = 16;           // of the one cluster that looks at all pages
constexpr int kSetWords = 16384;         // of 32 pages, of a block
constexpr int kMaxSetPages = kSetBlocks * kSetWords * 32;
constexpr int kMaxForks = 65536;

cudaError_t launch_page_copy(const CopyParts& c, const int32_t* src, const int32_t* dst, int n, int from_pages,
                             int to_pages, cudaStream_t s);
cudaError_t launch_page_fork(const TablesView& t, const int32_t* parent, int n, const int32_t* free_pages, int nfree,
                             int32_t* out_table, int32_t* out_lens, int32_t* src, int32_t* dst, int32_t* used,
                             cudaStream_t s);
cudaError_t launch_page_free(const TablesView& t, int32_t* lens, const int32_t* drop, int ndrop, int npages,
                             int32_t* free_pages, int32_t* count, cudaStream_t s);
cudaError_t launch_page_compact(const TablesView& t, int npages, int32_t* out_table, int32_t* src, int32_t* dst,
                                int32_t* ids, int32_t* used, cudaStream_t s);
// npages: of the cache (the largest int where it is not known)
cudaError_t launch_validate_set(const TablesView& t, int npages, const int32_t* list, int n, int bound, const int32_t* more,
                                int more_bound, WsHeader* hdr, cudaStream_t s);

}  // namespace slnr
