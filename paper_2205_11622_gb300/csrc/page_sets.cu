// Whole pages between the steps of a program: copies of them, requests that go on
// from others, the pages that no request holds, and pages packed to the front.
#include "launch.h"
#include "page_sets.cuh"

namespace slnr {
namespace {

// ---------------------------------------------------------------------------
// Copies.  An item is 256 units of a page's tensor (4 KB of 16-byte units), and a
// warp's: 8 loads a lane in flight, then 8 stores.  Warp g of W takes items g, g +
// W, ... of all pages; its lanes look at 32 of them at once for the ones whose
// entries name pages, so that long lists of which few are used cost little.  600 pages of
// 64 slots, 8 heads of 128 (315 MB in and out) 52 us, 6.0 TB/s.
constexpr int kCopyThreads = 256;

template <typename U>
__device__ __forceinline__ void copy_item(const CopyPart& a, int64_t src, int64_t dst, int item) {
  const int lane = threadIdx.x & 31;
  U x[kCopyLoads];
  int64_t to[kCopyLoads];
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k) {
    const int p = item * kCopyItem + k * 32 + lane;
    to[k] = -1;
    if (p < a.pieces) {
      const int row = a.row.div(p), outer = a.inner.div(row), inner = row - outer * a.inner.d;
      const int64_t off = (int64_t)(p - row * a.row.d) * sizeof(U);
      to[k] = dst * a.to_page + outer * a.to_outer + inner * a.to_inner + off;
      x[k] = *reinterpret_cast<const U*>(a.from + src * a.from_page + outer * a.from_outer + inner * a.from_inner + off);
    }
  }
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k)
    if (to[k] >= 0) *reinterpret_cast<U*>(a.to + to[k]) = x[k];
}

__global__ void __launch_bounds__(kCopyThreads)
k_page_copy(const __grid_constant__ CopyParts c, const int32_t* src, const int32_t* dst, int n, int from_pages, int to_pages) {
  const int lane = threadIdx.x & 31;
  const int64_t all = (int64_t)n * c.items, warps = (int64_t)gridDim.x * (kCopyThreads / 32);
  const int64_t first = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
  for (int64_t w0 = first; w0 < all; w0 += 32 * warps) {
    const int64_t w = w0 + lane * warps;
    int from = -1, to = -1, item = 0;
    if (w < all) {
      const int e = (int)(w / c.items);
      item = (int)(w - (int64_t)e * c.items);
      from = src[e];
      to = dst[e];
    }
    const bool on = (unsigned)from < (unsigned)from_pages && (unsigned)to < (unsigned)to_pages;
    for (uint32_t left = __ballot_sync(0xffffffffu, on); left; left &= left - 1) {
      const int l = __ffs(left) - 1;
      const int64_t f = __shfl_sync(0xffffffffu, from, l), t = __shfl_sync(0xffffffffu, to, l);
      const int i = __shfl_sync(0xffffffffu, item, l);
      int k = 0;
#pragma unroll
      for (int j = 1; j < kCopyParts; ++j)
        if (j < c.n && i >= c.part[j].first) k = j;
      const CopyPart& a = c.part[k];
      if (a.unit == 16) copy_item<uint4>(a, f, t, i - a.first);
      else if (a.unit == 8) copy_item<uint2>(a, f, t, i - a.first);
      else copy_item<uint32_t>(a, f, t, i - a.first);
    }
  }
}

// ---------------------------------------------------------------------------
// Sets of pages: one cluster of 16 blocks.  Each block has a sixteenth of the
// pages, a bit each, in its shared memory, and reads a sixteenth of the tables.  Up to
// 2^20 pages a block sets the bits of what it reads in a set of all pages of its own,
// and the sets are joined (512 requests, 150k pages, 27 -> 16 us); above, where
// those do not fit, it sets them where they belong.  Counts go through shared memory
// too, so one launch does it, without a workspace, and lists come out in the pages' order.
constexpr int kSetThreads = 1024;
constexpr int kSetWarps = kSetBlocks * kSetThreads / 32;
constexpr int kRun = 256;  // entries of a row that a warp takes at once

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t address_in(const void* local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(r)
               : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
  return r;
}
__device__ __forceinline__ int load_far(uint32_t at) {
  int v;
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void or_far(uint32_t at, uint32_t bits) {
  asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(at), "r"(bits) : "memory");
}

// Pages of a request of n keys, as many as its row of the table has.
__device__ __forceinline__ int held_pages(int n, const TablesView& t) {
  return n > 0 ? min(t.page.div(n - 1) + 1, t.width) : 0;
}

// Exclusive sum over the block's threads; `total` gets the whole.
__device__ __forceinline__ int block_before(int x, int& total, int* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int y = s_warp[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  total = __shfl_sync(0xffffffffu, y, 31);
  const int before = __shfl_sync(0xffffffffu, y, (warp + 31) & 31);
  return x - mine + (warp > 0 ? before : 0);
}

// The sums of a number of each block: of the blocks before this one, and of all.
// s_mine: the block's, which stays until the next cluster_sync after this.
__device__ __forceinline__ int cluster_before(const int* s_mine, int& total) {
  const int rank = (int)cluster_rank(), lane = threadIdx.x & 31;
  cluster_sync();
  const int x = lane < kSetBlocks ? load_far(address_in(s_mine, lane)) : 0;
  const int before = __reduce_add_sync(0xffffffffu, lane < rank ? x : 0);
  total = __reduce_add_sync(0xffffffffu, x);
  return before;
}

// Calls f(request, first entry, entries of its row that are its) for runs of entries, a warp each.
template <typename F>
__device__ __forceinline__ void each_run(int rows, int width, F f) {
  const int runs = width > 0 ? (width - 1) / kRun + 1 : 1;
  const int64_t all = (int64_t)rows * runs;
  for (int64_t i = (int64_t)cluster_rank() * (kSetThreads / 32) + (threadIdx.x >> 5); i < all; i += kSetWarps) {
    const int r = (int)(i / runs);
    f(r, (int)(i - (int64_t)r * runs) * kRun);
  }
}

struct SetShared {
  int warp[32];
  int count, count2;
};

// Sets the bits of the pages that requests hold; words: of each block.  all: LOCAL,
// the block's set of all pages.
template <bool LOCAL>
__device__ __forceinline__ void mark_held(const TablesView& t, uint32_t* bits, uint32_t* all, int words, int npages) {
  const int lane = threadIdx.x & 31;
  if (LOCAL)
    for (int i = threadIdx.x; i < kSetBlocks * words; i += kSetThreads) all[i] = 0;
  else
    for (int i = threadIdx.x; i < words; i += kSetThreads) bits[i] = 0;
  cluster_sync();
  each_run(t.nreq, t.width, [&](int r, int at) {
    const int n = held_pages(__ldcg(t.lens + r), t);
    if (at >= n) return;
    const int32_t* row = t.table + r * t.stride;
    int p[kRun / 32];
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k) {
      const int j = at + k * 32 + lane;
      p[k] = j < n ? __ldg(row + j) : -1;
    }
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k)
      if ((unsigned)p[k] < (unsigned)npages) {
        const int w = p[k] >> 5;
        if (LOCAL) {
          atomicOr(all + w, 1u << (p[k] & 31));
        } else {
          const int block = w / words;
          or_far(address_in(bits + (w - block * words), block), 1u << (p[k] & 31));
        }
      }
  });
  cluster_sync();
  if (!LOCAL) return;
  const int rank = (int)cluster_rank();
  for (int w = threadIdx.x; w < words; w += kSetThreads) {
    uint32_t x = 0;
#pragma unroll
    for (int k = 0; k < kSetBlocks; ++k) x |= (uint32_t)load_far(address_in(all + rank * words + w, k));
    bits[w] = x;
  }
  __syncthreads();
}

// Bits before each word of the block, in its order; returns their number.
template <typename F>
__device__ __forceinline__ int count_words(int words, int* prefix, SetShared& sh, F bits_of) {
  int sum = 0;
  for (int w0 = 0; w0 < words; w0 += kSetThreads) {
    const int w = w0 + threadIdx.x;
    int total;
    const int before = block_before(w < words ? __popc(bits_of(w)) : 0, total, sh.warp);
    if (w < words) prefix[w] = sum + before;
    sum += total;
  }
  return sum;
}

// Bits of word w (of all pages) that are pages.
__device__ __forceinline__ uint32_t pages_of_word(int w, int npages) {
  const int left = npages - w * 32;
  return left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1 : 0;
}

template <bool LOCAL>
__global__ void __cluster_dims__(kSetBlocks, 1, 1) __launch_bounds__(kSetThreads)
k_page_free(TablesView t, int32_t* lens, const int32_t* __restrict__ drop, int ndrop, int npages, int words,
            int32_t* free_pages, int32_t* count) {
  extern __shared__ uint32_t bits[];
  __shared__ SetShared sh;
  int* prefix = reinterpret_cast<int*>(bits + words);
  const int rank = (int)cluster_rank(), tid = threadIdx.x;
  for (int64_t i = rank * kSetThreads + tid; i < ndrop; i += kSetBlocks * kSetThreads) {
    const int r = __ldg(drop + i);
    if ((unsigned)r < (unsigned)t.nreq) lens[r] = 0;
  }
  mark_held<LOCAL>(t, bits, bits + 2 * words, words, npages);  // its first barrier makes the lengths seen
  auto unused = [&](int w) { return ~bits[w] & pages_of_word(rank * words + w, npages); };
  const int mine = count_words(words, prefix, sh, unused);
  if (tid == 0) sh.count = mine;
  int total;
  const int before = cluster_before(&sh.count, total);
  for (int i = tid; i < words * 32; i += kSetThreads) {
    const int w = i >> 5, p = (rank * words + w) * 32 + (i & 31);
    const uint32_t b = unused(w);
    if ((b >> (i & 31)) & 1) free_pages[before + prefix[w] + __popc(b & ((1u << (i & 31)) - 1))] = p;
  }
  for (int i = total + rank * kSetThreads + tid; i < npages; i += kSetBlocks * kSetThreads) free_pages[i] = -1;
  if (rank == 0 && tid == 0) count[0] = total;
  cluster_sync();  // a block's shared memory stays until the others have read it
}

template <bool LOCAL>
__global__ void __cluster_dims__(kSetBlocks, 1, 1) __launch_bounds__(kSetThreads)
k_page_compact(TablesView t, int npages, int words, int32_t* out_table, int32_t* src, int32_t* dst, int32_t* ids,
               int32_t* used) {
  extern __shared__ uint32_t bits[];
  __shared__ SetShared sh;
  int* prefix = reinterpret_cast<int*>(bits + words);
  const int rank = (int)cluster_rank(), tid = threadIdx.x, lane = tid & 31;
  mark_held<LOCAL>(t, bits, bits + 2 * words, words, npages);
  const int mine = count_words(words, prefix, sh, [&](int w) { return bits[w]; });
  if (tid == 0) sh.count = mine;
  int total;
  const int before = cluster_before(&sh.count, total);
  // pages in use before page `total`: as many stay where they are
  const int w_cut = total >> 5;
  if (tid == 0) {
    sh.count2 = 0;
    if (w_cut / words == rank && w_cut < kSetBlocks * words) {
      const int w = w_cut - rank * words;
      sh.count2 = before + prefix[w] + __popc(bits[w] & ((1u << (total & 31)) - 1));
    }
  }
  int stay;
  cluster_before(&sh.count2, stay);
  if (total >= npages) stay = total;  // nothing lies behind
  const int moves = total - stay, bound = npages / 2;
  for (int i = tid; i < words * 32; i += kSetThreads) {
    const int w = i >> 5, p = (rank * words + w) * 32 + (i & 31);
    if (p >= npages) continue;
    const uint32_t b = bits[w];
    const bool on = (b >> (i & 31)) & 1;
    const int in_use = before + prefix[w] + __popc(b & ((1u << (i & 31)) - 1));  // before p
    if (p < total) {
      if (!on) dst[p - in_use] = p;
      ids[p] = on ? p : -1;
    } else {
      if (on) src[in_use - stay] = p;
      else ids[p] = -1;
    }
  }
  for (int i = moves + rank * kSetThreads + tid; i < bound; i += kSetBlocks * kSetThreads) src[i] = dst[i] = -1;
  cluster_sync();
  for (int i = rank * kSetThreads + tid; i < moves; i += kSetBlocks * kSetThreads) ids[__ldcg(src + i)] = __ldcg(dst + i);
  if (rank == 0 && tid == 0) used[0] = total;
  cluster_sync();
  each_run(t.nreq, t.width, [&](int r, int at) {
    const int n = held_pages(__ldcg(t.lens + r), t);
    const int32_t* row = t.table + r * t.stride;
    int p[kRun / 32];
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k) {
      const int j = at + k * 32 + lane;
      p[k] = j < n ? __ldg(row + j) : -1;
    }
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k) {
      const int j = at + k * 32 + lane;
      if (j < t.width) out_table[(int64_t)r * t.width + j] = (unsigned)p[k] < (unsigned)npages ? __ldcg(ids + p[k]) : -1;
    }
  });
}

// ---------------------------------------------------------------------------
// Requests that go on from others.  Child i takes the pages of parent[i]; of a
// parent's children the first takes its last page too where that is not full, the
// others get copies of it.  The block of a child finds out whether an earlier one
// has the same parent by looking (a warp a child, 128 at a time), which needs no
// memory of the parents' number, and takes time with the children's number squared
// where few of them share a parent (us of the GPU, of as many parents: 512 children
// 11, 4096 81, 16384 840, 65536 42600; of one parent 9, 17, 45, 157).
constexpr int kForkChildren = kMaxForks / kSetBlocks;

__global__ void __cluster_dims__(kSetBlocks, 1, 1) __launch_bounds__(kSetThreads)
k_page_fork(TablesView t, const int32_t* __restrict__ parent, int n, const int32_t* __restrict__ free_pages, int nfree,
            int32_t* out_table, int32_t* out_lens, int32_t* src, int32_t* dst, int32_t* used) {
  __shared__ SetShared sh;
  __shared__ int s_dst[kForkChildren];  // 1 where the last page is copied, then the page that it goes to; -2: it is not
  const int rank = (int)cluster_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (n + kSetBlocks - 1) / kSetBlocks, c0 = min(rank * per, n), c1 = min(c0 + per, n);
  const int64_t slots = (int64_t)t.width * t.page.d;
  const int most = slots < INT32_MAX ? (int)slots : INT32_MAX;  // keys of a request
  auto length = [&](int p) { return (unsigned)p < (unsigned)t.nreq ? min(max(__ldg(t.lens + p), 0), most) : 0; };
  for (int i = c0 + warp; i < c1; i += kSetThreads / 32) {
    const int p = __ldg(parent + i), len = length(p), full = t.page.div(len);
    // a last page that is not full; an entry that is no page (free pages had run out) stays what it is
    const bool part = len - full * t.page.d != 0 && full < t.width && __ldg(t.table + p * t.stride + full) >= 0;
    bool found = false;
    for (int j = 0; part && !found && j < i; j += 128) {
      bool same = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) same = same || (j + 32 * k + lane < i && __ldg(parent + j + 32 * k + lane) == p);
      found = __any_sync(0xffffffffu, same);
    }
    if (lane == 0) {
      s_dst[i - c0] = found;
      out_lens[i] = len;
    }
  }
  __syncthreads();
  // each thread's children are neighbours
  const int each = (per + kSetThreads - 1) / kSetThreads, m0 = min(tid * each, c1 - c0), m1 = min(m0 + each, c1 - c0);
  int mine = 0, total;
  for (int m = m0; m < m1; ++m) mine += s_dst[m];
  int at = block_before(mine, total, sh.warp);
  if (tid == 0) sh.count = total;
  at += cluster_before(&sh.count, total);
  for (int m = m0; m < m1; ++m) {
    int to = -1, from = -1;
    if (s_dst[m]) {
      const int p = __ldg(parent + c0 + m);
      from = __ldg(t.table + p * t.stride + t.page.div(length(p)));
      to = at < nfree ? __ldg(free_pages + at) : -1;
      ++at;
    }
    src[c0 + m] = to >= 0 ? from : -1;
    dst[c0 + m] = to;
    s_dst[m] = s_dst[m] ? to : -2;
  }
  if (rank == 0 && tid == 0) used[0] = total;
  __syncthreads();
  const int runs = t.width > 0 ? (t.width - 1) / kRun + 1 : 0;
  const int64_t all = (int64_t)(c1 - c0) * runs;
  for (int64_t w = warp; w < all; w += kSetThreads / 32) {
    const int m = (int)(w / runs), first = (int)(w - (int64_t)m * runs) * kRun, i = c0 + m;
    const int p = __ldg(parent + i), len = length(p), held = held_pages(len, t);
    const int copy = s_dst[m], last = copy == -2 ? -1 : held - 1;
    const int32_t* row = t.table + (held > 0 ? p * t.stride : 0);
    int x[kRun / 32];
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k) {
      const int j = first + k * 32 + lane;
      x[k] = j < held ? __ldg(row + j) : -1;
      if (j == last) x[k] = copy;
    }
#pragma unroll
    for (int k = 0; k < kRun / 32; ++k) {
      const int j = first + k * 32 + lane;
      if (j < t.width) out_table[(int64_t)i * t.width + j] = x[k];
    }
  }
  cluster_sync();  // a block's shared memory stays until the others have read it
}

// ---------------------------------------------------------------------------
// Validate mode: lengths that fit their rows, entries of the tables that are pages,
// and lists whose entries are below a bound.
__global__ void k_validate_set(TablesView t, int npages, const int32_t* list, int n, int bound, const int32_t* more,
                               int more_bound, WsHeader* hdr) {
  const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  int bad = 0;
  for (int64_t r = id; r < t.nreq; r += step) {
    const int len = t.lens[r];
    if (len < 0 || len > (int64_t)t.width * t.page.d) bad |= kErrPos;
    else
      for (int i = 0; i < held_pages(len, t); ++i)
        if ((unsigned)t.table[r * t.stride + i] >= (unsigned)npages) bad |= kErrCrdRange;
  }
  for (int64_t i = id; i < n; i += step) {
    if (list && list[i] >= bound) bad |= kErrCrdRange;
    if (more && more[i] >= more_bound) bad |= kErrCrdRange;
  }
  if (bad) atomicOr(&hdr->error, bad);
}

template <typename K>
cudaError_t prepare(K kernel, size_t smem) {
  cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (r == cudaSuccess && smem) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  return r;
}

constexpr int kLocalWords = 2048;  // of a block, 2^20 pages in all
// Shared memory of a block: its words, the bits before each; a set of all pages.
size_t set_bytes(int words, bool local) { return (size_t)4 * words * (local ? 2 + kSetBlocks : 2); }

int words_of(int npages) { return npages > 0 ? pieces(pieces(npages, 32), kSetBlocks) : 1; }

}  // namespace

cudaError_t launch_page_copy(const CopyParts& c, const int32_t* src, const int32_t* dst, int n, int from_pages,
                             int to_pages, cudaStream_t s) {
  const int64_t blocks = ((int64_t)n * c.items + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  const unsigned grid = (unsigned)(blocks < 152 * 8 ? blocks : 152 * 8);
  k_page_copy<<<SLNR_COUNTED(grid), kCopyThreads, 0, s>>>(c, src, dst, n, from_pages, to_pages);
  return cudaGetLastError();
}

cudaError_t launch_page_fork(const TablesView& t, const int32_t* parent, int n, const int32_t* free_pages, int nfree,
                             int32_t* out_table, int32_t* out_lens, int32_t* src, int32_t* dst, int32_t* used,
                             cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = once([&] { return prepare(k_page_fork, 0); });
  if (e != cudaSuccess) return e;
  k_page_fork<<<SLNR_COUNTED(kSetBlocks), kSetThreads, 0, s>>>(t, parent, n, free_pages, nfree, out_table, out_lens, src, dst,
                                                              used);
  return cudaGetLastError();
}

cudaError_t launch_page_free(const TablesView& t, int32_t* lens, const int32_t* drop, int ndrop, int npages,
                             int32_t* free_pages, int32_t* count, cudaStream_t s) {
  static OncePerDevice once[2];
  const int words = words_of(npages);
  const bool local = words <= kLocalWords;
  auto kernel = local ? k_page_free<true> : k_page_free<false>;
  const cudaError_t e = once[local]([&] { return prepare(kernel, local ? set_bytes(kLocalWords, true) : set_bytes(kSetWords, false)); });
  if (e != cudaSuccess) return e;
  kernel<<<SLNR_COUNTED(kSetBlocks), kSetThreads, set_bytes(words, local), s>>>(t, lens, drop, ndrop, npages, words, free_pages,
                                                                              count);
  return cudaGetLastError();
}

cudaError_t launch_page_compact(const TablesView& t, int npages, int32_t* out_table, int32_t* src, int32_t* dst,
                                int32_t* ids, int32_t* used, cudaStream_t s) {
  static OncePerDevice once[2];
  const int words = words_of(npages);
  const bool local = words <= kLocalWords;
  auto kernel = local ? k_page_compact<true> : k_page_compact<false>;
  const cudaError_t e = once[local]([&] { return prepare(kernel, local ? set_bytes(kLocalWords, true) : set_bytes(kSetWords, false)); });
  if (e != cudaSuccess) return e;
  kernel<<<SLNR_COUNTED(kSetBlocks), kSetThreads, set_bytes(words, local), s>>>(t, npages, words, out_table, src, dst, ids,
                                                                              used);
  return cudaGetLastError();
}

cudaError_t launch_validate_set(const TablesView& t, int npages, const int32_t* list, int n, int bound, const int32_t* more,
                                int more_bound, WsHeader* hdr, cudaStream_t s) {
  k_validate_set<<<SLNR_COUNTED(304), 256, 0, s>>>(t, npages, list, n, bound, more, more_bound, hdr);
  return cudaGetLastError();
}

}  // namespace slnr
