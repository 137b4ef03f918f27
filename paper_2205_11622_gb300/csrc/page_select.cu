// The cheap score: for each new token and key head, the pages that its
// attention will look at.
//
// u = sum of the group's query rows (fp32, in the heads' order), coded as
// c = round(u f), f = 127 (1 / max|u|), each step rounded in fp32; score(page) = (sum_d c_d code_d) * scale.  The sum
// is a whole number below 2^24 and the product is rounded once, so the score,
// and with it the selection, does not depend on the order of summation.
#include "launch.h"
#include "paged.cuh"

namespace slnr {
namespace {

constexpr int kSelThreads = 256;
constexpr int kSelMaxTokens = 16;
constexpr int kSelMaxWidth = 128;
constexpr int kSelSmem = 200 * 1024;

template <typename T>
__device__ __forceinline__ float as_float(T x);
template <>
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }

// Whole numbers in the order of the scores; every score's is above 0 (0: not a candidate).
__device__ __forceinline__ uint32_t key_of(float score) {
  const uint32_t b = __float_as_uint(score + 0.f);  // -0 as 0
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// A block takes `ntile` consecutive tokens and one head.  Scores: a thread
// holds the codes of one page in registers and multiplies them by each token's
// codes out of shared memory, four products an instruction.  Selection: a warp
// a token finds the key of the last page to take by halving the keys' range
// (32 counts over the token's keys in shared memory), then writes the pages in
// order.
template <typename T>
__global__ void __launch_bounds__(kSelThreads)
k_page_select(PagesView p, CacheView c, RowsView q, int group, int ntile, int npages, int32_t* picked, int npicked,
              int first, int last) {
  extern __shared__ __align__(16) unsigned char smem[];
  int* s_code = reinterpret_cast<int*>(smem);                             // [ntile][width / 4]
  uint32_t* s_key = reinterpret_cast<uint32_t*>(smem) + ntile * (kSelMaxWidth / 4);  // [ntile][npages]
  __shared__ int s_req[kSelMaxTokens], s_own[kSelMaxTokens];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.y, t0 = blockIdx.x * ntile, n = min(ntile, p.ntok - t0);
  const int words = c.width / 4;

  // codes of the tokens' queries: a warp a token, 4 columns a lane
  for (int i = warp; i < n; i += kSelThreads / 32) {
    const int t = t0 + i;
    const int r = __ldg(p.req + t);
    if (lane == 0) {
      int own = -1;
      if (r >= 0) {
        const int pos = p.k_len[r] - (p.q_pos[r + 1] - t);
        own = pos < 0 ? -1 : min(c.page.div(pos), npages - 1);
      }
      s_req[i] = r;
      s_own[i] = own;
    }
    float u[4] = {0.f, 0.f, 0.f, 0.f};
    if (lane < words) {
      const T* row = (const T*)q.p + (int64_t)t * q.tok + (int64_t)h * group * q.head + 4 * lane;
      for (int g = 0; g < group; ++g, row += q.head) {
        T x[4];
        *reinterpret_cast<uint2*>(x) = __ldg(reinterpret_cast<const uint2*>(row));
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __fadd_rn(u[e], as_float(x[e]));
      }
    }
    float most = fmaxf(fmaxf(fabsf(u[0]), fabsf(u[1])), fmaxf(fabsf(u[2]), fabsf(u[3])));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const float f = most > 0.f ? __fmul_rn(127.f, __fdiv_rn(1.f, most)) : 0.f;
    int code = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int x = min(max(__float2int_rn(__fmul_rn(u[e], f)), -127), 127);
      code |= (x & 0xff) << (8 * e);
    }
    if (lane < words) s_code[i * (kSelMaxWidth / 4) + lane] = code;
  }
  __syncthreads();

  // scores of runs of tokens of one request
  for (int i0 = 0; i0 < n;) {
    const int r = s_req[i0];
    int i1 = i0 + 1, most = s_own[i0];
    while (i1 < n && s_req[i1] == r) most = max(most, s_own[i1++]);
    for (int pg = tid; pg <= most; pg += kSelThreads) {
      const int id = __ldg(p.table + r * p.table_stride + pg);
      const bool ok = (unsigned)id < (unsigned)c.npages;
      const int64_t at = ok ? (int64_t)id * c.nheads + h : 0;
      const int2* code = reinterpret_cast<const int2*>(c.codes + at * c.width);
      int2 x[kSelMaxWidth / 8];
#pragma unroll
      for (int w = 0; w < kSelMaxWidth / 8; ++w) x[w] = 2 * w < words && ok ? __ldg(code + w) : make_int2(0, 0);
      const float scale = ok ? __ldg(c.scales + at) : 0.f;
      for (int i = i0; i < i1; ++i) {
        const int2* y = reinterpret_cast<const int2*>(s_code + i * (kSelMaxWidth / 4));
        int dot = 0;
#pragma unroll
        for (int w = 0; w < kSelMaxWidth / 8; ++w)
          if (2 * w < words) {
            const int2 b = y[w];
            dot = __dp4a(x[w].x, b.x, dot);
            dot = __dp4a(x[w].y, b.y, dot);
          }
        s_key[i * npages + pg] = key_of(__fmul_rn((float)dot, scale));
      }
    }
    i0 = i1;
  }
  __syncthreads();

  for (int i = warp; i < n; i += kSelThreads / 32) {
    uint32_t* key = s_key + i * npages;
    int32_t* out = picked + ((int64_t)(t0 + i) * c.nheads + h) * npicked;
    const int own = s_own[i];
    // always taken: pages [0, lead) and [tail, own]; between them by score
    const int lead = min(first, own + 1), tail = max(own + 1 - last, lead);
    int want = min(npicked - lead - (own + 1 - tail), tail - lead);
    uint32_t v = 0;  // the least key taken
    int ties = 0;    // of the pages with that key, how many
    if (want > 0 && want < tail - lead) {
      uint32_t lo = 1, hi = 0xffffffffu;  // count(key >= lo) >= want
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        int cnt = 0;
        for (int pg = lead + lane; pg < tail; pg += 32) cnt += key[pg] >= mid;
        cnt = __reduce_add_sync(0xffffffffu, cnt);
        if (cnt >= want) lo = mid;
        else hi = mid - 1;
      }
      v = lo;
      int above = 0;
      for (int pg = lead + lane; pg < tail; pg += 32) above += key[pg] > v;
      ties = want - __reduce_add_sync(0xffffffffu, above);
    } else if (want > 0) {
      ties = want;
    }
    const bool all = want > 0 && want == tail - lead, none = want <= 0;
    int at = 0;
    for (int base = 0; base <= own; base += 32) {
      const int pg = base + lane;
      bool take = pg <= own && (pg < lead || pg >= tail);
      bool tie = false;
      if (pg >= lead && pg < tail && !none) {
        const uint32_t x = key[pg];
        take = all || x > v;
        tie = !all && x == v;
      }
      const unsigned tied = __ballot_sync(0xffffffffu, tie);
      if (tie && __popc(tied & ((1u << lane) - 1)) < ties) take = true;
      ties = max(ties - __popc(tied), 0);
      const unsigned m = __ballot_sync(0xffffffffu, take);
      const int where = at + __popc(m & ((1u << lane) - 1));
      if (take && where < npicked) out[where] = pg;
      at += __popc(m);
    }
    for (int w = at + lane; w < npicked; w += 32) out[w] = -1;
  }
}

}  // namespace

int select_tokens(int pages) {
  for (int n = kSelMaxTokens; n > 0; n /= 2)
    if ((int64_t)n * (kSelMaxWidth + 4 * (int64_t)pages) <= kSelSmem) return n;
  return 0;
}

cudaError_t launch_page_select(const PagesView& p, const CacheView& c, const RowsView& q, int dtype, int nheads_q,
                               int32_t* picked, int npicked, int first, int last, cudaStream_t s) {
  if (p.ntok == 0) return cudaSuccess;
  const int npages = p.max_k > 0 ? (p.max_k - 1) / c.page.d + 1 : 1;
  // one token a block where requests have one: more blocks, and no two tokens share a page's codes
  const int ntile = p.max_q <= 1 ? 1 : select_tokens(npages);
  const size_t smem = (size_t)ntile * (kSelMaxWidth + 4 * (size_t)npages);
  auto kernel = dtype == SLNR_FP16 ? k_page_select<__half> : k_page_select<__nv_bfloat16>;
  static OncePerDevice once[2];
  cudaError_t e = once[dtype == SLNR_FP16](
      [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelSmem); });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)pieces(p.ntok, ntile), (unsigned)c.nheads);
  kernel<<<(SLNR_COUNTED(grid)), kSelThreads, smem, s>>>(p, c, q, nheads_q / c.nheads, ntile, npages, picked, npicked,
                                                        first, last);
  return cudaGetLastError();
}

}  // namespace slnr
