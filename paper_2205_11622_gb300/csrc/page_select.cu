// The cheap score: for each new token and key head, the pages that its
// attention will look at.
//
// u = sum of the group's query rows (fp32, in the heads' order), coded as
// c = round(u f), f = 127 (1 / max|u|), each step rounded in fp32;
// score(page) = (sum_d c_d code_d) * scale.  The sum is a whole number below 2^24
// and the product is rounded once, so the score, and with it the selection, does
// not depend on the order of summation.
#include "launch.h"
#include "mma16.cuh"
#include "paged.cuh"

namespace slnr {
namespace {

constexpr int kSelMaxTokens = 16;
constexpr int kSelMaxWidth = 128;
constexpr int kSelSmem = 200 * 1024;

template <typename T>
__device__ __forceinline__ float as_float(T x);
template <>
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }

// Keys of a token's row in shared memory: 8 mod 32, so that the rows that a product's lanes write fall on different
// banks, and whole groups of 8 pages.
__host__ __device__ __forceinline__ int key_pitch(int npages) { return (npages + 23) / 32 * 32 + 8; }

// Whole numbers in the order of the scores.
__device__ __forceinline__ uint32_t key_of(float score) {
  const uint32_t b = __float_as_uint(score + 0.f);  // -0 as 0
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// The `want` highest of n keys (0 < want < n), the lower index first where keys
// are equal: v = the least key taken, and how many of the keys equal to v.  A
// warp halves the range [least, highest] of the keys until as many as wanted lie
// at or above its middle (some ten steps; 32 at most, where keys are equal).
struct Cut {
  uint32_t v;
  int ties;
};
template <typename Count>
__device__ __forceinline__ Cut find_cut(uint32_t lo, uint32_t hi, int want, Count count) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    const int c = count(mid);
    if (c == want) return Cut{mid - 1, 0};  // all keys above mid - 1, none of those equal to it
    if (c > want) lo = mid;
    else hi = mid - 1;
  }
  return Cut{lo, want - (lo == 0xffffffffu ? 0 : count(lo + 1))};
}
// The same where the maxima of parts of the keys leave few of them: of 32 K parts
// (every 32 K-th key each) the want-th highest maximum is at or below the cut, so
// what lies below it is out.  The others, 32 K ln(32 K / (32 K - want)) of keys in
// no order, go to `found` in theirs, and the cut is found among them alone.  Writes
// the indexes of the keys taken, in order, plus `base`, to out; false (nothing
// written) where more than FOUND are left.
constexpr int kFound = 256;
template <int K, int FOUND>
__device__ __forceinline__ bool take_few(const uint32_t* key, int n, int want, int base, uint16_t* found, int32_t* out) {
  const int lane = threadIdx.x & 31;
  const unsigned below = (1u << lane) - 1;
  uint32_t part[K], most = 0, least = 0xffffffffu;
#pragma unroll
  for (int k = 0; k < K; ++k) part[k] = 0;
#pragma unroll 8 / K
  for (int i = lane; i < n; i += 32 * K) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (i + 32 * k < n) part[k] = max(part[k], key[i + 32 * k]);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    most = max(most, part[k]);
    least = min(least, part[k]);
  }
  const uint32_t top = __reduce_max_sync(0xffffffffu, most);
  uint32_t lo = __reduce_min_sync(0xffffffffu, least), hi = top;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) c += __popc(__ballot_sync(0xffffffffu, part[k] >= mid));
    if (c >= want) lo = mid;
    else hi = mid - 1;
    if (c == want) break;
  }
  if (lo == 0) return false;  // a score of NaN can have a key of 0
  int total = 0;
#pragma unroll 8
  for (int i = 0; i < n; i += 32) {
    const bool in = i + lane < n && key[i + lane] >= lo;
    const unsigned m = __ballot_sync(0xffffffffu, in);
    const int at = total + __popc(m & below);
    if (in && at < FOUND) found[at] = (uint16_t)(i + lane);
    total += __popc(m);
  }
  if (total > FOUND) return false;
  __syncwarp();
  uint32_t f[FOUND / 32];
#pragma unroll
  for (int i = 0; i < FOUND / 32; ++i) f[i] = 32 * i + lane < total ? key[found[32 * i + lane]] : 0;
  Cut cut{lo - 1, 0};  // all of them
  if (total > want)
    cut = find_cut(lo, top, want, [&](uint32_t mid) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < FOUND / 32; ++i)
        if (32 * i < total) c += __popc(__ballot_sync(0xffffffffu, f[i] >= mid));  // mid > 0
      return c;
    });
  int at = 0;
#pragma unroll
  for (int i = 0; i < FOUND / 32; ++i) {
    if (32 * i >= total) break;
    const bool on = 32 * i + lane < total, tie = on && f[i] == cut.v;
    const unsigned tied = __ballot_sync(0xffffffffu, tie);
    const bool take = on && (f[i] > cut.v || (tie && __popc(tied & below) < cut.ties));
    cut.ties = max(cut.ties - __popc(tied), 0);
    const unsigned m = __ballot_sync(0xffffffffu, take);
    if (take) out[at + __popc(m & below)] = base + found[32 * i + lane];
    at += __popc(m);
  }
  __syncwarp();
  return true;
}
__device__ __forceinline__ Cut cut_in_memory(const uint32_t* key, int n, int want) {
  const int lane = threadIdx.x & 31;
  return find_cut(0, 0xffffffffu, want, [&](uint32_t mid) {
    int c = 0;
    for (int i = lane; i < n; i += 32) c += key[i] >= mid;
    return (int)__reduce_add_sync(0xffffffffu, c);
  });
}

// Four codes as two pairs of fp16: 1024 + (code + 128) is the fp16 whose low byte
// is code + 128.  Exact, as whole numbers up to 2048 are.
__device__ __forceinline__ uint2 halves_of(uint32_t codes) {
  const uint32_t x = codes ^ 0x80808080u;
  const __half2 bias = __float2half2_rn(1152.f);
  uint2 r;
  r.x = __byte_perm(x, 0x64646464u, 0x4140);
  r.y = __byte_perm(x, 0x64646464u, 0x4342);
  *reinterpret_cast<__half2*>(&r.x) = __hsub2(*reinterpret_cast<__half2*>(&r.x), bias);
  *reinterpret_cast<__half2*>(&r.y) = __hsub2(*reinterpret_cast<__half2*>(&r.y), bias);
  return r;
}

// Keys of up to 16 tokens' scores, for runs of tokens of one request.  Lane: columns
// [quarter, quarter + 4 STEPS) of tokens lane / 4 and + 8, or of page lane / 4.
template <int THREADS>
__device__ __forceinline__ void score_many(const PagesView& p, const CacheView& c, int h, int n, const int* s_req,
                                           const int* s_own, const int* s_code, uint32_t* s_key, int pitch) {
  constexpr int WARPS = THREADS / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int STEPS = kSelMaxWidth / 16;
  const int steps = (c.width + 15) / 16, quarter = (lane & 3) * 4 * steps, row = lane >> 2;
  uint32_t fa[STEPS][4];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int w = (lane & 3) * steps + i;
    const bool on = i < steps && 4 * w < c.width;
    const uint2 x0 = halves_of(on && row < n ? s_code[row * (kSelMaxWidth / 4) + w] : 0);
    const uint2 x1 = halves_of(on && row + 8 < n ? s_code[(row + 8) * (kSelMaxWidth / 4) + w] : 0);
    fa[i][0] = x0.x;
    fa[i][1] = x1.x;
    fa[i][2] = x0.y;
    fa[i][3] = x1.y;
  }
  for (int i0 = 0; i0 < n;) {
    const int r = s_req[i0];
    int i1 = i0 + 1, most = s_own[i0];
    while (i1 < n && s_req[i1] == r) most = max(most, s_own[i1++]);
    for (int base = 8 * warp; base <= most; base += 8 * WARPS) {
      const int pg = base + row;
      const int id = pg <= most ? __ldg(p.table + r * p.table_stride + pg) : -1;
      const bool ok = (unsigned)id < (unsigned)c.npages;
      const int64_t at = ok ? (int64_t)id * c.nheads + h : 0;
      const int8_t* code = c.codes + at * c.width + quarter;
      uint32_t x[STEPS];
      if (c.width == kSelMaxWidth) {  // two 16-byte loads a lane
        const uint4 y0 = ok ? __ldg(reinterpret_cast<const uint4*>(code)) : make_uint4(0, 0, 0, 0);
        const uint4 y1 = ok ? __ldg(reinterpret_cast<const uint4*>(code) + 1) : make_uint4(0, 0, 0, 0);
        x[0] = y0.x; x[1] = y0.y; x[2] = y0.z; x[3] = y0.w;
        x[4] = y1.x; x[5] = y1.y; x[6] = y1.z; x[7] = y1.w;
      } else {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
          x[i] = ok && i < steps && quarter + 4 * i < c.width ? __ldg(reinterpret_cast<const uint32_t*>(code) + i) : 0u;
      }
      const float scale = ok ? __ldg(c.scales + at) : 0.f;
      float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
        if (i < steps) {
          const uint2 b = halves_of(x[i]);
          Half2<__half>::mma(dot, fa[i], b.x, b.y);
        }
      // dot[e]: token lane / 4 + 8 (e / 2), page 2 (lane % 4) + e % 2, whose scale lane 4 (page) holds
      const int col = 2 * (lane & 3);
      const float f0 = __shfl_sync(0xffffffffu, scale, 4 * col), f1 = __shfl_sync(0xffffffffu, scale, 4 * col + 4);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const int i = row + 4 * e;
        if (i >= i0 && i < i1)
          *reinterpret_cast<uint2*>(s_key + i * pitch + base + col) =
              make_uint2(key_of(__fmul_rn(dot[e], f0)), key_of(__fmul_rn(dot[e + 1], f1)));
      }
    }
    i0 = i1;
  }
}

// Keys of one token's scores.  8 lanes a page, 16 columns a lane, in four-way integer
// products: with one token a sixteenth of a matrix product's work is wanted.  A warp
// has 16 pages on their way, their numbers are read one turn earlier: 32 tokens of
// long requests 15.9 -> 12.8 us in the kernel, 64 requests of 2048 pages (8 heads of
// 128, 134 MB) 70 -> 36 a call, 3.7 TB/s with its selection.
template <int THREADS>
__device__ __forceinline__ void score_one(const PagesView& p, const CacheView& c, int h, int r, int most,
                                          const int* s_code, uint32_t* s_key) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane & 7, words = c.width / 4;
  if (r < 0) return;
  const int* table = p.table + r * p.table_stride;
  const bool wide = c.width % 16 == 0;  // else rows start on 8 bytes
  int u[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = 4 * part + e < words ? s_code[4 * part + e] : 0;
  int id[4];
  uint4 x[4];
  float scale;
  // page base + 4 i + lane / 8
  const auto find = [&](int base) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pg = base + 4 * i + (lane >> 3);
      id[i] = pg <= most ? __ldg(table + pg) : -1;
    }
  };
  const auto load = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool ok = (unsigned)id[i] < (unsigned)c.npages;
      const int8_t* code = c.codes + (ok ? (int64_t)id[i] * c.nheads + h : 0) * c.width + 16 * part;
      x[i] = make_uint4(0, 0, 0, 0);
      if (wide) {
        if (ok && 4 * part < words) x[i] = __ldg(reinterpret_cast<const uint4*>(code));
      } else {
        if (ok && 4 * part < words) {
          const uint2 y = __ldg(reinterpret_cast<const uint2*>(code));
          x[i].x = y.x, x[i].y = y.y;
        }
        if (ok && 4 * part + 2 < words) {
          const uint2 y = __ldg(reinterpret_cast<const uint2*>(code) + 1);
          x[i].z = y.x, x[i].w = y.y;
        }
      }
    }
    const int mine = lane & 2 ? (lane & 1 ? id[3] : id[2]) : (lane & 1 ? id[1] : id[0]);
    scale = (unsigned)mine < (unsigned)c.npages ? __ldg(c.scales + (int64_t)mine * c.nheads + h) : 0.f;
  };
  constexpr int TURN = THREADS / 32 * 16;
  find(16 * warp);
  load();
  find(16 * warp + TURN);
  for (int base = 16 * warp; base <= most; base += TURN) {
    int dot[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      dot[i] = __dp4a((int)x[i].w, u[3],
                      __dp4a((int)x[i].z, u[2], __dp4a((int)x[i].y, u[1], __dp4a((int)x[i].x, u[0], 0))));
    const float f = scale;
    load();
    find(base + 2 * TURN);
    // sums over the 8 lanes: lane i of them ends with that of page i % 4
    const bool odd = lane & 1, high = lane & 2;
    const int a = (odd ? dot[1] : dot[0]) + __shfl_xor_sync(0xffffffffu, odd ? dot[0] : dot[1], 1);
    const int b = (odd ? dot[3] : dot[2]) + __shfl_xor_sync(0xffffffffu, odd ? dot[2] : dot[3], 1);
    int sum = (high ? b : a) + __shfl_xor_sync(0xffffffffu, high ? a : b, 2);
    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
    const int pg = base + 4 * (lane & 3) + (lane >> 3);
    if ((lane & 4) == 0 && pg <= most) s_key[pg] = key_of(__fmul_rn((float)sum, f));
  }
}

// A block takes `ntile` consecutive tokens and one head.  Scores of several tokens:
// fp16 matrix products of 16 tokens and 8 pages, exact as all their sums are whole numbers
// below 2^24; a warp a group of 8 pages, codes straight from memory into the
// product's registers (the columns of a row in an order of their own, the same
// for both operands).  Selection: a warp a token, then the pages written in order.
// Bound by instructions (60% of the issue slots): 2048 tokens over up to 512
// pages, 8 heads of 128, 43 us.  Four-way integer products of a page a thread
// took 88 where these took 58; all keys of a token halved in shared memory 152
// where a cut in registers took 88, and few candidates 44 where that took 53.  One
// token a block (ONE): score_one.
template <typename T, int THREADS, bool ONE>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
k_page_select(PagesView p, CacheView c, RowsView q, int group, int ntile, int npages, int32_t* picked, int npicked,
              int first, int last) {
  extern __shared__ __align__(16) unsigned char smem[];
  int* s_code = reinterpret_cast<int*>(smem);                             // [ntile][width / 4]
  uint32_t* s_key = reinterpret_cast<uint32_t*>(smem) + ntile * (kSelMaxWidth / 4);  // [ntile][pitch]
  __shared__ int s_req[kSelMaxTokens], s_own[kSelMaxTokens];
  constexpr int WARPS = THREADS / 32;
  __shared__ uint16_t s_found[ONE ? 1 : WARPS][kFound];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.y, t0 = blockIdx.x * ntile, n = min(ntile, p.ntok - t0);
  const int words = c.width / 4, pitch = key_pitch(npages);

  // codes of the tokens' queries: a warp a token, 4 columns a lane
  for (int i = warp; i < n; i += WARPS) {
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
        alignas(8) T x[4];
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

  if constexpr (ONE)
    score_one<THREADS>(p, c, h, s_req[0], s_own[0], s_code, s_key);
  else
    score_many<THREADS>(p, c, h, n, s_req, s_own, s_code, s_key, pitch);
  __syncthreads();

  for (int i = warp; i < n; i += WARPS) {
    const uint32_t* key = s_key + i * pitch;
    int32_t* out = picked + ((int64_t)(t0 + i) * c.nheads + h) * npicked;
    const int own = s_own[i];
    // always taken: pages [0, lead) and [tail, own]; between them by score
    const int lead = min(first, own + 1), tail = max(own + 1 - last, lead);
    const int want = min(npicked - lead - (own + 1 - tail), tail - lead);
    const int among = tail - lead;
    Cut cut{0, 0};
    if (want > 0 && want < among) {
      const uint32_t* k = key + lead;
      uint16_t* found = s_found[warp];
      // 16 of 32 parts leave some 22 keys, 96 of 128 some 180.  64 of 1024 pages for 2048
      // tokens: 132 us from memory, 95 so
      const bool done = want <= 16   ? take_few<1, 128>(k, among, want, lead, found, out + lead)
                        : want <= 96 ? take_few<4, kFound>(k, among, want, lead, found, out + lead)
                                     : false;
      if (done) {
        for (int w = lane; w < npicked; w += 32) {
          if (w < lead) out[w] = w;
          if (w >= lead + want) out[w] = w - lead - want <= own - tail ? tail + w - lead - want : -1;
        }
        continue;
      }
      cut = cut_in_memory(k, among, want);
    }
    const uint32_t v = cut.v;
    int ties = cut.ties;
    const bool all = want > 0 && want == tail - lead, none = want <= 0;
    int at = 0;
    for (int base = 0; base <= own; base += 32) {
      const int pg = base + lane;
      const bool scored = pg >= lead && pg < tail;
      const uint32_t x = scored ? key[pg] : 0;
      bool take = pg <= own && (scored ? !none && (all || x > v) : true);
      if (ties > 0) {
        const bool tie = scored && !none && !all && x == v;
        const unsigned tied = __ballot_sync(0xffffffffu, tie);
        if (tie && __popc(tied & ((1u << lane) - 1)) < ties) take = true;
        ties = max(ties - __popc(tied), 0);
      }
      const unsigned m = __ballot_sync(0xffffffffu, take);
      const int where = at + __popc(m & ((1u << lane) - 1));
      if (take && where < npicked) out[where] = pg;
      at += __popc(m);
    }
    for (int w = at + lane; w < npicked; w += 32) out[w] = -1;
  }
}

template <typename T, int THREADS, bool ONE>
cudaError_t launch_select(const PagesView& p, const CacheView& c, const RowsView& q, int group, int ntile, int npages,
                          int32_t* picked, int npicked, int first, int last, cudaStream_t s) {
  auto kernel = k_page_select<T, THREADS, ONE>;
  static OncePerDevice once;
  cudaError_t e =
      once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelSmem); });
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)pieces(p.ntok, ntile), (unsigned)c.nheads);
  const size_t smem = (size_t)ntile * (kSelMaxWidth + 4 * (size_t)key_pitch(npages));
  kernel<<<(SLNR_COUNTED(grid)), THREADS, smem, s>>>(p, c, q, group, ntile, npages, picked, npicked, first, last);
  return cudaGetLastError();
}

template <typename T, typename... A>
cudaError_t launch_select_as(int threads, bool one, const A&... args) {
  if (one) return threads == 1024 ? launch_select<T, 1024, true>(args...) : launch_select<T, 256, true>(args...);
  return threads == 512 ? launch_select<T, 512, false>(args...) : launch_select<T, 256, false>(args...);
}

}  // namespace

int select_tokens(int pages) {
  for (int n = kSelMaxTokens; n > 0; n /= 2)
    if ((int64_t)n * (kSelMaxWidth + 4 * (int64_t)key_pitch(pages)) <= kSelSmem) return n;
  return 0;
}

cudaError_t launch_page_select(const PagesView& p, const CacheView& c, const RowsView& q, int dtype, int nheads_q,
                               int32_t* picked, int npicked, int first, int last, cudaStream_t s) {
  if (p.ntok == 0) return cudaSuccess;
  const int npages = p.max_k > 0 ? (p.max_k - 1) / c.page.d + 1 : 1;
  // one token a block where requests have one: more blocks, and no two tokens share a page's codes
  const bool one = p.max_q <= 1;
  const int ntile = one ? 1 : select_tokens(npages);
  // Larger blocks where there would be few warps on an SM (us, key heads of 128, with
  // 256 threads and with more): few single tokens of many pages, 16 requests of 2048,
  // 8 heads, 21 and 18, one of 8192 53 and 36, but 64 of 2048 37 and 62 and one of 256
  // as long either way; chunks whose scores fill the shared memory, 2048 tokens over
  // 2048 pages 263 and 161, but over 512 44 and 50.
  int threads = 256;
  if (one && (int64_t)p.ntok * c.nheads <= 152 && npages > 512) threads = 1024;
  if (!one && ntile * (int64_t)key_pitch(npages) * 4 > 56 * 1024) threads = 512;
  const auto launch = dtype == SLNR_FP16 ? launch_select_as<__half, PagesView, CacheView, RowsView, int, int, int, int32_t*,
                                                            int, int, int, cudaStream_t>
                                         : launch_select_as<__nv_bfloat16, PagesView, CacheView, RowsView, int, int, int,
                                                            int32_t*, int, int, int, cudaStream_t>;
  return launch(threads, one, p, c, q, nheads_q / c.nheads, ntile, npages, picked, npicked, first, last, s);
}

}  // namespace slnr
