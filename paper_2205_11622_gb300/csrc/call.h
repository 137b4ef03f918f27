// What the C entry points share: the last error, the per-launch timing of a
// call (both defined in api.cu), and argument checks.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "slnr.h"

namespace slnr {

// Sets the calling thread's slnr_last_error() text and returns st.
slnr_status fail(slnr_status st, const char* fmt, ...);

void timing_begin();
void timing_mark(const char* name, cudaStream_t s);
void timing_end(cudaStream_t s);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

inline slnr_status check_ws(const slnr_opts* o, size_t need) {
  if (!o->workspace) return fail(SLNR_ERR_WORKSPACE, "workspace is NULL (needs %zu bytes)", need);
  if ((reinterpret_cast<uintptr_t>(o->workspace) & 255u) != 0)
    return fail(SLNR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (o->workspace_bytes < need)
    return fail(SLNR_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", o->workspace_bytes, need);
  return SLNR_OK;
}

}  // namespace slnr

// A failure is reported by the call that met it: the runtime's copy, which the next
// launch would return again, is taken out.
#define SLNR_CUDA(expr)                                                                   \
  do {                                                                                    \
    cudaError_t e_ = (expr);                                                              \
    if (e_ != cudaSuccess) {                                                              \
      (void)cudaGetLastError();                                                           \
      return ::slnr::fail(SLNR_ERR_CUDA, "%s: %s", #expr, cudaGetErrorString(e_));        \
    }                                                                                     \
  } while (0)

// A kernel launch of the call: timing mark, then the launch, then its status.
#define SLNR_LAUNCH(name, expr)     \
  do {                              \
    ::slnr::timing_mark(name, s);   \
    SLNR_CUDA(expr);                \
  } while (0)

#define SLNR_CHECK(expr)            \
  do {                              \
    slnr_status st_ = (expr);       \
    if (st_ != SLNR_OK) return st_; \
  } while (0)
