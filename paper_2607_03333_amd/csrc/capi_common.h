// What the C entry points share: error reporting, the guard that keeps C++
// exceptions inside, argument checks of shapes, and kernel timing.
#pragma once

#include <cmath>
#include <exception>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "spork.h"

namespace spork {
namespace capi {

inline thread_local std::string g_last_error;

inline int fail(int code, const std::string& msg) {
  g_last_error = msg;
  return code;
}

// Per-thread kernel timing: event pairs recorded around each launch.
struct Timing {
  bool on = false;
  std::vector<hipEvent_t> pool;  // created lazily, reused across reads
  size_t used = 0;
  std::vector<std::pair<int, size_t>> marks;  // (kind, index of the begin event)
};
inline thread_local Timing g_timing;

inline hipEvent_t next_event() {
  if (g_timing.used == g_timing.pool.size()) {
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    g_timing.pool.push_back(e);
  }
  return g_timing.pool[g_timing.used++];
}

// Launch `f` on `stream`, bracketed by timing events of `kind` when enabled.
template <typename F>
hipError_t timed(int kind, hipStream_t stream, F&& f) {
  if (!g_timing.on) return f();
  const size_t at = g_timing.used;
  hipEvent_t b = next_event(), e = next_event();
  if (b == nullptr || e == nullptr) return hipErrorOutOfMemory;
  hipError_t rc = hipEventRecord(b, stream);
  if (rc != hipSuccess) return rc;
  rc = f();
  if (rc != hipSuccess) return rc;
  rc = hipEventRecord(e, stream);
  if (rc == hipSuccess) g_timing.marks.push_back({kind, at});
  return rc;
}

inline int elem_bytes(int32_t dtype) { return dtype == SPORK_DTYPE_BF16 ? 2 : (dtype == SPORK_DTYPE_F32 ? 4 : 0); }

inline int check_shape(const spork_shape* sh) {
  if (sh == nullptr) return fail(SPORK_E_INVAL, "shape is NULL");
  if (sh->hq <= 0 || sh->hkv <= 0 || sh->hq % sh->hkv != 0)
    return fail(SPORK_E_INVAL, "hq and hkv must be positive and hq a multiple of hkv");
  if (sh->head_dim <= 0 || sh->block_size <= 0) return fail(SPORK_E_INVAL, "head_dim and block_size must be positive");
  if (elem_bytes(sh->dtype) == 0) return fail(SPORK_E_UNSUPPORTED, "dtype must be SPORK_DTYPE_F32 or SPORK_DTYPE_BF16");
  if (!std::isfinite(sh->sm_scale)) return fail(SPORK_E_INVAL, "sm_scale must be finite");
  return SPORK_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(SPORK_E_INVAL, "host allocation failed");
  } catch (const std::exception& e) {
    return fail(SPORK_E_INVAL, e.what());
  } catch (...) {
    return fail(SPORK_E_INVAL, "unknown error");
  }
}

inline int hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return SPORK_OK;
  return fail(SPORK_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace capi
}  // namespace spork
