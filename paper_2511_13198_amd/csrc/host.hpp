// Host helpers that the library's translation units share: error text, kernel
// timing, argument checks.
#pragma once
#include "../../include/pdyattn.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <vector>

namespace pdy_host {

inline thread_local char g_err[512] = "";

inline pdy_status fail(pdy_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

inline pdy_status hip_fail(hipError_t e, const char* what) {
  return fail(PDY_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ---------------------------------------------------------------------------
// Optional per-thread kernel timing: while enabled, every launch is bracketed
// by two events on its own stream; pdy_profile_stop reduces them per kernel.
// ---------------------------------------------------------------------------
enum KernelId { K_PLAN = 0, K_FWD, K_DKDV, K_DQ, K_SPLIT_MERGE, K_SPLIT_SUM, K_CROSS_LIST,
                K_CROSS_FWD, K_CROSS_MERGE, K_CROSS_DQ, K_CROSS_DKDV, K_CROSS_SUM, K_ROTARY,
                K_COUNT };
const char* const kKernelNames[K_COUNT] = {"plan_kernel",     "fwd_kernel",
                                           "bwd_dkdv_kernel", "bwd_dq_kernel",
                                           "split_merge_kernel", "split_sum_kernel",
                                           "cross_list_kernel", "cross_fwd_kernel",
                                           "cross_merge_kernel", "cross_dq_kernel",
                                           "cross_dkdv_kernel", "cross_sum_kernel",
                                           "rotary_kernel"};
struct ProfRec {
  int kid;
  hipEvent_t a, b;
};
inline thread_local bool g_prof_on = false;
inline thread_local std::vector<ProfRec> g_prof_recs;
inline thread_local std::vector<hipEvent_t> g_prof_pool;

inline hipError_t prof_event(hipEvent_t* ev) {
  if (!g_prof_pool.empty()) {
    *ev = g_prof_pool.back();
    g_prof_pool.pop_back();
    return hipSuccess;
  }
  return hipEventCreate(ev);
}

// Launch through `fn` (which enqueues exactly one kernel on `st`), timing it
// when profiling is on.  Returns the launch error, if any.
template <typename F>
hipError_t launch_timed(int kid, hipStream_t st, F fn) {
  if (!g_prof_on) {
    fn();
    return hipGetLastError();
  }
  ProfRec r;
  r.kid = kid;
  hipError_t e = prof_event(&r.a);
  if (e == hipSuccess) e = prof_event(&r.b);
  if (e == hipSuccess) e = hipEventRecord(r.a, st);
  if (e != hipSuccess) return e;
  fn();
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = hipEventRecord(r.b, st);
  if (e == hipSuccess) g_prof_recs.push_back(r);
  return e;
}

template <typename K>
hipError_t set_lds(K kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

inline pdy_status check_scale(float scale, int32_t causal) {
  if (causal != 0 && causal != 1) return fail(PDY_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (!std::isfinite(scale) || !(scale > 0.f))
    return fail(PDY_ERR_INVALID_ARG, "scale must be finite and > 0");
  return PDY_OK;
}

inline pdy_status check_ptr(const void* p, const char* name) {
  if (p == nullptr) return fail(PDY_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(PDY_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return PDY_OK;
}

}  // namespace pdy_host
