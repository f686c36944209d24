// Host-side helpers of the entry points that need no layer handle.
#pragma once

#include "eat_internal.cuh"

namespace eat {

inline eat_status bad_arg(const char* fn, const char* what) {
  return thread_fail(EAT_ERR_INVALID_ARG, "%s: %s", fn, what);
}
inline eat_status launched(const char* fn, cudaError_t e) {
  if (e == cudaSuccess) return EAT_OK;
  return thread_fail(EAT_ERR_CUDA, "%s launch: %s", fn, cudaGetErrorString(e));
}
inline bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b + m && b < a + n;
}
inline bool misaligned(const void* p, int n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) != 0; }

}  // namespace eat
