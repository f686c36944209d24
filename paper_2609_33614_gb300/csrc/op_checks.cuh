// Host-side helpers of the entry points that need no layer handle.
#pragma once

#include "eat_internal.cuh"

#include <initializer_list>

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
// An array of a call: its bytes (a null one has none).
struct Span {
  const void* p;
  size_t n;
};
inline bool overlap(const Span& a, const Span& b) {
  return a.p && b.p && a.n > 0 && b.n > 0 && overlap(a.p, a.n, b.p, b.n);
}
// Whether one of the outputs overlaps an input or another output.
inline bool overlaps(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* o = outs.begin(); o != outs.end(); ++o) {
    for (const Span& i : ins)
      if (overlap(*o, i)) return true;
    for (const Span* p = o + 1; p != outs.end(); ++p)
      if (overlap(*o, *p)) return true;
  }
  return false;
}
// SMs of the current device (1 where it cannot tell: the launch that follows then says why).
inline int num_sms() {
  int device = 0, n = 0;
  if (cudaGetDevice(&device) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1)
    return 1;
  return n;
}
inline bool misaligned(const void* p, int n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) != 0; }

}  // namespace eat
