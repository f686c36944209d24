// RMS norm of the residual stream (what stands between two layers), with an optional e4m3 output,
// and its gradient.
//   h = x + r;  rstd = 1 / sqrt(sum h^2 / d + eps);  y = h rstd gamma
//   e4m3: s = max |y| / 448, q = round(y / s).  max |y| = rstd max |h gamma|, so the row's sum of
//   squares and its maximum come out of one reduction and y / s = (h gamma) (448 / max |h gamma|).
//   gradient, n = h rstd:  dx = dres + rstd (gamma dy - n mean(gamma dy n));  dgamma = sum_t dy n
#include "eat_internal.cuh"

#include <cuda_fp8.h>

#include <string>

namespace eat {

namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f(float v) { return v; }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }

// Sum and maximum over the block, in every thread.
__device__ float2 block_sum_max(float s, float m) {
  __shared__ float2 red[kThreads / 32];
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(s, m);
  __syncthreads();
  s = 0.f;
  m = 0.f;
  for (int i = 0; i < kThreads / 32; ++i) {
    s += red[i].x;
    m = fmaxf(m, red[i].y);
  }
  return make_float2(s, m);
}

// One block per row.
template <typename T, bool F8>
__global__ void __launch_bounds__(kThreads)
rms_norm_kernel(const T* __restrict__ x, const T* r, int d, const float* __restrict__ gamma,
                float eps, T* h, void* y, float* __restrict__ y_scale) {
  pdl_wait();
  pdl_launch_dependents();
  const size_t row = (size_t)blockIdx.x * d;
  float ss = 0.f, mx = 0.f;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = to_f(x[row + c]) + (r ? to_f(r[row + c]) : 0.f);
    ss += v * v;
    mx = fmaxf(mx, fabsf(v * gamma[c]));
  }
  const float2 a = block_sum_max(ss, mx);
  const float rstd = 1.0f / sqrtf(a.x / (float)d + eps);
  const float top = a.y * rstd;
  const float scale = top > 0.f ? top / 448.0f : 1.0f;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = to_f(x[row + c]) + (r ? to_f(r[row + c]) : 0.f);
    if (r) h[row + c] = from_f<T>(v);
    const float o = v * rstd * gamma[c];
    if (F8) ((__nv_fp8_e4m3*)y)[row + c] = __nv_fp8_e4m3(o / scale);
    else ((T*)y)[row + c] = from_f<T>(o);
  }
  if (F8 && threadIdx.x == 0) y_scale[blockIdx.x] = scale;
}

// Block b takes rows b, b + gridDim.x, ...: dx of each row, and the block's part of dgamma
// (part[b], every column of which belongs to one thread).
template <typename T>
__global__ void __launch_bounds__(kThreads)
rms_norm_grad_kernel(const T* __restrict__ h, int rows, int d, const float* __restrict__ gamma,
                     float eps, const T* dy, const T* dres, T* dx, float* __restrict__ part) {
  pdl_wait();
  pdl_launch_dependents();
  float* mine = part + (size_t)blockIdx.x * d;
  for (int t = blockIdx.x; t < rows; t += gridDim.x) {
    const size_t row = (size_t)t * d;
    float ss = 0.f, dot = 0.f;
    for (int c = threadIdx.x; c < d; c += kThreads) {
      const float v = to_f(h[row + c]);
      ss += v * v;
      dot += gamma[c] * to_f(dy[row + c]) * v;
    }
    const float rstd = 1.0f / sqrtf(block_sum_max(ss, 0.f).x / (float)d + eps);
    const float m = block_sum_max(dot, 0.f).x * rstd / (float)d;
    for (int c = threadIdx.x; c < d; c += kThreads) {
      const float n = to_f(h[row + c]) * rstd, g = to_f(dy[row + c]);
      mine[c] = (t == (int)blockIdx.x ? 0.f : mine[c]) + g * n;
      const float v = rstd * (gamma[c] * g - n * m);
      dx[row + c] = from_f<T>(v + (dres ? to_f(dres[row + c]) : 0.f));
    }
  }
}

__global__ void __launch_bounds__(kThreads)
rms_norm_dgamma_kernel(const float* __restrict__ part, int n_parts, int d,
                       float* __restrict__ dgamma) {
  pdl_wait();
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= d) return;
  float s = 0.f;
  for (int i = 0; i < n_parts; ++i) s += part[(size_t)i * d + c];
  dgamma[c] = s;
}

int grad_blocks(int T) { return T < 608 ? T : 608; }

eat_status bad(const char* fn, const char* what) {
  set_thread_error((std::string(fn) + ": " + what).c_str());
  return EAT_ERR_INVALID_ARG;
}
eat_status launched(const char* fn, cudaError_t e) {
  if (e == cudaSuccess) return EAT_OK;
  set_thread_error((std::string(fn) + " launch: " + cudaGetErrorString(e)).c_str());
  return EAT_ERR_CUDA;
}
bool misaligned(const void* p, int n) { return ((uintptr_t)p & (uintptr_t)(n - 1)) != 0; }

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" eat_status eat_rms_norm(const void* x, const void* residual, int32_t T, int32_t d,
                                   int32_t xdtype, const float* gamma, double eps, void* h,
                                   void* y, int32_t ydtype, float* y_scale, void* stream) {
  const char* fn = "eat_rms_norm";
  if (!x || !gamma || !y) return bad(fn, "x, gamma and y must be non-NULL");
  if (residual && !h) return bad(fn, "a residual needs h");
  if (T < 1 || d < 1 || d > 65536) return bad(fn, "need T >= 1 and 1 <= d <= 65536");
  if (xdtype != EAT_F32 && xdtype != EAT_BF16) return bad(fn, "xdtype must be F32 or BF16");
  if (ydtype != xdtype && ydtype != EAT_FP8_E4M3)
    return bad(fn, "ydtype must be xdtype or FP8_E4M3");
  if (ydtype == EAT_FP8_E4M3 && !y_scale) return bad(fn, "an e4m3 output needs y_scale");
  if (!((float)eps > 0.0f) || !(eps <= 1e30)) return bad(fn, "eps must be positive");
  const int al = xdtype == EAT_BF16 ? 2 : 4;
  if (misaligned(x, al) || misaligned(residual, al) || (residual && misaligned(h, al)) ||
      misaligned(gamma, 4) || (ydtype == EAT_FP8_E4M3 ? misaligned(y_scale, 4) : misaligned(y, al)))
    return bad(fn, "misaligned pointer");
  auto run = [&](auto* tag, auto f8) {
    using E = std::remove_pointer_t<decltype(tag)>;
    return launch_pdl(rms_norm_kernel<E, decltype(f8)::value>, dim3(T), dim3(kThreads), 0,
                      (cudaStream_t)stream, (const E*)x, (const E*)residual, d, gamma, (float)eps,
                      (E*)h, y, y_scale);
  };
  const bool f8 = ydtype == EAT_FP8_E4M3;
  cudaError_t e;
  if (xdtype == EAT_BF16)
    e = f8 ? run((__nv_bfloat16*)nullptr, std::true_type()) : run((__nv_bfloat16*)nullptr, std::false_type());
  else
    e = f8 ? run((float*)nullptr, std::true_type()) : run((float*)nullptr, std::false_type());
  return launched(fn, e);
}

extern "C" int64_t eat_rms_norm_grad_workspace(int32_t T, int32_t d) {
  return T < 1 || d < 1 ? 0 : (int64_t)grad_blocks(T) * d * 4;
}

extern "C" eat_status eat_rms_norm_grad(const void* h, int32_t T, int32_t d, int32_t xdtype,
                                        const float* gamma, double eps, const void* dy,
                                        const void* dres, void* dx, float* dgamma, void* work,
                                        void* stream) {
  const char* fn = "eat_rms_norm_grad";
  if (!h || !gamma || !dy || !dx || !dgamma || !work)
    return bad(fn, "h, gamma, dy, dx, dgamma and work must be non-NULL");
  if (T < 1 || d < 1 || d > 65536) return bad(fn, "need T >= 1 and 1 <= d <= 65536");
  if (xdtype != EAT_F32 && xdtype != EAT_BF16) return bad(fn, "xdtype must be F32 or BF16");
  if (!((float)eps > 0.0f) || !(eps <= 1e30)) return bad(fn, "eps must be positive");
  const int al = xdtype == EAT_BF16 ? 2 : 4;
  if (misaligned(h, al) || misaligned(dy, al) || misaligned(dres, al) || misaligned(dx, al) ||
      misaligned(gamma, 4) || misaligned(dgamma, 4) || misaligned(work, 16))
    return bad(fn, "misaligned pointer");
  const cudaStream_t st = (cudaStream_t)stream;
  auto run = [&](auto* tag) {
    using E = std::remove_pointer_t<decltype(tag)>;
    const int blocks = grad_blocks(T);
    cudaError_t e = launch_pdl(rms_norm_grad_kernel<E>, dim3(blocks), dim3(kThreads), 0, st,
                               (const E*)h, T, d, gamma, (float)eps, (const E*)dy, (const E*)dres,
                               (E*)dx, (float*)work);
    if (e != cudaSuccess) return e;
    return launch_pdl(rms_norm_dgamma_kernel, dim3((d + kThreads - 1) / kThreads), dim3(kThreads),
                      0, st, (const float*)work, blocks, d, dgamma);
  };
  return launched(fn, xdtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr));
}
