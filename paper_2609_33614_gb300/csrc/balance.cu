// Load-balancing loss of a router with per-expert counts, and its gradient to the logits.
//   counts[e] = entries of idx equal to e;  f_e = counts[e] / sum counts;  p_t = softmax(logits_t)
//   loss = E sum_e f_e (1/n) sum_t p_te;   dlogits_te = g E / n p_te (f_e - sum_j f_j p_tj)
#include "eat_internal.cuh"

#include <string>

namespace eat {

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kPer = kMaxExperts / 32;  // experts per lane
constexpr int kMaxBlocks = 304;

__device__ __forceinline__ float warp_sum(float v) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// softmax of a row of E logits; lane l holds the experts l, l + 32, ... (0 beyond E)
__device__ __forceinline__ void row_softmax(const float* z, int E, int lane, float (&p)[kPer]) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    p[i] = i * 32 + lane < E ? z[i * 32 + lane] : -INFINITY;
    m = fmaxf(m, p[i]);
  }
  m = warp_max(m);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    p[i] = i * 32 + lane < E ? __expf(p[i] - m) : 0.f;
    s += p[i];
  }
  s = 1.0f / warp_sum(s);
#pragma unroll
  for (int i = 0; i < kPer; ++i) p[i] *= s;
}

// A warp per token; part[b][e] = {sum of p, count} of block b, its last entry the tokens counted.
__global__ void __launch_bounds__(kThreads)
balance_part_kernel(const float* __restrict__ logits, int T, int E, int K,
                    const int32_t* __restrict__ idx, const uint8_t* __restrict__ mask,
                    float* __restrict__ psum, int32_t* __restrict__ cnt) {
  __shared__ int s_cnt[kMaxExperts + 1];
  __shared__ float s_p[kWarps][kMaxExperts];
  pdl_wait();
  pdl_launch_dependents();
  for (int i = threadIdx.x; i <= E; i += kThreads) s_cnt[i] = 0;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float acc[kPer] = {};
  for (int t = blockIdx.x * kWarps + warp; t < T; t += gridDim.x * kWarps) {
    if (mask && !mask[t]) continue;
    float p[kPer];
    row_softmax(logits + (size_t)t * E, E, lane, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += p[i];
    if (lane < K) {
      const int e = idx[(size_t)t * K + lane];
      if (e >= 0 && e < E) atomicAdd(&s_cnt[e], 1);
    }
    if (lane == 0) atomicAdd(&s_cnt[E], 1);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (i * 32 + lane < E) s_p[warp][i * 32 + lane] = acc[i];
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) {
    float s = 0.f;
    for (int w = 0; w < kWarps; ++w) s += s_p[w][e];
    psum[(size_t)blockIdx.x * E + e] = s;
  }
  for (int e = threadIdx.x; e <= E; e += kThreads)
    cnt[(size_t)blockIdx.x * (E + 1) + e] = s_cnt[e];
}

__global__ void __launch_bounds__(kThreads)
balance_join_kernel(const float* __restrict__ psum, const int32_t* __restrict__ cnt, int parts,
                    int E, float* __restrict__ loss, int32_t* __restrict__ counts,
                    int32_t* __restrict__ n_tokens) {
  __shared__ float red[kThreads];
  __shared__ float red_c[kThreads];
  __shared__ int s_n;
  pdl_wait();
  float s = 0.f;
  int c = 0;
  const int e = threadIdx.x;
  if (e < E) {
    for (int b = 0; b < parts; ++b) {
      s += psum[(size_t)b * E + e];
      c += cnt[(size_t)b * (E + 1) + e];
    }
    counts[e] = c;
  }
  if (threadIdx.x == 0) {
    int n = 0;
    for (int b = 0; b < parts; ++b) n += cnt[(size_t)b * (E + 1) + E];
    s_n = n;
    *n_tokens = n;
  }
  red[threadIdx.x] = s * (float)c;
  red_c[threadIdx.x] = (float)c;
  __syncthreads();
  for (int w = kThreads / 2; w > 0; w >>= 1) {
    if (threadIdx.x < w) {
      red[threadIdx.x] += red[threadIdx.x + w];
      red_c[threadIdx.x] += red_c[threadIdx.x + w];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0)
    *loss = red_c[0] > 0.f ? (float)E * red[0] / (red_c[0] * (float)s_n) : 0.f;
}

__global__ void __launch_bounds__(kThreads)
balance_grad_kernel(const float* logits, int T, int E, const uint8_t* __restrict__ mask,
                    const int32_t* __restrict__ counts, const int32_t* __restrict__ n_tokens,
                    const float* __restrict__ g, float* dlogits) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float f[kPer], total = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    f[i] = i * 32 + lane < E ? (float)counts[i * 32 + lane] : 0.f;
    total += f[i];
  }
  total = warp_sum(total);
  const float scale = total > 0.f ? *g * (float)E / ((float)*n_tokens) : 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) f[i] = total > 0.f ? f[i] / total : 0.f;
  for (int t = blockIdx.x * kWarps + warp; t < T; t += gridDim.x * kWarps) {
    const bool on = total > 0.f && !(mask && !mask[t]);
    float p[kPer], dot = 0.f;
    row_softmax(logits + (size_t)t * E, E, lane, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) dot += f[i] * p[i];
    dot = warp_sum(dot);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 32 + lane < E)
        dlogits[(size_t)t * E + i * 32 + lane] = on ? scale * p[i] * (f[i] - dot) : 0.f;
  }
}

int part_blocks(int T) {
  const int b = (T + kWarps - 1) / kWarps;
  return b < kMaxBlocks ? b : kMaxBlocks;
}

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

extern "C" int64_t eat_balance_workspace(int32_t T, int32_t E) {
  return T < 1 || E < 1 ? 0 : (int64_t)part_blocks(T) * (2 * E + 1) * 4;
}

extern "C" eat_status eat_balance_loss(const float* logits, int32_t T, int32_t E, int32_t K,
                                       const int32_t* idx, const uint8_t* mask, float* loss,
                                       int32_t* counts, int32_t* n_tokens, void* work,
                                       void* stream) {
  const char* fn = "eat_balance_loss";
  if (!logits || !idx || !loss || !counts || !n_tokens || !work)
    return bad(fn, "logits, idx, loss, counts, n_tokens and work must be non-NULL");
  if (T < 1 || E < 1 || E > kMaxExperts || K < 1 || K > kMaxK)
    return bad(fn, "need T >= 1, 1 <= E <= 256 and 1 <= K <= 16");
  if (misaligned(logits, 4) || misaligned(idx, 4) || misaligned(loss, 4) ||
      misaligned(counts, 4) || misaligned(n_tokens, 4) || misaligned(work, 16))
    return bad(fn, "misaligned pointer");
  const cudaStream_t st = (cudaStream_t)stream;
  const int parts = part_blocks(T);
  float* psum = (float*)work;
  int32_t* cnt = (int32_t*)(psum + (size_t)parts * E);
  cudaError_t e = launch_pdl(balance_part_kernel, dim3(parts), dim3(kThreads), 0, st, logits, T, E,
                             K, idx, mask, psum, cnt);
  if (e == cudaSuccess)
    e = launch_pdl(balance_join_kernel, dim3(1), dim3(kThreads), 0, st, (const float*)psum,
                   (const int32_t*)cnt, parts, E, loss, counts, n_tokens);
  return launched(fn, e);
}

extern "C" eat_status eat_balance_grad(const float* logits, int32_t T, int32_t E,
                                       const uint8_t* mask, const int32_t* counts,
                                       const int32_t* n_tokens, const float* g, float* dlogits,
                                       void* stream) {
  const char* fn = "eat_balance_grad";
  if (!logits || !counts || !n_tokens || !g || !dlogits)
    return bad(fn, "logits, counts, n_tokens, g and dlogits must be non-NULL");
  if (T < 1 || E < 1 || E > kMaxExperts) return bad(fn, "need T >= 1 and 1 <= E <= 256");
  if (misaligned(logits, 4) || misaligned(counts, 4) || misaligned(n_tokens, 4) ||
      misaligned(g, 4) || misaligned(dlogits, 4))
    return bad(fn, "misaligned pointer");
  return launched(fn, launch_pdl(balance_grad_kernel, dim3(part_blocks(T)), dim3(kThreads), 0,
                                 (cudaStream_t)stream, logits, T, E, mask, counts, n_tokens, g,
                                 dlogits));
}
