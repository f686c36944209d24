// Vocabulary head: softmax cross entropy of hidden states against a vocabulary matrix, in pieces
// of the vocabulary, without holding the logits; and its gradient.
//   l_tv = s_t s_v <x_t, w_v>;  r = log sum_{v != y} exp l_v - l_y;  nll = log(1 + exp r)
//   lse = l_y + nll;  P_tv = g_t (exp(l_tv - lse_t) - [v = y_t]);  dx = P w;  dw = P^T x
#include "eat_internal.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <new>
#include <string>

struct eat_head {
  eat_head_desc desc;
  char* mem = nullptr;
  float2* part = nullptr;          // [vocabulary tiles][max_tokens] {max, sum of exp}
  float* ly = nullptr;             // [max_tokens] target logits
  float* lse = nullptr;            // [max_tokens]
  __nv_bfloat16* p = nullptr;      // [max_tokens, piece] P of a piece of the vocabulary
  float* dx = nullptr;             // [max_tokens, d] dx over the pieces so far
  int piece = 0;
};

namespace eat {

namespace {

constexpr int kTile = 64, kStep = 16;
constexpr int kPieceBytes = 64 << 20;

__device__ __forceinline__ float val(const __nv_bfloat16* p, size_t i) {
  return __bfloat162float(p[i]);
}
__device__ __forceinline__ float val(const __nv_fp8_e4m3* p, size_t i) { return (float)p[i]; }

// acc = 64 x 64 tile of A B^T at (m0, n0): A(m, k) = a[m am + k ak] for m < M, B(n, k) = b[n bn + k
// bk] for n < N, summed over k < K; thread (tx, ty) holds rows ty + 16 i and columns tx + 16 j.
template <typename TA, typename TB>
__device__ void tile_product(const TA* a, size_t am, size_t ak, int M, int m0, const TB* b,
                             size_t bn, size_t bk, int N, int n0, int K, float (&acc)[4][4]) {
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  for (int k0 = 0; k0 < K; k0 += kStep) {
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
      const int ka = ak == 1 ? i % kStep : i / kTile, ma = ak == 1 ? i / kStep : i % kTile;
      const int kb = bk == 1 ? i % kStep : i / kTile, nb = bk == 1 ? i / kStep : i % kTile;
      sa[ka][ma] = m0 + ma < M && k0 + ka < K ? val(a, (m0 + ma) * am + (k0 + ka) * ak) : 0.f;
      sb[kb][nb] = n0 + nb < N && k0 + kb < K ? val(b, (n0 + nb) * bn + (k0 + kb) * bk) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][ty + 16 * i] * sb[k][tx + 16 * j];
  }
}

// part[v tile][t]: maximum and sum of exp over the tile's rows other than the target
template <typename E>
__global__ void __launch_bounds__(256)
head_part_kernel(const E* __restrict__ x, const float* __restrict__ xs, const E* __restrict__ w,
                 const float* __restrict__ ws, int T, int V, int d,
                 const int32_t* __restrict__ target, float2* __restrict__ part,
                 float* __restrict__ ly) {
  pdl_wait();
  pdl_launch_dependents();
  const int v0 = blockIdx.x * kTile, t0 = blockIdx.y * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4];
  tile_product(x, d, 1, T, t0, w, d, 1, V, v0, d, acc);
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + ty + 16 * i;
    const int y = t < T ? target[t] : -1;
    const float st = xs && t < T ? xs[t] : 1.f;
    float m = -INFINITY, s = 0.f;
    for (int j = 0; j < 4; ++j) {
      const int v = v0 + tx + 16 * j;
      if (v < V) acc[i][j] *= st * (ws ? ws[v] : 1.f);
      if (v < V && v == y) ly[t] = acc[i][j];
      if (v >= V || v == y) acc[i][j] = -INFINITY;
      m = fmaxf(m, acc[i][j]);
    }
    for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    for (int j = 0; j < 4; ++j) s += acc[i][j] == -INFINITY ? 0.f : expf(acc[i][j] - m);
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (tx == 0 && t < T) part[(size_t)blockIdx.x * T + t] = make_float2(m, s);
  }
}

__global__ void __launch_bounds__(256)
head_join_kernel(const float2* __restrict__ part, int tiles, const float* __restrict__ ly, int T,
                 int V, const int32_t* __restrict__ target, float* __restrict__ nll,
                 float* __restrict__ lse, float* __restrict__ lse_opt) {
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= T) return;
  float m = -INFINITY, s = 0.f;
  for (int i = 0; i < tiles; ++i) {
    const float2 q = part[(size_t)i * T + t];
    const float n = fmaxf(m, q.x);
    if (!(n == -INFINITY)) s = s * expf(m - n) + q.y * expf(q.x - n);
    m = n;
  }
  const int y = target[t];
  float a = 0.f, b = 0.f;
  if (y >= V) {
    a = b = NAN;
  } else if (y >= 0) {
    const float r = m + logf(s) - ly[t];
    a = fmaxf(r, 0.f) + log1pf(expf(-fabsf(r)));
    if (isnan(r)) a = r;
    b = ly[t] + a;
  }
  nll[t] = a;
  lse[t] = b;
  if (lse_opt) lse_opt[t] = b;
}

// P of the vocabulary rows [vp, vp + n) (columns of p), as bf16
__global__ void __launch_bounds__(256)
head_p_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ w, int T,
              int V, int d, int vp, int n, const int32_t* __restrict__ target,
              const float* __restrict__ lse, const float* __restrict__ g,
              __nv_bfloat16* __restrict__ p, int ld) {
  pdl_wait();
  pdl_launch_dependents();
  const int c0 = blockIdx.x * kTile, t0 = blockIdx.y * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4];
  tile_product(x, d, 1, T, t0, w + (size_t)vp * d, d, 1, n, c0, d, acc);
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + ty + 16 * i;
    if (t >= T) continue;
    const int y = target[t];
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + tx + 16 * j;
      if (c >= n) continue;
      float v = 0.f;
      if (y >= 0 && y < V) v = g[t] * (expf(acc[i][j] - lse[t]) - (vp + c == y ? 1.f : 0.f));
      p[(size_t)t * ld + c] = __float2bfloat16_rn(v);
    }
  }
}

// dx (+)= P w[vp ...]; the last piece writes the rounded result
__global__ void __launch_bounds__(256)
head_dx_kernel(const __nv_bfloat16* __restrict__ p, int ld, int n,
               const __nv_bfloat16* __restrict__ w, int T, int d, int first, int last,
               float* __restrict__ sum, __nv_bfloat16* __restrict__ dx) {
  pdl_wait();
  pdl_launch_dependents();
  const int c0 = blockIdx.x * kTile, t0 = blockIdx.y * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4];
  tile_product(p, ld, 1, T, t0, w, 1, d, d, c0, n, acc);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + ty + 16 * i, c = c0 + tx + 16 * j;
      if (t >= T || c >= d) continue;
      const size_t o = (size_t)t * d + c;
      const float v = acc[i][j] + (first ? 0.f : sum[o]);
      if (last) dx[o] = __float2bfloat16_rn(v);
      else sum[o] = v;
    }
}

// The hidden states with zero rows for the tokens that carry no loss
struct Rows {
  const __nv_bfloat16* x;
  const int32_t* target;
  int V, d;
};
__device__ __forceinline__ float val(const Rows r, size_t i) {
  const int y = r.target[i / r.d];
  return y >= 0 && y < r.V ? __bfloat162float(r.x[i]) : 0.f;
}

__global__ void __launch_bounds__(256)
head_dw_kernel(const __nv_bfloat16* __restrict__ p, int ld, int n,
               const __nv_bfloat16* __restrict__ x, const int32_t* __restrict__ target, int T,
               int V, int d, __nv_bfloat16* __restrict__ dw) {
  pdl_wait();
  pdl_launch_dependents();
  const int c0 = blockIdx.x * kTile, v0 = blockIdx.y * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4];
  __shared__ float sa[kStep][kTile + 1], sb[kStep][kTile + 1];
  const Rows r{x, target, V, d};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  for (int k0 = 0; k0 < T; k0 += kStep) {
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
      const int k = i / kTile, m = i % kTile;
      sa[k][m] = v0 + m < n && k0 + k < T ? val(p, (size_t)(k0 + k) * ld + v0 + m) : 0.f;
      sb[k][m] = c0 + m < d && k0 + k < T ? val(r, (size_t)(k0 + k) * d + c0 + m) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][ty + 16 * i] * sb[k][tx + 16 * j];
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int v = v0 + ty + 16 * i, c = c0 + tx + 16 * j;
      if (v < n && c < d) dw[(size_t)v * d + c] = __float2bfloat16_rn(acc[i][j]);
    }
}

eat_status fail(eat_status s, const std::string& msg) {
  set_thread_error(msg.c_str());
  return s;
}

void free_head(eat_head* h) {
  if (!h) return;
  if (h->mem) cudaFree(h->mem);
  delete h;
}

int tiles(int n) { return (n + kTile - 1) / kTile; }

eat_status check_call(const char* fn, eat_head* h, const void* x, int32_t T,
                      const int32_t* target, const float* nll) {
  const std::string f(fn);
  if (!h) return fail(EAT_ERR_INVALID_ARG, f + ": null handle");
  if (!x || !target || !nll)
    return fail(EAT_ERR_INVALID_ARG, f + ": x, target and nll must be non-NULL");
  if (T < 1 || T > h->desc.max_tokens)
    return fail(EAT_ERR_INVALID_ARG, f + ": T outside [1, max_tokens]");
  if ((uintptr_t)x & 15) return fail(EAT_ERR_INVALID_ARG, f + ": x must be 16-byte aligned");
  if (((uintptr_t)target | (uintptr_t)nll) & 3)
    return fail(EAT_ERR_INVALID_ARG, f + ": misaligned pointer");
  return EAT_OK;
}

cudaError_t run_nll(eat_head* h, const void* x, const float* xs, int T, const int32_t* target,
                    float* nll, float* lse_opt, cudaStream_t st) {
  const int V = h->desc.vocab, d = h->desc.d_model;
  const dim3 grid(tiles(V), tiles(T));
  cudaError_t e;
  if (h->desc.dtype == EAT_BF16)
    e = launch_pdl(head_part_kernel<__nv_bfloat16>, grid, dim3(256), 0, st,
                   (const __nv_bfloat16*)x, (const float*)nullptr,
                   (const __nv_bfloat16*)h->desc.w, (const float*)nullptr, T, V, d, target,
                   h->part, h->ly);
  else
    e = launch_pdl(head_part_kernel<__nv_fp8_e4m3>, grid, dim3(256), 0, st,
                   (const __nv_fp8_e4m3*)x, xs, (const __nv_fp8_e4m3*)h->desc.w, h->desc.w_scale,
                   T, V, d, target, h->part, h->ly);
  if (e != cudaSuccess) return e;
  return launch_pdl(head_join_kernel, dim3((T + 255) / 256), dim3(256), 0, st,
                    (const float2*)h->part, tiles(V), (const float*)h->ly, T, V, target, nll,
                    h->lse, lse_opt);
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" {

eat_status eat_head_create(const eat_head_desc* desc, eat_head** out) {
  if (!out) return fail(EAT_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!desc) return fail(EAT_ERR_INVALID_ARG, "desc is NULL");
  const eat_head_desc& D = *desc;
  if (D.dtype != EAT_BF16 && D.dtype != EAT_FP8_E4M3)
    return fail(EAT_ERR_UNSUPPORTED, "head dtype must be BF16 or FP8_E4M3");
  if (D.d_model < 64 || D.d_model % 64 || D.d_model > 16384)
    return fail(EAT_ERR_UNSUPPORTED, "d_model must be a multiple of 64 up to 16384");
  if (D.vocab < 1 || D.vocab > (1 << 20))
    return fail(EAT_ERR_UNSUPPORTED, "vocab must be in [1, 2^20]");
  if (D.max_tokens < 1 || D.max_tokens > 65536)
    return fail(EAT_ERR_INVALID_ARG, "max_tokens must be in [1, 65536]");
  if (!D.w) return fail(EAT_ERR_INVALID_ARG, "w is NULL");
  if ((uintptr_t)D.w & 15) return fail(EAT_ERR_INVALID_ARG, "w must be 16-byte aligned");
  if (D.dtype == EAT_FP8_E4M3 && (!D.w_scale || ((uintptr_t)D.w_scale & 3)))
    return fail(EAT_ERR_INVALID_ARG, "an e4m3 head needs w_scale, 4-byte aligned");
  if (D.with_grad && D.dtype != EAT_BF16)
    return fail(EAT_ERR_UNSUPPORTED, "gradients need a BF16 head");
  eat_head* h = new (std::nothrow) eat_head();
  if (!h) return fail(EAT_ERR_OOM, "host allocation failed");
  h->desc = D;
  const size_t T = (size_t)D.max_tokens;
  h->piece = (int)std::min<size_t>((size_t)tiles(D.vocab) * kTile,
                                   std::max<size_t>(kPieceBytes / 2 / T / kTile * kTile, kTile));
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t n_part = up(sizeof(float2) * tiles(D.vocab) * T), n_t = up(4 * T);
  const size_t n_p = D.with_grad ? up(2 * T * h->piece) : 0;
  const size_t n_dx = D.with_grad ? up(4 * T * D.d_model) : 0;
  const size_t total = n_part + 2 * n_t + n_p + n_dx;
  const cudaError_t e = cudaMalloc((void**)&h->mem, total);
  if (e != cudaSuccess) {
    cudaGetLastError();  // a failed allocation leaves the context usable: clear its error
    free_head(h);
    return fail(EAT_ERR_OOM, "cudaMalloc of " + std::to_string(total) + " bytes failed: " +
                                 cudaGetErrorString(e));
  }
  char* at = h->mem;
  h->part = (float2*)at;
  h->ly = (float*)(at += n_part);
  h->lse = (float*)(at += n_t);
  h->p = (__nv_bfloat16*)(at += n_t);
  h->dx = (float*)(at += n_p);
  *out = h;
  return EAT_OK;
}

eat_status eat_head_destroy(eat_head* h) {
  if (!h) return EAT_OK;
  cudaDeviceSynchronize();
  free_head(h);
  return EAT_OK;
}

eat_status eat_head_reset(eat_head* h, void* stream) {
  if (!h) return fail(EAT_ERR_INVALID_ARG, "eat_head_reset: null handle");
  const cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess)
    return fail(EAT_ERR_CUDA, std::string("eat_head_reset: ") + cudaGetErrorString(e));
  return EAT_OK;
}

eat_status eat_head_nll(eat_head* h, const void* x, const float* x_scale, int32_t T,
                        const int32_t* target, float* nll, float* lse, void* stream) {
  const eat_status s = check_call("eat_head_nll", h, x, T, target, nll);
  if (s != EAT_OK) return s;
  if (h->desc.dtype == EAT_FP8_E4M3 && (!x_scale || ((uintptr_t)x_scale & 3)))
    return fail(EAT_ERR_INVALID_ARG, "eat_head_nll: an e4m3 head needs x_scale, 4-byte aligned");
  const cudaError_t e = run_nll(h, x, x_scale, T, target, nll, lse, (cudaStream_t)stream);
  if (e != cudaSuccess)
    return fail(EAT_ERR_CUDA, std::string("eat_head_nll launch: ") + cudaGetErrorString(e));
  return EAT_OK;
}

eat_status eat_head_nll_grad(eat_head* h, const void* x, int32_t T, const int32_t* target,
                             const float* g, float* nll, float* lse, void* dx, void* dw,
                             void* stream) {
  const eat_status s = check_call("eat_head_nll_grad", h, x, T, target, nll);
  if (s != EAT_OK) return s;
  if (!h->desc.with_grad)
    return fail(EAT_ERR_INVALID_ARG, "eat_head_nll_grad: the handle was created without with_grad");
  if (!g || !dx || !dw)
    return fail(EAT_ERR_INVALID_ARG, "eat_head_nll_grad: g, dx and dw must be non-NULL");
  if (((uintptr_t)dx | (uintptr_t)dw) & 15)
    return fail(EAT_ERR_INVALID_ARG, "eat_head_nll_grad: dx and dw must be 16-byte aligned");
  if (dx == x) return fail(EAT_ERR_INVALID_ARG, "eat_head_nll_grad: dx must not alias x");
  const cudaStream_t st = (cudaStream_t)stream;
  const int V = h->desc.vocab, d = h->desc.d_model;
  const __nv_bfloat16* w = (const __nv_bfloat16*)h->desc.w;
  cudaError_t e = run_nll(h, x, nullptr, T, target, nll, lse, st);
  for (int vp = 0; vp < V && e == cudaSuccess; vp += h->piece) {
    const int n = std::min(h->piece, V - vp);
    e = launch_pdl(head_p_kernel, dim3(tiles(n), tiles(T)), dim3(256), 0, st,
                   (const __nv_bfloat16*)x, w, T, V, d, vp, n, target, (const float*)h->lse, g,
                   h->p, h->piece);
    if (e == cudaSuccess)
      e = launch_pdl(head_dx_kernel, dim3(tiles(d), tiles(T)), dim3(256), 0, st,
                     (const __nv_bfloat16*)h->p, h->piece, n, w + (size_t)vp * d, T, d, vp == 0,
                     vp + n == V, h->dx, (__nv_bfloat16*)dx);
    if (e == cudaSuccess)
      e = launch_pdl(head_dw_kernel, dim3(tiles(d), tiles(n)), dim3(256), 0, st,
                     (const __nv_bfloat16*)h->p, h->piece, n, (const __nv_bfloat16*)x, target, T,
                     V, d, (__nv_bfloat16*)dw + (size_t)vp * d);
  }
  if (e != cudaSuccess)
    return fail(EAT_ERR_CUDA, std::string("eat_head_nll_grad launch: ") + cudaGetErrorString(e));
  return EAT_OK;
}

}  // extern "C"
