// RMS norm of the residual stream (what stands between two layers), with an optional e4m3 output,
// and its gradient.
//   h = x + r;  rstd = 1 / sqrt(sum h^2 / d + eps);  y = h rstd gamma
//   e4m3: s = max |y| / 448, q = round(y / s).  max |y| = rstd max |h gamma|, so the row's sum of
//   squares and its maximum come out of one reduction and y / s = (h gamma) (rstd / s).
//   gradient, n = h rstd:  dx = dres + rstd (gamma dy - n mean(gamma dy n));  dgamma = sum_t dy n
// Bound: HBM (a row is read once and kept in registers between the reduction and the outputs).
// A thread holds NV vectors of 16 bytes of a row; a row is taken by a warp (up to 64 vectors) or by a
// block of as many warps as it needs.  Rows whose length is no multiple of a vector begin at any
// element: their vectors are the aligned ones of memory, and the first and the last of a row are
// shared with its neighbours (read whole, masked, and stored element by element).  All sums are
// fp32; a value is rounded once, when it is stored.
#include "op_checks.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

namespace eat {

namespace {

constexpr int kThreads = 256;  // of a block whose warps take a row each, and of the plain kernels
constexpr int kWarps = kThreads / 32;
constexpr int kMaxRows = 1 << 30;  // row numbers and their strides ahead stay within an int
constexpr int kMaxThreads = 512;  // of a block that takes a row
constexpr int kMaxWarps = kMaxThreads / 32;
// e4m3 rows whose largest value is not above this get the scale 1 (and bytes 0): max / 448 and its
// reciprocal stay away from fp32's ends
constexpr float kTiny = 1e-35f;

// What the products h gamma are multiplied by for an e4m3 row, one after the other: rstd / scale and 1,
// or, where that quotient (448 / max |h gamma|) is beyond fp32, rstd and 1 / scale.
__device__ __forceinline__ float2 e4m3_factors(float rstd, float scale) {
  const float k = rstd / scale;
  return isinf(k) ? make_float2(rstd, 1.0f / scale) : make_float2(k, 1.0f);
}

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int kN = 4;  // elements of 16 bytes
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
  static __device__ __forceinline__ void unpack(uint4 u, float* v) {
    v[0] = __uint_as_float(u.x);
    v[1] = __uint_as_float(u.y);
    v[2] = __uint_as_float(u.z);
    v[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3]));
  }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
  static __device__ __forceinline__ void unpack(uint4 u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *(const uint32_t*)&b;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Elements [c, c + kN) of a row as they lie in memory.  With ALIGNED the row begins at a vector and c
// never leaves it; else the vector may begin in the row before and end in the one behind (their
// elements are there to be masked), and `left` elements from the row's begin on are the matrix's.
template <typename T, bool ALIGNED>
__device__ __forceinline__ uint4 load_vec(const T* row, int c, long long left) {
  constexpr int N = Elem<T>::kN;
  if (ALIGNED || c + N <= left) return *(const uint4*)(row + c);
  union {
    uint4 u;
    T e[N];
  } v;
  v.u = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (c + j < left) v.e[j] = row[c + j];
  return v.u;
}
// The elements outside the row become 0.
template <int N, bool ALIGNED>
__device__ __forceinline__ void mask_vec(float (&v)[N], int c, int d) {
  if (ALIGNED || (c >= 0 && c + N <= d)) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (c + j < 0 || c + j >= d) v[j] = 0.f;
}
template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_vec(T* row, int c, int d, const float* v) {
  constexpr int N = Elem<T>::kN;
  if (ALIGNED || (c >= 0 && c + N <= d)) {
    *(uint4*)(row + c) = Elem<T>::pack(v);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (c + j >= 0 && c + j < d) row[c + j] = Elem<T>::put(v[j]);
}
// Elements [c, c + N) of gamma.  A row that begins anywhere has c anywhere, but the same remainder of
// four in all its threads: whole vectors around the elements are loaded, and shifted by it.  (Loads
// element by element made 16384 rows of 2047 take twice the time of 2048.)
template <int N, bool ALIGNED>
__device__ __forceinline__ void load_gamma(const float* g, int c, int d, float* v) {
  if (ALIGNED) {
#pragma unroll
    for (int j = 0; j < N; j += 4) *(float4*)(v + j) = __ldg((const float4*)(g + c + j));
    return;
  }
  const int a = c & 3;
  if (c - a >= 0 && c - a + N + 4 <= d) {
    float w[N + 4];
#pragma unroll
    for (int j = 0; j < N + 4; j += 4) *(float4*)(w + j) = __ldg((const float4*)(g + c - a + j));
#pragma unroll
    for (int j = 0; j < N; ++j)
      v[j] = a == 0 ? w[j] : a == 1 ? w[j + 1] : a == 2 ? w[j + 2] : w[j + 3];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = c + j >= 0 && c + j < d ? __ldg(g + c + j) : 0.f;
  }
}

// Sums (or maxima) over the threads of a row, in every one of them: a warp, or the whole block; `red`
// alternates between two buffers, so one barrier per row is enough.
template <bool WARP, bool MAX>
__device__ __forceinline__ float2 row_reduce(float a, float b, float2 (*red)[kMaxWarps],
                                             int turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    const float b2 = __shfl_xor_sync(0xffffffffu, b, o);
    b = MAX ? fmaxf(b, b2) : b + b2;
  }
  if (WARP) return make_float2(a, b);
  if ((threadIdx.x & 31) == 0) red[turn & 1][threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  const int warps = blockDim.x >> 5;
  float2 s = red[turn & 1][0];
#pragma unroll
  for (int i = 1; i < kMaxWarps; ++i) {
    if (i >= warps) break;
    const float2 q = red[turn & 1][i];
    s.x += q.x;
    s.y = MAX ? fmaxf(s.y, q.y) : s.y + q.y;
  }
  return s;
}

template <typename T, bool F8, bool WARP, int NV, bool ALIGNED>
__global__ void __launch_bounds__(kMaxThreads)
rms_norm_kernel(const T* x, const T* r, int rows, int d, const float* __restrict__ gamma, float eps,
                T* h, void* y, float* __restrict__ y_scale) {
  constexpr int N = Elem<T>::kN;
  __shared__ float2 red[2][kMaxWarps];
  pdl_wait();
  pdl_launch_dependents();
  const int t = WARP ? blockIdx.x * kWarps + (threadIdx.x >> 5) : blockIdx.x;
  if (t >= rows) return;
  const int lane = WARP ? threadIdx.x & 31 : threadIdx.x, ROW = WARP ? 32 : blockDim.x;
  const size_t at = (size_t)t * d;
  const int shift = ALIGNED ? 0 : (int)(at % N);
  const long long left = (long long)(rows - t) * d;
  uint4 ux[NV], ur[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * ROW) * N - shift;
    if (c < d) {
      ux[i] = load_vec<T, ALIGNED>(x + at, c, left);
      if (r) ur[i] = load_vec<T, ALIGNED>(r + at, c, left);
    }
  }
  float v[NV][N];
  float ss = 0.f, top = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * ROW) * N - shift;
    if (c < d) {
      Elem<T>::unpack(ux[i], v[i]);
      if (r) {
        float w[N];
        Elem<T>::unpack(ur[i], w);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] += w[j];
        store_vec<T, ALIGNED>(h + at, c, d, v[i]);
      }
      mask_vec<N, ALIGNED>(v[i], c, d);
#pragma unroll
      for (int j = 0; j < N; ++j) ss = fmaf(v[i][j], v[i][j], ss);
      float g[N];
      load_gamma<N, ALIGNED>(gamma, c, d, g);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[i][j] *= g[j];
        if (F8) top = fmaxf(top, fabsf(v[i][j]));
      }
    }
  }
  const float2 a = row_reduce<WARP, true>(ss, top, red, 0);
  const float rstd = 1.0f / sqrtf(a.x / (float)d + eps);
  float2 k = make_float2(rstd, 1.0f);
  if (F8) {
    const float m = a.y * rstd, scale = m > kTiny ? m / 448.0f : 1.0f;
    k = e4m3_factors(rstd, scale);
    if (lane == 0) y_scale[t] = scale;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * ROW) * N - shift;
    if (c < d) {
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = F8 ? v[i][j] * k.x * k.y : v[i][j] * k.x;
      if (!F8) {
        store_vec<T, ALIGNED>((T*)y + at, c, d, v[i]);
      } else {
        uint32_t q[N / 4];
#pragma unroll
        for (int j = 0; j < N; j += 4)
          q[j / 4] = __nv_fp8x4_e4m3(make_float4(v[i][j], v[i][j + 1], v[i][j + 2], v[i][j + 3])).__x;
        // (at + c is a multiple of N in either case)
        uint8_t* o = (uint8_t*)y + at + c;
        if (ALIGNED || (c >= 0 && c + N <= d)) {
          if (N == 8) *(uint2*)o = make_uint2(q[0], q[N / 4 - 1]);
          else *(uint32_t*)o = q[0];
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (c + j >= 0 && c + j < d) o[j] = (uint8_t)(q[j / 4] >> (8 * (j & 3)));
        }
      }
    }
  }
}

// Threads of the gradient's blocks at most, and blocks that are to fit an SM.
__host__ __device__ constexpr int grad_threads(int nv) { return nv <= 2 ? kThreads : kMaxThreads; }
// Rows of a group on their way or at work: 32 KB each of h, dy and dres (24 KB of it on the way) at 256
// threads and two vectors, 96 KB a block.
__host__ __device__ constexpr int grad_stages(int nv) { return nv <= 2 ? 4 : 2; }

// Dynamic shared memory of a block at most: all stages (a warp's sums take less, kWarps rows of up to 64
// vectors of bf16).
constexpr int grad_smem_limit(int nv) { return grad_stages(nv) * 3 * nv * grad_threads(nv) * 16; }
static_assert(kWarps * 64 * 8 * 4 <= grad_smem_limit(1), "the warps' sums fit the stages");

// Group b of threads (a warp or the block) takes rows b, b + groups, ... (the number of groups is a
// multiple of a vector's elements, so these rows begin alike): dx, and in registers the group's sum of
// dy n, which the block adds up and leaves in part[block].
// Rows are copied ahead into shared memory; each thread waits for, and reads, its own vectors only.
// (Rows ahead in registers reach one row: 4095 x 4096 with a residual's gradient 31 us, so 22.)
template <typename T, bool WARP, int NV, bool ALIGNED>
__global__ void __launch_bounds__(grad_threads(NV), NV <= 2 ? 2 : 1)
rms_norm_grad_kernel(const T* __restrict__ h, int rows, int d, const float* __restrict__ gamma,
                     float eps, const T* dy, const T* dres, T* dx, float* __restrict__ part) {
  constexpr int N = Elem<T>::kN, S = grad_stages(NV);
  constexpr int kGroups = WARP ? kWarps : 1;  // per block
  __shared__ float2 red[2][kMaxWarps];
  extern __shared__ uint4 ring[];  // [stage][h, dy, dres][NV][thread]; at the end the warps' sums (WARP)
  pdl_wait();
  pdl_launch_dependents();
  const int lane = WARP ? threadIdx.x & 31 : threadIdx.x, ROW = WARP ? 32 : blockDim.x;
  const int t0 = blockIdx.x * kGroups + (WARP ? threadIdx.x >> 5 : 0);
  const int step = gridDim.x * kGroups;
  const int shift = ALIGNED ? 0 : (int)((size_t)t0 * d % N);
  auto slot = [&](int stage, int a, int i) {
    return ring + ((stage * 3 + a) * NV + i) * blockDim.x + threadIdx.x;
  };
  auto copy = [&](const T* m, int t, int a, int stage) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * ROW) * N - shift;
      if (c >= d) continue;
      const T* row = m + (size_t)t * d;
      uint4* to = slot(stage, a, i);
      const long long left = (long long)(rows - t) * d;
      if (ALIGNED || c + N <= left)
        cp_async16((uint32_t)__cvta_generic_to_shared(to), row + c);
      else
        *to = load_vec<T, ALIGNED>(row, c, left);
    }
  };
  auto fetch = [&](int t, int stage) {
    if (t < rows) {
      copy(h, t, 0, stage);
      copy(dy, t, 1, stage);
      if (dres) copy(dres, t, 2, stage);
    }
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fetch(t0 + k * step, k);
  float acc[NV][N], gm[NV][N];  // sums of dy n; gamma, alike for all rows
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (lane + i * ROW) * N - shift;
#pragma unroll
    for (int j = 0; j < N; ++j) acc[i][j] = 0.f;
    if (c < d) load_gamma<N, ALIGNED>(gamma, c, d, gm[i]);
  }
  int turn = 0;
  for (int t = t0; t < rows; t += step, ++turn) {
    const size_t at = (size_t)t * d;
    const int stage = turn % S;
    fetch(t + (S - 1) * step, (turn + S - 1) % S);
    cp_async_wait<S - 1>();
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * ROW) * N - shift;
      if (c < d) {
        float v[N], w[N];
        Elem<T>::unpack(*slot(stage, 0, i), v);
        Elem<T>::unpack(*slot(stage, 1, i), w);
        mask_vec<N, ALIGNED>(v, c, d);
        mask_vec<N, ALIGNED>(w, c, d);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          ss = fmaf(v[j], v[j], ss);
          dot = fmaf(gm[i][j] * w[j], v[j], dot);
        }
      }
    }
    const float2 a = row_reduce<WARP, false>(ss, dot, red, turn);
    const float rstd = 1.0f / sqrtf(a.x / (float)d + eps);
    const float m = a.y * rstd / (float)d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * ROW) * N - shift;
      if (c < d) {
        float v[N], w[N], o[N];
        Elem<T>::unpack(*slot(stage, 0, i), v);
        Elem<T>::unpack(*slot(stage, 1, i), w);
        mask_vec<N, ALIGNED>(v, c, d);
        mask_vec<N, ALIGNED>(w, c, d);
        if (dres) Elem<T>::unpack(*slot(stage, 2, i), o);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float n = v[j] * rstd;
          acc[i][j] = fmaf(w[j], n, acc[i][j]);
          const float k = rstd * (gm[i][j] * w[j] - n * m);
          o[j] = dres ? o[j] + k : k;
        }
        store_vec<T, ALIGNED>(dx + at, c, d, o);
      }
    }
  }
  cp_async_wait<0>();
  float* mine = part + (size_t)blockIdx.x * d;
  if (WARP) {
    float* const s_part = (float*)ring;  // [kWarps][d]
    __syncthreads();
    float* w = s_part + (threadIdx.x >> 5) * d;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = (lane + i * ROW) * N - shift + j;
        if (c >= 0 && c < d) w[c] = acc[i][j];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += kThreads) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) s += s_part[i * d + c];
      mine[c] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (lane + i * ROW) * N - shift;
      if (ALIGNED) {
#pragma unroll
        for (int j = 0; j < N; j += 4)
          if (c < d) *(uint4*)(mine + c + j) = Elem<float>::pack(acc[i] + j);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (c + j >= 0 && c + j < d) mine[c + j] = acc[i][j];
      }
    }
  }
}

// Rows that no vector kernel takes (longer than 16384 bf16 or 8192 fp32, or in memory that is not aligned
// to vectors, such as a view one element in): a block per row, element by element, reading the row twice.
// With a residual, bf16: 4096 x 20000 261 us, 2.5 TB/s; 4096 x 4096 one element in 36 us, where aligned
// rows take 21.
template <typename T, bool F8>
__global__ void __launch_bounds__(kThreads)
rms_norm_any_kernel(const T* x, const T* r, int d, const float* __restrict__ gamma, float eps, T* h,
                    void* y, float* __restrict__ y_scale) {
  __shared__ float2 red[2][kMaxWarps];
  pdl_wait();
  pdl_launch_dependents();
  const size_t row = (size_t)blockIdx.x * d;
  auto sum = [&](int c) {
    return Elem<T>::get(x[row + c]) + (r ? Elem<T>::get(r[row + c]) : 0.f);
  };
  float ss = 0.f, top = 0.f;
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = sum(c);
    ss = fmaf(v, v, ss);
    top = fmaxf(top, fabsf(v * gamma[c]));
  }
  const float2 a = row_reduce<false, true>(ss, top, red, 0);
  const float rstd = 1.0f / sqrtf(a.x / (float)d + eps);
  const float m = a.y * rstd, scale = m > kTiny ? m / 448.0f : 1.0f;
  const float2 k = F8 ? e4m3_factors(rstd, scale) : make_float2(rstd, 1.0f);
  for (int c = threadIdx.x; c < d; c += kThreads) {
    const float v = sum(c);
    if (r) h[row + c] = Elem<T>::put(v);
    const float o = v * gamma[c] * k.x * k.y;
    if (F8) ((__nv_fp8_e4m3*)y)[row + c] = __nv_fp8_e4m3(o);
    else ((T*)y)[row + c] = Elem<T>::put(o);
  }
  if (F8 && threadIdx.x == 0) y_scale[blockIdx.x] = scale;
}
// Block b takes rows b, b + gridDim.x, ...; every column of part[b] belongs to one thread, which adds each
// row's term to it in memory.  Bound by that: 4096 x 20000 1215 us, 0.5 TB/s; 4096 x 4096 one element in
// 219 us, where aligned rows take 28.
template <typename T>
__global__ void __launch_bounds__(kThreads)
rms_norm_grad_any_kernel(const T* __restrict__ h, int rows, int d, const float* __restrict__ gamma,
                         float eps, const T* dy, const T* dres, T* dx, float* __restrict__ part) {
  __shared__ float2 red[2][kMaxWarps];
  pdl_wait();
  pdl_launch_dependents();
  float* mine = part + (size_t)blockIdx.x * d;
  int turn = 0;
  for (int t = blockIdx.x; t < rows; t += gridDim.x, ++turn) {
    const size_t row = (size_t)t * d;
    float ss = 0.f, dot = 0.f;
    for (int c = threadIdx.x; c < d; c += kThreads) {
      const float v = Elem<T>::get(h[row + c]);
      ss = fmaf(v, v, ss);
      dot = fmaf(gamma[c] * Elem<T>::get(dy[row + c]), v, dot);
    }
    const float2 a = row_reduce<false, false>(ss, dot, red, turn);
    const float rstd = 1.0f / sqrtf(a.x / (float)d + eps);
    const float m = a.y * rstd / (float)d;
    for (int c = threadIdx.x; c < d; c += kThreads) {
      const float n = Elem<T>::get(h[row + c]) * rstd, g = Elem<T>::get(dy[row + c]);
      mine[c] = fmaf(g, n, turn ? mine[c] : 0.f);
      const float v = rstd * (gamma[c] * g - n * m);
      dx[row + c] = Elem<T>::put(dres ? Elem<T>::get(dres[row + c]) + v : v);
    }
  }
}

// dgamma: 32 columns per block, its warps over the blocks' sums, added in a fixed order.
__global__ void __launch_bounds__(1024)
rms_norm_dgamma_kernel(const float* __restrict__ part, int n_parts, int d,
                       float* __restrict__ dgamma) {
  __shared__ float s_w[32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int i = warp; i < n_parts; i += 32) s += part[(size_t)i * d + c];
  }
  s_w[warp][lane] = s;
  __syncthreads();
  s = s_w[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0 && blockIdx.x * 32 + warp < d) dgamma[blockIdx.x * 32 + warp] = s;
}

// Blocks of the gradient's first kernel: as many as fit this chip's 152 SMs (512 threads each) at most,
// a multiple of a vector's elements unless every group has one row.
constexpr int kGradBlocks = 1216;
int grad_blocks(int T, int groups, int threads) {
  return std::min((T + groups - 1) / groups, 152 * std::max(1, std::min(8, 512 / threads)));
}

// The kernel for rows of d elements of type E in memory aligned to vectors: pick(WARP, NV, ALIGNED,
// threads) with the first three as types; false when no vector kernel takes the row.  The gradient
// takes two vectors a thread where the norm takes one: it holds three matrices' rows and a barrier
// per row, and blocks of half the threads overlap better (16384 x 2048: 81 -> 51 us).
template <typename E, bool GRAD, typename F>
bool pick_rows(int d, F&& pick) {
  constexpr int N = Elem<E>::kN;
  const bool aligned = d % N == 0;
  const int vecs = aligned ? d / N : (d + 2 * N - 2) / N;  // of a row that begins anywhere
  auto go = [&](auto warp, auto nv) {
    constexpr int NV = decltype(nv)::value;
    const int threads =
        decltype(warp)::value ? kThreads : ((vecs + NV - 1) / NV + 31) / 32 * 32;
    if (aligned) pick(warp, nv, std::true_type(), threads);
    else pick(warp, nv, std::false_type(), threads);
    return true;
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Four = std::integral_constant<int, 4>;
  if (vecs <= 32) return go(std::true_type(), One());
  if (vecs <= 64) return go(std::true_type(), Two());
  if constexpr (!GRAD) {
    if (vecs <= 320) return go(std::false_type(), One());
  }
  if (vecs <= 512) return go(std::false_type(), Two());
  if (vecs <= 4 * kMaxThreads) return go(std::false_type(), Four());
  return false;
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" eat_status eat_rms_norm(const void* x, const void* residual, int32_t T, int32_t d,
                                   int32_t xdtype, const float* gamma, double eps, void* h,
                                   void* y, int32_t ydtype, float* y_scale, void* stream) {
  const char* fn = "eat_rms_norm";
  if (!x || !gamma || !y) return bad_arg(fn, "x, gamma and y must be non-NULL");
  if (residual && !h) return bad_arg(fn, "a residual needs h");
  if (T < 1 || T > kMaxRows || d < 1 || d > 65536)
    return bad_arg(fn, "need T >= 1, T <= 2^30 and 1 <= d <= 65536");
  if (xdtype != EAT_F32 && xdtype != EAT_BF16) return bad_arg(fn, "xdtype must be F32 or BF16");
  if (ydtype != xdtype && ydtype != EAT_FP8_E4M3)
    return bad_arg(fn, "ydtype must be xdtype or FP8_E4M3");
  if (ydtype == EAT_FP8_E4M3 && !y_scale) return bad_arg(fn, "an e4m3 output needs y_scale");
  if (!((float)eps > 0.0f) || !(eps <= 1e30)) return bad_arg(fn, "eps must be positive");
  const int al = xdtype == EAT_BF16 ? 2 : 4;
  if (misaligned(x, al) || misaligned(residual, al) || (residual && misaligned(h, al)) ||
      misaligned(gamma, 4) || (ydtype == EAT_FP8_E4M3 ? misaligned(y_scale, 4) : misaligned(y, al)))
    return bad_arg(fn, "misaligned pointer");
  const bool vec = !(misaligned(x, 16) || misaligned(residual, 16) || misaligned(gamma, 16) ||
                     misaligned(y, 16) || (residual && misaligned(h, 16)));
  const cudaStream_t st = (cudaStream_t)stream;
  auto run = [&](auto* tag, auto f8) {
    using E = std::remove_pointer_t<decltype(tag)>;
    constexpr bool F8 = decltype(f8)::value;
    cudaError_t e = cudaSuccess;
    if (vec && pick_rows<E, false>(d, [&](auto warp, auto nv, auto al, int threads) {
          constexpr bool WARP = decltype(warp)::value;
          const unsigned blocks = WARP ? ((unsigned)T + kWarps - 1) / kWarps : (unsigned)T;
          e = launch_pdl(rms_norm_kernel<E, F8, WARP, decltype(nv)::value, decltype(al)::value>,
                         dim3(blocks), dim3(threads), 0, st, (const E*)x, (const E*)residual, T, d,
                         gamma, (float)eps, (E*)h, y, y_scale);
        }))
      return e;
    return launch_pdl(rms_norm_any_kernel<E, F8>, dim3(T), dim3(kThreads), 0, st, (const E*)x,
                      (const E*)residual, d, gamma, (float)eps, (E*)h, y, y_scale);
  };
  const bool f8 = ydtype == EAT_FP8_E4M3;
  cudaError_t e;
  if (xdtype == EAT_BF16)
    e = f8 ? run((__nv_bfloat16*)nullptr, std::true_type())
           : run((__nv_bfloat16*)nullptr, std::false_type());
  else
    e = f8 ? run((float*)nullptr, std::true_type()) : run((float*)nullptr, std::false_type());
  return launched(fn, e);
}

extern "C" int64_t eat_rms_norm_grad_workspace(int32_t T, int32_t d) {
  return T < 1 || d < 1 ? 0 : (int64_t)std::min(T, kGradBlocks) * d * 4;
}

extern "C" eat_status eat_rms_norm_grad(const void* h, int32_t T, int32_t d, int32_t xdtype,
                                        const float* gamma, double eps, const void* dy,
                                        const void* dres, void* dx, float* dgamma, void* work,
                                        void* stream) {
  const char* fn = "eat_rms_norm_grad";
  if (!h || !gamma || !dy || !dx || !dgamma || !work)
    return bad_arg(fn, "h, gamma, dy, dx, dgamma and work must be non-NULL");
  if (T < 1 || T > kMaxRows || d < 1 || d > 65536)
    return bad_arg(fn, "need T >= 1, T <= 2^30 and 1 <= d <= 65536");
  if (xdtype != EAT_F32 && xdtype != EAT_BF16) return bad_arg(fn, "xdtype must be F32 or BF16");
  if (!((float)eps > 0.0f) || !(eps <= 1e30)) return bad_arg(fn, "eps must be positive");
  const int al = xdtype == EAT_BF16 ? 2 : 4;
  if (misaligned(h, al) || misaligned(dy, al) || misaligned(dres, al) || misaligned(dx, al) ||
      misaligned(gamma, 4) || misaligned(dgamma, 4) || misaligned(work, 16))
    return bad_arg(fn, "misaligned pointer");
  const cudaStream_t st = (cudaStream_t)stream;
  const bool vec = !(misaligned(h, 16) || misaligned(dy, 16) || misaligned(dres, 16) ||
                     misaligned(dx, 16) || misaligned(gamma, 16));
  auto run = [&](auto* tag) {
    using E = std::remove_pointer_t<decltype(tag)>;
    cudaError_t e = cudaSuccess;
    int blocks = grad_blocks(T, 1, kThreads);
    if (!(vec && pick_rows<E, true>(d, [&](auto warp, auto nv, auto al, int threads) {
            constexpr bool WARP = decltype(warp)::value;
            constexpr int NV = decltype(nv)::value;
            blocks = grad_blocks(T, WARP ? kWarps : 1, threads);
            // a group with one row needs one stage
            const bool one = (long long)blocks * (WARP ? kWarps : 1) >= T;
            const size_t stage = (size_t)3 * NV * threads * 16;
            const size_t smem = std::max(one ? stage : grad_stages(NV) * stage,
                                         WARP ? (size_t)kWarps * d * 4 : 0);
            auto* kernel = rms_norm_grad_kernel<E, WARP, NV, decltype(al)::value>;
            // (per call: it holds for the current device and context, and takes less than a launch.  The
            // limit is the function's, not the call's: the largest that any of its calls needs, so
            // that calls of other threads cannot lower it before the launch)
            if (smem > 47 * 1024)
              e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       grad_smem_limit(NV));
            if (e == cudaSuccess)
              e = launch_pdl(kernel, dim3(blocks), dim3(threads), smem, st, (const E*)h, T, d,
                             gamma, (float)eps, (const E*)dy, (const E*)dres, (E*)dx,
                             (float*)work);
          })))
      e = launch_pdl(rms_norm_grad_any_kernel<E>, dim3(blocks), dim3(kThreads), 0, st, (const E*)h,
                     T, d, gamma, (float)eps, (const E*)dy, (const E*)dres, (E*)dx, (float*)work);
    if (e != cudaSuccess) return e;
    return launch_pdl(rms_norm_dgamma_kernel, dim3((d + 31) / 32), dim3(1024), 0, st,
                      (const float*)work, blocks, d, dgamma);
  };
  return launched(fn, xdtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr));
}
