// Elements of the operators' rows: fp32 and bf16, one by one and in 16-byte vectors, and e4m3 with the
// scales of their blocks.
#pragma once

#include "eat_internal.cuh"

#include <cuda_fp8.h>

namespace eat {

// e4m3 values whose largest magnitude is not above this get the scale 1 (and bytes 0): max / 448 and its
// reciprocal stay away from fp32's ends
constexpr float kTiny = 1e-35f;

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

// N elements of a row as floats: in whole 16-byte vectors (N a multiple of kN, aligned), or, where rows
// begin anywhere, one by one and S apart (so that S lanes side by side read what lies side by side); of
// the row's `left` > 0 from p on, those that do not exist read as 0 and are not written.
template <typename T, int N, bool VEC, int S = 1>
__device__ __forceinline__ void load_elems(const T* p, int left, float* v) {
  if (VEC) {
#pragma unroll
    for (int j = 0; j < N; j += Elem<T>::kN) Elem<T>::unpack(*(const uint4*)(p + j), v + j);
  } else {
    // (all loads, then their use: a load under a condition of its own would be waited for)
    T t[N];
#pragma unroll
    for (int j = 0; j < N; ++j) t[j] = p[j * S < left ? j * S : 0];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j * S < left ? Elem<T>::get(t[j]) : 0.f;
  }
}
template <typename T, int N, bool VEC, int S = 1>
__device__ __forceinline__ void store_elems(T* p, int left, const float* v) {
  if (VEC) {
#pragma unroll
    for (int j = 0; j < N; j += Elem<T>::kN) *(uint4*)(p + j) = Elem<T>::pack(v + j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j * S < left) p[j * S] = Elem<T>::put(v[j]);
  }
}
// Where lane l of S begins in a piece of S kN elements.
template <typename T, bool VEC>
__device__ __forceinline__ int lane_at(int l) {
  return VEC ? l * Elem<T>::kN : l;
}

// kN elements of a row as they were loaded (a 16-byte vector, four registers, where rows begin at
// vectors), and as floats when they are needed.
template <typename T, bool VEC, int S>
struct RowVec {
  static constexpr int kN = Elem<T>::kN;
  uint4 u;
  T f[VEC ? 1 : kN];
  int n;  // of f
  // the elements from p on, of which `left` exist; zeros if not live
  __device__ __forceinline__ void load(const T* p, int left, bool live) {
    if (VEC) {
      u = live && left > 0 ? *(const uint4*)p : make_uint4(0, 0, 0, 0);
    } else {
      n = live ? left : 0;
      if (n > 0) {
#pragma unroll
        for (int j = 0; j < kN; ++j) f[VEC ? 0 : j] = p[j * S < n ? j * S : 0];
      }
    }
  }
  __device__ __forceinline__ void get(float* v) const {
    if (VEC) {
      Elem<T>::unpack(u, v);
    } else {
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] = j * S < n ? Elem<T>::get(f[VEC ? 0 : j]) : 0.f;
    }
  }
};

// ---- e4m3 in blocks: a block's scale is its largest magnitude / 448, and a byte stands for scale times
// its value.  A block that holds an infinity has an infinite scale, so all of it reads as NaN; a NaN
// leaves the others as they are.
constexpr int kBlock = 128;  // elements of a block along its axis
constexpr long long blocks_of(long long n) { return (n + kBlock - 1) / kBlock; }

// (within 2^-23 of the quotient)
__device__ __forceinline__ float block_scale(float top) {
  return top > kTiny ? top * (1.0f / 448.0f) : 1.0f;
}
// What a block's values are divided by: its scale, and the scale's rounded reciprocal.  With both, a
// product and two fused steps give the rounded quotient (Markstein, IBM J. R&D 34, 1990), where a
// division would cost ten instructions an element, and a product alone would take values that lie between
// two e4m3 values, which quotients of bf16 values often do, to the wrong side.
struct BlockDiv {
  float scale, recip;
  __device__ __forceinline__ explicit BlockDiv(float top)
      : scale(block_scale(top)), recip(top > kTiny ? 1.0f / scale : 0.0f) {}
  __device__ __forceinline__ BlockDiv(float s, float r) : scale(s), recip(r) {}
  __device__ __forceinline__ float operator()(float v) const {
    const float t = v * recip;
    return fmaf(fmaf(-t, scale, v), recip, t);
  }
};
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t e4m3x4(const float* v) {
  return e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16;
}
// N = 4 or 8 bytes of a row.
template <int N, bool VEC, int S = 1>
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, const uint32_t* w) {
  if (VEC) {
    if (N == 8) *(uint2*)p = make_uint2(w[0], w[N / 4 - 1]);
    else *(uint32_t*)p = w[0];
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j * S < left) p[j * S] = (uint8_t)(w[j / 4] >> 8 * (j % 4));
  }
}
// The same of quotients.
template <int N, bool VEC, int S = 1>
__device__ __forceinline__ void store_e4m3(uint8_t* p, int left, const float* v) {
  uint32_t w[N / 4];
#pragma unroll
  for (int j = 0; j < N / 4; ++j) w[j] = e4m3x4(v + 4 * j);
  store_bytes<N, VEC, S>(p, left, w);
}
template <int N, bool VEC, int S = 1>
__device__ __forceinline__ void store_e4m3(uint8_t* p, int left, const float* v, const BlockDiv& div) {
  float t[N];
#pragma unroll
  for (int j = 0; j < N; ++j) t[j] = div(v[j]);
  store_e4m3<N, VEC, S>(p, left, t);
}
// Rows [lo, hi) of the experts of 32 lanes, held to be in order and apart from each other whatever the
// offsets say, so that they never add up to more than there are; before: the largest end so far.
__device__ __forceinline__ void in_order(int& lo, int& hi, int& before) {
  const int lane = threadIdx.x & 31;
  int top = hi;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, top, o);
    if (lane >= o) top = max(top, u);
  }
  const int prev = __shfl_up_sync(0xffffffffu, top, 1);
  lo = max(lo, max(before, lane > 0 ? prev : 0));
  hi = max(hi, lo);
  before = max(before, __shfl_sync(0xffffffffu, top, 31));
}
// The largest magnitude over groups of G lanes, in all of them.
template <int G>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

}  // namespace eat
