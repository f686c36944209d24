// Tensor-core kernels of the vocabulary head (head_tc.cu) and what its host side (head.cu) calls.
#pragma once

#include "eat_internal.cuh"

#include <cuda.h>
#include <cuda_fp8.h>

namespace eat {

constexpr int kHeadSmallT = 128;  // calls of up to this many tokens stream the vocabulary once
constexpr int kHeadTile = 256;    // tokens, vocabulary rows and columns of an SM pair's tile
// a partial maximum that no logit has set; finite, so that differences of it are not NaN
constexpr float kHeadLow = -3.0e38f;
// what a maximum is held to, so that a logit of +inf minus it is +inf and not NaN
constexpr float kHeadHigh = 3.402823466e38f;
// Exponentials of the gradient's pass are taken relative to the token's target logit.  A token with
// a logit more than this many powers of two above it is taken again, relative to its largest logit.
constexpr float kHeadFar = 40.0f;

// A gradient over n counted tokens, 1 <= n <= 128, multiplies X' in two bf16 parts: the tokens' rows
// come a second time head_lo(n) rows further, where X' holds what its first part left over.  (A row of
// dW often is one token's; with one part it would carry two roundings, and the second costs nothing
// where a tile of 256 rows, and for 32 tokens a k-block of 64, is there anyway.)
__host__ __device__ __forceinline__ int head_lo(int n) {
  return n < 1 || n > 128 ? 0 : n <= 32 ? 32 : n <= 64 ? 64 : 128;
}
__host__ __device__ __forceinline__ int head_rows(int n) { return n + head_lo(n); }

struct HeadStatus {
  unsigned int* err;     // device status word
  unsigned int* mirror;  // device address of its host-mapped copy
  unsigned long long limit_ns;  // of a kernel's wait
};

// Loss of up to kHeadSmallT tokens.  part: each CTA's maximum and sum of exp2 relative to it of the base-2
// logits of its vocabulary rows, without the targets, per column; ly[t] the base-2 target logit.  With
// few columns the CTA that takes the last ticket joins them (tickets: a word that is 0 between calls),
// else part is [CTA][column] for the kernel that does.
struct HeadSmallArgs {
  int T, V, d, kblocks;
  const int32_t* target;
  const void* x;    // the matrices themselves, for the target logits
  const void* w;
  const float* xs;  // e4m3: [T]
  const float* ws;  // e4m3: [V]
  float2* part;
  float* ly;
  unsigned int* tickets;
  float* nll;
  float* lse;       // or null
  HeadStatus st;
};
int head_small_n(int T);
bool head_small_joins(int n);  // the kernel of n columns writes nll and lse itself
int head_small_ctas(int num_sms, int V);
cudaError_t head_launch_small(bool w8, const CUtensorMap& w128, const CUtensorMap& w16,
                              const CUtensorMap& x, const HeadSmallArgs& a, int ctas,
                              cudaStream_t st);

// Loss of more tokens (exp == false): part2[128-row piece of the vocabulary][T] as above, ly[t] the
// base-2 target logit.  Gradient's first pass (exp == true): e[row][v] = exp2(l - ref) as bf16 (0 in
// the target's column, beyond V and in rows beyond the counted tokens), part[piece][cap] its sums.
struct HeadPairArgs {
  int T, V, d, kblocks;
  const int32_t* target;
  const void* x;  // exp == false: the matrices themselves, for the target logits
  const void* w;
  const float* xs;
  const float* ws;
  float2* part2;
  float* ly;
  // gradient's first pass, over the counted tokens [t0, t0 + cap)
  const int32_t* n_counted;  // device
  int t0, cap, ld;
  const float* ref;          // [tokens] base-2 target logits
  uint32_t* row_max;         // [tokens] ordered bits of a far token's largest base-2 logit, or 0
  int32_t* far;              // [tiles] a token of the tile is far
  int redo;                  // only the tiles with far tokens, relative to their largest logits
  float* part;
  __nv_bfloat16* e;
  HeadStatus st;
};
cudaError_t head_launch_pair(bool w8, bool exp, const CUtensorMap& x, const CUtensorMap& w,
                             const HeadPairArgs& a, int max_pairs, cudaStream_t st);

// dx = f (E W) and dW = E^T X of the counted tokens [t0, t0 + cap): both products' tiles in one
// launch.  Pieces of tokens after the first add to dw_sum; the last one rounds.
struct HeadGradArgs {
  int V, d;
  const int32_t* n_counted;
  int t0, cap;
  const float* f;        // [tokens] factors of the rows of dx
  const int32_t* rows;   // [tokens] rows of dx
  __nv_bfloat16* dx;
  __nv_bfloat16* dw;
  float* dw_sum;         // [V, d], or null when one piece holds every token
  int slices;            // of dx's sums over the vocabulary
  float* dx_part;        // slices > 1: [slice][cap][d] unscaled sums instead of dx
  HeadStatus st;
};
// Slices of dx's sums for a piece of cap tokens (a multiple of kHeadTile).
int head_dx_slices(int cap, int V, int d, int max_pairs);
cudaError_t head_launch_grad(const CUtensorMap& e, const CUtensorMap& w, const CUtensorMap& x,
                             const HeadGradArgs& a, int max_pairs, cudaStream_t st);

// The kernels' shared-memory limits on the current device, and the SM pairs that can be resident.
cudaError_t head_configure(int num_sms, int* max_pairs);
// Row-major [rows, cols] matrix in boxes of box_rows rows of 128 bytes, 128-byte swizzle, zeros
// outside.
bool head_encode(CUtensorMap* m, bool w8, const void* ptr, long long rows, long long cols,
                 int box_rows);

// 16 bytes of a row as floats: 8 bf16 or 16 e4m3
template <bool W8>
struct Vec {
  static constexpr int kN = W8 ? 16 : 8;
  float v[kN];
  __device__ explicit Vec(uint4 u) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (W8) {
        __nv_fp8x4_e4m3 q;
        q.__x = w[i];
        const float4 f = (float4)q;
        v[4 * i] = f.x;
        v[4 * i + 1] = f.y;
        v[4 * i + 2] = f.z;
        v[4 * i + 3] = f.w;
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
};
template <bool W8>
__device__ __forceinline__ float dot16(uint4 a, uint4 b, float s) {
  const Vec<W8> x(a), w(b);
#pragma unroll
  for (int i = 0; i < Vec<W8>::kN; ++i) s = fmaf(x.v[i], w.v[i], s);
  return s;
}

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// nll and lse of a token from the base-2 target logit and the sum of the others' exp2 relative to m
__device__ __forceinline__ float2 token_loss(float m, float s, float ly) {
  const float r = (m - ly + log2f(s)) * kLn2;
  float a = fmaxf(r, 0.f) + log1pf(expf(-fabsf(r)));
  if (isnan(r)) a = r;
  // (a target of logit -inf: the others' sum alone)
  return make_float2(a, ly == -INFINITY ? (m + log2f(s)) * kLn2 : fmaf(ly, kLn2, a));
}

// Ordered bits of a float: larger floats have larger bits, and no float has 0 (other than NaNs).
__device__ __forceinline__ uint32_t ordered_bits(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
// What a token's exponentials are relative to.
__device__ __forceinline__ float head_ref(float ref, uint32_t row_max) {
  return row_max ? from_ordered(row_max) : ref;
}

}  // namespace eat
