// Load-balancing loss of a router with per-expert counts, and its gradient to the logits.
//   counts[e] = entries of idx equal to e;  f_e = counts[e] / sum counts;  p_t = softmax(logits_t)
//   loss = E sum_e f_e (1/n) sum_t p_te;   dlogits_te = g E / n p_te (f_e - sum_j f_j p_tj)
// Bound: latency (a router's logits are a few MB at most, which L2 holds).  A warp takes kTok tokens
// at a time, lane l the experts l, l + 32, ..., so that the tokens' loads and shuffles overlap.
// Counts are integers (shared-memory atomics, any order gives the same); probabilities are summed in
// fp32 in a fixed order: a lane over its warp's tokens, the block's warps, then the blocks.
#include "op_checks.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

namespace eat {

namespace {

constexpr int kMaxTokens = 1 << 26;  // times 16 selections: counts stay within an int
constexpr int kTok = 4;
constexpr int kWarps = 16;
constexpr int kThreads = 32 * kWarps;
constexpr int kCluster = 8;
// Calls of up to kOneBlockT tokens run in one block and up to kOneClusterT in one cluster, whose
// blocks add up in shared memory: one launch and no sums in memory, 6.4 us of the host a call, as long
// as the device takes no more (512 x 64: 4.7 us; 2000 x 64: 9.4).  Larger ones are joined by a second
// launch: 8.4 us of the host (device: 2000 x 64 4.7, 16384 x 64 8.6; in clusters, joined twice, 12.0).
constexpr int kOneBlockT = kWarps * kTok;
constexpr int kOneClusterT = 1024;
constexpr int kMaxBlocks = 304;  // two per SM

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// softmax of the tokens t0 .. t0 + kTok - 1 (those for which on[k]; others: all zeros)
// (expf: with __expf probabilities of exp(-60) were off by 22 x 2^-23 of themselves; the call takes 0.1 us
// longer.  Quotients instead of the reciprocal's products: 1 to 3 us more.)
template <int PER>
__device__ __forceinline__ void softmax_rows(const float* logits, long long t0, int E, int lane,
                                             const bool (&on)[kTok], float (&p)[kTok][PER]) {
#pragma unroll
  for (int k = 0; k < kTok; ++k)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = i * 32 + lane;
      p[k][i] = on[k] && e < E ? logits[(t0 + k) * E + e] : -INFINITY;
    }
  float m[kTok], s[kTok];
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    m[k] = p[k][0];
#pragma unroll
    for (int i = 1; i < PER; ++i) m[k] = fmaxf(m[k], p[k][i]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < kTok; ++k) m[k] = fmaxf(m[k], __shfl_xor_sync(0xffffffffu, m[k], o));
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    s[k] = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      p[k][i] = on[k] && i * 32 + lane < E ? expf(p[k][i] - m[k]) : 0.f;
      s[k] += p[k][i];
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < kTok; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
#pragma unroll
  for (int k = 0; k < kTok; ++k) {
    s[k] = on[k] ? 1.0f / s[k] : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) p[k][i] *= s[k];
  }
}

// loss, counts and the number of counted tokens from the sums of a block's threads: thread e < E
// has expert e's sum of p and count, n the counted tokens
__device__ void write_loss(float s, int c, int n, int E, float* loss, int32_t* counts,
                           int32_t* n_tokens) {
  __shared__ float2 red[kMaxExperts / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((int)threadIdx.x < E) counts[threadIdx.x] = c;
  const float a = warp_sum(s * (float)c), b = warp_sum((float)c);
  if (lane == 0 && warp < kMaxExperts / 32) red[warp] = make_float2(a, b);
  __syncthreads();
  if (threadIdx.x == 0) {
    float x = 0.f, y = 0.f;
    for (int i = 0; i < kMaxExperts / 32; ++i) {
      x += red[i].x;
      y += red[i].y;
    }
    *loss = y > 0.f ? (float)E * x / (y * (float)n) : 0.f;
    *n_tokens = n;
  }
}

// A launch of one cluster writes the call's results; with blocks of their own, block b leaves its sums
// in psum[b][E] and cnt[b][E + 1] (the last: the tokens counted).
template <int PER>
__global__ void __launch_bounds__(kThreads)
balance_sum_kernel(const float* __restrict__ logits, int T, int E, int K,
                   const int32_t* __restrict__ idx, const uint8_t* __restrict__ mask,
                   float* __restrict__ psum, int32_t* __restrict__ cnt, float* __restrict__ loss,
                   int32_t* __restrict__ counts, int32_t* __restrict__ n_tokens) {
  namespace cg = cooperative_groups;
  __shared__ int s_cnt[kMaxExperts + 1];
  __shared__ float s_p[kWarps][32 * PER];
  __shared__ float s_sum[32 * PER];
  const cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks();
  pdl_wait();
  pdl_launch_dependents();
  for (int i = threadIdx.x; i <= E; i += kThreads) s_cnt[i] = 0;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float acc[PER] = {};
  for (long long t0 = (long long)(blockIdx.x * kWarps + warp) * kTok; t0 < T;
       t0 += (long long)gridDim.x * kWarps * kTok) {
    bool on[kTok];
    int e[kTok];
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      on[k] = t0 + k < T && !(mask && !mask[t0 + k]);
      e[k] = on[k] && lane < K ? idx[(t0 + k) * K + lane] : -1;
    }
    float p[kTok][PER];
    softmax_rows<PER>(logits, t0, E, lane, on, p);
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
#pragma unroll
      for (int i = 0; i < PER; ++i) acc[i] += p[k][i];
      if (e[k] >= 0 && e[k] < E) atomicAdd(&s_cnt[e[k]], 1);
    }
    if (lane == 0) atomicAdd(&s_cnt[E], (int)on[0] + (int)on[1] + (int)on[2] + (int)on[3]);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) s_p[warp][i * 32 + lane] = acc[i];
  __syncthreads();
  const int e = threadIdx.x;
  if (e < 32 * PER) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += s_p[w][e];
    s_sum[e] = s;
  }
  cluster.sync();
  if (cluster.block_rank() == 0) {
    float s = 0.f;
    int c = 0, n = 0;
#pragma unroll
    for (int r = 0; r < kCluster; ++r) {
      if (r >= blocks) break;
      const int* rc = cluster.map_shared_rank(s_cnt, r);
      if (e < E) {
        s += cluster.map_shared_rank(s_sum, r)[e];
        c += rc[e];
      }
      n += rc[E];
    }
    if ((int)gridDim.x == blocks) {
      write_loss(s, c, n, E, loss, counts, n_tokens);
    } else {
      if (e < E) {
        psum[(size_t)blockIdx.x * E + e] = s;
        cnt[(size_t)blockIdx.x * (E + 1) + e] = c;
      }
      if (e == 0) cnt[(size_t)blockIdx.x * (E + 1) + E] = n;
    }
  }
  cluster.sync();  // no block leaves while another reads its sums
}

// The blocks' sums joined: a warp takes every 32nd block, its lanes the experts.
constexpr int kJoinWarps = 32;
template <int PER>
__global__ void __launch_bounds__(32 * kJoinWarps)
balance_join_kernel(const float* __restrict__ psum, const int32_t* __restrict__ cnt, int parts,
                    int E, float* __restrict__ loss, int32_t* __restrict__ counts,
                    int32_t* __restrict__ n_tokens) {
  __shared__ float s_p[kJoinWarps][32 * PER];
  __shared__ int s_cnt[32 * PER], s_n;
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < 32 * PER) s_cnt[threadIdx.x] = 0;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  float s[PER] = {};
  int c[PER] = {}, n = 0;
#pragma unroll 5
  for (int b = warp; b < parts; b += kJoinWarps) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = i * 32 + lane;
      if (e < E) {
        s[i] += psum[(size_t)b * E + e];
        c[i] += cnt[(size_t)b * (E + 1) + e];
      }
    }
    if (lane == 0) n += cnt[(size_t)b * (E + 1) + E];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    s_p[warp][i * 32 + lane] = s[i];
    if (c[i]) atomicAdd(&s_cnt[i * 32 + lane], c[i]);
  }
  if (lane == 0) atomicAdd(&s_n, n);
  __syncthreads();
  float sum = 0.f;
  if ((int)threadIdx.x < E) {
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += s_p[w][threadIdx.x];
  }
  write_loss(sum, (int)threadIdx.x < E ? s_cnt[threadIdx.x] : 0, s_n, E, loss, counts, n_tokens);
}

template <int PER>
__global__ void __launch_bounds__(kThreads)
balance_grad_kernel(const float* logits, int T, int E, const uint8_t* __restrict__ mask,
                    const int32_t* __restrict__ counts, const int32_t* __restrict__ n_tokens,
                    const float* __restrict__ g, float* dlogits) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float f[PER], total = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    f[i] = i * 32 + lane < E ? (float)counts[i * 32 + lane] : 0.f;
    total += f[i];
  }
  total = warp_sum(total);
  const float scale = total > 0.f ? *g * (float)E / (float)*n_tokens : 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) f[i] = total > 0.f ? f[i] / total : 0.f;
  for (long long t0 = (long long)(blockIdx.x * kWarps + warp) * kTok; t0 < T;
       t0 += (long long)gridDim.x * kWarps * kTok) {
    bool on[kTok];
#pragma unroll
    for (int k = 0; k < kTok; ++k)
      on[k] = t0 + k < T && total > 0.f && !(mask && !mask[t0 + k]);
    float p[kTok][PER], dot[kTok];
    softmax_rows<PER>(logits, t0, E, lane, on, p);
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      dot[k] = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) dot[k] = fmaf(f[i], p[k][i], dot[k]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < kTok; ++k) dot[k] += __shfl_xor_sync(0xffffffffu, dot[k], o);
#pragma unroll
    for (int k = 0; k < kTok; ++k)
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (t0 + k < T && i * 32 + lane < E)
          dlogits[(t0 + k) * E + i * 32 + lane] = on[k] ? scale * p[k][i] * (f[i] - dot[k]) : 0.f;
  }
}

int blocks_for(int T) {
  return (int)std::min(((long long)T + kOneBlockT - 1) / kOneBlockT, (long long)kMaxBlocks);
}

// go(PER): experts per lane
template <typename F>
cudaError_t pick_per(int E, F&& go) {
  if (E <= 32) return go(std::integral_constant<int, 1>());
  if (E <= 64) return go(std::integral_constant<int, 2>());
  if (E <= 128) return go(std::integral_constant<int, 4>());
  return go(std::integral_constant<int, 8>());
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" int64_t eat_balance_workspace(int32_t T, int32_t E) {
  if (T < 1 || E < 1) return 0;
  return T <= kOneClusterT ? 16 : (int64_t)blocks_for(T) * (2 * E + 1) * 4;
}

extern "C" eat_status eat_balance_loss(const float* logits, int32_t T, int32_t E, int32_t K,
                                       const int32_t* idx, const uint8_t* mask, float* loss,
                                       int32_t* counts, int32_t* n_tokens, void* work,
                                       void* stream) {
  const char* fn = "eat_balance_loss";
  if (!logits || !idx || !loss || !counts || !n_tokens || !work)
    return bad_arg(fn, "logits, idx, loss, counts, n_tokens and work must be non-NULL");
  if (T < 1 || T > kMaxTokens || E < 1 || E > kMaxExperts || K < 1 || K > kMaxK)
    return bad_arg(fn, "need T >= 1, T <= 2^26, 1 <= E <= 256 and 1 <= K <= 16");
  if (misaligned(logits, 4) || misaligned(idx, 4) || misaligned(loss, 4) ||
      misaligned(counts, 4) || misaligned(n_tokens, 4) || misaligned(work, 16))
    return bad_arg(fn, "misaligned pointer");
  const cudaStream_t st = (cudaStream_t)stream;
  const bool one = T <= kOneClusterT;
  const int cluster = one && T > kOneBlockT ? kCluster : 1, blocks = one ? cluster : blocks_for(T);
  float* psum = (float*)work;
  int32_t* cnt = (int32_t*)(psum + (size_t)blocks * E);
  return launched(fn, pick_per(E, [&](auto per) {
    constexpr int PER = decltype(per)::value;
    const cudaError_t e =
        launch_pdl_cluster(balance_sum_kernel<PER>, dim3(blocks), cluster, dim3(kThreads), 0, st,
                           logits, T, E, K, idx, mask, psum, cnt, loss, counts, n_tokens);
    if (e != cudaSuccess || one) return e;
    return launch_pdl(balance_join_kernel<PER>, dim3(1), dim3(32 * kJoinWarps), 0, st,
                      (const float*)psum, (const int32_t*)cnt, blocks, E, loss, counts, n_tokens);
  }));
}

extern "C" eat_status eat_balance_grad(const float* logits, int32_t T, int32_t E,
                                       const uint8_t* mask, const int32_t* counts,
                                       const int32_t* n_tokens, const float* g, float* dlogits,
                                       void* stream) {
  const char* fn = "eat_balance_grad";
  if (!logits || !counts || !n_tokens || !g || !dlogits)
    return bad_arg(fn, "logits, counts, n_tokens, g and dlogits must be non-NULL");
  if (T < 1 || T > kMaxTokens || E < 1 || E > kMaxExperts)
    return bad_arg(fn, "need T >= 1, T <= 2^26 and 1 <= E <= 256");
  if (misaligned(logits, 4) || misaligned(counts, 4) || misaligned(n_tokens, 4) ||
      misaligned(g, 4) || misaligned(dlogits, 4))
    return bad_arg(fn, "misaligned pointer");
  return launched(fn, pick_per(E, [&](auto per) {
    return launch_pdl(balance_grad_kernel<decltype(per)::value>, dim3(blocks_for(T)),
                      dim3(kThreads), 0, (cudaStream_t)stream, logits, T, E, mask, counts, n_tokens,
                      g, dlogits);
  }));
}
