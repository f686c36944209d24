// Tokens sorted by expert and back (what a layer's experts read and what becomes of their rows), and
// the gradients of both.
//   sort:    offsets[e] = number of selections of experts below e; slot[t][k] = the row of selection
//            (t, k), rows of an expert in the selections' order (t, then k); -1 where there is none
//   gather:  rows[slot[t][k]] = x[t], in x's type or in e4m3 with a scale for each 128 elements
//   combine: y[t] = sum_k w[t][k] rows[slot[t][k]]  (w = 1: the gradient of gather)
//   combine's gradient: drows[slot[t][k]] = w[t][k] dy[t];  dw[t][k] = <dy[t], rows[slot[t][k]]>
// Bound: HBM; the sort itself: latency.  The copies go by token: a row of x (or dy) is read once and
// written to all of its slots.  Rows behind the last selection are written as zeros by the same warps:
// token t takes the t-th of them and every T-th further, at most K.  All sums are fp32, in the order of
// k and of the lanes, so the same inputs give the same bits; a value is rounded when it is stored.
#include "elem.cuh"
#include "op_checks.cuh"
#include "tc_ptx.cuh"

#include <algorithm>
#include <type_traits>

namespace eat {

namespace {

// ------------------------------------------------------------------------------------- sort
// A block sorts a chunk of consecutive selections; a warp takes PER times 32 of them in order and
// counts per expert as it goes (lanes of the same expert find each other by __match_any_sync), so a
// selection's row is its expert's first + the chunks' and warps' before + its rank in the warp.
constexpr int kSortThreads = 1024;
constexpr int kSortCtas = 8;   // of a cluster
constexpr int kPer = 8;        // of a chunk of the calls that no cluster holds
constexpr int kChunkLen = kSortThreads * kPer;
constexpr int kClusterMost = kSortCtas * kSortThreads * 16;

// kCluster: the launch's one cluster holds all selections.  Otherwise chunk[c][e]: kCount writes the
// chunks' counts, kAssign reads the sums of the chunks before, and total[e].
enum : int { kCluster = 0, kCount = 1, kAssign = 2 };

template <int MODE, int PER>
__global__ void __launch_bounds__(kSortThreads)
sort_kernel(const int32_t* __restrict__ idx, int n, int K, int E, const uint8_t* __restrict__ mask,
            int32_t* chunk, const int32_t* __restrict__ total, int32_t* __restrict__ offsets,
            int32_t* __restrict__ slot) {
  extern __shared__ int s_cnt[];  // [warps][E], then [E] first rows, [E] this CTA's counts
  __shared__ int s_sum[kMaxExperts / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
  int* const s_base = s_cnt + warps * E;
  int* const s_mine = s_base + E;
  for (int i = tid; i < warps * E; i += blockDim.x) s_cnt[i] = 0;
  pdl_wait();
  pdl_launch_dependents();
  const int first = (blockIdx.x * warps + warp) * 32 * PER + lane;
  int ex[PER], rank[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = first + 32 * i;
    int e = at < n ? idx[at] : -1;
    if (mask && at < n && !mask[at / K]) e = -1;
    ex[i] = e >= 0 && e < E ? e : -1;
  }
  __syncthreads();
  int* const mine = s_cnt + warp * E;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const unsigned same = __match_any_sync(0xffffffffu, ex[i]);
    const int below = __popc(same & ((1u << lane) - 1u));
    int c = 0;
    if (ex[i] >= 0) c = mine[ex[i]];
    rank[i] = c + below;
    __syncwarp();
    if (ex[i] >= 0 && below == 0) mine[ex[i]] = c + __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = tid; e < E; e += blockDim.x) {
    int sum = 0;
    for (int w0 = 0; w0 < warps; w0 += 8) {
      int c[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) c[w] = w0 + w < warps ? s_cnt[(w0 + w) * E + e] : 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        if (w0 + w < warps) s_cnt[(w0 + w) * E + e] = sum;
        sum += c[w];
      }
    }
    if (MODE == kCount) chunk[(size_t)blockIdx.x * E + e] = sum;
    s_mine[e] = sum;
  }
  if (MODE == kCount) return;
  int before = 0;  // expert tid's: in the CTAs or chunks before this one
  int all = 0;
  if (MODE == kCluster) {
    if (gridDim.x > 1) ptx::cluster_sync_all();
    else __syncthreads();
    if (tid < E) {
      if (gridDim.x == 1) {
        all = s_mine[tid];
      } else {
        int c[kSortCtas];
#pragma unroll
        for (int r = 0; r < kSortCtas; ++r) {
          c[r] = 0;
          if (r < (int)gridDim.x)
            asm volatile("ld.shared::cluster.s32 %0, [%1];"
                         : "=r"(c[r])
                         : "r"(ptx::map_rank(ptx::smem_u32(s_mine + tid), (uint32_t)r)));
        }
#pragma unroll
        for (int r = 0; r < kSortCtas; ++r) {
          if (r < (int)blockIdx.x) before += c[r];
          all += c[r];
        }
      }
    }
    // (no CTA leaves while another may still read its counts)
    if (gridDim.x > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  } else if (tid < E) {
    all = total[tid];
    before = chunk[(size_t)blockIdx.x * E + tid];
  }
  // first rows of the experts: scans of 32 of them, then of those sums (a block has at least E threads,
  // or 256)
  int v = all;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  if (lane == 31 && warp < kMaxExperts / 32) s_sum[warp] = v;
  __syncthreads();
  if (tid < E) {
    int at = v - all;
    for (int w = 0; w < warp; ++w) at += s_sum[w];
    s_base[tid] = at + before;
    if (blockIdx.x == 0) {
      offsets[tid] = at;
      if (tid == E - 1) offsets[E] = at + all;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = first + 32 * i;
    if (at < n) slot[at] = ex[i] < 0 ? -1 : s_base[ex[i]] + mine[ex[i]] + rank[i];
  }
  if (MODE == kCluster && gridDim.x > 1)
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A warp per expert: chunk[c][e] becomes the sum of the chunks before c, total[e] the sum of all.
__global__ void __launch_bounds__(32) sort_scan_kernel(int32_t* chunk, int chunks, int E,
                                                       int32_t* __restrict__ total) {
  pdl_wait();
  pdl_launch_dependents();
  const int e = blockIdx.x, lane = threadIdx.x;
  int before = 0;
  for (int b = 0; b < chunks; b += 32) {
    const int at = b + lane;
    const int c = at < chunks ? chunk[(size_t)at * E + e] : 0;
    int v = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    if (at < chunks) chunk[(size_t)at * E + e] = before + v - c;
    before += __shfl_sync(0xffffffffu, v, 31);
  }
  if (lane == 0) total[e] = before;
}

// ------------------------------------------------------------------------------ there and back
constexpr int kWarps = 8;  // of a block whose warps take pieces of tokens
constexpr int kLoads = 4;  // vectors of a lane at a time

// Rows behind the last selection, as offsets says (any value is held to the buffer).
__device__ __forceinline__ int rows_used(const int32_t* offsets, int E, int rows) {
  return max(0, min(offsets[E], rows));
}

// V: what a row is copied in (16 bytes where the rows begin at multiples of it, else less).
template <typename V>
__global__ void __launch_bounds__(32 * kWarps)
gather_kernel(const V* __restrict__ x, const int32_t* __restrict__ slot,
              const int32_t* __restrict__ offsets, int T, int K, int E, int len, int pieces,
              V* __restrict__ rows) {
  pdl_wait();
  pdl_launch_dependents();
  const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, t = (int)(w / pieces), c0 = (int)(w % pieces) * 32 * kLoads;
  if (t >= T) return;
  const int M = T * K, used = rows_used(offsets, E, M);
  const int mine = lane < K ? slot[(size_t)t * K + lane] : -1;
  V v[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int c = c0 + 32 * i + lane;
    if (c < len) v[i] = x[(size_t)t * len + c];
  }
  for (int k = 0; k < K; ++k) {
    const int r = __shfl_sync(0xffffffffu, mine, k);
    if (r < 0 || r >= M) continue;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = c0 + 32 * i + lane;
      if (c < len) rows[(size_t)r * len + c] = v[i];
    }
  }
  for (long long r = (long long)used + t; r < M; r += T) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = c0 + 32 * i + lane;
      if (c < len) rows[(size_t)r * len + c] = V{};
    }
  }
}

// The same in e4m3: a block of 128 elements is taken by as many lanes as it has 16-byte vectors.
template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kWarps)
gather_fp8_kernel(const T* __restrict__ x, const int32_t* __restrict__ slot,
                  const int32_t* __restrict__ offsets, int tokens, int K, int E, int d, int pieces,
                  uint8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int N = Elem<T>::kN, G = kBlock / N, U = 2;
  pdl_wait();
  pdl_launch_dependents();
  const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, t = (int)(w / pieces);
  const int c0 = (int)(w % pieces) * 32 * N * U + lane / G * kBlock + lane_at<T, VEC>(lane % G);
  if (t >= tokens) return;
  const int M = tokens * K, used = rows_used(offsets, E, M);
  const int mine = lane < K ? slot[(size_t)t * K + lane] : -1;
  float v[U][N], s[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = c0 + 32 * N * i;
    float top = 0.f;
    if (c < d) load_elems<T, N, VEC, G>(x + (size_t)t * d + c, d - c, v[i]);
    if (c < d)
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(v[i][j]));
    top = group_max<G>(top);
    const BlockDiv div(top);
    s[i] = div.scale;
#pragma unroll
    for (int j = 0; j < N; ++j) v[i][j] = div(v[i][j]);
  }
  for (int k = 0; k < K; ++k) {
    const int r = __shfl_sync(0xffffffffu, mine, k);
    if (r < 0 || r >= M) continue;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = c0 + 32 * N * i;
      if (c >= d) continue;
      store_e4m3<N, VEC, G>(q + (size_t)r * d + c, d - c, v[i]);
      if (lane % G == 0) scale[(size_t)(c / kBlock) * M + r] = s[i];
    }
  }
  const float zero[N] = {};
  for (long long r = (long long)used + t; r < M; r += tokens) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = c0 + 32 * N * i;
      if (c >= d) continue;
      store_e4m3<N, VEC, G>(q + (size_t)r * d + c, d - c, zero);
      if (lane % G == 0) scale[(size_t)(c / kBlock) * M + r] = 1.0f;
    }
  }
}

// y[t]: a warp takes a vector a lane of one token at a time, the loads of kAhead rows before their use, and
// loads the next token's slots meanwhile.  Bound: HBM (8191 tokens x 8 of 2048 bf16: 33 us, 5.2 TB/s; with
// eight rows ahead 41, with two vectors a lane 36, as fewer warps fit).
constexpr int kAhead = 4;          // rows
constexpr int kCombineBlocks = 4;  // of an SM
template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kWarps, VEC ? kCombineBlocks : 1)
combine_kernel(const T* __restrict__ rows, const int32_t* __restrict__ slot,
               const float* __restrict__ weight, int tokens, int K, int d, int pieces,
               T* __restrict__ y) {
  constexpr int N = Elem<T>::kN;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, M = tokens * K;
  // units of (token, piece of its row), and the step between a warp's
  const long long first = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int step = gridDim.x * kWarps, dt = step / pieces, dp = step - dt * pieces;
  int nt = (int)(first / pieces), np = (int)(first - (long long)nt * pieces);
  int next = -1;
  float next_wt = 1.0f;
  auto prefetch = [&] {
    next = -1;
    if (nt < tokens && lane < K) {
      const size_t at = (size_t)nt * K + lane;
      next = slot[at];
      if (weight) next_wt = weight[at];
    }
  };
  prefetch();
  while (nt < tokens) {
    const int mine = next < M ? next : -1, t = nt;
    const int c = np * (32 * N) + lane_at<T, VEC>(lane), left = d - c;
    const float wt = next_wt;
    nt += dt;
    np += dp;
    if (np >= pieces) {
      np -= pieces;
      ++nt;
    }
    prefetch();
    float sum[N] = {};
    for (int k0 = 0; k0 < K; k0 += kAhead) {
      RowVec<T, VEC, 32> in[kAhead];
      int r[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        r[k] = __shfl_sync(0xffffffffu, mine, (k0 + k) & 31);
        in[k].load(rows + (size_t)max(r[k], 0) * d + c, left, r[k] >= 0);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float f = __shfl_sync(0xffffffffu, wt, (k0 + k) & 31);
        if (r[k] < 0) continue;
        float v[N];
        in[k].get(v);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = fmaf(f, v[j], sum[j]);
      }
    }
    if (left > 0) store_elems<T, N, VEC, 32>(y + (size_t)t * d + c, left, sum);
  }
}

// A block takes a token: its warps share the row, and add their parts of dw in their order.
template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kWarps)
combine_grad_kernel(const T* __restrict__ dy, const T* __restrict__ rows,
                    const int32_t* __restrict__ slot, const int32_t* __restrict__ offsets,
                    const float* __restrict__ weight, int tokens, int K, int E, int d,
                    T* __restrict__ drows, float* __restrict__ dw) {
  constexpr int N = Elem<T>::kN;
  __shared__ float s_part[kWarps][kMaxK];
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int M = tokens * K, used = rows_used(offsets, E, M);
  int mine = lane < K ? slot[(size_t)t * K + lane] : -1;
  if (mine >= M) mine = -1;
  const float wt = lane < K ? weight[(size_t)t * K + lane] : 0.f;
  float part = 0.f;  // lane k's: the warp's part of dw[t][k]
  for (int k0 = 0; k0 < K; k0 += kAhead) {
    float dot[kAhead] = {};
    for (int c0 = warp * 32 * N; c0 < d; c0 += blockDim.x * N) {
      const int c = c0 + lane_at<T, VEC>(lane), left = d - c;
      RowVec<T, VEC, 32> own, in[kAhead];
      int r[kAhead];
      own.load(dy + (size_t)t * d + c, left, true);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        r[k] = __shfl_sync(0xffffffffu, mine, (k0 + k) & 31);
        in[k].load(rows + (size_t)max(r[k], 0) * d + c, left, r[k] >= 0);
      }
      float g[N];
      own.get(g);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float f = __shfl_sync(0xffffffffu, wt, (k0 + k) & 31);
        if (r[k] < 0 || left <= 0) continue;
        float v[N], o[N];
        in[k].get(v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          dot[k] = fmaf(g[j], v[j], dot[k]);
          o[j] = f * g[j];
        }
        store_elems<T, N, VEC, 32>(drows + (size_t)r[k] * d + c, left, o);
      }
      if (k0 == 0 && left > 0) {
        const float zero[N] = {};
        for (long long r = (long long)used + t; r < M; r += tokens)
          store_elems<T, N, VEC, 32>(drows + (size_t)r * d + c, left, zero);
      }
    }
    // lanes exchange the halves that they do not keep: lane l ends with the sum of the (l % kAhead)-th
#pragma unroll
    for (int h = kAhead / 2; h > 0; h >>= 1) {
      const bool upper = lane & h;
#pragma unroll
      for (int i = 0; i < h; ++i) {
        const float give = upper ? dot[i] : dot[i + h], keep = upper ? dot[i + h] : dot[i];
        dot[i] = keep + __shfl_xor_sync(0xffffffffu, give, h);
      }
    }
#pragma unroll
    for (int o = kAhead; o < 32; o <<= 1) dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], o);
    if (lane / kAhead == k0 / kAhead) part = dot[0];
  }
  if (lane < K) s_part[warp][lane] = part;
  __syncthreads();
  if (threadIdx.x < K) {
    float s = 0.f;
    for (int i = 0; i < (int)blockDim.x / 32; ++i) s += s_part[i][threadIdx.x];
    dw[(size_t)t * K + threadIdx.x] = s;
  }
}

int sort_chunks(int n) { return (n + kChunkLen - 1) / kChunkLen; }
dim3 warp_grid(long long warps) { return dim3((unsigned)((warps + kWarps - 1) / kWarps)); }

// What the calls on sorted rows have in common; empty when they may go on.
const char* bad_rows(int32_t T, int32_t K, int32_t E, int32_t d, int32_t dtype) {
  if (T < 1 || K < 1 || K > kMaxK || (long long)T * K > 1 << 30)
    return "need T >= 1, 1 <= K <= 16 and T K <= 2^30";
  if (E < 1 || E > kMaxExperts) return "need 1 <= E <= 256";
  if (d < 1 || d > 65536) return "need 1 <= d <= 65536";
  if (dtype != EAT_F32 && dtype != EAT_BF16) return "dtype must be F32 or BF16";
  return nullptr;
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" int64_t eat_expert_sort_workspace(int32_t T, int32_t K, int32_t E) {
  if (T < 1 || K < 1 || K > kMaxK || E < 1 || E > kMaxExperts || (long long)T * K > 1 << 30) return 0;
  return T * K <= kClusterMost ? 0 : (int64_t)(sort_chunks(T * K) + 1) * E * 4;
}

extern "C" eat_status eat_expert_sort(const int32_t* idx, int32_t T, int32_t K, int32_t E,
                                      const uint8_t* mask, int32_t* offsets, int32_t* slot,
                                      void* work, void* stream) {
  const char* fn = "eat_expert_sort";
  if (!idx || !offsets || !slot) return bad_arg(fn, "idx, offsets and slot must be non-NULL");
  if (const char* why = bad_rows(T, K, E, 1, EAT_F32)) return bad_arg(fn, why);
  if (!work && eat_expert_sort_workspace(T, K, E) > 0) return bad_arg(fn, "a call of this size needs work");
  if (misaligned(idx, 4) || misaligned(offsets, 4) || misaligned(slot, 4) || misaligned(work, 16))
    return bad_arg(fn, "misaligned pointer");
  const size_t bytes_n = 4 * (size_t)T * K;
  if (overlaps({{offsets, 4 * (size_t)(E + 1)},
                {slot, bytes_n},
                {work, (size_t)eat_expert_sort_workspace(T, K, E)}},
               {{idx, bytes_n}, {mask, (size_t)T}}))
    return bad_arg(fn, "an output or work overlaps another array");
  const cudaStream_t st = (cudaStream_t)stream;
  const int n = T * K, chunks = sort_chunks(n);
  auto smem = [&](int threads) { return (size_t)(threads / 32 + 2) * E * 4; };  // at most 35 KB
  if (n <= kClusterMost) {
    // One launch.  Two selections a thread in as many CTAs as that takes, up to a cluster's; more of them
    // only where it holds no more threads (65528 selections of 64 experts: 10.5 us, 25 in the three launches
    // that larger calls take)
    const int per = n <= 2 * kSortCtas * kSortThreads ? 2 : n <= 8 * kSortCtas * kSortThreads ? 8 : 16;
    const int ctas = (n + per * kSortThreads - 1) / (per * kSortThreads);
    // (a small call's block has no warps that only add to its sums, but a thread for each expert)
    const int need = ctas > 1 ? kSortThreads : (n + 2 * 32 - 1) / (2 * 32) * 32;
    const int threads = std::max(need, (E + 31) / 32 * 32);
    auto* kernel = per == 2   ? sort_kernel<kCluster, 2>
                   : per == 8 ? sort_kernel<kCluster, 8>
                              : sort_kernel<kCluster, 16>;
    return launched(fn, launch_pdl_cluster(kernel, dim3(ctas), ctas, dim3(threads), smem(threads), st, idx,
                                           n, K, E, mask, (int32_t*)nullptr, (const int32_t*)nullptr,
                                           offsets, slot));
  }
  int32_t *chunk = (int32_t*)work, *total = chunk + (size_t)chunks * E;
  const size_t bytes = smem(kSortThreads);
  cudaError_t e = launch_pdl(sort_kernel<kCount, kPer>, dim3(chunks), dim3(kSortThreads), bytes, st, idx, n,
                             K, E, mask, chunk, (const int32_t*)nullptr, (int32_t*)nullptr,
                             (int32_t*)nullptr);
  if (e == cudaSuccess)
    e = launch_pdl(sort_scan_kernel, dim3(E), dim3(32), 0, st, chunk, chunks, E, total);
  if (e == cudaSuccess)
    e = launch_pdl(sort_kernel<kAssign, kPer>, dim3(chunks), dim3(kSortThreads), bytes, st, idx, n, K, E,
                   mask, chunk, (const int32_t*)total, offsets, slot);
  return launched(fn, e);
}

extern "C" eat_status eat_expert_gather(const void* x, int32_t T, int32_t K, int32_t E, int32_t d,
                                        int32_t dtype, const int32_t* slot, const int32_t* offsets,
                                        void* rows, int32_t rows_dtype, float* scale,
                                        void* stream) {
  const char* fn = "eat_expert_gather";
  if (!x || !slot || !offsets || !rows)
    return bad_arg(fn, "x, slot, offsets and rows must be non-NULL");
  if (const char* why = bad_rows(T, K, E, d, dtype)) return bad_arg(fn, why);
  if (rows_dtype != dtype && rows_dtype != EAT_FP8_E4M3)
    return bad_arg(fn, "rows_dtype must be dtype or FP8_E4M3");
  const bool fp8 = rows_dtype == EAT_FP8_E4M3;
  if (fp8 && !scale) return bad_arg(fn, "e4m3 rows need scale");
  const int eb = dtype == EAT_BF16 ? 2 : 4;
  if (misaligned(x, eb) || misaligned(rows, fp8 ? 1 : eb) || misaligned(slot, 4) ||
      misaligned(offsets, 4) || (fp8 && misaligned(scale, 4)))
    return bad_arg(fn, "misaligned pointer");
  const size_t n = (size_t)T * d;
  if (overlaps({{rows, n * K * (fp8 ? 1 : eb)}, {fp8 ? scale : nullptr, 4 * (size_t)blocks_of(d) * T * K}},
               {{x, n * eb}, {slot, 4 * (size_t)T * K}, {offsets, 4 * (size_t)(E + 1)}}))
    return bad_arg(fn, "rows or scale overlaps another array");
  const cudaStream_t st = (cudaStream_t)stream;
  if (fp8) {
    auto run = [&](auto* tag) {
      using X = std::remove_pointer_t<decltype(tag)>;
      constexpr int N = Elem<X>::kN;
      const int pieces = (d + 64 * N - 1) / (64 * N);
      const bool vec = d % N == 0 && !misaligned(x, 16) && !misaligned(rows, N);
      return launch_pdl(vec ? gather_fp8_kernel<X, true> : gather_fp8_kernel<X, false>,
                        warp_grid((long long)T * pieces), dim3(32 * kWarps), 0, st, (const X*)x,
                        slot, offsets, T, K, E, d, pieces, (uint8_t*)rows, scale);
    };
    return launched(fn, dtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr));
  }
  auto run = [&](auto* tag) {
    using V = std::remove_pointer_t<decltype(tag)>;
    const int len = (int)((long long)d * eb / (int)sizeof(V));
    const int pieces = (len + 32 * kLoads - 1) / (32 * kLoads);
    return launch_pdl(gather_kernel<V>, warp_grid((long long)T * pieces), dim3(32 * kWarps), 0, st,
                      (const V*)x, slot, offsets, T, K, E, len, pieces, (V*)rows);
  };
  auto fits = [&](int n) { return (long long)d * eb % n == 0 && !misaligned(x, n) && !misaligned(rows, n); };
  return launched(fn, fits(16)  ? run((uint4*)nullptr)
                      : fits(4) ? run((uint32_t*)nullptr)
                                : run((uint16_t*)nullptr));
}

extern "C" eat_status eat_expert_combine(const void* rows, int32_t T, int32_t K, int32_t d,
                                         int32_t dtype, const int32_t* slot, const float* w, void* y,
                                         void* stream) {
  const char* fn = "eat_expert_combine";
  if (!rows || !slot || !y) return bad_arg(fn, "rows, slot and y must be non-NULL");
  if (const char* why = bad_rows(T, K, 1, d, dtype)) return bad_arg(fn, why);
  const int eb = dtype == EAT_BF16 ? 2 : 4;
  if (misaligned(rows, eb) || misaligned(y, eb) || misaligned(slot, 4) || misaligned(w, 4))
    return bad_arg(fn, "misaligned pointer");
  const size_t sel = (size_t)T * K;
  if (overlaps({{y, (size_t)T * d * eb}}, {{rows, sel * d * eb}, {slot, 4 * sel}, {w, 4 * sel}}))
    return bad_arg(fn, "y overlaps rows, slot or w");
  auto run = [&](auto* tag) {
    using X = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<X>::kN;
    const bool vec = d % N == 0 && !misaligned(rows, 16) && !misaligned(y, 16);
    const int pieces = (d + 32 * N - 1) / (32 * N);
    // (as many blocks as run at a time, so that a warp has a next token)
    const unsigned most = (unsigned)(kCombineBlocks * num_sms());
    const unsigned all = warp_grid((long long)T * pieces).x;
    return launch_pdl(vec ? combine_kernel<X, true> : combine_kernel<X, false>, dim3(std::min(most, all)),
                      dim3(32 * kWarps), 0, (cudaStream_t)stream, (const X*)rows, slot, w, T, K, d,
                      pieces, (X*)y);
  };
  return launched(fn, dtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr));
}

extern "C" eat_status eat_expert_combine_grad(const void* dy, const void* rows, int32_t T, int32_t K,
                                              int32_t E, int32_t d, int32_t dtype,
                                              const int32_t* slot, const int32_t* offsets,
                                              const float* w, void* drows, float* dw, void* stream) {
  const char* fn = "eat_expert_combine_grad";
  if (!dy || !rows || !slot || !offsets || !w || !drows || !dw)
    return bad_arg(fn, "dy, rows, slot, offsets, w, drows and dw must be non-NULL");
  if (const char* why = bad_rows(T, K, E, d, dtype)) return bad_arg(fn, why);
  const int eb = dtype == EAT_BF16 ? 2 : 4;
  if (misaligned(dy, eb) || misaligned(rows, eb) || misaligned(drows, eb) || misaligned(slot, 4) ||
      misaligned(offsets, 4) || misaligned(w, 4) || misaligned(dw, 4))
    return bad_arg(fn, "misaligned pointer");
  const size_t sel = (size_t)T * K, n = sel * d * eb;
  if (overlaps({{drows, n}, {dw, 4 * sel}}, {{rows, n},
                                             {dy, n / K},
                                             {slot, 4 * sel},
                                             {offsets, 4 * (size_t)(E + 1)},
                                             {w, 4 * sel}}))
    return bad_arg(fn, "drows or dw overlaps another array");
  auto run = [&](auto* tag) {
    using X = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<X>::kN;
    const bool vec =
        d % N == 0 && !misaligned(dy, 16) && !misaligned(rows, 16) && !misaligned(drows, 16);
    // Many tokens: two warps each, so that more tokens' loads are under way (8191 tokens x 8 of 2048:
    // 71 us, 107 with eight, cold; no other size was measured); few: as many as the row has vectors for.
    const int most = T >= 16 * num_sms() ? 2 : kWarps;
    const int warps = std::min(most, (d + 32 * N - 1) / (32 * N));
    return launch_pdl(vec ? combine_grad_kernel<X, true> : combine_grad_kernel<X, false>, dim3(T),
                      dim3(32 * warps), 0, (cudaStream_t)stream, (const X*)dy, (const X*)rows, slot,
                      offsets, w, T, K, E, d, (X*)drows, dw);
  };
  return launched(fn, dtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr));
}
