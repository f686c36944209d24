// Tensor-core kernels of the vocabulary head: logits l_tv = <x_t, w_v> that live in TMEM only.
//
//  small_kernel (loss, up to 128 tokens): a tile is 256 vocabulary rows (two MMAs of M = 128) x the
//      call's tokens (N = 16 .. 128), so a decode call streams the vocabulary matrix once, the tokens
//      (which every CTA reads again for each tile, from L2) half as often, and its MMAs stay below that.
//      Bound: HBM.  Each CTA takes an equal run of 16-row groups, in tiles of equal heights; its warps
//      keep a running maximum and sum of exponentials per token, joined across the CTA at its end,
//      and across the CTAs by the one that finishes last.  The steps of a k-block go to up to four
//      accumulators in turn, added in fp32: a tensor-core sum truncates at every step (at 4096 terms a logit
//      is off by 6e-6, biased towards zero), and shorter sums keep a decode token's loss within 1e-6.
//      One token, 50257 x 2048 bf16: 35 us a call, 5.9 TB/s; 16 tokens, 100000 x 4096: 126 us,
//      6.5 TB/s; 64 tokens, 100003 x 4096 e4m3: 65 us, 6.3 TB/s.
//  pair_kernel: 256 tokens (M, on an SM pair, cta_group::2) x 256 vocabulary rows (N).  A thread
//      owns a token's row of the tile, so sums over the vocabulary stay within a thread.  Bound:
//      tensor pipe.  kNll: running maximum and sum; kExp: exponentials relative to the target's
//      logit, stored as bf16 for the gradient's products, and their sums; kGrad: dx = f (E W) and
//      dW = E^T X, operands taken from the row-major matrices as they are (K-major or MN-major).
//      8192 tokens, 65536 x 2048: kExp 1.95, kGrad 1.88 PFLOP/s, 3.86 ms the whole call; e4m3 loss of
//      4096 tokens, 65536 x 4096: 649 us, 3.4 PFLOP/s.
// Warp roles as in the expert kernels: warp 0 one elected lane issues TMA, warp 1 owns TMEM and one
// elected lane issues MMAs, the others drain TMEM (double-buffered accumulators).  Every wait is
// bounded; on expiry the kernel records it, lets copies and MMAs land, frees TMEM and returns.
#include "head_tc.cuh"

#include <cudaTypedefs.h>

#include <algorithm>
#include <mutex>

#include "tc_ptx.cuh"

namespace eat {

namespace {

using namespace ptx;

constexpr int kRowBytes = 128;             // bytes of a k-block's row: 64 bf16 or 128 e4m3
constexpr int kOperand = 128 * kRowBytes;  // 128 rows of a k-block
constexpr int kBoxBytes = 64 * kRowBytes;  // a box of 64 rows

__device__ __forceinline__ void report(const HeadStatus& st, volatile int* abort_flag) {
  if (*abort_flag) *(volatile unsigned int*)st.mirror = *(volatile unsigned int*)st.err;
}

// (m, s) += (m2, s2): sums of exp2 relative to their maxima
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float n = fmaxf(m, m2);
  s = s * ex2(m - n) + s2 * ex2(m2 - n);
  m = n;
}

// A warp: the target logits of tokens t0, t0 + step, ... as fp32 sums of their own.  A tensor-core sum
// truncates at every step, which a logit that grows steadily, as a target's does, shows most.
template <bool W8, typename Args>
__device__ __forceinline__ void target_logits(const Args& a, int t0, int step, int lane) {
  const int vecs = a.d / (W8 ? 16 : 8);  // 16-byte pieces of a row
  for (int t = t0; t < a.T; t += step) {
    const int y = a.target[t];
    if (y < 0 || y >= a.V) continue;
    const uint4* x = (const uint4*)a.x + (size_t)t * vecs;
    const uint4* w = (const uint4*)a.w + (size_t)y * vecs;
    float d = 0.f;
#pragma unroll 4
    for (int c = lane; c < vecs; c += 32) d = dot16<W8>(x[c], w[c], d);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    if (lane == 0) a.ly[t] = d * kLog2e * (W8 ? a.xs[t] * a.ws[y] : 1.0f);
  }
}

// Sums of W values a lane over the warp's lanes: lane l gets the sum of the l % W-th values.  Lanes
// exchange the halves that they do not keep, so W values take W - 1 shuffles (and one more for 16).
template <int W>
__device__ __forceinline__ float column_sums(float (&v)[W], int lane) {
#pragma unroll
  for (int h = W / 2; h > 0; h >>= 1) {
    const bool upper = lane & h;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float give = upper ? v[i] : v[i + h], keep = upper ? v[i + h] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, h);
    }
  }
  if (W == 16) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
  return v[0];
}

// ------------------------------------------------------------------------------ small calls
constexpr int kSmallCtas = 160;  // at most (the last one's lanes take five each)
constexpr int kSmallRows = 256;  // vocabulary rows of a tile at most: two M = 128 halves
// The ring of stages of a small call: as many k-blocks of its tiles as fit, up to kSmallStages.
constexpr int kSmallStages = 16;
constexpr int kSmallRing = 216 * 1024;
constexpr int kSmallStageBytes = 50 * 1024;  // of a stage at most, unless one k-block is larger
template <int N>
struct SmallCfg {
  static constexpr int kSmem = 1024 + kSmallRing;
  static constexpr int kSplits = 128 / N < 4 ? 128 / N : 4;      // accumulators of a half tile
  static constexpr int kHalfCols = kSplits * N;
  static constexpr int kAccCols = 2 * kHalfCols;
  static constexpr int kTmemCols = 2 * kAccCols;
  static constexpr int kCols = N < 64 ? N : 64;                  // token columns of a warp
  static constexpr int kChunk = N < 32 ? N : 32;                 // of them at a time
  static constexpr int kEpiWarps = 4 * (N / kCols);
  static constexpr int kDotWarp = 2 + kEpiWarps;  // the target logits
  static constexpr int kThreads = 32 * (kDotWarp + 1);
  // Up to 32 columns the CTA that finishes last joins the sums of all; of more, a kernel of its own
  // (40 tokens, 20000 x 1024: 16.0 us that way, 17.8 with the last CTA; 128 columns: 5 us less;
  // 16: no less, and the host saves a launch)
  static constexpr bool kJoins = N <= 32;  // (head_small_joins)
};

template <int N, bool W8>
__global__ void __launch_bounds__(SmallCfg<N>::kThreads, 1)
small_kernel(const __grid_constant__ CUtensorMap map_w128, const __grid_constant__ CUtensorMap map_w16,
             const __grid_constant__ CUtensorMap map_x, const HeadSmallArgs a) {
  using C = SmallCfg<N>;
  constexpr int kElems = W8 ? 128 : 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t full[kSmallStages], empty[kSmallStages], tfull[2], tempty[2], mma_done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ int32_t s_target[N];
  __shared__ float s_xs[N];
  __shared__ float2 s_fin[4][N];
  __shared__ float s_max[C::kEpiWarps][C::kChunk];
  __shared__ int s_last;
  volatile int* abort_flag = &abort_word;
  const WaitCtx wc{abort_flag, a.st.err};

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSmallStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], C::kEpiWarps);
    }
    mbar_init(&mma_done, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_w128);
    prefetch_map(&map_x);
  }
  if (warp == 1) tmem_alloc<false>(&tmem_slot, C::kTmemCols);
  // this CTA's vocabulary rows (worked out before the wait: the divisions take 0.5 us)
  const unsigned groups = (unsigned)(a.V + 15) / 16;
  const int row0 = 16 * (int)(groups * blockIdx.x / gridDim.x);
  const int row1 = min(a.V, 16 * (int)(groups * (blockIdx.x + 1) / gridDim.x));
  // in tiles of equal heights, whose stages hold no more than they need: a call is bound by the bytes
  // in flight
  const int rows = row1 - row0, tiles = (rows + kSmallRows - 1) / kSmallRows;
  const int height = ((rows + tiles - 1) / tiles + 15) / 16 * 16;
  const int a_bytes = height * kRowBytes, sub_bytes = a_bytes + N * kRowBytes;
  // k-blocks of a stage: a stage costs a round of barriers however little it holds
  const int kps = max(1, min(8, kSmallStageBytes / sub_bytes)), stage_bytes = kps * sub_bytes;
  // (an MMA reads its 128 rows whole: the last k-block's reach past a low tile stays inside the ring)
  const int reach = (height > 128 ? 2 : 1) * kOperand;
  const int S = min(kSmallStages, (kSmallRing - max(0, reach - sub_bytes)) / stage_bytes);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  if (warp == 0) {
    if (elect_one()) {
      const uint64_t once = policy_evict_first();
      int stage = 0;
      uint32_t phase = 0;
      long long issued = 0;
      bool ok = true;
      for (int r = row0; r < row1 && ok; r += height) {
        const int boxes = min(height, row1 - r + 15) / 16;  // 16-row boxes of the tile
        for (int kb = 0; kb < a.kblocks; kb += kps) {
          const int nk = min(kps, a.kblocks - kb);
          if (!mbar_wait(&empty[stage], phase ^ 1u, wc, 1u)) {
            ok = false;
            break;
          }
          mbar_expect_tx(&full[stage], nk * (boxes * 16 + N) * kRowBytes);
          for (int j = 0; j < nk; ++j) {
            uint8_t* st = smem + stage * stage_bytes + j * sub_bytes;
            const int kx = (kb + j) * kElems;
            tma_load(st + a_bytes, &map_x, &full[stage], kx, 0);
            int b = 0;
            for (; b + 8 <= boxes; b += 8)
              tma_load_hint(st + b * 16 * kRowBytes, &map_w128, &full[stage], kx, r + 16 * b,
                            once);
            for (; b < boxes; ++b)
              tma_load_hint(st + b * 16 * kRowBytes, &map_w16, &full[stage], kx, r + 16 * b, once);
          }
          ++issued;
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      // copies in flight land before the CTA may exit
      for (long long i = issued > S ? issued - S : 0; i < issued; ++i)
        mbar_wait(&full[i % S], (uint32_t)((i / S) & 1), wc, 2u, false);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t id = idesc(W8, 128, N);
      int stage = 0, local = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int r = row0; r < row1 && ok; r += height, ++local) {
        const int buf = local & 1;
        if (!mbar_wait(&tempty[buf], ((local >> 1) & 1) ^ 1u, wc, 4u)) break;
        tc_fence_after();
        const bool two = min(height, row1 - r) > 128;
        for (int kb = 0; kb < a.kblocks; kb += kps) {
          const int nk = min(kps, a.kblocks - kb);
          if (!mbar_wait(&full[stage], phase, wc, 8u)) {
            ok = false;
            break;
          }
          tc_fence_after();
          for (int j = 0; j < nk; ++j) {
            const uint32_t d = tmem_base + (uint32_t)(buf * C::kAccCols);
            const uint32_t sa = smem_u32(smem + stage * stage_bytes + j * sub_bytes);
            const uint64_t da = sdesc_k(sa), d2 = sdesc_k(sa + kOperand);
            const uint64_t db = sdesc_k(sa + a_bytes);
            // (an accumulator's first step is among the first k-block's four)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t dk = d + (k % C::kSplits) * N;
              const uint32_t acc = kb + j > 0 || k >= C::kSplits;
              mma<false, W8>(dk, da + 2 * k, db + 2 * k, id, acc);
              if (two) mma<false, W8>(dk + C::kHalfCols, d2 + 2 * k, db + 2 * k, id, acc);
            }
          }
          mma_commit<false>(&empty[stage]);
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok) mma_commit<false>(&tfull[buf]);
      }
      mma_commit<false>(&mma_done);  // no MMA may run when TMEM is freed
    }
    if (lane == 0) mbar_wait(&mma_done, 0u, wc, 16u, false);
  } else if (warp == C::kDotWarp) {
    target_logits<W8>(a, blockIdx.x, gridDim.x, lane);  // beside the MMAs
  } else {
    // A lane has vocabulary row 32 q + lane of each half of the tile; per kChunk token columns the warp
    // takes their maximum and the sum of exponentials over its rows, which lane l then joins to the
    // l-th column's so far.  (State in registers, a lane per row, needs the columns unrolled: code
    // that is fetched once per call for 10 us of 64 columns.)
    constexpr int W = C::kChunk;
    const int q = warp & 3, half = (warp - 2) >> 2, col0 = half * C::kCols;
    float2* const state = s_fin[q] + col0;
    float* const s_m = s_max[warp - 2];
    for (int c = lane; c < C::kCols; c += 32) state[c] = make_float2(kHeadLow, 0.f);
    // (by these warps alone: the loads of the vocabulary do not wait for the targets)
    for (int i = threadIdx.x - 64; i < N; i += 32 * C::kEpiWarps) {
      s_target[i] = i < a.T ? a.target[i] : -1;
      s_xs[i] = kLog2e * (W8 && i < a.T ? a.xs[i] : 1.0f);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kEpiWarps) : "memory");
    int local = 0;
    for (int r = row0; r < row1; r += height, ++local) {
      const int buf = local & 1;
      if (!warp_wait(&tfull[buf], (local >> 1) & 1, wc, 32u)) break;
      tc_fence_after();
#pragma unroll 1
      for (int p = 0; p < 2 && 128 * p < min(height, row1 - r); ++p) {
        const int v = r + 128 * p + 32 * q + lane;
        const bool live = v < min(r + height, row1);
        const float sv = W8 && live ? a.ws[v] : 1.0f;
        const uint32_t t0 = tmem_base + ((uint32_t)(32 * q) << 16) +
                            (uint32_t)(buf * C::kAccCols + p * C::kHalfCols + col0);
#pragma unroll 1
        for (int c0 = 0; c0 < C::kCols; c0 += W) {
          uint32_t w[W];
          __syncwarp();
#pragma unroll
          for (int j = 0; j < W; j += 16) tmem_ld16(t0 + c0 + j, w + j);
          tmem_wait_ld();
#pragma unroll 1
          for (int i = 1; i < C::kSplits; ++i) {
            uint32_t w2[W];
#pragma unroll
            for (int j = 0; j < W; j += 16) tmem_ld16(t0 + i * N + c0 + j, w2 + j);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < W; ++j)
              w[j] = __float_as_uint(__uint_as_float(w[j]) + __uint_as_float(w2[j]));
          }
          float l[W];
#pragma unroll
          for (int j = 0; j < W; ++j) {
            l[j] = __uint_as_float(w[j]) * (W8 ? sv * s_xs[col0 + c0 + j] : kLog2e);
            if (!live) l[j] = kHeadLow;
          }
          // a column whose target is one of the warp's rows leaves that row out
          const int o = lane < W ? s_target[col0 + c0 + lane] - (v - lane) : -1;
          unsigned hits = __ballot_sync(0xffffffffu, o >= 0 && o < 32);
          if (hits) {
#pragma unroll
            for (int j = 0; j < W; ++j)
              if ((hits >> j & 1u) && s_target[col0 + c0 + j] == v) l[j] = kHeadLow;
          }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < W; ++j) {
            // (finite where all are -inf, or one is +inf)
            const float m = fminf(fmaxf(warp_max(l[j]), kHeadLow), kHeadHigh);
            l[j] = ex2(l[j] - m);
            if (lane == 0) s_m[j] = m;
          }
          const float s = column_sums<W>(l, lane);
          __syncwarp();
          if (lane < W) {
            float2 f = state[c0 + lane];
            join(f.x, f.y, s_m[lane], s);
            state[c0 + lane] = f;
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty[buf]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc<false>(tmem_base, C::kTmemCols);
  for (int c = threadIdx.x; c < a.T; c += C::kThreads) {
    float2 f = s_fin[0][c];
    for (int i = 1; i < 4; ++i) join(f.x, f.y, s_fin[i][c].x, s_fin[i][c].y);
    // [CTA][column] for the kernel that joins them, [column][CTA] for the last CTA's warps
    a.part[C::kJoins ? (size_t)c * gridDim.x + blockIdx.x : (size_t)blockIdx.x * N + c] = f;
  }
  if (threadIdx.x == 0) report(a.st, abort_flag);
  if (!C::kJoins) return;
  // the CTA that finishes last joins the sums of all (in their order, whichever CTA it is)
  __syncthreads();
  if (threadIdx.x == 0) {
    // releases what the CTA wrote (the barrier above orders it), and acquires what the others did
    unsigned int old;
    asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;"
                 : "=r"(old)
                 : "l"(a.tickets), "r"(gridDim.x - 1)
                 : "memory");
    s_last = old == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  // a warp takes every kWarps-th token, all of its loads first
  constexpr int kWarps = C::kThreads / 32, kTok = (N + kWarps - 1) / kWarps;
  constexpr int kLoads = kSmallCtas / 32;
  float2 v[kTok][kLoads];
  float ly[kTok];
  const unsigned int err = __ldcg(a.st.err);
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const int t = warp + i * kWarps;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int cta = k * 32 + lane;
      v[i][k] = make_float2(kHeadLow, 0.f);
      if (t < a.T && cta < (int)gridDim.x)
        v[i][k] = __ldcg(a.part + (size_t)t * gridDim.x + cta);
    }
    ly[i] = t < a.T ? __ldcg(a.ly + t) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const int t = warp + i * kWarps;
    if (t >= a.T) break;
    float2 f = v[i][0];
#pragma unroll
    for (int k = 1; k < kLoads; ++k) join(f.x, f.y, v[i][k].x, v[i][k].y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float m = __shfl_xor_sync(0xffffffffu, f.x, o);
      const float s = __shfl_xor_sync(0xffffffffu, f.y, o);
      join(f.x, f.y, m, s);
    }
    if (lane == 0) {
      const int y = s_target[t];
      float2 r = make_float2(0.f, 0.f);
      if (y >= a.V) r = make_float2(NAN, NAN);
      else if (y >= 0) r = token_loss(f.x, f.y, ly[i]);
      if (y >= 0 && err) r = make_float2(NAN, NAN);
      if (err && t == 0) *a.st.mirror = err;
      a.nll[t] = r.x;
      if (a.lse) a.lse[t] = r.y;
    }
  }
}

// --------------------------------------------------------------------------------- SM pairs
enum : int { kNll = 0, kExp = 1, kGrad = 2 };

template <int MODE>
struct PairCfg {
  // a stage is one k-block: 128 rows of A and of B of each CTA (six stages of 32 KB; three of two
  // k-blocks measured 0 to 2 % slower from 12 to 8192 tokens)
  static constexpr int kStage = 2 * kOperand;
  static constexpr int kStages = 6;
  // kExp, kGrad: 32 rows of 64 bytes per epilogue warp, on their way to memory
  static constexpr int kOut = MODE == kNll ? 0 : 8 * 32 * 64;
  static constexpr int kSmem = 1024 + kStages * kStage + kOut;
  static constexpr int kEpiWarps = 8;
  static constexpr int kDotWarp = 2 + kEpiWarps;  // kNll: the target logits
  static constexpr int kThreads = 64 + 32 * kEpiWarps + (MODE == kNll ? 32 : 0);
  static constexpr int kAccCols = 256;
};

struct PairParams {
  HeadPairArgs p;
  HeadGradArgs g;
};

// One tile of a launch: 256 rows of A from m0, 256 rows of B from n0, kb k-blocks.
struct Tile {
  int m0, n0, kb;
  int k0;   // first k-block
  bool dw;  // kGrad: a tile of dW
};

// The gradient's tiles in the order in which equal workers would take them: first the product with
// the longer sums (n1 tiles of k1 k-blocks each, dealt round), then the other one (n2 tiles of k2),
// whose j-th tile of a worker is the one that it would reach in time order.
struct GradTiles {
  int n1, k1, n2, k2, pairs, pair;
  bool dw_first;
  __device__ int first_count() const { return n1 / pairs + (pair < n1 % pairs ? 1 : 0); }
  // the i-th tile of this pair: its number, and in `second` whether it is of the second product;
  // -1 when there is none
  __device__ int at(int i, bool& second) const {
    const int own = first_count();
    second = i >= own;
    if (!second) return i * pairs + pair;
    const int j = i - own, r = n1 % pairs;
    long long t;
    if (r == 0) {
      t = (long long)j * pairs + pair;
    } else if (pair >= r) {  // free one tile of the first product earlier
      const long long ahead = (long long)j * k2 - k1;  // time after the others begin
      t = (long long)j * (pairs - r) + (pair - r) + (ahead > 0 ? (ahead + k2 - 1) / k2 * r : 0);
    } else {
      t = (long long)j * r + pair + (long long)(j + k1 / max(k2, 1) + 1) * (pairs - r);
    }
    return t < n2 ? (int)t : -1;
  }
};

// k-blocks of a slice of the vocabulary
__host__ __device__ __forceinline__ int slice_blocks(int V, int slices) {
  return ((V + 63) / 64 + slices - 1) / slices;
}

// A warp's 32 rows of 64 bytes, as four 16-byte pieces each, between the layout of TMEM (lane: row) and
// that of memory (four lanes a row, eight rows at a time, so that stores fill whole sectors).  The
// piece's place is exchanged by row, which spreads both accesses over the banks.  Lanes that stored
// their rows' 64 bytes themselves took 9.5 us per 256 x 256 bf16 tile, four times the tile's products
// over 64 tokens.
__device__ __forceinline__ int out_slot(int row, int piece) {
  return row * 4 + (piece ^ ((row >> 1) & 3));
}
__device__ __forceinline__ void out_put(uint4* buf, int lane, const uint32_t* w) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j)
    buf[out_slot(lane, j)] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  __syncwarp();
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&v;
}

template <int MODE, bool W8>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairCfg<MODE>::kThreads, 1)
pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
            const __grid_constant__ CUtensorMap map_x, const __grid_constant__ PairParams prm) {
  using C = PairCfg<MODE>;
  constexpr int S = C::kStages;
  constexpr int kElems = W8 ? 128 : 64;
  const HeadPairArgs& p = prm.p;
  const HeadGradArgs& g = prm.g;
  const HeadStatus status = MODE == kGrad ? g.st : p.st;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t full[S], empty[S], tfull[2], tempty[2], mma_done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ float s_ws[W8 ? C::kEpiWarps : 1][W8 ? 128 : 1];
  volatile int* abort_flag = &abort_word;
  const WaitCtx wc{abort_flag, status.err};

  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (MODE == kExp && p.redo) {  // as a rule no token is far: the launch ends here
    pdl_wait();
    int any = 0;
    for (int i = threadIdx.x; i < p.cap / kHeadTile; i += C::kThreads)
      any |= p.far[p.t0 / kHeadTile + i];
    if (!__syncthreads_or(any)) return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 2 * C::kEpiWarps);  // the epilogue warps of both CTAs (rank 0's)
    }
    mbar_init(&mma_done, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    if (MODE == kGrad) prefetch_map(&map_x);
  }
  if (warp == 1) tmem_alloc<true>(&tmem_slot, 512);
  tc_fence_before();
  cluster_sync_all();  // both CTAs' barriers exist before either signals the other
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  // the launch's tokens (kNll), or the counted ones of its piece
  int rows = p.T, n_counted = 0;  // (rows: those of E; n_counted: those of dx)
  if (MODE != kNll) {
    n_counted = MODE == kGrad ? *g.n_counted : *p.n_counted;
    const int t0 = MODE == kGrad ? g.t0 : p.t0, cap = MODE == kGrad ? g.cap : p.cap;
    rows = max(0, min(cap, head_rows(n_counted) - t0));
  }
  const int row_tiles = (rows + kHeadTile - 1) / kHeadTile;
  const int V = MODE == kGrad ? g.V : p.V;
  const int v_tiles = (V + kHeadTile - 1) / kHeadTile;
  const int units = row_tiles * v_tiles;
  GradTiles gt{};
  const int d_tiles = MODE == kGrad ? (g.d + kHeadTile - 1) / kHeadTile : 1;
  if (MODE == kGrad) {
    const int nx = row_tiles * d_tiles * g.slices, kx = slice_blocks(V, g.slices);
    // a piece without tokens adds nothing, but the first one still writes dW
    const int nw = rows > 0 || g.t0 == 0 ? v_tiles * d_tiles : 0, kw = (rows + 63) / 64;
    gt.dw_first = kw > kx;
    gt.n1 = gt.dw_first ? nw : nx;
    gt.k1 = gt.dw_first ? kw : kx;
    gt.n2 = gt.dw_first ? nx : nw;
    gt.k2 = gt.dw_first ? kx : kw;
    gt.pairs = n_pairs;
    gt.pair = pair;
  }
  // the next tile of this pair after step i (i is left at the step that follows it)
  auto next_tile = [&](int& i, Tile& t) -> bool {
    if (MODE == kGrad) {
      bool second;
      const int n = gt.at(i, second);
      if (n < 0 || (!second && n >= gt.n1)) return false;
      ++i;
      t.dw = second != gt.dw_first;
      t.n0 = n % d_tiles * kHeadTile;
      const int r = n / d_tiles;
      if (t.dw) {
        t.m0 = r * kHeadTile;
        t.k0 = 0;
        t.kb = second ? gt.k2 : gt.k1;
      } else {
        const int per = slice_blocks(V, g.slices), all = (V + 63) / 64;
        t.m0 = r % row_tiles * kHeadTile;
        t.k0 = r / row_tiles * per;
        t.kb = max(0, min(per, all - t.k0));
      }
      return true;
    }
    for (;;) {
      const long long u = (long long)i * n_pairs + pair;
      if (u >= units) return false;
      ++i;
      const int rt = (int)(u % row_tiles);
      if (MODE == kExp && p.redo && !p.far[(p.t0 / kHeadTile) + rt]) continue;
      t.dw = false;
      t.m0 = rt * kHeadTile;
      t.n0 = (int)(u / row_tiles) * kHeadTile;
      t.k0 = 0;
      t.kb = p.kblocks;
      return true;
    }
  };
  const uint32_t full0 = map_rank(smem_u32(full), 0);
  const uint32_t tempty0 = map_rank(smem_u32(tempty), 0);

  if (warp == 0) {
    if (elect_one()) {
      int stage = 0, i = 0;
      uint32_t phase = 0;
      long long issued = 0;
      bool ok = true;
      Tile t;
      while (ok && next_tile(i, t)) {
        // dX: A = E (K-major), B = W (MN-major); dW: A = E, B = X (both MN-major); scores: A = X,
        // B = W (both K-major)
        const CUtensorMap* mb = MODE == kGrad && t.dw ? &map_x : &map_b;
        const int ra = t.m0 + (int)rank * 128 + (MODE == kExp ? p.t0 : 0);
        const int rb = t.n0 + (int)rank * 128;
        for (int kb = 0; kb < t.kb; ++kb) {
          if (!mbar_wait(&empty[stage], phase ^ 1u, wc, 1u)) {
            ok = false;
            break;
          }
          uint8_t* sa = smem + stage * C::kStage;
          uint8_t* sb = sa + kOperand;
          const uint32_t fb = full0 + 8u * (uint32_t)stage;
          if (leader) mbar_expect_tx(&full[stage], 2 * C::kStage);
          const int kx = (t.k0 + kb) * kElems;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if (MODE == kGrad) {
              if (t.dw) tma_load_pair(sa + b * kBoxBytes, &map_a, fb, ra + 64 * b, kx);
              else tma_load_pair(sa + b * kBoxBytes, &map_a, fb, kx, ra + 64 * b);
              tma_load_pair(sb + b * kBoxBytes, mb, fb, rb + 64 * b, kx + (t.dw ? g.t0 : 0));
            } else {
              tma_load_pair(sa + b * kBoxBytes, &map_a, fb, kx, ra + 64 * b);
              tma_load_pair(sb + b * kBoxBytes, mb, fb, kx, rb + 64 * b);
            }
          }
          ++issued;
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      // rank 0: the copies of both CTAs still in flight land before the pair may exit
      if (leader)
        for (long long n = issued > S ? issued - S : 0; n < issued; ++n)
          mbar_wait(&full[n % S], (uint32_t)((n / S) & 1), wc, 2u, false);
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      int stage = 0, i = 0, local = 0;
      uint32_t phase = 0;
      bool ok = true;
      Tile t;
      for (; ok && next_tile(i, t); ++local) {
        const int buf = local & 1;
        if (!mbar_wait(&tempty[buf], ((local >> 1) & 1) ^ 1u, wc, 4u)) break;
        tc_fence_after();
        const uint32_t d0 = tmem_base + (uint32_t)(buf * C::kAccCols);
        const uint32_t id = idesc(W8, 256, 256, MODE == kGrad && t.dw, MODE == kGrad);
        const bool a_mn = MODE == kGrad && t.dw;
        const int step_a = a_mn ? 128 : 2, step_b = MODE == kGrad ? 128 : 2;
        for (int kb = 0; kb < t.kb; ++kb) {
          if (!mbar_wait(&full[stage], phase, wc, 8u)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem + stage * C::kStage);
          const uint64_t da = a_mn ? sdesc_mn(sa) : sdesc_k(sa);
          const uint64_t db = MODE == kGrad ? sdesc_mn(sa + kOperand) : sdesc_k(sa + kOperand);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma<true, W8>(d0, da + k * step_a, db + k * step_b, id, kb > 0 || k > 0);
          mma_commit<true>(&empty[stage]);
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok) mma_commit<true>(&tfull[buf]);
      }
      mma_commit<true>(&mma_done);
    }
    if (lane == 0) mbar_wait(&mma_done, 0u, wc, 16u, false);
  } else if (MODE == kNll && warp == C::kDotWarp) {
    target_logits<W8>(p, blockIdx.x, gridDim.x, lane);  // beside the MMAs
  } else {
    // a thread: row 128 rank + 32 q + lane of the tile, columns [128 ch, 128 ch + 128)
    const int q = warp & 3, ch = (warp - 2) >> 2;
    const int my_row = (int)rank * 128 + 32 * q + lane;
    int i = 0, local = 0;
    Tile t;
    for (; next_tile(i, t); ++local) {
      const int buf = local & 1;
      const int row = t.m0 + my_row, n0 = t.n0 + 128 * ch;
      // what the rows and columns need, loaded while the MMAs run
      int y = -1;
      float xs = kLog2e, ref = INFINITY;
      if (MODE != kGrad && row < rows) {
        y = p.target[(MODE == kExp ? p.t0 : 0) + row];
        if (W8) xs *= p.xs[row];
        if (MODE == kExp) {
          ref = p.ref[p.t0 + row];
          if (p.redo) ref = head_ref(ref, p.row_max[p.t0 + row]);
        }
      }
      if (W8) {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          const int v = n0 + c + lane;
          s_ws[W8 ? warp - 2 : 0][c + lane] = v < V ? p.ws[v] : 0.f;
        }
        __syncwarp();
      }
      if (!warp_wait(&tfull[buf], (local >> 1) & 1, wc, 32u)) break;
      tc_fence_after();
      const uint32_t tb =
          tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * C::kAccCols + 128 * ch);
      float m = kHeadLow, s = 0.f;
      // kGrad: where the tile goes: fp32 sums (dX's slices, dW's pieces of tokens but the last), or
      // bf16 rows.  Lane l stores piece l % 4 of the rows l / 4 + 8 i of its warp's 32.
      float factor = 1.f;
      float* sum = nullptr;
      __nv_bfloat16* out = nullptr;
      bool add = false;
      int dst[4], limit = 0;  // rows of the destination, -1: none
      uint4* const box = (uint4*)(smem + S * C::kStage) + (warp - 2) * 128;
      if (MODE == kGrad) {
        limit = t.dw ? V : min(rows, n_counted - g.t0);
        if (t.dw) {
          const bool last = g.t0 + g.cap >= n_counted;
          add = g.t0 > 0;
          if (add || !last) sum = g.dw_sum;
          if (last) out = g.dw;
        } else if (g.slices > 1) {
          sum = g.dx_part + (size_t)(t.k0 / slice_blocks(V, g.slices)) * g.cap * g.d;
        } else {
          out = g.dx;
          if (row < limit) factor = g.f[g.t0 + row];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = t.m0 + (int)rank * 128 + 32 * q + 8 * k + (lane >> 2);
          dst[k] = r >= limit ? -1 : !t.dw && out ? g.rows[g.t0 + r] : r;
        }
      }
#pragma unroll 1
      for (int c0 = 0; c0 < 128; c0 += 32) {
        uint32_t w[32];
        __syncwarp();
        tmem_ld16(tb + c0, w);
        tmem_ld16(tb + c0 + 16, w + 16);
        tmem_wait_ld();
        const int nc = n0 + c0;
        if (MODE == kGrad) {
          if (nc >= g.d) continue;
          if (t.kb == 0) {
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = 0;
          }
          if (sum) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              out_put(box, lane, w + 16 * half);
              const int c = nc + 16 * half + 4 * (lane & 3);
              float4 v[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (add && dst[k] >= 0) v[k] = *(const float4*)(sum + (size_t)dst[k] * g.d + c);
                else v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint4 u = box[out_slot(8 * k + (lane >> 2), lane & 3)];
                v[k].x += __uint_as_float(u.x);
                v[k].y += __uint_as_float(u.y);
                v[k].z += __uint_as_float(u.z);
                v[k].w += __uint_as_float(u.w);
                if (dst[k] < 0) continue;
                if (out)
                  *(uint2*)(out + (size_t)dst[k] * g.d + c) =
                      make_uint2(pack_bf16(v[k].x, v[k].y), pack_bf16(v[k].z, v[k].w));
                else
                  *(float4*)(sum + (size_t)dst[k] * g.d + c) = v[k];
              }
            }
            continue;
          }
          uint32_t b[16];
#pragma unroll
          for (int j = 0; j < 16; ++j)
            b[j] = pack_bf16(__uint_as_float(w[2 * j]) * factor,
                             __uint_as_float(w[2 * j + 1]) * factor);
          out_put(box, lane, b);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4 u = box[out_slot(8 * k + (lane >> 2), lane & 3)];
            if (dst[k] >= 0)
              *(uint4*)(out + (size_t)dst[k] * g.d + nc + 8 * (lane & 3)) = u;
          }
          continue;
        }
        // scores: base-2 logits
        float l[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float sc = W8 ? xs * s_ws[W8 ? warp - 2 : 0][c0 + j] : kLog2e;
          l[j] = MODE == kExp ? __uint_as_float(w[j]) : __uint_as_float(w[j]) * sc;
        }
        const int hit = y - nc;  // the target's column, if among these
        if (MODE == kNll) {
          if (hit >= 0 && hit < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == hit) l[j] = kHeadLow;
          }
          if (nc + 32 > V) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (nc + j >= V) l[j] = kHeadLow;
          }
          float n = m;
#pragma unroll
          for (int j = 0; j < 32; ++j) n = fmaxf(n, l[j]);
          n = fminf(n, kHeadHigh);
          float s0 = s * ex2(m - n), s1 = 0.f;
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            s0 += ex2(l[j] - n);
            s1 += ex2(l[j + 1] - n);
          }
          s = s0 + s1;
          m = n;
        } else {
          float s0 = 0.f, s1 = 0.f;
          // (columns past the vocabulary, which loads fill with zeros, are no logits)
          if (nc + 32 > V) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (nc + j >= V) l[j] = kHeadLow;
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) m = fmaxf(m, l[j]);
#pragma unroll
          for (int j = 0; j < 32; ++j) l[j] = ex2(fmaf(l[j], kLog2e, -ref));
          // (a row that stands for no token has x = 0, and with a vocabulary row that holds an
          // infinity a logit of NaN, which X' = 0 would not take out of dW)
          if (y < 0) {
#pragma unroll
            for (int j = 0; j < 32; ++j) l[j] = 0.f;
          }
          if (hit >= 0 && hit < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == hit) l[j] = 0.f;
          }
          if (nc + 32 > V) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (nc + j >= V) l[j] = 0.f;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            s0 += l[j];
            s1 += l[j + 1];
          }
          s += s0 + s1;
          uint32_t b[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) b[j] = pack_bf16(l[2 * j], l[2 * j + 1]);
          out_put(box, lane, b);
          // (rows up to the tile's end exist)
          __nv_bfloat16* e = p.e + (size_t)(t.m0 + (int)rank * 128 + 32 * q) * p.ld + nc;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = 8 * k + (lane >> 2);
            *(uint4*)(e + (size_t)r * p.ld + 8 * (lane & 3)) = box[out_slot(r, lane & 3)];
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (leader) mbar_arrive(&tempty[buf]);
        else mbar_arrive_remote(tempty0 + 8u * (uint32_t)buf);
      }
      if (MODE == kNll && row < rows)
        p.part2[(size_t)(n0 / 128) * p.T + row] = make_float2(m, s);
      if (MODE == kExp) {
        p.part[(size_t)(n0 / 128) * p.cap + row] = s;
        if (!p.redo && row < rows && m * kLog2e > ref + kHeadFar) {
          atomicMax(&p.row_max[p.t0 + row], ordered_bits(fminf(m * kLog2e, kHeadHigh)));
          p.far[(p.t0 + row) / kHeadTile] = 1;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while the other may still signal it
  tc_fence_after();
  if (warp == 1) tmem_dealloc<true>(tmem_base, 512);
  if (threadIdx.x == 0) report(status, abort_flag);
}

// -------------------------------------------------------------------------------- host side
PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = (PFN_cuTensorMapEncodeTiled_v12000)p;
  });
  return fn;
}

template <int N, bool W8>
cudaError_t launch_small(const CUtensorMap& w128, const CUtensorMap& w16, const CUtensorMap& x,
                         const HeadSmallArgs& a, int ctas, cudaStream_t st) {
  return launch_pdl(small_kernel<N, W8>, dim3(ctas), dim3(SmallCfg<N>::kThreads),
                    SmallCfg<N>::kSmem, st, w128, w16, x, a);
}
template <bool W8>
cudaError_t launch_small_n(const CUtensorMap& w128, const CUtensorMap& w16, const CUtensorMap& x,
                           const HeadSmallArgs& a, int ctas, cudaStream_t st) {
  switch (head_small_n(a.T)) {
    case 16: return launch_small<16, W8>(w128, w16, x, a, ctas, st);
    case 32: return launch_small<32, W8>(w128, w16, x, a, ctas, st);
    case 64: return launch_small<64, W8>(w128, w16, x, a, ctas, st);
    default: return launch_small<128, W8>(w128, w16, x, a, ctas, st);
  }
}
template <int MODE, bool W8>
cudaError_t launch_pair(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& x,
                        const PairParams& p, int pairs, cudaStream_t st) {
  return launch_pdl(pair_kernel<MODE, W8>, dim3(2 * pairs), dim3(PairCfg<MODE>::kThreads),
                    PairCfg<MODE>::kSmem, st, a, b, x, p);
}

template <typename K>
cudaError_t limit(K kernel, int smem) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
}
template <bool W8>
cudaError_t configure_small() {
  cudaError_t e = limit(small_kernel<16, W8>, SmallCfg<16>::kSmem);
  if (e == cudaSuccess) e = limit(small_kernel<32, W8>, SmallCfg<32>::kSmem);
  if (e == cudaSuccess) e = limit(small_kernel<64, W8>, SmallCfg<64>::kSmem);
  if (e == cudaSuccess) e = limit(small_kernel<128, W8>, SmallCfg<128>::kSmem);
  return e;
}
template <int MODE, bool W8>
cudaError_t configure_pair(int num_sms, int* max_pairs) {
  const cudaError_t e = limit(pair_kernel<MODE, W8>, PairCfg<MODE>::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(num_sms & ~1);
  cfg.blockDim = dim3(PairCfg<MODE>::kThreads);
  cfg.dynamicSmemBytes = PairCfg<MODE>::kSmem;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, pair_kernel<MODE, W8>, &cfg) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    n = num_sms / 2;
  }
  *max_pairs = std::max(1, std::min(*max_pairs, n));
  return cudaSuccess;
}

}  // namespace

int head_small_n(int T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128; }
bool head_small_joins(int n) { return n <= 32; }
int head_small_ctas(int num_sms, int V) {
  return std::min(std::min(num_sms, kSmallCtas), (V + 15) / 16);
}

cudaError_t head_launch_small(bool w8, const CUtensorMap& w128, const CUtensorMap& w16,
                              const CUtensorMap& x, const HeadSmallArgs& a, int ctas,
                              cudaStream_t st) {
  return w8 ? launch_small_n<true>(w128, w16, x, a, ctas, st)
            : launch_small_n<false>(w128, w16, x, a, ctas, st);
}

cudaError_t head_launch_pair(bool w8, bool exp, const CUtensorMap& x, const CUtensorMap& w,
                             const HeadPairArgs& a, int max_pairs, cudaStream_t st) {
  PairParams p{};
  p.p = a;
  const long long tokens = exp ? a.cap : a.T;
  const long long units =
      (tokens + kHeadTile - 1) / kHeadTile * ((a.V + kHeadTile - 1) / kHeadTile);
  if (exp)
    return launch_pair<kExp, false>(x, w, w, p, (int)std::min<long long>(max_pairs, units), st);
  // (a small vocabulary leaves pairs without tiles, but with target logits: 16 tokens a pair)
  const int pairs = (int)std::min<long long>(max_pairs, std::max<long long>(units, a.T / 16));
  return w8 ? launch_pair<kNll, true>(x, w, w, p, pairs, st)
            : launch_pair<kNll, false>(x, w, w, p, pairs, st);
}

// A piece whose tiles of dx are few, and whose sums run over the whole vocabulary, would leave most
// SM pairs waiting for them: the sums are cut so that a slice takes at most half of what every pair
// has to do anyway (a tile costs about 12 k-blocks besides its own), and not below 12 k-blocks, about
// what the launch that adds the slices, in order, costs.
int head_dx_slices(int cap, int V, int d, int max_pairs) {
  const long long dt = (d + kHeadTile - 1) / kHeadTile, kx = (V + 63) / 64, kw = (cap + 63) / 64;
  const long long nx = cap / kHeadTile * dt, nw = (V + kHeadTile - 1) / kHeadTile * dt, fix = 12;
  if (nx >= 2LL * max_pairs) return 1;
  const long long share = (nx * (kx + fix) + nw * (kw + fix)) / max_pairs;
  const long long len = std::max(12LL, share / 2);
  const long long n = std::min((kx + len - 1) / len, 2LL * max_pairs / nx + 1);
  // (no slice is empty)
  const long long per = (kx + n - 1) / n;
  return (int)((kx + per - 1) / per);
}

cudaError_t head_launch_grad(const CUtensorMap& e, const CUtensorMap& w, const CUtensorMap& x,
                             const HeadGradArgs& a, int max_pairs, cudaStream_t st) {
  PairParams p{};
  p.g = a;
  const long long units =
      ((long long)a.cap / kHeadTile * a.slices + (a.V + kHeadTile - 1) / kHeadTile) *
      ((a.d + kHeadTile - 1) / kHeadTile);
  const int pairs = (int)std::min<long long>(max_pairs, units);
  return launch_pair<kGrad, false>(e, w, x, p, pairs, st);
}

cudaError_t head_configure(int num_sms, int* max_pairs) {
  *max_pairs = std::max(1, num_sms / 2);
  cudaError_t e = configure_small<false>();
  if (e == cudaSuccess) e = configure_small<true>();
  if (e == cudaSuccess) e = configure_pair<kNll, false>(num_sms, max_pairs);
  if (e == cudaSuccess) e = configure_pair<kNll, true>(num_sms, max_pairs);
  if (e == cudaSuccess) e = configure_pair<kExp, false>(num_sms, max_pairs);
  if (e == cudaSuccess) e = configure_pair<kGrad, false>(num_sms, max_pairs);
  return e;
}

bool head_encode(CUtensorMap* m, bool w8, const void* ptr, long long rows, long long cols,
                 int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)cols * (w8 ? 1 : 2)};
  cuuint32_t box[2] = {(cuuint32_t)(w8 ? 128 : 64), (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, w8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
            const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace eat
