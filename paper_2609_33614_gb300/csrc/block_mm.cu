// Matrix products of e4m3 operands with a scale for each block of 128 along the sums (quant.cu makes
// them), for one matrix or for the experts' matrices on rows sorted by expert:
//   y[r][n]  = sum_b xs[b][r] ws[n / 128][b] sum_{k in b} x[r][k] w[n][k]
//   y[r][k]  = the same with w as it lies, summed over n (transposed: the gradient to x)
//   dw[n][k] = sum_b gs[b][n] xs[b][k] sum_{r in b} g[r][n] x[r][k], b the blocks of 128 rows of an expert
//
// A k-block of 128 is up to four MMAs into an accumulator of its own in TMEM; the epilogue's warps read it,
// multiply by the block's scales and add it to fp32 sums in registers while the next k-blocks run.
//   block_mm_kernel: a tile of the output is up to NT of its rows x 128 of its columns, as the transposed
//      product: the 128 columns (w's; dw: x's) are the MMA's M, the rows (x's; dw: g's) its N.  So a matrix
//      is read once for up to NT rows of x, however few there are, and an expert's rows are cut into
//      tiles of equal heights.  In the 16x256b layout a thread has two neighbouring rows of the output for each
//      of its columns, so a scale's pair is one load.  Bound: HBM with few rows an expert (1 token, 2 of 8
//      matrices of 28672 x 4096: 41 us, 5.7 TB/s; 32 tokens, 8 of 64 of 2048 x 2048: 42 us, 6.4 TB/s); dw
//      of 18432 rows, 64 matrices of 2048 x 2048: 205 us, of which writing dw is 79.
//   wide_kernel: on SM pairs, 256 rows (M) x 256 columns (N), for many rows an expert: half the operand bytes
//      from L2 for each MMA, and a k-block's scales are one product a thread.  Bound: the accumulator's way
//      through TMEM (two buffers: an MMA of 530 cycles, then 500 of reading and adding, then the
//      hand-over).  8192 x 2048 x 8192: 137 us, 2.0 PFLOP/s; 60 matrices of 2816 x 2048, 170 rows
//      each: 97 us; a router's 10240 rows, 30 to 500 each: 122.
// Operands come by TMA as they lie (K-major, or MN-major where the sum runs over their rows): w serves
// both directions, and the gradient reads both operands by rows.
// Warps: 0 issues TMA, 1 owns TMEM and issues MMAs, 2 copies the blocks' scales into a ring (block_mm_kernel)
// and clears the rows behind the last expert's, 3 has no role (registers are shared out by fours), the others
// drain TMEM.  Every wait is bounded; where one
// expires the CTA's tiles that are not done become NaN, copies and MMAs land, TMEM is freed and the kernel ends.
#include "elem.cuh"
#include "op_checks.cuh"
#include "tc_ptx.cuh"

#include "tensor_map.cuh"

#include <algorithm>
#include <atomic>

namespace eat {

namespace {

using namespace ptx;

enum : int { kForward = 0, kBack = 1, kGrad = 2 };

// A call's bounded waits: their limit, and for the tests of what follows when one expires a CTA whose copies
// end after so many k-blocks, and a device word that takes the codes of the waits that gave up (or null).
struct Waits {
  unsigned long long limit_ns = kWaitLimitNs;
  int held_cta = -1;
  long long held_after = 0;
  unsigned int* status = nullptr;
};

struct Args {
  const float *xs, *ws;  // kGrad: g's and x's
  const int32_t* offsets;
  int E, M, N, K;  // N, K: w's shape; M: x's rows (kGrad: the operands' padded rows)
  int blocks;      // kGrad: rows of the scales
  void* out;
  int vec;         // rows of the output begin at multiples of 16 bytes
  Waits waits;
};

constexpr int kOperand = kBlock * kBlock;  // bytes of 128 rows of a k-block
constexpr int kAhead = 4;                  // k-blocks whose scales are on their way
constexpr int kFirstEpi = 4;               // warps before the epilogue's

template <int NT>
struct Cfg {
  static constexpr int kEpiWarps = NT >= 64 ? 8 : 4;
  static constexpr int kCols = NT >= 64 ? NT / 2 : NT;  // of the accumulator, for a warp
  static constexpr int kChunks = kCols / 16;  // of 16, which the warp reads at a time
  static constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
  static constexpr int kBufs = NT == 256 ? 2 : NT == 128 ? 4 : 8;  // accumulators
  static constexpr int kTmemCols = NT * kBufs;
  static constexpr int kStage = kOperand + NT * kBlock;
  static constexpr int kStages = NT == 256 ? 4 : NT == 128 ? 6 : NT == 64 ? 8 : 10;
  static constexpr int kBox = NT < 64 ? NT : 64;  // rows of x that a copy takes
  static constexpr int kSlots = kAhead + kBufs;  // of the ring of scales
  static constexpr int kSlotFloats = NT + kBlock;
  static constexpr int kOut = kEpiWarps * 32 * 64;  // 32 rows of 64 bytes per warp
  static constexpr int kSmem =
      1024 + kStages * kStage + kOut + kSlots * kSlotFloats * 4;
  // Registers of the first four warps and of the epilogue's once they are shared out (NT = 256: 168 a thread
  // at launch, 384 (168) = 128 (88) + 256 (208)); 0: as launched.
  static constexpr int kFewRegs = NT == 256 ? 88 : 0, kManyRegs = NT == 256 ? 208 : 0;
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int c0,
                                            int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// 16 lanes x 16 columns: registers 4 g .. 4 g + 3 of lane l hold columns 8 g + 2 (l % 4), + 1 of lane
// l / 4, and the same columns of lane l / 4 + 8.
__device__ __forceinline__ void tmem_ld_pairs(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7])
      : "r"(taddr));
}
// MN-major e4m3, 128-byte swizzle: a row of 128 bytes holds 128 consecutive M (or N) elements of one k;
// groups of 8 k lie 1024 B apart (stride offset), the next 128 elements 16384 B further (leading offset);
// 32 k further is + 256.
__device__ __forceinline__ uint64_t sdesc_mn8(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)(kOperand >> 4) << 16 |
         (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// Pairs of floats
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, float b) {
  uint64_t r;
  asm("{\n .reg .b64 t;\n mov.b64 t, {%2, %2};\n mul.rn.f32x2 %0, %1, t;\n}\n"
      : "=l"(r)
      : "l"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 floats(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint32_t bf16x2(uint64_t v) {
  const float2 f = floats(v);
  const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
  return *(const uint32_t*)&b;
}
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&v;
}
// 16 bytes of a row that may begin anywhere, of which `left` elements exist.
template <typename Out>
__device__ __forceinline__ void store_some(Out* p, int left, uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(Out); ++i) {
    if (i >= left) break;
    if (sizeof(Out) == 4) ((uint32_t*)p)[i] = w[i & 3];
    else ((uint16_t*)p)[i] = (uint16_t)(w[i / 2 & 3] >> 16 * (i & 1));
  }
}
// Four 8 x 8 matrices of 16-bit values whose fragments the lanes hold, transposed into rows of 16 bytes.
__device__ __forceinline__ void stmatrix_t(uint32_t dst, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(dst),
               "r"(a), "r"(b), "r"(c), "r"(d)
               : "memory");
}

// Operands landed and the accumulator free.  Both are asked at once: a wait that need not wait takes 180
// cycles where its answer is waited for, and the accumulator's, which every k-block waits for, comes last.
__device__ __forceinline__ bool both(uint64_t* full, uint32_t fp, uint64_t* tempty, uint32_t tp, WaitCtx wc) {
  const bool f = mbar_test_wait(full, fp), t = mbar_test_wait(tempty, tp);
  if (!f && !mbar_wait_inline(full, fp, wc, 8u)) return false;
  return t || mbar_wait_inline(tempty, tp, wc, 4u);
}

// The experts of a call, in shared memory: rows row[e] .. end[e] - 1 (held to [0, M]) and the row tiles of
// the experts below e; kGrad: first padded row, number of rows (-1: not all there), first block.
struct Experts {
  int row[kMaxExperts], end[kMaxExperts], tile0[kMaxExperts + 1];
};
// One tile: `rows` output rows from row0 (x's rows, or dw's n), columns from c0 on, of expert e; its sums'
// length and number of k-blocks (kGrad: from padded row k0, block b0).
struct Tile {
  int e, row0, rows, c0, nkb, k0, b0, sums;
};

// By a full warp: fills ex for row tiles of up to NT rows.
template <int MODE, int NT>
__device__ __forceinline__ void list_experts(const Args& a, Experts& ex) {
  const int lane = threadIdx.x & 31;
  // prefix sums over the experts; what follows the last one is in [E]
  int tiles = 0, padded = 0, blocks = 0, before = 0;
  const int cap = MODE == kGrad ? 1 << 30 : a.M;
  for (int e0 = 0; e0 < a.E; e0 += 32) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e < a.E) {
      lo = a.offsets ? max(0, min(a.offsets[e], cap)) : 0;
      hi = a.offsets ? max(lo, min(a.offsets[e + 1], cap)) : a.M;
    }
    in_order(lo, hi, before);
    const int n = hi - lo;
    int vt = (n + NT - 1) / NT, vp = (n + 31) & ~31, vb = (n + kBlock - 1) / kBlock;
    const int t = vt, p = vp, b = vb;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int ut = __shfl_up_sync(0xffffffffu, vt, o), up = __shfl_up_sync(0xffffffffu, vp, o),
                ub = __shfl_up_sync(0xffffffffu, vb, o);
      if (lane >= o) {
        vt += ut;
        vp += up;
        vb += ub;
      }
    }
    if (e < a.E) {
      if (MODE == kGrad) {
        // (offsets that are not those of the operands reach nothing outside of them: -1 rows, and a sum of NaN)
        const int k0 = padded + vp - p, b0 = blocks + vb - b;
        const bool fits = k0 >= 0 && b0 >= 0 && (long long)k0 + p <= a.M && (long long)b0 + b <= a.blocks;
        ex.row[e] = k0;
        ex.end[e] = fits || n == 0 ? n : -1;
        ex.tile0[e] = b0;
      } else {
        ex.row[e] = lo;
        ex.end[e] = hi;
        ex.tile0[e] = tiles + vt - t;
      }
    }
    tiles += __shfl_sync(0xffffffffu, vt, 31);
    padded += __shfl_sync(0xffffffffu, vp, 31);
    blocks += __shfl_sync(0xffffffffu, vb, 31);
  }
  if (lane == 0) ex.tile0[a.E] = tiles;
}

// Tile u of x's rows, in the order (expert, columns, rows): tiles that read the same part of a matrix
// follow each other.  The rows of an expert are cut into tiles of equal heights, a multiple of 16.
template <int COLS>
__device__ __forceinline__ Tile row_tile(const Args& a, const Experts& ex, int col_tiles, int inner,
                                         long long u) {
  Tile t;
  // the last expert whose tiles begin at or before u (its first column's, so that the search compares ints)
  const int q = u >> 32 ? (int)(u / col_tiles) : (int)((unsigned)u / (unsigned)col_tiles);
  int lo = 0, hi = a.E;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ex.tile0[mid] <= q) lo = mid;
    else hi = mid;
  }
  t.e = lo;
  const unsigned n = ex.end[lo] - ex.row[lo], count = ex.tile0[lo + 1] - ex.tile0[lo];
  const unsigned v = (unsigned)(u - (long long)ex.tile0[lo] * col_tiles);
  const unsigned h = ((n + count - 1) / count + 15) & ~15u;
  const unsigned c = v / count, i = v - c * count;
  t.row0 = ex.row[lo] + (int)(i * h);
  t.rows = (int)min(h, n - i * h);
  t.c0 = (int)c * COLS;
  t.sums = inner;
  t.k0 = t.b0 = 0;
  t.nkb = (inner + kBlock - 1) / kBlock;
  return t;
}

// The rows behind the last expert's, in pieces of 512 bytes of which every CTA takes its share: a warp
// clears some whenever it has time.
template <typename Out>
struct Behind {
  uint4* at = nullptr;
  long long pieces = 0, piece = 0;
  __device__ __forceinline__ Behind(const Args& a, const Experts& ex, int cols, bool any) {
    if (!any || !a.offsets) return;
    const int lane = threadIdx.x & 31;
    int end = 0;
    for (int e = lane; e < a.E; e += 32) end = max(end, ex.end[e]);
    end = (int)__reduce_max_sync(0xffffffffu, (unsigned)end);
    Out* const first = (Out*)a.out + (size_t)end * cols;
    Out* const last = (Out*)a.out + (size_t)a.M * cols;
    uint4* const begin = (uint4*)(((uintptr_t)first + 15) & ~(uintptr_t)15);
    uint4* const stop = (uint4*)((uintptr_t)last & ~(uintptr_t)15);
    if (blockIdx.x == 0) {  // what lies before and behind whole vectors
      const long long n = last - first, head = min(n, (long long)((Out*)begin - first));
      if (lane < head) first[lane] = Elem<Out>::put(0.f);
      const long long tail = stop >= begin ? last - (Out*)stop : 0;
      if (lane < tail) last[-1 - lane] = Elem<Out>::put(0.f);
    }
    at = begin + lane;
    piece = blockIdx.x;
    pieces = stop > begin ? ((long long)(stop - begin) + 31) / 32 : 0;
    if (pieces > 0 && at + (pieces - 1) * 32 >= stop) --pieces;  // this lane has none in the last
  }
  __device__ __forceinline__ void clear(int n) {
    for (; n > 0 && piece < pieces; --n, piece += gridDim.x) at[piece * 32] = make_uint4(0, 0, 0, 0);
  }
};

// By one thread, after the CTA's last wait.
__device__ __forceinline__ void report(const Args& a, const volatile unsigned int& err) {
  if (a.waits.status && err) atomicOr(a.waits.status, err);
}

template <int MODE, int NT, typename Out>
__global__ void __launch_bounds__(Cfg<NT>::kThreads, 1)
block_mm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const Args a) {
  using C = Cfg<NT>;
  static_assert(MODE != kGrad || C::kCols == kBlock, "columns of 128 bytes");
  constexpr int S = C::kStages, B = C::kBufs;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* const s_out = smem + S * C::kStage;
  float* const s_scale = (float*)(s_out + C::kOut);
  __shared__ uint64_t full[S], empty[S], tfull[B], tempty[B], mma_done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ unsigned int err_word;
  __shared__ Experts ex;
  volatile int* const abort_flag = &abort_word;
  const WaitCtx wc{abort_flag, &err_word, a.waits.limit_ns};

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < B; ++b) {
      mbar_init(&tfull[b], 2);  // the products and the scales
      mbar_init(&tempty[b], C::kEpiWarps);
    }
    mbar_init(&mma_done, 1);
    abort_word = 0;
    err_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_a);
    prefetch_map(&map_b);
  }
  if (warp == 1) tmem_alloc<false>(&tmem_slot, C::kTmemCols);
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) list_experts<MODE, NT>(a, ex);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;

  const int cols = MODE == kForward ? a.N : a.K, inner = MODE == kForward ? a.K : a.N;
  const int col_tiles = (cols + kBlock - 1) / kBlock;
  const int n_tiles = (a.N + NT - 1) / NT;  // kGrad, and their rows
  const int grad_rows = ((a.N + n_tiles - 1) / n_tiles + 15) & ~15;
  const long long units = (long long)(MODE == kGrad ? a.E * n_tiles : ex.tile0[a.E]) * col_tiles;
  auto tile_at = [&](long long u) {
    Tile t;
    if (MODE == kGrad) {
      // (below 2^25 tiles: 32-bit divisions)
      const unsigned per = n_tiles * col_tiles, e = (unsigned)u / per, v = (unsigned)u - e * per;
      const unsigned c = v / (unsigned)n_tiles, i = v - c * n_tiles;
      t.e = (int)e;
      t.row0 = (int)i * grad_rows;
      t.rows = min(grad_rows, a.N - t.row0);
      t.c0 = (int)c * kBlock;
      t.sums = ex.end[t.e];
      t.k0 = ex.row[t.e];
      t.b0 = ex.tile0[t.e];
    } else {
      return row_tile<kBlock>(a, ex, col_tiles, inner, u);
    }
    t.nkb = (t.sums + kBlock - 1) / kBlock;
    return t;
  };

  if (warp < kFirstEpi) {
    if constexpr (C::kFewRegs > 0)
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kFewRegs));
    if (warp == 0) {
      if (elect_one()) {
        int stage = 0;
        uint32_t phase = 0;
        long long issued = 0;
        const long long held = (int)blockIdx.x == a.waits.held_cta ? a.waits.held_after : -1;
        bool ok = true;
        for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
          const Tile t = tile_at(u);
          for (int kb = 0; kb < t.nkb; ++kb) {
            if (issued == held || !mbar_wait_inline(&empty[stage], phase ^ 1u, wc, 1u)) {
              ok = false;
              break;
            }
            uint8_t* const sa = smem + stage * C::kStage;
            uint8_t* const sb = sa + kOperand;
            uint64_t* const bar = &full[stage];
            if (MODE == kGrad) {
              const int k = t.k0 + kb * kBlock, boxes = (min(kBlock, t.sums - kb * kBlock) + 31) / 32;
              const int chunks = (t.rows + kBlock - 1) / kBlock;
              mbar_expect_tx(bar, (1 + chunks) * boxes * 32 * kBlock);
              for (int i = 0; i < boxes; ++i) {
                tma_load(sa + i * 32 * kBlock, &map_a, bar, t.c0, k + 32 * i);
                for (int c = 0; c < chunks; ++c)
                  tma_load(sb + c * kOperand + i * 32 * kBlock, &map_b, bar, t.row0 + c * kBlock, k + 32 * i);
              }
            } else {
              const int k = kb * kBlock, boxes = (t.rows + C::kBox - 1) / C::kBox;
              mbar_expect_tx(bar, kOperand + boxes * C::kBox * kBlock);
              if (MODE == kForward) tma_load_3d(sa, &map_a, bar, k, t.c0, t.e);
              else tma_load_3d(sa, &map_a, bar, t.c0, k, t.e);
              for (int i = 0; i < boxes; ++i)
                tma_load(sb + i * C::kBox * kBlock, &map_b, bar, k, t.row0 + i * C::kBox);
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
        int stage = 0, buf = 0;
        uint32_t phase = 0, bphase = 0;
        bool ok = true;
        for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
          const Tile t = tile_at(u);
          const uint32_t id = idesc(true, kBlock, (t.rows + 15) & ~15, MODE != kForward, MODE == kGrad);
          for (int kb = 0; kb < t.nkb; ++kb) {
            if (!both(&full[stage], phase, &tempty[buf], bphase ^ 1u, wc)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem + stage * C::kStage);
            const uint64_t da = MODE == kForward ? sdesc_k(sa) : sdesc_mn8(sa);
            const uint64_t db = MODE == kGrad ? sdesc_mn8(sa + kOperand) : sdesc_k(sa + kOperand);
            const uint32_t d = tmem_base + (uint32_t)(buf * NT);
            const int steps = (min(kBlock, t.sums - kb * kBlock) + 31) / 32;
            for (int k = 0; k < steps; ++k)
              mma<false, true>(d, da + k * (MODE == kForward ? 2 : 256), db + k * (MODE == kGrad ? 256 : 2),
                               id, k > 0);
            mma_commit<false>(&empty[stage]);
            mma_commit<false>(&tfull[buf]);
            if (++stage == S) {
              stage = 0;
              phase ^= 1u;
            }
            if (++buf == B) {
              buf = 0;
              bphase ^= 1u;
            }
          }
        }
        mma_commit<false>(&mma_done);  // no MMA may run when TMEM is freed
      }
      // (the whole warp: the wait's limit counts from the last MMA's issue, whichever lane issues)
      __syncwarp();
      if (lane == 0) mbar_wait(&mma_done, 0u, wc, 16u, false);
    } else if (warp == 2) {
      Behind<Out> behind(a, ex, cols, MODE != kGrad);
      // The copies of k-block i are issued kAhead before those of i - kAhead are handed over, which is once
      // the accumulator that goes with them is free: then so is the slot that comes kBufs before it.
      long long u = blockIdx.x;
      Tile t{};
      int kb = 0, copy = 0, buf = 0;
      uint32_t bphase = 0;
      auto next = [&] {  // the tile of the next k-block to copy; false behind the last
        while (kb == t.nkb) {
          if (u >= units) return false;
          t = tile_at(u);
          u += gridDim.x;
          kb = 0;
        }
        return true;
      };
      const int nb = (a.N + kBlock - 1) / kBlock, kbs = (a.K + kBlock - 1) / kBlock;
      int pending = 0;
      for (int i = 0;; ++i) {
        if (i >= kAhead) {
          if (pending == 0) break;
          cp_async_wait<kAhead - 1>();
          __syncwarp();
          if (!warp_wait(&tempty[buf], bphase ^ 1u, wc, 64u)) break;
          if (lane == 0) mbar_arrive(&tfull[buf]);
          --pending;
          if (++buf == B) {
            buf = 0;
            bphase ^= 1u;
          }
        }
        if (next()) {
          const uint32_t dst = smem_u32(s_scale + copy * C::kSlotFloats);
          const float* rs =
              (MODE == kGrad ? a.xs + (size_t)(t.b0 + kb) * a.N : a.xs + (size_t)kb * a.M) + t.row0;
#pragma unroll
          for (int j = 0; j < NT; j += 32)
            if (j + lane < t.rows) cp_async4(dst + (j + lane) * 4, rs + j + lane);
          if (MODE == kGrad) {
            const float* cs = a.ws + (size_t)(t.b0 + kb) * a.K;
#pragma unroll
            for (int j = 0; j < kBlock; j += 32)
              cp_async4(dst + (NT + j + lane) * 4, cs + min(t.c0 + j + lane, a.K - 1));
          } else if (lane == 0) {
            const size_t at = MODE == kForward ? ((size_t)t.e * nb + t.c0 / kBlock) * kbs + kb
                                               : ((size_t)t.e * nb + kb) * kbs + t.c0 / kBlock;
            cp_async4(dst + NT * 4, a.ws + at);
          }
          ++kb;
          ++pending;
          if (++copy == C::kSlots) copy = 0;
        }
        cp_async_commit();  // (one group an iteration, whether it holds a copy or not)
        if (MODE != kGrad) behind.clear(8);
      }
      if (MODE != kGrad) behind.clear(1 << 30);
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else {
    if constexpr (C::kManyRegs > 0)
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kManyRegs));
    const int q = warp & 3, ch = (warp - kFirstEpi) >> 2;  // quarter of the columns, half of the rows
    const uint32_t tq = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(ch * C::kCols);
    uint4* const box = (uint4*)(s_out + (warp - kFirstEpi) * 32 * 64);
    int slot = 0, buf = 0;
    uint32_t bphase = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
      const Tile t = tile_at(u);
      // acc[g][i]: rows 8 g + 2 (lane % 4), + 1, column 8 i + lane / 4 of the warp's
      uint64_t acc[C::kCols / 8][4];
#pragma unroll
      for (int g = 0; g < C::kCols / 8; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[g][i] = 0;
      const int live = t.rows - ch * C::kCols;  // rows of this warp
      for (int kb = 0; ok && kb < t.nkb; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait_inline(&tfull[buf], bphase, wc, 32u))) {
          ok = false;
          break;
        }
        tc_fence_after();
        const float* const sc = s_scale + slot * C::kSlotFloats;
        const uint32_t tb = tq + (uint32_t)(buf * NT);
        float f[4];  // of the thread's columns
        if (MODE == kGrad) {
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = sc[NT + 32 * q + 8 * i + (lane >> 2)];
        } else {
          f[0] = sc[NT];
        }
        // a chunk's loads run while the one before it is added
        uint32_t w[2][2][8];
        tmem_ld_pairs(tb, w[0][0]);
        tmem_ld_pairs(tb + (16u << 16), w[0][1]);
#pragma unroll
        for (int c = 0; c < C::kChunks; ++c) {
          uint64_t s[2];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            s[g] = *(const uint64_t*)(sc + ch * C::kCols + 16 * c + 8 * g + 2 * (lane & 3));
            if (MODE != kGrad) s[g] = mul2(s[g], f[0]);
          }
          tmem_wait_ld();
          if (c + 1 < C::kChunks) {
            tmem_ld_pairs(tb + (uint32_t)(16 * (c + 1)), w[(c + 1) & 1][0]);
            tmem_ld_pairs(tb + (uint32_t)(16 * (c + 1)) + (16u << 16), w[(c + 1) & 1][1]);
          }
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t* const v = &w[c & 1][i >> 1][4 * g + 2 * (i & 1)];
              uint64_t& d = acc[2 * c + g][i];
              d = fma2(pair(v[0], v[1]), MODE == kGrad ? mul2(s[g], f[i]) : s[g], d);
            }
          if (16 * (c + 1) >= live) break;
        }
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&tempty[buf]);
        if (++slot == C::kSlots) slot = 0;
        if (++buf == B) {
          buf = 0;
          bphase ^= 1u;
        }
      }
      // (here and not where the sums begin, which cost dw of 64 matrices of 2048 x 2048 207 -> 221 us)
      if (!ok || (MODE == kGrad && t.sums < 0)) {
#pragma unroll
        for (int g = 0; g < C::kCols / 8; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[g][i] = pair(0x7fc00000u, 0x7fc00000u);
      }
      // out[row][column]: rows of 32 columns of this warp
      const size_t row0 = (MODE == kGrad ? (size_t)t.e * a.N : 0) + t.row0 + ch * C::kCols;
      const int col = t.c0 + 32 * q;
      Out* const out = (Out*)a.out + row0 * cols + col;
      if (sizeof(Out) == 4) {
        // eight lanes with the same lane % 4 store a sector of a row
#pragma unroll
        for (int g = 0; g < C::kCols / 8; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = floats(acc[g][i]);
            const int r = 8 * g + 2 * (lane & 3), c = 8 * i + (lane >> 2);
            if (col + c < cols) {
              if (r < live) out[(size_t)r * cols + c] = Elem<Out>::put(v.x);
              if (r + 1 < live) out[(size_t)(r + 1) * cols + c] = Elem<Out>::put(v.y);
            }
          }
      } else {
        // 32 rows at a time through shared memory, whose pieces of 16 bytes are exchanged by row
        constexpr int kRows = C::kCols < 32 ? C::kCols : 32;
#pragma unroll
        for (int r0 = 0; r0 < C::kCols; r0 += kRows) {
          if (r0 >= live) break;
          __syncwarp();
#pragma unroll
          for (int g = 0; g < kRows / 8; ++g) {
            const int r = 8 * g + (lane & 7), piece = lane >> 3;
            const uint64_t(&v)[4] = acc[r0 / 8 + g];
            stmatrix_t(smem_u32(box + r * 4 + (piece ^ ((r >> 1) & 3))), bf16x2(v[0]), bf16x2(v[1]),
                       bf16x2(v[2]), bf16x2(v[3]));
          }
          __syncwarp();
          const int c = 8 * (lane & 3);
          uint4 v[kRows / 8];
#pragma unroll
          for (int k = 0; k < kRows / 8; ++k) {
            const int r = 8 * k + (lane >> 2);
            v[k] = box[r * 4 + ((lane & 3) ^ ((r >> 1) & 3))];
          }
          Out* p = out + (size_t)(r0 + (lane >> 2)) * cols + c;
          const int rows = live - r0 - (lane >> 2);
          if (a.vec && col + 32 <= cols) {
#pragma unroll
            for (int k = 0; k < kRows / 8; ++k)
              if (8 * k < rows) *(uint4*)(p + (size_t)(8 * k) * cols) = v[k];
          } else {
#pragma unroll
            for (int k = 0; k < kRows / 8; ++k)
              if (8 * k < rows) store_some(p + (size_t)(8 * k) * cols, cols - col - c, v[k]);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0) report(a, err_word);
  if (warp == 1) tmem_dealloc<false>(tmem_base, C::kTmemCols);
}

// ------------------------------------------------------------------------------ many rows an expert
// On an SM pair (cta_group::2): up to 256 of x's rows (M, half of them each CTA's) x 256 columns (N).  A
// thread owns a row of 128 columns, so a k-block's scales are one product a thread: its row's times the
// columns' block's, loaded kLead k-blocks ahead.
struct Wide {
  static constexpr int kRows = 256, kCols = 256;
  static constexpr int kStage = 2 * kOperand, kStages = 6;
  static constexpr int kEpiWarps = 8, kThreads = 32 * (kFirstEpi + kEpiWarps);
  static constexpr int kOut = kEpiWarps * 32 * 64;
  static constexpr int kSmem = 1024 + kStages * kStage + kOut;
  static constexpr int kLead = 4;
  static constexpr int kFewRegs = 88, kManyRegs = 208;  // as above
};

__device__ __forceinline__ void tma_load_pair_3d(void* dst, const CUtensorMap* map, uint32_t bar, int c0,
                                                 int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}

template <int MODE, typename Out>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Wide::kThreads, 1)
wide_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
            const Args a) {
  using C = Wide;
  constexpr int S = C::kStages, L = C::kLead;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t full[S], empty[S], tfull[2], tempty[2], mma_done;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ unsigned int err_word;
  __shared__ Experts ex;
  volatile int* const abort_flag = &abort_word;
  const WaitCtx wc{abort_flag, &err_word, a.waits.limit_ns};

  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], 2 * C::kEpiWarps);  // the epilogue's warps of both CTAs (rank 0's)
    }
    mbar_init(&mma_done, 1);
    abort_word = 0;
    err_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&map_w);
    prefetch_map(&map_x);
  }
  if (warp == 1) tmem_alloc<true>(&tmem_slot, 512);
  pdl_wait();
  pdl_launch_dependents();
  if (warp == 0) list_experts<MODE, C::kRows>(a, ex);
  tc_fence_before();
  cluster_sync_all();  // both CTAs' barriers exist before either signals the other
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;

  const int cols = MODE == kForward ? a.N : a.K, inner = MODE == kForward ? a.K : a.N;
  const int col_tiles = (cols + C::kCols - 1) / C::kCols;
  const long long units = (long long)ex.tile0[a.E] * col_tiles;
  const long long first = blockIdx.x >> 1, step = gridDim.x >> 1;
  auto tile_at = [&](long long u) { return row_tile<C::kCols>(a, ex, col_tiles, inner, u); };
  // rows of a CTA: rank 0's half is a multiple of 16
  auto half = [](int rows) { return min(rows, ((rows + 1) / 2 + 15) & ~15); };
  const uint32_t full0 = map_rank(smem_u32(full), 0), tempty0 = map_rank(smem_u32(tempty), 0);

  if (warp < kFirstEpi) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kFewRegs));
    if (warp == 0) {
      if (elect_one()) {
        int stage = 0;
        uint32_t phase = 0;
        long long issued = 0;
        const long long held = (int)blockIdx.x == a.waits.held_cta ? a.waits.held_after : -1;
        bool ok = true;
        for (long long u = first; ok && u < units; u += step) {
          const Tile t = tile_at(u);
          const int h = half(t.rows), box0 = (h + 31) / 32, box1 = (t.rows - h + 31) / 32;
          const int boxes = leader ? box0 : box1, row0 = t.row0 + (leader ? 0 : h);
          const int c0 = t.c0 + (int)rank * kBlock;
          const uint32_t bytes = (uint32_t)(2 * kOperand + (box0 + box1) * 32 * kBlock);
          for (int kb = 0; kb < t.nkb; ++kb) {
            if (issued == held || !mbar_wait_inline(&empty[stage], phase ^ 1u, wc, 1u)) {
              ok = false;
              break;
            }
            uint8_t* const sa = smem + stage * C::kStage;
            uint8_t* const sb = sa + kOperand;
            const uint32_t bar = full0 + 8u * (uint32_t)stage;
            if (leader) mbar_expect_tx(&full[stage], bytes);
            const int k = kb * kBlock;
            if (MODE == kForward) tma_load_pair_3d(sb, &map_w, bar, k, c0, t.e);
            else tma_load_pair_3d(sb, &map_w, bar, c0, k, t.e);
            for (int i = 0; i < boxes; ++i)
              tma_load_pair(sa + i * 32 * kBlock, &map_x, bar, k, row0 + 32 * i);
            ++issued;
            if (++stage == S) {
              stage = 0;
              phase ^= 1u;
            }
          }
        }
        // rank 0: the copies of both CTAs still in flight land before the pair may exit
        if (leader)
          for (long long i = issued > S ? issued - S : 0; i < issued; ++i)
            mbar_wait(&full[i % S], (uint32_t)((i / S) & 1), wc, 2u, false);
      }
    } else if (warp == 1) {
      if (leader && elect_one()) {
        constexpr uint32_t id = idesc(true, C::kRows, C::kCols, false, MODE == kBack);
        int stage = 0, buf = 0;
        uint32_t phase = 0, bphase = 0;
        bool ok = true;
        for (long long u = first; ok && u < units; u += step) {
          const Tile t = tile_at(u);
          for (int kb = 0; kb < t.nkb; ++kb) {
            if (!both(&full[stage], phase, &tempty[buf], bphase ^ 1u, wc)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem + stage * C::kStage);
            const uint64_t da = sdesc_k(sa);
            const uint64_t db = MODE == kBack ? sdesc_mn8(sa + kOperand) : sdesc_k(sa + kOperand);
            const uint32_t d = tmem_base + (uint32_t)(buf * C::kCols);
            const int steps = (min(kBlock, inner - kb * kBlock) + 31) / 32;
            for (int k = 0; k < steps; ++k)
              mma<true, true>(d, da + 2 * k, db + k * (MODE == kBack ? 256 : 2), id, k > 0);
            mma_commit<true>(&empty[stage]);
            mma_commit<true>(&tfull[buf]);
            if (++stage == S) {
              stage = 0;
              phase ^= 1u;
            }
            if (++buf == 2) {
              buf = 0;
              bphase ^= 1u;
            }
          }
        }
        mma_commit<true>(&mma_done);
      }
      __syncwarp();
      if (leader && lane == 0) mbar_wait(&mma_done, 0u, wc, 16u, false);
    } else if (warp == 2) {
      Behind<Out> behind(a, ex, cols, true);
      behind.clear(1 << 30);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kManyRegs));
    const int q = warp & 3, ch = (warp - kFirstEpi) >> 2;  // quarter of the rows, half of the columns
    const uint32_t tq = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(ch * kBlock);
    uint4* const box = (uint4*)(smem + S * C::kStage) + (warp - kFirstEpi) * 128;
    const int nb = (a.N + kBlock - 1) / kBlock, kbs = (a.K + kBlock - 1) / kBlock;
    int buf = 0;
    uint32_t bphase = 0;
    bool ok = true;
    Tile t{};
    float xs[L], ws[L];
    const float *px = nullptr, *pw = nullptr;
    int live = 0, row0 = 0;  // of this CTA's rows
    size_t wstep = 0;
    auto begin = [&](long long u) {  // the tile and its first scales
      t = tile_at(u);
      const int h = half(t.rows);
      row0 = t.row0 + (leader ? 0 : h);
      live = leader ? h : t.rows - h;
      const int cb = min(t.c0 / kBlock + ch, (cols + kBlock - 1) / kBlock - 1);
      px = a.xs + min(row0 + 32 * q + lane, a.M - 1);
      pw = a.ws + (size_t)t.e * nb * kbs + (MODE == kForward ? (size_t)cb * kbs : (size_t)cb);
      wstep = MODE == kForward ? 1 : (size_t)kbs;
      // (the k-blocks behind the last are not used: they repeat it)
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if (i > 0) {
          px += i < t.nkb ? a.M : 0;
          pw += i < t.nkb ? wstep : 0;
        }
        xs[i] = *px;
        ws[i] = *pw;
      }
    };
    bool ready = false;
    if (first < units) begin(first);
    for (long long u = first; u < units;) {
      float acc[kBlock];
#pragma unroll
      for (int j = 0; j < kBlock; ++j) acc[j] = 0.f;
      const bool mine = live > 32 * q && t.c0 + ch * kBlock < cols;  // of the warp's quarter and half
      // What a k-block costs beside its products counts as much as they do (110 cycles a barrier whose
      // answer is waited for, of 500): the next accumulator is asked for before this one is added, the
      // scales' loads have no branch, and the loop is unrolled, so that a scale stays in the register that
      // it is loaded into (a move would wait for it).
      for (int kb0 = 0; ok && kb0 < t.nkb; kb0 += L) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
          if (kb0 + i >= t.nkb) break;
          if (!__all_sync(0xffffffffu, ready) &&
              !__all_sync(0xffffffffu, mbar_wait_inline(&tfull[buf], bphase, wc, 32u))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t tb = tq + (uint32_t)(buf * C::kCols), free_bar = tempty0 + 8u * (uint32_t)buf;
          buf ^= 1;
          bphase ^= buf ^ 1u;
          ready = mbar_test_wait(&tfull[buf], bphase);
          if (mine) {
            const float f = xs[i] * ws[i];
#pragma unroll
            for (int c = 0; c < kBlock; c += 32) {
              uint32_t w[32];
              tmem_ld16(tb + c, w);
              tmem_ld16(tb + c + 16, w + 16);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; ++j) acc[c + j] = fmaf(__uint_as_float(w[j]), f, acc[c + j]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(free_bar);
          const bool more = kb0 + i + L < t.nkb;
          px += more ? a.M : 0;
          pw += more ? wstep : 0;
          xs[i] = *px;
          ws[i] = *pw;
        }
      }
      if (!ok) {
#pragma unroll
        for (int j = 0; j < kBlock; ++j) acc[j] = NAN;
      }
      // The warp's rows, 64 bytes of each at a time through shared memory (lane: row, then four lanes a row):
      // pieces of 16 bytes whose place is exchanged by row.
      const int last = live - 32 * q, col = t.c0 + ch * kBlock;
      Out* const out = (Out*)a.out + (size_t)(row0 + 32 * q) * cols + col;
      const bool store = mine;
      u += step;
      if (u < units) begin(u);  // (its scales come while this tile is stored)
      if (!store) continue;
      constexpr int kPer = 64 / sizeof(Out), kVec = 16 / sizeof(Out);
#pragma unroll
      for (int c = 0; c < kBlock; c += kPer) {
        if (col + c >= cols) break;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float* const v = acc + c + j * kVec;
          uint4 p;
          if (sizeof(Out) == 4)
            p = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                           __float_as_uint(v[3]));
          else
            p = make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4 % kVec], v[5 % kVec]),
                           bf16x2(v[6 % kVec], v[7 % kVec]));
          box[lane * 4 + (j ^ ((lane >> 1) & 3))] = p;
        }
        __syncwarp();
        const int cc = c + (lane & 3) * kVec, rows = last - (lane >> 2);
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 8 * k + (lane >> 2);
          v[k] = box[r * 4 + ((lane & 3) ^ ((r >> 1) & 3))];
        }
        Out* p = out + (size_t)(lane >> 2) * cols + cc;
        if (a.vec && col + c + kPer <= cols) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (8 * k < rows) *(uint4*)(p + (size_t)(8 * k) * cols) = v[k];
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (8 * k < rows) store_some(p + (size_t)(8 * k) * cols, cols - col - cc, v[k]);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // Rank 1 issues no MMA, so its wait for the pair's last one begins where its own tiles are done: from the
  // kernel's begin its limit would bound the whole call, not a step (5e5 rows of 65536 x 65536 take longer).
  if (!leader && warp == 1) {
    if (lane == 0) mbar_wait(&mma_done, 0u, wc, 16u, false);
    __syncwarp();
  }
  cluster_sync_all();  // neither CTA leaves while the other may still signal it
  tc_fence_after();
  if (threadIdx.x == 0) report(a, err_word);
  if (warp == 1) tmem_dealloc<true>(tmem_base, 512);
}

// -------------------------------------------------------------------------------- host side
// Whether a kernel was launched with the registers that its warps share out (setmaxnreg would wait for the
// rest forever).  Once per kernel: it is a property of the code.
template <typename K>
cudaError_t shares_registers(K* kernel, int threads, int few, int many) {
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, kernel);
  if (e != cudaSuccess || few == 0) return e;
  const int first = 32 * kFirstEpi;
  return at.numRegs * threads >= few * first + many * (threads - first) ? cudaSuccess
                                                                      : cudaErrorInvalidKernelImage;
}

template <int MODE>
cudaError_t run_wide(const CUtensorMap& mw, const CUtensorMap& mx, const Args& a, int out_dtype, int sms,
                     cudaStream_t st) {
  const int cols = MODE == kForward ? a.N : a.K;
  const long long tiles = std::min((long long)a.M, (a.M + (long long)a.E * (Wide::kRows - 1)) / Wide::kRows) *
                          ((cols + Wide::kCols - 1) / Wide::kCols);
  const int pairs = (int)std::min<long long>(std::max(1, sms / 2), tiles);
  auto go = [&](auto* kernel) {
    static std::atomic<bool> seen[2];
    std::atomic<bool>& checked = seen[out_dtype == EAT_BF16];
    cudaError_t e = cudaSuccess;
    if (!checked.load(std::memory_order_relaxed)) {
      e = shares_registers(kernel, Wide::kThreads, Wide::kFewRegs, Wide::kManyRegs);
      if (e == cudaSuccess) checked.store(true, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Wide::kSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(2 * pairs), dim3(Wide::kThreads), Wide::kSmem, st, mw, mx, a);
  };
  return out_dtype == EAT_BF16 ? go(wide_kernel<MODE, __nv_bfloat16>) : go(wide_kernel<MODE, float>);
}

template <int MODE, int NT>
cudaError_t run_nt(const CUtensorMap& ma, const CUtensorMap& mb, const Args& a, int out_dtype, int ctas,
                   cudaStream_t st) {
  auto go = [&](auto* kernel) {
    // (the kernel's own limit, whatever the call: it cannot be lowered between this and the launch)
    using C = Cfg<NT>;
    static std::atomic<bool> seen[2];  // (the two output types' kernels)
    std::atomic<bool>& checked = seen[out_dtype == EAT_BF16];
    cudaError_t e = cudaSuccess;
    if (!checked.load(std::memory_order_relaxed)) {
      e = shares_registers(kernel, C::kThreads, C::kFewRegs, C::kManyRegs);
      if (e == cudaSuccess) checked.store(true, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(ctas), dim3(Cfg<NT>::kThreads), Cfg<NT>::kSmem, st, ma, mb, a);
  };
  return out_dtype == EAT_BF16 ? go(block_mm_kernel<MODE, NT, __nv_bfloat16>)
                               : go(block_mm_kernel<MODE, NT, float>);
}

template <int MODE>
eat_status run(const char* fn, const void* x, const void* w, const Args& a, int out_dtype,
               cudaStream_t st) {
  int device = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return launched(fn, e);
  const int cols = MODE == kForward ? a.N : a.K, col_tiles = (cols + kBlock - 1) / kBlock;
  // at most, for tiles of up to n rows
  auto tiles_of = [&](int n) {
    if (MODE == kGrad) return (long long)a.E * ((a.N + n - 1) / n) * col_tiles;
    return std::min((long long)a.M, (a.M + (long long)a.E * (n - 1)) / n) * col_tiles;
  };
  // Rows of a tile: what an expert has on average, with room.  32 matrices of 2048 x 2048, 48 rows each: tiles
  // of 64 28.4 us, 128 31.5, 256 36.0; 96 rows: 44.5, 38.7, 43.0, on pairs 43.5; 128 rows: 50.7, 40.7,
  // 46.9, 44.8; 160 rows: 62.4, 48.0, 48.2, 45.7; 256 rows: 97.0, 69.4, 59.0, 55.1.
  int nt = 256;  // (kGrad: its operands come in columns of 128, a warp's half)
  bool wide = false;
  if (MODE != kGrad) {
    const int rows = (a.M + a.E - 1) / a.E;
    nt = rows <= 16 ? 32 : rows <= 48 ? 64 : 128;
    wide = rows > 144;
    // Where tiles are few, the lowest that all run at the same time: a tile's time is mostly latency and its
    // share of the epilogue (1000 rows, 512 x 2048: 32 to 64 rows 8.6 us, 128 10.1, 256 14.6, on pairs 13.3).
    // Of 256 rows only short sums, as pairs start 1 us later and take less for each k-block (777 rows, 4096 x
    // 1408: 11.7 us, on pairs 12.6; 531 rows, 4096 x 4096: 23.1 and 21.1; between 11 and 32 k-blocks nothing was
    // measured).  M counts the rows behind the last expert's too: with 60 % of them live the best tile of 160 and
    // 192 rows of 64 experts is 4 to 5 % faster than this rule's.
    const int nkb = ((MODE == kForward ? a.K : a.N) + kBlock - 1) / kBlock;
    for (int n = 32; n <= (nkb <= 12 ? 256 : 128); n *= 2)
      if (tiles_of(n) <= sms) {
        nt = n;
        wide = false;
        break;
      }
  }
  const int box = MODE == kGrad || wide ? 32 : std::min(nt, 64);
  CUtensorMap ma, mb;
  bool ok;
  if (MODE == kGrad)
    ok = encode_bytes(&ma, 2, w, a.K, a.M, 1, box) && encode_bytes(&mb, 2, x, a.N, a.M, 1, box);
  else
    ok = encode_bytes(&ma, 3, w, a.K, a.N, a.E, kBlock) &&
         encode_bytes(&mb, 2, x, MODE == kForward ? a.K : a.N, a.M, 1, box);
  if (!ok) return thread_fail(EAT_ERR_CUDA, "%s: tensor map", fn);
  if constexpr (MODE != kGrad)
    if (wide) return launched(fn, run_wide<MODE>(ma, mb, a, out_dtype, sms, st));
  const int ctas = (int)std::min<long long>(sms, tiles_of(nt));
  if (nt == 256) e = run_nt<MODE, 256>(ma, mb, a, out_dtype, ctas, st);
  else if constexpr (MODE != kGrad)
    e = nt == 128  ? run_nt<MODE, 128>(ma, mb, a, out_dtype, ctas, st)
        : nt == 64 ? run_nt<MODE, 64>(ma, mb, a, out_dtype, ctas, st)
                   : run_nt<MODE, 32>(ma, mb, a, out_dtype, ctas, st);
  return launched(fn, e);
}

const char* bad_shape(int32_t E, int32_t M, int32_t N, int32_t K, const void* offsets,
                      int32_t out_dtype) {
  if (E < 1 || E > kMaxExperts) return "need 1 <= E <= 256";
  if (M < 1 || M > 1 << 30) return "need between 1 and 2^30 rows";
  if (N < 1 || N > 65536 || K < 1 || K > 65536) return "need N and K between 1 and 65536";
  if (!offsets && E != 1) return "several experts need offsets";
  if (out_dtype != EAT_BF16 && out_dtype != EAT_F32) return "the output's dtype must be F32 or BF16";
  return nullptr;
}

}  // namespace
}  // namespace eat

using namespace eat;

namespace {

eat_status product(const char* fn, const void* xq, const float* xs, const void* wq, const float* ws,
                   const int32_t* offsets, int32_t E, int32_t M, int32_t N, int32_t K, int32_t transposed,
                   void* y, int32_t ydtype, const Waits& waits, void* stream) {
  if (!xq || !xs || !wq || !ws || !y) return bad_arg(fn, "xq, xs, wq, ws and y must be non-NULL");
  if (const char* why = bad_shape(E, M, N, K, offsets, ydtype)) return bad_arg(fn, why);
  if (K % 16 || (transposed && N % 16))
    return thread_fail(EAT_ERR_UNSUPPORTED, "%s: K (transposed: and N) must be multiples of 16", fn);
  if (misaligned(xq, 16) || misaligned(wq, 16) || misaligned(xs, 4) || misaligned(ws, 4) ||
      misaligned(offsets, 4) || misaligned(y, ydtype == EAT_BF16 ? 2 : 4))
    return bad_arg(fn, "misaligned pointer");
  const size_t out = (size_t)M * (transposed ? K : N) * (ydtype == EAT_BF16 ? 2 : 4);
  const int inner = transposed ? N : K;
  if (overlaps({{y, out}}, {{xq, (size_t)M * inner},
                            {xs, 4 * (size_t)blocks_of(inner) * M},
                            {wq, (size_t)E * N * K},
                            {ws, 4 * (size_t)E * blocks_of(N) * blocks_of(K)},
                            {offsets, 4 * (size_t)(E + 1)}}))
    return bad_arg(fn, "y overlaps another array");
  const int vec = !misaligned(y, 16) && (transposed ? K : N) % 8 == 0;
  const Args a{xs, ws, offsets, E, M, N, K, 0, y, vec, waits};
  const cudaStream_t st = (cudaStream_t)stream;
  return transposed ? run<kBack>(fn, xq, wq, a, ydtype, st) : run<kForward>(fn, xq, wq, a, ydtype, st);
}

eat_status product_grad(const char* fn, const void* gq, const float* gs, const void* xq, const float* xs,
                        const int32_t* offsets, int32_t E, int32_t rows, int32_t blocks, int32_t N,
                        int32_t K, void* dw, int32_t dtype, const Waits& waits, void* stream) {
  if (!gq || !gs || !xq || !xs || !dw) return bad_arg(fn, "gq, gs, xq, xs and dw must be non-NULL");
  if (const char* why = bad_shape(E, rows, N, K, offsets, dtype)) return bad_arg(fn, why);
  // (eat_quant_columns makes no others; an expert whose rows or blocks are not all there would count as empty)
  if (rows % 32) return bad_arg(fn, "rows must be a multiple of 32");
  if (blocks < (rows + kBlock - 1) / kBlock) return bad_arg(fn, "need blocks >= rows / 128");
  if (N % 16 || K % 16)
    return thread_fail(EAT_ERR_UNSUPPORTED, "%s: N and K must be multiples of 16", fn);
  if (misaligned(gq, 16) || misaligned(xq, 16) || misaligned(gs, 4) || misaligned(xs, 4) ||
      misaligned(offsets, 4) || misaligned(dw, dtype == EAT_BF16 ? 2 : 4))
    return bad_arg(fn, "misaligned pointer");
  const size_t out = (size_t)E * N * K * (dtype == EAT_BF16 ? 2 : 4);
  if (overlaps({{dw, out}}, {{gq, (size_t)rows * N},
                             {gs, 4 * (size_t)blocks * N},
                             {xq, (size_t)rows * K},
                             {xs, 4 * (size_t)blocks * K},
                             {offsets, 4 * (size_t)(E + 1)}}))
    return bad_arg(fn, "dw overlaps another array");
  const Args a{gs, xs, offsets, E, rows, N, K, blocks, dw, !misaligned(dw, 16), waits};
  return run<kGrad>(fn, gq, xq, a, dtype, (cudaStream_t)stream);
}

// (copies that nothing waits for have landed long before a millisecond is over)
const char* bad_waits(int64_t limit_ns, int32_t cta, int64_t copies, const void* status) {
  if (limit_ns < 1000000 || limit_ns > 1000000000) return "limit_ns must be in [1e6, 1e9]";
  if (cta >= 0 && copies < 0) return "copies must not be negative";
  if (!status || misaligned(status, 4)) return "status must be a device word";
  return nullptr;
}

}  // namespace

extern "C" eat_status eat_block_mm(const void* xq, const float* xs, const void* wq, const float* ws,
                                   const int32_t* offsets, int32_t E, int32_t M, int32_t N, int32_t K,
                                   int32_t transposed, void* y, int32_t ydtype, void* stream) {
  return product("eat_block_mm", xq, xs, wq, ws, offsets, E, M, N, K, transposed, y, ydtype, Waits{}, stream);
}

extern "C" eat_status eat_block_mm_selftest(const void* xq, const float* xs, const void* wq,
                                            const float* ws, const int32_t* offsets, int32_t E, int32_t M,
                                            int32_t N, int32_t K, int32_t transposed, void* y,
                                            int32_t ydtype, int64_t limit_ns, int32_t cta, int64_t copies,
                                            uint32_t* status, void* stream) {
  const char* fn = "eat_block_mm_selftest";
  if (const char* why = bad_waits(limit_ns, cta, copies, status)) return bad_arg(fn, why);
  return product(fn, xq, xs, wq, ws, offsets, E, M, N, K, transposed, y, ydtype,
                 Waits{(unsigned long long)limit_ns, cta, copies, status}, stream);
}

extern "C" eat_status eat_block_mm_grad(const void* gq, const float* gs, const void* xq,
                                        const float* xs, const int32_t* offsets, int32_t E,
                                        int32_t rows, int32_t blocks, int32_t N, int32_t K, void* dw,
                                        int32_t dtype, void* stream) {
  return product_grad("eat_block_mm_grad", gq, gs, xq, xs, offsets, E, rows, blocks, N, K, dw, dtype, Waits{},
                      stream);
}

extern "C" eat_status eat_block_mm_grad_selftest(const void* gq, const float* gs, const void* xq,
                                                 const float* xs, const int32_t* offsets, int32_t E,
                                                 int32_t rows, int32_t blocks, int32_t N, int32_t K, void* dw,
                                                 int32_t dtype, int64_t limit_ns, int32_t cta,
                                                 int64_t copies, uint32_t* status, void* stream) {
  const char* fn = "eat_block_mm_grad_selftest";
  if (const char* why = bad_waits(limit_ns, cta, copies, status)) return bad_arg(fn, why);
  return product_grad(fn, gq, gs, xq, xs, offsets, E, rows, blocks, N, K, dw, dtype,
                      Waits{(unsigned long long)limit_ns, cta, copies, status}, stream);
}
