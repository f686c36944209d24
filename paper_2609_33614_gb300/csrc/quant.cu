// e4m3 operands with a scale for each block of 128 (block_mm.cu multiplies them), and the gated
// activation between two such products.
//   rows:    a scale for each 128 elements of a row, [ceil(K / 128)][M]
//   columns: a scale for each 128 rows of a column, [blocks][K]: what the weights' gradient, a sum over
//            an expert's rows, reads.  Each expert's rows begin at a multiple of 32 (what one MMA
//            sums), zeros behind its last.
//   tiles:   weights, a scale for each 128 x 128 tile, so one copy serves both directions
//   swiglu:  h = gate up / (1 + exp(-gate)) of rows [gate | up]; its gradient:
//            s = 1 / (1 + exp(-gate)):  dgate = dh up s (1 + gate (1 - s)),  dup = dh gate s
// Bound: HBM; each input is read once and kept in registers between a block's maximum and its bytes.
// swiglu's e4m3 form takes the maximum of the unrounded fp32 values.
#include "elem.cuh"
#include "op_checks.cuh"

#include <algorithm>
#include <type_traits>

namespace eat {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// 1 / (1 + exp(-g)) for g >= kFarGate, where the exponential is finite.  CUDA's tables give expf 2 units in the last
// place and __expf 2 + |1.173 g|, so that it is within 3 2^-23 of itself (EXACT: fp32 results), or within
// (4 + 1.173 |g|) 2^-23, below 2^-16, far less than what bf16 or e4m3 keep of it.
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float g) {
  if (EXACT) return __frcp_rn(1.0f + expf(-g));
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.0f + __expf(-g)));
  return r;
}
// Below it exp(-g) would overflow long before gate * sigmoid * up is 0 (-89: -2e-37 up).  There the sigmoid is exp(g)
// to within 2^-92 of itself, and exp(g / 2), which each of two factors takes, is a normal number down to -174.
constexpr float kFarGate = -64.0f;
template <bool EXACT>
__device__ __forceinline__ float far_root(float g) {
  return EXACT ? expf(0.5f * g) : __expf(0.5f * g);
}
// Whether any of a thread's gates is: as a rule none, so that there is one test for all of them.  (Without a
// branch, both forms at once, 16383 x 1408 bf16 took 24.7 for 20.9 us and its gradient 34.7 for 28.8.)
template <int N>
__device__ __forceinline__ bool any_far(const float* g) {
  float lo = g[0];
#pragma unroll
  for (int j = 1; j < N; ++j) lo = fminf(lo, g[j]);
  return lo < kFarGate;
}

// ------------------------------------------------------------------------------------- rows
constexpr int kMostRows = 8;  // of a unit: their scales fill a sector of [blocks][M]

// A unit is kRows rows of one block of 128 columns, taken by as many lanes as the block has 16-byte
// vectors.  GLU: the values are swiglu of rows of twice the length.
template <typename T, bool VEC, bool GLU, int kRows>
__global__ void __launch_bounds__(kThreads, VEC ? 4 : 1)
quant_rows_kernel(const T* __restrict__ x, int M, int K, int blocks, uint8_t* __restrict__ q,
                  float* __restrict__ scale) {
  constexpr int N = Elem<T>::kN, G = kBlock / N, U = GLU && kRows > 4 ? 4 : kRows;
  pdl_wait();
  pdl_launch_dependents();
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / G;
  const int kb = (int)(unit % blocks), l = threadIdx.x % G;
  const long long r0 = unit / blocks * kRows;
  const int c = kb * kBlock + lane_at<T, VEC>(l), left = K - c;
  const size_t pitch = GLU ? 2 * (size_t)K : (size_t)K;
  float s = 1.0f;  // lane l: of the l-th row
#pragma unroll
  for (int i0 = 0; i0 < kRows; i0 += U) {
    // (kept as they were loaded until their row's turn: four blocks an SM)
    RowVec<T, VEC, G> in[U], up[GLU ? U : 1];
    const T* const p = x + (r0 + i0) * pitch + c;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      in[i].load(p + i * pitch, left, r0 + i0 + i < M);
      if (GLU) up[GLU ? i : 0].load(p + i * pitch + K, left, r0 + i0 + i < M);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const long long r = r0 + i0 + i;
      float v[N], top = 0.f;
      if (!GLU) {
        in[i].get(v);
      } else {
        float g[N], u[N];
        in[i].get(g);
        up[GLU ? i : 0].get(u);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = g[j] * sigmoid<false>(g[j]) * u[j];
        if (any_far<N>(g)) {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (g[j] < kFarGate) {
              const float h = far_root<false>(g[j]);
              v[j] = (g[j] * h) * (u[j] * h);
            }
        }
      }
      // (elements that do not exist are 0)
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(v[j]));
      const BlockDiv div(group_max<G>(top));
      if (r < M && left > 0) store_e4m3<N, VEC, G>(q + (size_t)r * K + c, left, v, div);
      if (l == i0 + i) s = div.scale;
    }
  }
  if (l < kRows && r0 + l < M) scale[(size_t)kb * M + r0 + l] = s;
}

// ---------------------------------------------------------------------------------- columns
constexpr int kTileThreads = 512, kTileWarps = kTileThreads / 32;  // of a block that takes 128 x 128
constexpr int kTilesOfBlock = 4;  // at most, of its rows: a thread block finds them once

// Block b of the experts' blocks of 128 rows: its rows in x, and where they go in the padded order.
struct RowBlock {
  int row, n, padded;  // first row, number (0: none), first padded row
};
// By a full warp; the same in all lanes.  Offsets are held to [0, M].  Blocks past the experts' last
// take the rows behind it: n is 0, and row the first of their 128 (M where there is none).
__device__ RowBlock find_block(const int32_t* offsets, int E, int M, int b) {
  constexpr int kRounds = kMaxExperts / 32;
  const int lane = threadIdx.x & 31;
  int lo[kRounds], hi[kRounds];  // (one latency for all of them)
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int e = 32 * i + lane;
    const bool in = e < E;
    lo[i] = in && offsets ? offsets[e] : 0;
    hi[i] = !in ? 0 : offsets ? offsets[e + 1] : M;
  }
  int blocks = 0, padded = 0, end = 0, before = 0;  // of the experts so far
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    if (32 * i >= E) break;
    int l = max(0, min(lo[i], M)), h = 32 * i + lane < E ? max(l, min(hi[i], M)) : l;
    in_order(l, h, before);
    const int c = (h - l + kBlock - 1) / kBlock, p = (h - l + 31) & ~31;
    int vc = c, vp = p;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int uc = __shfl_up_sync(0xffffffffu, vc, o), up = __shfl_up_sync(0xffffffffu, vp, o);
      if (lane >= o) {
        vc += uc;
        vp += up;
      }
    }
    const int at = b - (blocks + vc - c);
    const unsigned who = __ballot_sync(0xffffffffu, at >= 0 && at < c);
    if (who) {
      const int src = __ffs(who) - 1;
      const RowBlock r{l + at * kBlock, min(kBlock, h - l - at * kBlock), padded + vp - p + at * kBlock};
      return RowBlock{__shfl_sync(0xffffffffu, r.row, src), __shfl_sync(0xffffffffu, r.n, src),
                      __shfl_sync(0xffffffffu, r.padded, src)};
    }
    blocks += __shfl_sync(0xffffffffu, vc, 31);
    padded += __shfl_sync(0xffffffffu, vp, 31);
    end = max(end, (int)__reduce_max_sync(0xffffffffu, (unsigned)h));
  }
  return RowBlock{(int)min((long long)M, end + (long long)(b - blocks) * kBlock), 0, 0};
}

// A tile of 128 rows and 128 columns at a time: thread (l, r) holds a vector of R consecutive rows.
// ROWS: the rows' own blocks as well (q, scale), which the same tile holds whole.
template <typename T, bool VEC, bool ROWS>
__global__ void __launch_bounds__(kTileThreads, VEC ? 2 : 1)
quant_columns_kernel(const T* __restrict__ x, int M, int K, const int32_t* __restrict__ offsets,
                     int E, int padded_rows, int blocks, int tiles, uint8_t* __restrict__ q,
                     float* __restrict__ scale, uint8_t* __restrict__ cq,
                     float* __restrict__ cscale) {
  constexpr int N = Elem<T>::kN, L = kBlock / N, R = kBlock * L / kTileThreads;
  __shared__ float s_top[kTileWarps][kBlock];
  __shared__ float s_scale[kBlock], s_recip[kBlock];
  pdl_wait();
  pdl_launch_dependents();
  const int b = blockIdx.x;
  const RowBlock rb = find_block(offsets, E, M, b);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int l = threadIdx.x % L, r = threadIdx.x / L * R;
  const int out_rows = (rb.n + 31) & ~31;
  if (rb.n > 0 && (b >= blocks || rb.padded + out_rows > padded_rows)) return;  // no such offsets
  if (rb.n == 0) {  // rows behind the last expert's
    if (ROWS)
      for (int i = blockIdx.y; i < tiles; i += gridDim.y) {
        const int c = i * kBlock + lane_at<T, VEC>(l), left = K - c;
        const float zero[N] = {};
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const int row = rb.row + r + k;
          if (row >= M) break;
          if (left > 0) store_e4m3<N, VEC, L>(q + (size_t)row * K + c, left, zero);
          if (l == 0) scale[(size_t)i * M + row] = 1.0f;
        }
      }
    return;
  }
  // (a tile's rows are kept as they were loaded, and the next tile's come while this one is taken)
  RowVec<T, VEC, L> in[R];
  auto load = [&](int i) {
    const int c = i * kBlock + lane_at<T, VEC>(l);
#pragma unroll
    for (int k = 0; k < R; ++k)
      in[k].load(x + (size_t)(rb.row + r + k) * K + c, K - c, r + k < rb.n && i < tiles);
  };
  load(blockIdx.y);
  for (int i = blockIdx.y; i < tiles; i += gridDim.y) {
    const int c = i * kBlock + lane_at<T, VEC>(l), left = K - c;
    float top[N] = {};
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float v[N], t = 0.f;
      in[k].get(v);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        top[j] = fmaxf(top[j], fabsf(v[j]));
        t = fmaxf(t, fabsf(v[j]));
      }
      if (ROWS) {
        const BlockDiv div(group_max<L>(t));
        if (r + k >= rb.n) continue;
        const size_t row = rb.row + r + k;
        if (left > 0) store_e4m3<N, VEC, L>(q + row * K + c, left, v, div);
        if (l == 0) scale[(size_t)i * M + row] = div.scale;
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
      for (int o = 16; o >= L; o >>= 1)
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
      if (lane < L) s_top[warp][lane_at<T, VEC>(lane) + (VEC ? j : j * L)] = top[j];
    }
    __syncthreads();
    if (threadIdx.x < kBlock) {
      float t = 0.f;
#pragma unroll
      for (int k = 0; k < kTileWarps; ++k) t = fmaxf(t, s_top[k][threadIdx.x]);
      const BlockDiv div(t);
      s_scale[threadIdx.x] = div.scale;
      s_recip[threadIdx.x] = div.recip;
      const int col = i * kBlock + threadIdx.x;
      if (col < K) cscale[(size_t)b * K + col] = div.scale;
    }
    __syncthreads();
    float fs[N], fr[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int at = lane_at<T, VEC>(l) + (VEC ? j : j * L);
      fs[j] = s_scale[at];
      fr[j] = s_recip[at];
    }
    uint32_t w[R][N / 4];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float v[N];
      in[k].get(v);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = BlockDiv(fs[j], fr[j])(v[j]);
#pragma unroll
      for (int j = 0; j < N / 4; ++j) w[k][j] = e4m3x4(v + 4 * j);
    }
    load(i + gridDim.y);
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (r + k < out_rows && left > 0)
        store_bytes<N, VEC, L>(cq + (size_t)(rb.padded + r + k) * K + c, left, w[k]);
  }
}

// ------------------------------------------------------------------------------------ tiles
// A block takes a tile; thread: N columns of R consecutive rows.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 3 : 1)
quant_tiles_kernel(const T* __restrict__ w, int n_rows, int K, uint8_t* __restrict__ q,
                   float* __restrict__ scale) {
  constexpr int N = Elem<T>::kN, L = kBlock / N, R = kBlock * L / kThreads;
  __shared__ float s_top[kWarps];
  pdl_wait();
  pdl_launch_dependents();
  const int kb = blockIdx.x, blocks = gridDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_blocks = (n_rows + kBlock - 1) / kBlock, nb = blockIdx.y;
  const size_t e = blockIdx.z, at = e * n_rows * K;
  const int l = threadIdx.x % L, r = threadIdx.x / L * R;
  const int c = kb * kBlock + lane_at<T, VEC>(l), left = K - c, row0 = nb * kBlock + r;
  RowVec<T, VEC, L> in[R];
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < R; ++k)
    in[k].load(w + at + (size_t)(row0 + k) * K + c, left, row0 + k < n_rows);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    float v[N];
    in[k].get(v);
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(v[j]));
  }
  top = group_max<32>(top);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWarps; ++k) top = fmaxf(top, s_top[k]);
  const BlockDiv div(top);
  if (threadIdx.x == 0) scale[(e * n_blocks + nb) * blocks + kb] = div.scale;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    float v[N];
    in[k].get(v);
    if (row0 + k < n_rows && left > 0)
      store_e4m3<N, VEC, L>(q + at + (size_t)(row0 + k) * K + c, left, v, div);
  }
}

// ----------------------------------------------------------------------------------- swiglu
// The gradient may be written over gu: a thread loads all that it needs before it stores, and stores where it alone
// loads (gu and out may be one array, so neither is __restrict__).
template <typename T, bool VEC>
__device__ __forceinline__ bool any_far(const RowVec<T, VEC, 32>& v, const float* g) {
  if (VEC && sizeof(T) == 2) {
    // (of 16-bit words the largest is the lowest gate, if one is negative; a NaN may count as far)
    const unsigned m = __vmaxu2(__vmaxu2(v.u.x, v.u.y), __vmaxu2(v.u.z, v.u.w));
    return (m & 0xffff) > 0xc280 || m > 0xc280ffffu;
  }
  return any_far<Elem<T>::kN>(g);
}
// Loaded here, whatever path uses it.
template <typename T, bool VEC>
__device__ __forceinline__ void loaded(RowVec<T, VEC, 32>& v) {
  if (VEC) asm volatile("" : "+r"(v.u.x), "+r"(v.u.y), "+r"(v.u.z), "+r"(v.u.w));
}

// A vector a thread; where rows begin anywhere a warp takes 32 vectors' elements of one row, lanes side by side
// (32000 x 721 bf16: 28.8 us, gradient 43.2; one element a thread, with a division for each, took over twice that).
// Bound: HBM, or the L2 that holds what was written (16383 x 1408 bf16: 20.9 us, gradient 28.8; fp32 38.5 and 60,
// of which expf and the rounded reciprocal are 2 of the first).
template <typename T, bool VEC, bool GRAD>
__global__ void __launch_bounds__(kThreads)
swiglu_kernel(const T* gu, const T* __restrict__ dh, long long n, int F, T* out) {
  constexpr int N = Elem<T>::kN;
  pdl_wait();
  pdl_launch_dependents();
  const long long thread = (long long)blockIdx.x * kThreads + threadIdx.x;
  long long r;
  int c;
  if (VEC) {
    if (thread * N >= n) return;
    r = thread * N / F;
    c = (int)(thread * N - r * F);
  } else {
    const int pieces = (F + 32 * N - 1) / (32 * N);
    r = (thread >> 5) / pieces;
    c = (int)((thread >> 5) - r * pieces) * (32 * N) + (threadIdx.x & 31);
    if (r * F >= n || c >= F) return;
  }
  const int left = F - c;
  const size_t at = (size_t)r * F + c, g0 = (size_t)r * 2 * F + c;
  constexpr bool EXACT = sizeof(T) == 4;
  RowVec<T, VEC, 32> rg, ru, rd;
  float g[N], u[N], o[N];
  if (VEC || GRAD) {
    rg.load(gu + g0, left, true);
    ru.load(gu + g0 + F, left, true);
  } else {
    load_elems<T, N, VEC, 32>(gu + g0, left, g);
    load_elems<T, N, VEC, 32>(gu + g0 + F, left, u);
  }
  if (GRAD) rd.load(dh + at, left, true);
  if (VEC) {  // all loads are under way before the branch (else the gradient takes 32 us for 29)
    loaded(ru);
    if (GRAD) loaded(rd);
  }
  if (VEC || GRAD) rg.get(g);
  if (any_far(rg, g)) {  // a path of its own, which holds no registers of the other
#pragma unroll 1
    for (int j = 0; j < N; ++j) {
      const int c_j = VEC ? j : 32 * j;
      if (c_j >= left) break;
      const float gj = Elem<T>::get(gu[g0 + c_j]), uj = Elem<T>::get(gu[g0 + F + c_j]);
      const bool f = gj < kFarGate;
      const float h = far_root<EXACT>(f ? gj : 0.0f), s = sigmoid<EXACT>(f ? 0.0f : gj);
      if (!GRAD) {
        out[at + c_j] = Elem<T>::put(f ? (gj * h) * (uj * h) : gj * s * uj);
      } else {
        const float dj = Elem<T>::get(dh[at + c_j]);  // (1 - the sigmoid is 1 far below 0)
        out[g0 + c_j] = Elem<T>::put(f ? (dj * h) * (uj * h) * (gj + 1.0f) : dj * uj * s * fmaf(gj, 1.0f - s, 1.0f));
        out[g0 + F + c_j] = Elem<T>::put(f ? (dj * h) * (gj * h) : dj * gj * s);
      }
    }
    return;
  }
  if (VEC || GRAD) ru.get(u);
  if (!GRAD) {
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = g[j] * sigmoid<EXACT>(g[j]) * u[j];
    store_elems<T, N, VEC, 32>(out + at, left, o);
    return;
  }
  float d[N], du[N];
  rd.get(d);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float s = sigmoid<EXACT>(g[j]);
    o[j] = d[j] * u[j] * s * fmaf(g[j], 1.0f - s, 1.0f);
    du[j] = d[j] * g[j] * s;
  }
  store_elems<T, N, VEC, 32>(out + g0, left, o);
  store_elems<T, N, VEC, 32>(out + g0 + F, left, du);
}

// Threads of a call of it.
long long swiglu_threads(int R, int F, int n, bool vec) {
  return vec ? ((long long)R * F + n - 1) / n : (long long)R * ((F + 32 * n - 1) / (32 * n)) * 32;
}

const char* bad_matrix(int32_t M, int32_t K, int32_t dtype) {
  if (M < 1 || M > 1 << 30) return "need between 1 and 2^30 rows";
  if (K < 1 || K > 65536) return "need between 1 and 65536 columns";
  if (dtype != EAT_F32 && dtype != EAT_BF16) return "dtype must be F32 or BF16";
  return nullptr;
}
int elem_bytes(int32_t dtype) { return dtype == EAT_BF16 ? 2 : 4; }

template <typename F>
cudaError_t by_type(int32_t dtype, F&& run) {
  return dtype == EAT_BF16 ? run((__nv_bfloat16*)nullptr) : run((float*)nullptr);
}

template <bool GLU>
cudaError_t quant_rows(const void* x, int M, int K, int dtype, void* q, float* scale,
                       cudaStream_t st) {
  return by_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<T>::kN;
    const int blocks = (K + kBlock - 1) / kBlock;
    const bool vec = K % N == 0 && !misaligned(x, 16) && !misaligned(q, N);
    auto go = [&](auto rows) {
      constexpr int R = decltype(rows)::value;
      const long long threads = (long long)((M + R - 1) / R) * blocks * (kBlock / N);
      return launch_pdl(vec ? quant_rows_kernel<T, true, GLU, R> : quant_rows_kernel<T, false, GLU, R>,
                        dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st,
                        (const T*)x, M, K, blocks, (uint8_t*)q, scale);
    };
    // Units of one row where longer ones would leave SMs without a block (8 rows of 14336, gated:
    // 2.6 us, 9.4 with eight)
    const long long units = (long long)((M + kMostRows - 1) / kMostRows) * blocks;
    if (units * (kBlock / N) < 2LL * kThreads * num_sms()) return go(std::integral_constant<int, 1>());
    return go(std::integral_constant<int, kMostRows>());
  });
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" eat_status eat_quant_rows(const void* x, int32_t M, int32_t K, int32_t dtype, void* q,
                                     float* scale, void* stream) {
  const char* fn = "eat_quant_rows";
  if (!x || !q || !scale) return bad_arg(fn, "x, q and scale must be non-NULL");
  if (const char* why = bad_matrix(M, K, dtype)) return bad_arg(fn, why);
  if (misaligned(x, elem_bytes(dtype)) || misaligned(scale, 4)) return bad_arg(fn, "misaligned pointer");
  const size_t n = (size_t)M * K;
  if (overlaps({{q, n}, {scale, 4 * (size_t)blocks_of(K) * M}}, {{x, n * elem_bytes(dtype)}}))
    return bad_arg(fn, "q or scale overlaps another array");
  return launched(fn, quant_rows<false>(x, M, K, dtype, q, scale, (cudaStream_t)stream));
}

extern "C" int64_t eat_quant_columns_rows(int32_t M, int32_t E) {
  if (M < 1 || M > 1 << 30 || E < 1 || E > kMaxExperts) return 0;
  // (an expert lacks at most 31 rows, and one without rows takes none)
  return std::min(((long long)M + 31 * E) / 32, (long long)M) * 32;
}
extern "C" int64_t eat_quant_columns_blocks(int32_t M, int32_t E) {
  if (M < 1 || M > 1 << 30 || E < 1 || E > kMaxExperts) return 0;
  return std::min(((long long)M + 127 * E) / kBlock, (long long)M);
}

extern "C" eat_status eat_quant_columns(const void* x, int32_t M, int32_t K, int32_t dtype,
                                        const int32_t* offsets, int32_t E, void* q, float* scale,
                                        void* cq, float* cscale, void* stream) {
  const char* fn = "eat_quant_columns";
  if (!x || !cq || !cscale) return bad_arg(fn, "x, cq and cscale must be non-NULL");
  if (!q != !scale) return bad_arg(fn, "q and scale come together");
  if (const char* why = bad_matrix(M, K, dtype)) return bad_arg(fn, why);
  if (E < 1 || E > kMaxExperts) return bad_arg(fn, "need 1 <= E <= 256");
  if (!offsets && E != 1) return bad_arg(fn, "several experts need offsets");
  if (misaligned(x, elem_bytes(dtype)) || misaligned(scale, 4) || misaligned(cscale, 4) ||
      misaligned(offsets, 4))
    return bad_arg(fn, "misaligned pointer");
  const long long padded = eat_quant_columns_rows(M, E);
  const int blocks = (int)eat_quant_columns_blocks(M, E), tiles = (K + kBlock - 1) / kBlock;
  if (padded > 1 << 30) return bad_arg(fn, "need at most 2^30 padded rows");
  const size_t n = (size_t)M * K * elem_bytes(dtype);
  if (overlaps({{q, (size_t)M * K},
                {scale, 4 * (size_t)tiles * M},
                {cq, (size_t)padded * K},
                {cscale, 4 * (size_t)blocks * K}},
               {{x, n}, {offsets, 4 * (size_t)(E + 1)}}))
    return bad_arg(fn, "an output overlaps another array");
  return launched(fn, by_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<T>::kN;
    const bool vec =
        K % N == 0 && !misaligned(x, 16) && !misaligned(cq, N) && !(q && misaligned(q, N));
    auto* kernel = q ? (vec ? quant_columns_kernel<T, true, true> : quant_columns_kernel<T, false, true>)
                     : (vec ? quant_columns_kernel<T, true, false>
                            : quant_columns_kernel<T, false, false>);
    // (one more block than the experts can have: the rows behind them)
    // Several tiles a block where there are more than run at a time: a block's life is mostly latency, so a
    // small call takes one each (two calls of 666 rows, 512 and 256 columns: 11 us, 26 with four a block of
    // 256 threads), a large one shares what finding the rows costs.
    const long long all = (long long)(blocks + 1) * tiles, run = 2LL * num_sms();
    const int per = (int)std::min((long long)kTilesOfBlock, (all + run - 1) / run);
    return launch_pdl(kernel, dim3(blocks + 1, (tiles + per - 1) / per), dim3(kTileThreads), 0,
                      (cudaStream_t)stream, (const T*)x, M, K, offsets, E, (int)padded, blocks, tiles,
                      (uint8_t*)q, scale, (uint8_t*)cq, cscale);
  }));
}

extern "C" eat_status eat_quant_tiles(const void* w, int32_t E, int32_t N, int32_t K, int32_t dtype,
                                      void* q, float* scale, void* stream) {
  const char* fn = "eat_quant_tiles";
  if (!w || !q || !scale) return bad_arg(fn, "w, q and scale must be non-NULL");
  if (E < 1 || E > kMaxExperts) return bad_arg(fn, "need 1 <= E <= 256");
  if (N < 1 || N > 65536) return bad_arg(fn, "need 1 <= N <= 65536");
  if (const char* why = bad_matrix(N, K, dtype)) return bad_arg(fn, why);
  if (misaligned(w, elem_bytes(dtype)) || misaligned(scale, 4)) return bad_arg(fn, "misaligned pointer");
  const size_t n = (size_t)E * N * K;
  if (overlaps({{q, n}, {scale, 4 * (size_t)E * blocks_of(N) * blocks_of(K)}}, {{w, n * elem_bytes(dtype)}}))
    return bad_arg(fn, "q or scale overlaps another array");
  return launched(fn, by_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int V = Elem<T>::kN;
    const bool vec = K % V == 0 && !misaligned(w, 16) && !misaligned(q, V);
    return launch_pdl(vec ? quant_tiles_kernel<T, true> : quant_tiles_kernel<T, false>,
                      dim3((K + kBlock - 1) / kBlock, (N + kBlock - 1) / kBlock, E), dim3(kThreads),
                      0, (cudaStream_t)stream, (const T*)w, N, K, (uint8_t*)q, scale);
  }));
}

extern "C" eat_status eat_swiglu(const void* gu, int32_t R, int32_t F, int32_t dtype, void* h,
                                 int32_t h_dtype, float* scale, void* stream) {
  const char* fn = "eat_swiglu";
  if (!gu || !h) return bad_arg(fn, "gu and h must be non-NULL");
  if (const char* why = bad_matrix(R, F, dtype)) return bad_arg(fn, why);
  if (h_dtype != dtype && h_dtype != EAT_FP8_E4M3)
    return bad_arg(fn, "h_dtype must be dtype or FP8_E4M3");
  const bool fp8 = h_dtype == EAT_FP8_E4M3;
  if (fp8 && !scale) return bad_arg(fn, "an e4m3 output needs scale");
  const int eb = elem_bytes(dtype);
  if (misaligned(gu, eb) || misaligned(h, fp8 ? 1 : eb) || (fp8 && misaligned(scale, 4)))
    return bad_arg(fn, "misaligned pointer");
  const size_t size = (size_t)R * F;
  if (overlaps({{h, size * (fp8 ? 1 : eb)}, {fp8 ? scale : nullptr, 4 * (size_t)blocks_of(F) * R}},
               {{gu, 2 * size * eb}}))
    return bad_arg(fn, "h or scale overlaps another array");
  const cudaStream_t st = (cudaStream_t)stream;
  if (fp8) return launched(fn, quant_rows<true>(gu, R, F, dtype, h, scale, st));
  return launched(fn, by_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<T>::kN;
    const bool vec = F % N == 0 && !misaligned(gu, 16) && !misaligned(h, 16);
    const long long threads = swiglu_threads(R, F, N, vec), n = (long long)R * F;
    return launch_pdl(vec ? swiglu_kernel<T, true, false> : swiglu_kernel<T, false, false>,
                      dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, (const T*)gu,
                      (const T*)nullptr, n, F, (T*)h);
  }));
}

extern "C" eat_status eat_swiglu_grad(const void* gu, const void* dh, int32_t R, int32_t F,
                                      int32_t dtype, void* dgu, void* stream) {
  const char* fn = "eat_swiglu_grad";
  if (!gu || !dh || !dgu) return bad_arg(fn, "gu, dh and dgu must be non-NULL");
  if (const char* why = bad_matrix(R, F, dtype)) return bad_arg(fn, why);
  const int eb = elem_bytes(dtype);
  if (misaligned(gu, eb) || misaligned(dh, eb) || misaligned(dgu, eb))
    return bad_arg(fn, "misaligned pointer");
  const size_t size = (size_t)R * F * eb;
  if (overlap(dgu, 2 * size, dh, size) || (dgu != gu && overlap(dgu, 2 * size, gu, 2 * size)))
    return bad_arg(fn, "dgu overlaps dh, or a part of gu");
  return launched(fn, by_type(dtype, [&](auto* tag) {
    using T = std::remove_pointer_t<decltype(tag)>;
    constexpr int N = Elem<T>::kN;
    const bool vec = F % N == 0 && !misaligned(gu, 16) && !misaligned(dh, 16) && !misaligned(dgu, 16);
    const long long threads = swiglu_threads(R, F, N, vec), n = (long long)R * F;
    return launch_pdl(vec ? swiglu_kernel<T, true, true> : swiglu_kernel<T, false, true>,
                      dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, (cudaStream_t)stream,
                      (const T*)gu, (const T*)dh, n, F, (T*)dgu);
  }));
}
