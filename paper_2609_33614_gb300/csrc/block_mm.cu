// Matrix products of e4m3 operands with a scale for each block of 128 along the sums (quant.cu makes
// them), for one matrix or for the experts' matrices on rows sorted by expert:
//   y[r][n]  = sum_b xs[b][r] ws[n / 128][b] sum_{k in b} x[r][k] w[n][k]
//   y[r][k]  = the same with w as it lies, summed over n (transposed: the gradient to x)
//   dw[n][k] = sum_b gs[b][n] xs[b][k] sum_{r in b} g[r][n] x[r][k], b the blocks of 128 rows of an expert
// All sums are fp32; each block's sum is scaled and added once; a value is rounded when it is stored.
#include "elem.cuh"
#include "op_checks.cuh"

namespace eat {

namespace {

enum : int { kForward = 0, kBack = 1, kGrad = 2 };

// out[i][j] = sum_k rows[i][k] cols[j][k]: rows are x's (of an expert), or dw's n; cols are what is left.
struct Args {
  const uint8_t *a, *w;      // rows' and columns' operand
  const float *as, *ws;
  const int32_t* offsets;    // or null: one expert with every row
  int E, M, N, K;            // N, K: w's shape; M: x's rows (kGrad: the operands' padded rows)
  int blocks;                // kGrad: rows of the scales
  void* out;
};

constexpr int kTile = 64, kStep = 32, kThreads = 256;

__device__ __forceinline__ float e4m3(uint8_t v) {
  __nv_fp8_e4m3 q;
  q.__x = v;
  return (float)q;
}

template <int MODE, typename T>
__global__ void __launch_bounds__(kThreads) block_mm_kernel(const Args a) {
  __shared__ float s_a[kStep][kTile + 1], s_b[kStep][kTile + 1];
  pdl_wait();
  pdl_launch_dependents();
  const int e = blockIdx.z, c0 = blockIdx.x * kTile, i0 = blockIdx.y * kTile;
  const int nb = (a.N + kBlock - 1) / kBlock, kb = (a.K + kBlock - 1) / kBlock;
  const int cols = MODE == kForward ? a.N : a.K, inner = MODE == kForward ? a.K : a.N;
  int lo = 0, hi = a.M, block0 = 0, padded0 = 0;
  if (a.offsets) {
    int end = 0;
    for (int f = 0; f <= e && f < a.E; ++f) {
      const int cap = MODE == kGrad ? 1 << 30 : a.M;
      if (MODE == kGrad && f > 0) {
        block0 += (hi - lo + kBlock - 1) / kBlock;
        padded0 += (hi - lo + 31) & ~31;
      }
      lo = max(0, min(a.offsets[f], cap));
      hi = max(lo, min(a.offsets[f + 1], cap));
      end = max(end, hi);
    }
    if (e == a.E) lo = end, hi = a.M;  // rows behind the last
  }
  const bool zero = e == a.E;
  int sums = inner, limit = hi - lo;
  size_t out0 = lo;
  if (MODE == kGrad) {
    sums = hi - lo;
    if (block0 + (sums + kBlock - 1) / kBlock > a.blocks || padded0 + sums > a.M) sums = 0;
    limit = a.N;
    out0 = (size_t)e * a.N;
  }
  if (zero) sums = 0;
  if (i0 >= limit) return;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int b = 0; b * kBlock < sums; ++b) {
    float p[4][4] = {};
    for (int k0 = b * kBlock; k0 < min(sums, (b + 1) * kBlock); k0 += kStep) {
      __syncthreads();
      for (int t = threadIdx.x; t < kStep * kTile; t += kThreads) {
        float va = 0.f, vb = 0.f;
        if (MODE == kGrad) {
          const int i = t % kTile, k = t / kTile;
          const size_t r = padded0 + k0 + k;
          if (k0 + k < sums && i0 + i < a.N) va = e4m3(a.a[r * a.N + i0 + i]);
          if (k0 + k < sums && c0 + i < a.K) vb = e4m3(a.w[r * a.K + c0 + i]);
          s_a[k][i] = va;
          s_b[k][i] = vb;
        } else {
          const int k = t % kStep, i = t / kStep;
          if (k0 + k < inner && i0 + i < limit)
            va = e4m3(a.a[(out0 + i0 + i) * (size_t)inner + k0 + k]);
          s_a[k][i] = va;
          if (MODE == kForward) {
            if (k0 + k < inner && c0 + i < cols)
              vb = e4m3(a.w[((size_t)e * a.N + c0 + i) * a.K + k0 + k]);
            s_b[k][i] = vb;
          } else {
            const int j = t % kTile, kk = t / kTile;
            if (k0 + kk < inner && c0 + j < cols)
              vb = e4m3(a.w[((size_t)e * a.N + k0 + kk) * a.K + c0 + j]);
            s_b[kk][j] = vb;
          }
        }
      }
      __syncthreads();
      for (int k = 0; k < kStep; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) p[i][j] = fmaf(s_a[k][ty * 4 + i], s_b[k][tx * 4 + j], p[i][j]);
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int row = i0 + ty * 4 + i, c = c0 + tx * 4 + j;
        if (row >= limit || c >= cols) continue;
        float s;
        if (MODE == kGrad)
          s = a.as[(size_t)(block0 + b) * a.N + row] * a.ws[(size_t)(block0 + b) * a.K + c];
        else
          s = a.as[(size_t)b * a.M + out0 + row] *
              a.ws[((size_t)e * nb + (MODE == kForward ? c / kBlock : b)) * kb +
                   (MODE == kForward ? b : c / kBlock)];
        acc[i][j] = fmaf(p[i][j], s, acc[i][j]);
      }
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int row = i0 + ty * 4 + i, c = c0 + tx * 4 + j;
      if (row < limit && c < cols) ((T*)a.out)[(out0 + row) * cols + c] = Elem<T>::put(acc[i][j]);
    }
}

template <int MODE>
cudaError_t run(const Args& a, int out_dtype, cudaStream_t st) {
  const int cols = MODE == kForward ? a.N : a.K, rows = MODE == kGrad ? a.N : a.M;
  const dim3 grid((cols + kTile - 1) / kTile, (rows + kTile - 1) / kTile,
                  a.E + (MODE == kGrad || !a.offsets ? 0 : 1));
  return launch_pdl(out_dtype == EAT_BF16 ? block_mm_kernel<MODE, __nv_bfloat16>
                                          : block_mm_kernel<MODE, float>,
                    grid, dim3(kThreads), 0, st, a);
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

extern "C" eat_status eat_block_mm(const void* xq, const float* xs, const void* wq, const float* ws,
                                   const int32_t* offsets, int32_t E, int32_t M, int32_t N, int32_t K,
                                   int32_t transposed, void* y, int32_t ydtype, void* stream) {
  const char* fn = "eat_block_mm";
  if (!xq || !xs || !wq || !ws || !y) return bad_arg(fn, "xq, xs, wq, ws and y must be non-NULL");
  if (const char* why = bad_shape(E, M, N, K, offsets, ydtype)) return bad_arg(fn, why);
  if (K % 16 || (transposed && N % 16))
    return thread_fail(EAT_ERR_UNSUPPORTED, "%s: K (transposed: and N) must be multiples of 16", fn);
  if (misaligned(xq, 16) || misaligned(wq, 16) || misaligned(xs, 4) || misaligned(ws, 4) ||
      misaligned(offsets, 4) || misaligned(y, ydtype == EAT_BF16 ? 2 : 4))
    return bad_arg(fn, "misaligned pointer");
  const Args a{(const uint8_t*)xq, (const uint8_t*)wq, xs, ws, offsets, E, M, N, K, 0, y};
  const cudaStream_t st = (cudaStream_t)stream;
  return launched(fn, transposed ? run<kBack>(a, ydtype, st) : run<kForward>(a, ydtype, st));
}

extern "C" eat_status eat_block_mm_grad(const void* gq, const float* gs, const void* xq,
                                        const float* xs, const int32_t* offsets, int32_t E,
                                        int32_t rows, int32_t blocks, int32_t N, int32_t K, void* dw,
                                        int32_t dtype, void* stream) {
  const char* fn = "eat_block_mm_grad";
  if (!gq || !gs || !xq || !xs || !dw) return bad_arg(fn, "gq, gs, xq, xs and dw must be non-NULL");
  if (const char* why = bad_shape(E, rows, N, K, offsets, dtype)) return bad_arg(fn, why);
  if (blocks < 1) return bad_arg(fn, "need blocks >= 1");
  if (N % 16 || K % 16)
    return thread_fail(EAT_ERR_UNSUPPORTED, "%s: N and K must be multiples of 16", fn);
  if (misaligned(gq, 16) || misaligned(xq, 16) || misaligned(gs, 4) || misaligned(xs, 4) ||
      misaligned(offsets, 4) || misaligned(dw, dtype == EAT_BF16 ? 2 : 4))
    return bad_arg(fn, "misaligned pointer");
  const Args a{(const uint8_t*)gq, (const uint8_t*)xq, gs, xs, offsets, E, rows, N, K, blocks, dw};
  return launched(fn, run<kGrad>(a, dtype, (cudaStream_t)stream));
}
