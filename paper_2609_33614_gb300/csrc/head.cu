// Vocabulary head: softmax cross entropy of hidden states against a vocabulary matrix, in pieces,
// without holding the logits; and its gradient.  Host side and the kernels around the products of
// head_tc.cu.
//   l_tv = s_t s_v <x_t, w_v>;  r = log sum_{v != y} exp l_v - l_y;  nll = log(1 + exp r)
//   (the target is left out of the sum, so that nll keeps its relative accuracy when it is small);
//   lse = l_y + nll;  P_tv = g_t (exp(l_tv - lse_t) - [v = y_t]);  dx = P w;  dw = P^T x.
// The gradient takes the counted tokens (target in [0, vocab)) in pieces of at most kPieceBytes of
// exponentials, and each product once:
//   E_tv = exp(l_tv - l_ty), stored as bf16 while its sum over v != y, Z', is taken in fp32;
//   then E_ty := -q with q = bf16(Z'), f_t = g_t / (1 + Z') (Z' / q), and
//   dx_t = f_t sum_v E_tv w_v (f in fp32),  dw = E^T X', X'_t = bf16(f_t x_t).
// P enters as f E: its target entry is exact in dx, as f_t q = g_t (1 - p_y); the other entries carry
// one bf16 rounding of E and that of q.  With up to 128 counted tokens X' has two bf16 parts (head_lo),
// and with them dw's target terms are exact too; with more they carry the rounding of X'.  A second pass that computed the logits again, now with lse at
// hand, would spend 8 instead of 6 T V d flops and round P once as well.
#include "head_tc.cuh"

#include "ffn_tc.cuh"
#include "op_checks.cuh"

#include <algorithm>
#include <cstring>
#include <new>

struct eat_head {
  eat_head_desc desc;
  bool w8 = false;
  int device = 0, num_sms = 0, max_pairs = 1;
  char* mem = nullptr;
  eat::HeadStatus st{nullptr, nullptr, eat::kWaitLimitNs};
  unsigned int* mirror_host = nullptr;
  bool failed = false;
  CUtensorMap w128, w64, w16, x64, e64;
  float2* part = nullptr;      // small calls [ctas][n]; larger ones [128-row pieces][T]
  float* ly = nullptr;         // [max_tokens] base-2 target logits
  unsigned int* tickets = nullptr;  // small calls (0 between calls)
  // gradient
  int cap = 0, ld = 0;         // tokens of a piece, columns of E
  int32_t* n_counted = nullptr;
  int32_t* rows = nullptr;     // [tokens] counted tokens, ascending
  int32_t* ytok = nullptr;     // [tokens] their targets
  float* f = nullptr;          // [tokens]
  uint32_t* row_max = nullptr;
  int32_t* far = nullptr;
  __nv_bfloat16* xc = nullptr;  // [tokens, d] their hidden states, then X'
  __nv_bfloat16* e = nullptr;   // [cap, ld]
  float* dw_sum = nullptr;
  float* dx_part = nullptr;     // slices of dx's sums over the vocabulary
};

namespace eat {

namespace {

constexpr size_t kPieceBytes = 512u << 20;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Joins the pieces' (or a small call's CTAs') sums of a loss, part[piece][stride]: 8 tokens per block, 64 threads each over the pieces of the vocabulary.
constexpr int kJoinT = 8;
__global__ void __launch_bounds__(512)
join_kernel(const float2* __restrict__ part, int pieces, int stride,
            const float* __restrict__ ly, int T, int V, const int32_t* __restrict__ target, float* __restrict__ nll,
            float* __restrict__ lse, const HeadStatus st) {
  __shared__ float2 s_p[16][kJoinT];
  pdl_wait();
  pdl_launch_dependents();
  const unsigned int err = *st.err;
  if (err && blockIdx.x == 0 && threadIdx.x == 0) *st.mirror = err;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x * kJoinT + (lane & 7);
  float m = kHeadLow, s = 0.f;
  if (t < T) {
#pragma unroll 8
    for (int i = warp * 4 + (lane >> 3); i < pieces; i += 64) {
      const float2 q = part[(size_t)i * stride + t];
      const float k = fmaxf(m, q.x);
      s = s * exp2f(m - k) + q.y * exp2f(q.x - k);
      m = k;
    }
  }
#pragma unroll
  for (int o = 8; o < 32; o <<= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
    const float k = fmaxf(m, m2);
    s = s * exp2f(m - k) + s2 * exp2f(m2 - k);
    m = k;
  }
  if (lane < kJoinT) s_p[warp][lane] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x >= kJoinT || t >= T) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    const float2 q = s_p[i][threadIdx.x];
    const float k = fmaxf(m, q.x);
    s = s * exp2f(m - k) + q.y * exp2f(q.x - k);
    m = k;
  }
  const int y = target[t];
  float2 r = make_float2(0.f, 0.f);
  if (y >= V || err) r = make_float2(NAN, NAN);
  else if (y >= 0) r = token_loss(m, s, ly[t]);
  if (y < 0) r = make_float2(0.f, 0.f);
  nll[t] = r.x;
  if (lse) lse[t] = r.y;
}

// ------------------------------------------------------------------------------- gradient
// 32 rows per block, a warp each: the i-th counted token's hidden state into xc (zeros up to the end
// of the last tile) and its base-2 target logit, of few tokens twice (head_lo); and for token i, if it
// does not count, its outputs.
// Every block finds its tokens itself: each thread counts a run of the targets (1 / 1024 of them),
// and the runs' prefix sums say which hold the block's rows.  (A launch of its own for the list took
// 14 us of 8192 tokens on one SM, and 3.5 us of any call.)
__global__ void __launch_bounds__(1024)
gather_kernel(const uint4* __restrict__ x, const uint4* __restrict__ w, int row_vecs, int T, int V,
              const int32_t* __restrict__ target, int32_t* __restrict__ rows,
              int32_t* __restrict__ ytok, int32_t* __restrict__ n_counted, uint4* __restrict__ xc,
              float* __restrict__ ly, uint32_t* __restrict__ row_max, int32_t* __restrict__ far,
              uint4* __restrict__ dx, float* __restrict__ nll, float* __restrict__ lse) {
  __shared__ int s_w[32], s_row[32];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i0 = blockIdx.x * 32;
  const int run = (T + 1023) / 1024, a = threadIdx.x * run, b = min(T, a + run);
  int mine = 0;
#pragma unroll 4
  for (int t = a; t < b; ++t) {
    const int y = target[t];
    mine += y >= 0 && y < V;
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) s_w[warp] = incl;
  __syncthreads();
  int before = 0, n = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    before += i < warp ? s_w[i] : 0;
    n += s_w[i];
  }
  int rank = before + incl - mine;  // of the run's first counted token
  const int lo = head_lo(n);        // where the tokens' rows come a second time, or 0
  if ((rank < i0 + 32 && rank + mine > i0) ||
      (lo && rank + lo < i0 + 32 && rank + lo + mine > i0)) {
    for (int t = a; t < b; ++t) {
      const int y = target[t];
      if (y >= 0 && y < V) {
        for (int at = rank; at <= rank + lo; at += max(lo, 1)) {
          if (at < i0 || at >= i0 + 32) continue;
          s_row[at - i0] = t;
          rows[at] = t;
          ytok[at] = y;
        }
        ++rank;
      }
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *n_counted = n;
  if (threadIdx.x == 0 && i0 % kHeadTile == 0) far[i0 / kHeadTile] = 0;
  __syncthreads();
  const int i = i0 + warp;
  if (i < n || (lo && i >= lo && i < lo + n)) {
    const int t = s_row[warp];
    const uint4* p = x + (size_t)t * row_vecs;
    const uint4* q = w + (size_t)target[t] * row_vecs;
    float d = 0.f;
#pragma unroll 8
    for (int c = lane; c < row_vecs; c += 32) {
      const uint4 v = p[c];
      xc[(size_t)i * row_vecs + c] = v;
      d = dot16<false>(v, q[c], d);
    }
    d = warp_sum(d);
    if (lane == 0) {
      ly[i] = d * kLog2e;
      row_max[i] = 0;
    }
  } else if (i < (n + kHeadTile - 1) / kHeadTile * kHeadTile) {
    for (int c = lane; c < row_vecs; c += 32) xc[(size_t)i * row_vecs + c] = make_uint4(0, 0, 0, 0);
    if (lane == 0) {  // (between the two)
      ly[i] = INFINITY;
      row_max[i] = 0;
      ytok[i] = -1;
    }
  }
  if (i < T) {
    const int y = target[i];
    if (y < 0 || y >= V) {
      for (int c = lane; c < row_vecs; c += 32) dx[(size_t)i * row_vecs + c] = make_uint4(0, 0, 0, 0);
      if (lane == 0) {
        nll[i] = y < 0 ? 0.f : NAN;
        if (lse) lse[i] = y < 0 ? 0.f : NAN;
      }
    }
  }
}

// After a piece's exponentials, kFinishT counted tokens per block: their sums, losses and factors; the
// target entries of E; X' in place of x.  (128 threads a token: with 32 tokens per block a call of a few
// tokens spent 11 to 16 us here, on one SM.)
constexpr int kFinishT = 8;
__global__ void __launch_bounds__(1024)
finish_kernel(const float* __restrict__ part, int pieces, int t0, int cap,
              const int32_t* __restrict__ n_counted, const int32_t* __restrict__ rows,
              const int32_t* __restrict__ ytok, const float* __restrict__ ly,
              const uint32_t* __restrict__ row_max, const float* __restrict__ g,
              __nv_bfloat16* __restrict__ e, int ld, float* __restrict__ f,
              uint4* __restrict__ xc, int row_vecs, float* __restrict__ nll,
              float* __restrict__ lse, const HeadStatus st) {
  __shared__ float s_p[32][kFinishT], s_f[kFinishT];
  pdl_wait();
  pdl_launch_dependents();
  const unsigned int err = *st.err;
  if (err && blockIdx.x == 0 && threadIdx.x == 0) *st.mirror = err;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int counted = *n_counted, n = min(cap, counted - t0), r0 = blockIdx.x * kFinishT;
  if (r0 >= n) return;
  const int lo = head_lo(counted);
  const int r = r0 + (lane & 7);  // row of the piece
  float s = 0.f;
  if (r < n) {
#pragma unroll 4
    for (int i = warp * 4 + (lane >> 3); i < pieces; i += 128) s += part[(size_t)i * cap + r];
  }
  s += __shfl_xor_sync(0xffffffffu, s, 8);
  s += __shfl_xor_sync(0xffffffffu, s, 16);
  if (lane < kFinishT) s_p[warp][lane] = s;
  __syncthreads();
  if (warp < kFinishT && r0 + warp < n) {  // warp j: token j
    const float sum = warp_sum(s_p[lane][warp]);
    if (lane == 0) {
      const int i = t0 + r0 + warp, t = rows[i], y = ytok[i];
      const float l2 = ly[i], ref = head_ref(l2, row_max[i]);
      float2 a = token_loss(ref, sum, l2);
      const float qf = __bfloat162float(__float2bfloat16_rn(sum));
      float k = g[t] / (sum + exp2f(l2 - ref));
      if (qf > 0.f) k *= sum / qf;
      if (err) {
        a = make_float2(NAN, NAN);
        k = NAN;
      }
      __nv_bfloat16* to = e + (size_t)(r0 + warp) * ld + y;
      to[0] = __float2bfloat16_rn(-qf);
      if (lo) to[(size_t)lo * ld] = __float2bfloat16_rn(-qf);
      f[i] = k;
      s_f[warp] = k;
      nll[t] = a.x;
      if (lse) lse[t] = a.y;
    }
  }
  __syncthreads();
  const int j = warp >> 2;  // four warps a token
  if (r0 + j >= n) return;
  const float k = s_f[j];
  uint4* row = xc + (size_t)(t0 + r0 + j) * row_vecs;
#pragma unroll 4
  for (int c = (warp & 3) * 32 + lane; c < row_vecs; c += 128) {
    const Vec<false> v(row[c]);
    uint32_t b[4], left[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = v.v[2 * i] * k, w = v.v[2 * i + 1] * k;
      const __nv_bfloat162 p = __floats2bfloat162_rn(u, w);
      const __nv_bfloat162 q = __floats2bfloat162_rn(u - __low2float(p), w - __high2float(p));
      b[i] = *(const uint32_t*)&p;
      left[i] = *(const uint32_t*)&q;
    }
    row[c] = make_uint4(b[0], b[1], b[2], b[3]);
    if (lo) row[(size_t)lo * row_vecs + c] = make_uint4(left[0], left[1], left[2], left[3]);
  }
}

// dx from the slices of its split sums: a warp per counted token and 256 columns.
__global__ void __launch_bounds__(256)
dx_join_kernel(const float* __restrict__ part, int slices, int t0, int cap, int d,
               const int32_t* __restrict__ n_counted, const int32_t* __restrict__ rows,
               const float* __restrict__ f, __nv_bfloat16* __restrict__ dx) {
  pdl_wait();
  pdl_launch_dependents();
  const int r = blockIdx.y * 8 + (threadIdx.x >> 5), c = blockIdx.x * 256 + (threadIdx.x & 31) * 8;
  if (r >= min(cap, *n_counted - t0) || c >= d) return;
  float s[8] = {};
#pragma unroll 4
  for (int i = 0; i < slices; ++i) {
    const float4* p = (const float4*)(part + ((size_t)i * cap + r) * d + c);
    const float4 a = p[0], b = p[1];
    s[0] += a.x;
    s[1] += a.y;
    s[2] += a.z;
    s[3] += a.w;
    s[4] += b.x;
    s[5] += b.y;
    s[6] += b.z;
    s[7] += b.w;
  }
  const float k = f[t0 + r];
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(s[2 * i] * k, s[2 * i + 1] * k);
    o[i] = *(const uint32_t*)&v;
  }
  *(uint4*)(dx + (size_t)rows[t0 + r] * d + c) = make_uint4(o[0], o[1], o[2], o[3]);
}

// -------------------------------------------------------------------------------- host side
void free_head(eat_head* h) {
  if (!h) return;
  if (h->mirror_host) cudaFreeHost(h->mirror_host);
  if (h->mem) cudaFree(h->mem);
  delete h;
}

int up(int n, int m) { return (n + m - 1) / m * m; }

// The handle's workspace and its kernels' shared-memory limits belong to the device it was created on.
eat_status check_device(const char* fn, const eat_head* h) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device)
    return thread_fail(EAT_ERR_INVALID_ARG, "%s: the handle is of device %d, the current one is %d",
                       fn, h->device, dev);
  return EAT_OK;
}

eat_status check_call(const char* fn, eat_head* h, const void* x, int32_t T,
                      const int32_t* target, const float* nll, const float* lse) {
  if (!h) return bad_arg(fn, "null handle");
  if (!x || !target || !nll) return bad_arg(fn, "x, target and nll must be non-NULL");
  if (T < 1 || T > h->desc.max_tokens) return bad_arg(fn, "T outside [1, max_tokens]");
  if (misaligned(x, 16)) return bad_arg(fn, "x must be 16-byte aligned");
  if (misaligned(target, 4) || misaligned(nll, 4) || misaligned(lse, 4))
    return bad_arg(fn, "misaligned pointer");
  const eat_status on_device = check_device(fn, h);
  if (on_device != EAT_OK) return on_device;
  if (!h->failed && *(volatile unsigned int*)h->mirror_host) h->failed = true;
  if (h->failed)
    return thread_fail(EAT_ERR_STATE,
                       "%s: a kernel of an earlier call gave up on a bounded wait; eat_head_reset "
                       "clears the state", fn);
  return EAT_OK;
}

cudaError_t run_small(eat_head* h, const void* x, const float* xs, int T, const int32_t* target,
                      float* nll, float* lse, cudaStream_t st) {
  const int V = h->desc.vocab, d = h->desc.d_model, n = head_small_n(T);
  CUtensorMap mx;
  if (!head_encode(&mx, h->w8, x, T, d, n)) return cudaErrorInvalidValue;
  const int ctas = head_small_ctas(h->num_sms, V), kb = h->w8 ? 128 : 64;
  HeadSmallArgs a{};
  a.T = T;
  a.V = V;
  a.d = d;
  a.kblocks = (d + kb - 1) / kb;
  a.target = target;
  a.x = x;
  a.w = h->desc.w;
  a.xs = xs;
  a.ws = h->desc.w_scale;
  a.part = h->part;
  a.ly = h->ly;
  a.tickets = h->tickets;
  a.nll = nll;
  a.lse = lse;
  a.st = h->st;
  const cudaError_t e = head_launch_small(h->w8, h->w128, h->w16, mx, a, ctas, st);
  if (e != cudaSuccess || head_small_joins(n)) return e;
  return launch_pdl(join_kernel, dim3((T + kJoinT - 1) / kJoinT), dim3(512), 0, st,
                    (const float2*)h->part, ctas, n, (const float*)h->ly, T, V, target, nll, lse,
                    h->st);
}

cudaError_t run_pair(eat_head* h, const void* x, const float* xs, int T, const int32_t* target,
                     float* nll, float* lse, cudaStream_t st) {
  const int V = h->desc.vocab, d = h->desc.d_model, kb = h->w8 ? 128 : 64;
  CUtensorMap mx;
  if (!head_encode(&mx, h->w8, x, T, d, 64)) return cudaErrorInvalidValue;
  HeadPairArgs a{};
  a.T = T;
  a.V = V;
  a.d = d;
  a.kblocks = (d + kb - 1) / kb;
  a.target = target;
  a.x = x;
  a.w = h->desc.w;
  a.xs = xs;
  a.ws = h->desc.w_scale;
  a.part2 = h->part;
  a.ly = h->ly;
  a.st = h->st;
  const cudaError_t e = head_launch_pair(h->w8, false, mx, h->w64, a, h->max_pairs, st);
  if (e != cudaSuccess) return e;
  return launch_pdl(join_kernel, dim3((T + kJoinT - 1) / kJoinT), dim3(512), 0, st,
                    (const float2*)h->part, up(V, kHeadTile) / 128, T, (const float*)h->ly, T, V,
                    target, nll, lse, h->st);
}

cudaError_t run_grad(eat_head* h, const void* x, int T, const int32_t* target, const float* g,
                     float* nll, float* lse, void* dx, void* dw, cudaStream_t st) {
  const int V = h->desc.vocab, d = h->desc.d_model, row_vecs = d / 8;
  const int t_pad = up(T, kHeadTile);
  cudaError_t e =
      launch_pdl(gather_kernel, dim3(t_pad / 32), dim3(1024), 0, st, (const uint4*)x,
                 (const uint4*)h->desc.w, row_vecs, T, V, target, h->rows, h->ytok, h->n_counted,
                 (uint4*)h->xc, h->ly, h->row_max, h->far, (uint4*)dx, nll, lse);
  for (int t0 = 0; t0 < T && e == cudaSuccess; t0 += h->cap) {
    const int cap = std::min(h->cap, t_pad - t0);
    HeadPairArgs a{};
    a.V = V;
    a.kblocks = d / 64;
    a.target = h->ytok;
    a.n_counted = h->n_counted;
    a.t0 = t0;
    a.cap = cap;
    a.ld = h->ld;
    a.ref = h->ly;
    a.row_max = h->row_max;
    a.far = h->far;
    a.part = (float*)h->part;
    a.e = h->e;
    a.st = h->st;
    e = head_launch_pair(false, true, h->x64, h->w64, a, h->max_pairs, st);
    if (e != cudaSuccess) break;
    a.redo = 1;
    e = head_launch_pair(false, true, h->x64, h->w64, a, h->max_pairs, st);
    if (e != cudaSuccess) break;
    e = launch_pdl(finish_kernel, dim3(cap / kFinishT), dim3(1024), 0, st, (const float*)h->part,
                   up(V, kHeadTile) / 128, t0, cap, (const int32_t*)h->n_counted,
                   (const int32_t*)h->rows, (const int32_t*)h->ytok, (const float*)h->ly,
                   (const uint32_t*)h->row_max, g, h->e, h->ld, h->f, (uint4*)h->xc, row_vecs, nll,
                   lse, h->st);
    if (e != cudaSuccess) break;
    const int slices = head_dx_slices(cap, V, d, h->max_pairs);
    const HeadGradArgs b{V, d, h->n_counted, t0, cap, h->f, h->rows, (__nv_bfloat16*)dx,
                         (__nv_bfloat16*)dw, h->dw_sum, slices, h->dx_part, h->st};
    e = head_launch_grad(h->e64, h->w64, h->x64, b, h->max_pairs, st);
    if (e == cudaSuccess && slices > 1)
      e = launch_pdl(dx_join_kernel, dim3((d + 255) / 256, (cap + 7) / 8), dim3(256), 0, st,
                     (const float*)h->dx_part, slices, t0, cap, d, (const int32_t*)h->n_counted,
                     (const int32_t*)h->rows, (const float*)h->f, (__nv_bfloat16*)dx);
  }
  return e;
}

}  // namespace
}  // namespace eat

using namespace eat;

extern "C" {

eat_status eat_head_create(const eat_head_desc* desc, eat_head** out) {
  if (!out) return bad_arg("eat_head_create", "out is NULL");
  *out = nullptr;
  if (!desc) return bad_arg("eat_head_create", "desc is NULL");
  const eat_head_desc& D = *desc;
  if (D.dtype != EAT_BF16 && D.dtype != EAT_FP8_E4M3)
    return thread_fail(EAT_ERR_UNSUPPORTED, "head dtype must be BF16 or FP8_E4M3");
  if (D.d_model < 64 || D.d_model % 64 || D.d_model > 16384)
    return thread_fail(EAT_ERR_UNSUPPORTED, "d_model must be a multiple of 64 up to 16384");
  if (D.vocab < 1 || D.vocab > (1 << 20))
    return thread_fail(EAT_ERR_UNSUPPORTED, "vocab must be in [1, 2^20]");
  if (D.max_tokens < 1 || D.max_tokens > 65536)
    return thread_fail(EAT_ERR_INVALID_ARG, "max_tokens must be in [1, 65536]");
  if (!D.w) return thread_fail(EAT_ERR_INVALID_ARG, "w is NULL");
  if ((uintptr_t)D.w & 15) return thread_fail(EAT_ERR_INVALID_ARG, "w must be 16-byte aligned");
  if (D.dtype == EAT_FP8_E4M3 && (!D.w_scale || ((uintptr_t)D.w_scale & 3)))
    return thread_fail(EAT_ERR_INVALID_ARG, "an e4m3 head needs w_scale, 4-byte aligned");
  if (D.with_grad && D.dtype != EAT_BF16)
    return thread_fail(EAT_ERR_UNSUPPORTED, "gradients need a BF16 head");

  int dev = 0;
  cudaDeviceProp prop;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaGetDeviceProperties(&prop, dev) != cudaSuccess) {
    cudaGetLastError();
    return thread_fail(EAT_ERR_CUDA, "no CUDA device");
  }
  if (prop.major != 10 || prop.minor != 3)
    return thread_fail(EAT_ERR_UNSUPPORTED, "the tensor-core kernels are built for sm_103a (GB300)");
  eat_head* h = new (std::nothrow) eat_head();
  if (!h) return thread_fail(EAT_ERR_OOM, "host allocation failed");
  h->desc = D;
  h->device = dev;
  h->w8 = D.dtype == EAT_FP8_E4M3;
  h->num_sms = prop.multiProcessorCount;
  cudaError_t e = head_configure(h->num_sms, &h->max_pairs);
  if (e != cudaSuccess) {
    free_head(h);
    return thread_fail(EAT_ERR_CUDA, "head kernels: %s", cudaGetErrorString(e));
  }

  const int V = D.vocab, t_pad = up(D.max_tokens, kHeadTile), pieces = up(V, kHeadTile) / 128;
  const size_t tokens = (size_t)t_pad;
  h->ld = up(V, kHeadTile);
  h->cap = (int)std::min<size_t>(
      tokens, std::max<size_t>(kPieceBytes / 2 / h->ld / kHeadTile * kHeadTile, kHeadTile));
  const size_t small_part = sizeof(float2) * (size_t)head_small_ctas(h->num_sms, V) * kHeadSmallT;
  const size_t large_part =
      D.max_tokens > kHeadSmallT ? sizeof(float2) * (size_t)pieces * D.max_tokens : 0;
  const size_t grad_part = D.with_grad ? sizeof(float) * (size_t)pieces * h->cap : 0;
  struct Part { void** p; size_t bytes; };
  Part parts[20];
  int np = 0;
  auto add = [&](void* p, size_t bytes) { parts[np++] = {(void**)p, bytes}; };
  add(&h->st.err, 16);
  add(&h->part, std::max({small_part, large_part, grad_part}));
  add(&h->ly, 4 * tokens);
  if (D.with_grad) {
    add(&h->n_counted, 4);
    add(&h->rows, 4 * tokens);
    add(&h->ytok, 4 * tokens);
    add(&h->f, 4 * tokens);
    add(&h->row_max, 4 * tokens);
    add(&h->far, 4 * (tokens / kHeadTile));
    add(&h->xc, 2 * tokens * D.d_model);
    add(&h->e, 2 * (size_t)h->cap * h->ld);
    if (h->cap < t_pad) add(&h->dw_sum, 4 * (size_t)V * D.d_model);
    // a call's last piece may be as short as one tile
    size_t most = 0;
    for (int c = kHeadTile; c <= h->cap; c += kHeadTile) {
      const int n = head_dx_slices(c, V, D.d_model, h->max_pairs);
      if (n > 1) most = std::max(most, 4 * (size_t)n * c * D.d_model);
    }
    if (most) add(&h->dx_part, most);
  }
  size_t total = 0;
  for (int i = 0; i < np; ++i) total += (parts[i].bytes + 255) / 256 * 256;
  e = cudaMalloc((void**)&h->mem, total);
  if (e == cudaSuccess) e = cudaHostAlloc((void**)&h->mirror_host, 16, cudaHostAllocMapped);
  if (e == cudaSuccess) {
    std::memset(h->mirror_host, 0, 16);
    e = cudaHostGetDevicePointer((void**)&h->st.mirror, h->mirror_host, 0);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();  // a failed allocation leaves the context usable: clear its error
    free_head(h);
    return thread_fail(EAT_ERR_OOM, "head workspace of %zu bytes: %s", total,
                       cudaGetErrorString(e));
  }
  char* at = h->mem;
  for (int i = 0; i < np; ++i) {
    *parts[i].p = at;
    at += (parts[i].bytes + 255) / 256 * 256;
  }
  h->tickets = h->st.err + 1;
  e = cudaMemset(h->st.err, 0, 16);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    free_head(h);
    return thread_fail(EAT_ERR_CUDA, "head workspace: %s", cudaGetErrorString(e));
  }
  bool ok = head_encode(&h->w128, h->w8, D.w, V, D.d_model, 128) &&
            head_encode(&h->w64, h->w8, D.w, V, D.d_model, 64) &&
            head_encode(&h->w16, h->w8, D.w, V, D.d_model, 16);
  if (ok && D.with_grad)
    ok = head_encode(&h->x64, false, h->xc, t_pad, D.d_model, 64) &&
         head_encode(&h->e64, false, h->e, h->cap, h->ld, 64);
  if (!ok) {
    free_head(h);
    return thread_fail(EAT_ERR_CUDA, "cuTensorMapEncodeTiled rejected a head tensor");
  }
  *out = h;
  return EAT_OK;
}

eat_status eat_head_destroy(eat_head* h) {
  if (!h) return EAT_OK;
  int dev = h->device;
  cudaGetDevice(&dev);
  if (dev != h->device) cudaSetDevice(h->device);
  cudaDeviceSynchronize();
  if (dev != h->device) cudaSetDevice(dev);
  free_head(h);
  return EAT_OK;
}

eat_status eat_head_reset(eat_head* h, void* stream) {
  const char* fn = "eat_head_reset";
  if (!h) return bad_arg(fn, "null handle");
  const eat_status on_device = check_device(fn, h);
  if (on_device != EAT_OK) return on_device;
  cudaError_t e = cudaMemsetAsync(h->st.err, 0, 16, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return thread_fail(EAT_ERR_CUDA, "%s: %s", fn, cudaGetErrorString(e));
  *(volatile unsigned int*)h->mirror_host = 0u;
  h->failed = false;
  return EAT_OK;
}

eat_status eat_head_selftest_expire_wait(eat_head* h, int64_t limit_ns, void* stream) {
  const char* fn = "eat_head_selftest_expire_wait";
  if (!h) return bad_arg(fn, "null handle");
  if (limit_ns < 1000 || limit_ns > 1000000000LL)
    return bad_arg(fn, "need 1 us <= limit_ns <= 1 s");
  const eat_status on_device = check_device(fn, h);
  if (on_device != EAT_OK) return on_device;
  return launched(fn, tc_selftest_bounded_wait((unsigned long long)limit_ns, h->st.err,
                                               (cudaStream_t)stream));
}

eat_status eat_head_selftest_wait_limit(eat_head* h, int64_t limit_ns) {
  const char* fn = "eat_head_selftest_wait_limit";
  if (!h) return bad_arg(fn, "null handle");
  if (limit_ns != 0 && (limit_ns < 1000000LL || limit_ns > 1000000000LL))
    return bad_arg(fn, "need 1 ms <= limit_ns <= 1 s, or 0");
  h->st.limit_ns = limit_ns ? (unsigned long long)limit_ns : kWaitLimitNs;
  return EAT_OK;
}

eat_status eat_head_nll(eat_head* h, const void* x, const float* x_scale, int32_t T,
                        const int32_t* target, float* nll, float* lse, void* stream) {
  const char* fn = "eat_head_nll";
  const eat_status s = check_call(fn, h, x, T, target, nll, lse);
  if (s != EAT_OK) return s;
  if (h->w8 && (!x_scale || misaligned(x_scale, 4)))
    return bad_arg(fn, "an e4m3 head needs x_scale, 4-byte aligned");
  const cudaStream_t st = (cudaStream_t)stream;
  return launched(fn, T <= kHeadSmallT ? run_small(h, x, x_scale, T, target, nll, lse, st)
                                       : run_pair(h, x, x_scale, T, target, nll, lse, st));
}

eat_status eat_head_nll_grad(eat_head* h, const void* x, int32_t T, const int32_t* target,
                             const float* g, float* nll, float* lse, void* dx, void* dw,
                             void* stream) {
  const char* fn = "eat_head_nll_grad";
  const eat_status s = check_call(fn, h, x, T, target, nll, lse);
  if (s != EAT_OK) return s;
  if (!h->desc.with_grad) return bad_arg(fn, "the handle was created without with_grad");
  if (!g || !dx || !dw) return bad_arg(fn, "g, dx and dw must be non-NULL");
  if (misaligned(dx, 16) || misaligned(dw, 16) || misaligned(g, 4))
    return bad_arg(fn, "dx and dw must be 16-byte aligned");
  // (x and w are read while dx and dw are written)
  const size_t row = 2 * (size_t)h->desc.d_model, tokens = T * row, vocab = h->desc.vocab * row;
  if (overlap(dx, tokens, x, tokens) || overlap(dx, tokens, h->desc.w, vocab))
    return bad_arg(fn, "dx must not overlap x or w");
  if (overlap(dw, vocab, x, tokens) || overlap(dw, vocab, h->desc.w, vocab) ||
      overlap(dw, vocab, dx, tokens))
    return bad_arg(fn, "dw must not overlap x, w or dx");
  return launched(fn, run_grad(h, x, T, target, g, nll, lse, dx, dw, (cudaStream_t)stream));
}

}  // extern "C"
