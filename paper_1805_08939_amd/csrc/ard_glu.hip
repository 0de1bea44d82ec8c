// Gated feed-forward layer under a row pattern on its hidden units:
//   g = W0 x + b0,  u = W1 x + b1,  h = scale act(g) u  on the kept units.
//
// Forward: both projections of the kept rows as one batched product, then the
// activation and the product. Backward: one pass writes the derivatives
//   dg = scale dh u act'(g),  du = scale dh act(g)
// of the kept rows (rounded to the element type once) and their row sums, the
// bias gradients, from the unrounded values; then dX = W0^T dg + W1^T du as one
// product over both halves, and dW as a batch of two. A pattern's kept rows are an
// arithmetic progression, so every gather is a row stride.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ard_gemm_fast.hpp"
#include "ard_internal.hpp"

namespace ard {
namespace {

// The activation and its derivative, in fp32.
struct Act {
  float f, d;
};
__device__ __forceinline__ Act act_of(int act, float g) {
  if (act == ARD_GLU_RELU) return {g > 0.0f ? g : (g == g ? 0.0f : g), g > 0.0f ? 1.0f : 0.0f};
  if (act == ARD_GLU_GELU) {
    const float cdf = 0.5f * erfcf(g * -0.70710678118654752440f);  // to its own last bits where it is small
    return {g * cdf, cdf + g * 0.39894228040143267794f * expf(-0.5f * g * g)};
  }
  const float s = 1.0f / (1.0f + expf(-g));
  if (act == ARD_GLU_SIGMOID) return {s, s * (1.0f - s)};
  return {g * s, s * (1.0f + g * (1.0f - s))};
}

struct GluShape {
  int32_t B, K, N, kept, period, offset;
  int64_t ldd;   // row length of the derivatives in the workspace
  size_t es;
  bool zero;     // dropped rows are written 0
};

// Joins the projections zf[2][kept][B] (fp32): a workgroup per hidden unit, a
// dropped one's row cleared if asked.
template <typename T>
__global__ void __launch_bounds__(256) glu_join_kernel(GluShape s, const float* __restrict__ zf,
                                                       const float* __restrict__ bias, int act, float scale,
                                                       T* __restrict__ Z, T* __restrict__ H) {
  const int64_t n = blockIdx.x;
  T* h = H + n * s.B;
  if (static_cast<int32_t>(n % s.period) != s.offset) {
    if (s.zero)
      for (int b = threadIdx.x; b < s.B; b += 256) h[b] = from_f32<T>(0.0f);
    return;
  }
  const int64_t i = (n - s.offset) / s.period;
  const float *gf = zf + i * s.B, *uf = gf + static_cast<int64_t>(s.kept) * s.B;
  const float b0 = bias ? bias[n] : 0.0f, b1 = bias ? bias[s.N + n] : 0.0f;
  for (int b = threadIdx.x; b < s.B; b += 256) {
    const float g = gf[b] + b0, u = uf[b] + b1;
    h[b] = from_f32<T>(scale * act_of(act, g).f * u);
    if (Z) {
      Z[n * s.B + b] = from_f32<T>(g);
      Z[(s.N + n) * s.B + b] = from_f32<T>(u);
    }
  }
}

// The derivatives D[2][kept][ldd] and their row sums: a workgroup per kept unit.
template <typename T>
__global__ void __launch_bounds__(256) glu_derive_kernel(GluShape s, const T* __restrict__ Z,
                                                         const T* __restrict__ dH, int act, float scale,
                                                         T* __restrict__ D, float* __restrict__ dbias) {
  const int64_t i = blockIdx.x, n = s.offset + i * s.period;
  const T *gp = Z + n * s.B, *up = Z + (s.N + n) * s.B, *hp = dH + n * s.B;
  T *dg = D + i * s.ldd, *du = D + (s.kept + i) * s.ldd;
  float sg = 0.0f, su = 0.0f;
  for (int b = threadIdx.x; b < s.B; b += 256) {
    const Act a = act_of(act, to_f32(gp[b]));
    const float d = scale * to_f32(hp[b]), g = d * to_f32(up[b]) * a.d, u = d * a.f;
    dg[b] = from_f32<T>(g);
    du[b] = from_f32<T>(u);
    sg += g;
    su += u;
  }
  if (!dbias) return;
  __shared__ float red[8];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sg += __shfl_down(sg, o, 64), su += __shfl_down(su, o, 64);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) red[wave] = sg, red[4 + wave] = su;
  __syncthreads();
  if (threadIdx.x == 0) {
    dbias[n] = (red[0] + red[1]) + (red[2] + red[3]);
    dbias[s.N + n] = (red[4] + red[5]) + (red[6] + red[7]);
  }
}

// Clears the dropped rows of dW[2][N][K] and entries of dbias[2][N].
template <typename T>
__global__ void __launch_bounds__(256) glu_clear_kernel(GluShape s, T* __restrict__ dW, float* __restrict__ dbias) {
  const int64_t n = blockIdx.x;  // of 2 N
  if (static_cast<int32_t>(n % s.N % s.period) == s.offset) return;
  if (dW)
    for (int64_t k = threadIdx.x; k < s.K; k += 256) dW[n * s.K + k] = from_f32<T>(0.0f);
  if (dbias && threadIdx.x == 0) dbias[n] = 0.0f;
}

// 0 to every 16 bytes and the rest behind them (a fill kernel: a caller may capture the call).
__global__ void __launch_bounds__(256) fill_zero_kernel(char* __restrict__ p, int64_t bytes) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256, first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  for (int64_t i = first; i < bytes / 16; i += step) reinterpret_cast<u32x4*>(p)[i] = u32x4{0u, 0u, 0u, 0u};
  for (int64_t i = bytes / 16 * 16 + first; i < bytes; i += step) p[i] = 0;
}
hipError_t fill_zero(void* p, size_t bytes, hipStream_t stream) {
  const unsigned blocks = static_cast<unsigned>(std::min<size_t>(2048, bytes / 4096 + 1));
  hipLaunchKernelGGL(fill_zero_kernel, dim3(blocks), dim3(256), 0, stream, static_cast<char*>(p),
                     static_cast<int64_t>(bytes));
  return hipGetLastError();
}

int need_ptr(const void* p, const char* name) {
  if (!p) return fail(ARD_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}
int may_ptr(const void* p, const char* name) {
  if (p && !aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}

int check_desc(const ard_glu_desc* d, GluShape* s) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->batch < 1 || d->in_features < 1 || d->hidden_features < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (batch %d, in %d, hidden %d)", d->batch, d->in_features,
                d->hidden_features);
  if (d->hidden_features >= 1 << 30) return fail(ARD_ERR_UNSUPPORTED, "at most 2^30 hidden units");
  if (d->act < ARD_GLU_SILU || d->act > ARD_GLU_SIGMOID)
    return fail(ARD_ERR_INVALID_ARG, "unknown activation %d", d->act);
  if (d->dropped != ARD_DROPPED_ZERO && d->dropped != ARD_DROPPED_SKIP)
    return fail(ARD_ERR_INVALID_ARG, "unknown dropped-output mode %d", d->dropped);
  if (d->grad_dtype != ARD_F32 && d->grad_dtype != d->dtype)
    return fail(ARD_ERR_INVALID_ARG, "grad_dtype must be ARD_F32 or dtype");
  if (!std::isfinite(d->scale)) return fail(ARD_ERR_INVALID_ARG, "scale must be finite");
  const int st = check_row_plan(d->hidden_plan, d->hidden_features, "hidden_plan", false);
  if (st != ARD_OK) return st;
  s->B = d->batch;
  s->K = d->in_features;
  s->N = d->hidden_features;
  const bool all = !d->hidden_plan || d->hidden_plan->period == 1;
  s->kept = all ? s->N : d->hidden_plan->kept;
  s->period = all ? 1 : d->hidden_plan->period;
  s->offset = all ? 0 : d->hidden_plan->offset;
  s->ldd = (static_cast<int64_t>(s->B) + 7) / 8 * 8;
  s->es = d->dtype == ARD_BF16 ? 2 : 4;
  s->zero = d->dropped == ARD_DROPPED_ZERO;
  return ARD_OK;
}

size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Floats of partial sums of a product, whichever kernel takes it.
template <typename T>
size_t partial_floats(int M, int N, int K, int kbatch, int batch) {
  int64_t s = plan_gemm<T>(M, N, K, kbatch, batch).splits;
  if constexpr (sizeof(T) == 4) {
    s = std::max<int64_t>(s, plan_fast_f32(M, N, K, kbatch, batch, kAnyRoom).splits);
    for (const auto& costs : kCostRegF32)
      s = std::max<int64_t>(s, plan_fast_f32(M, N, K, kbatch, batch, kAnyRoom, false, costs).splits);
  } else {
    s = std::max<int64_t>(s, plan_fast_bf16(M, N, K, kbatch, batch).splits);
  }
  return s > 1 ? static_cast<size_t>(s) * batch * M * N : 0;
}

// The workspace: what the products read or write first, their partial sums behind it.
struct Space {
  size_t head, part;
  size_t bytes() const { return head + part; }
};
template <typename T>
Space fwd_space(const GluShape& s) {
  if (s.kept == 0) return {0, 0};
  return {al256(static_cast<size_t>(2) * s.kept * s.B * 4), al256(4 * partial_floats<T>(s.kept, s.B, s.K, 1, 2))};
}
template <typename T>
Space bwd_space(const GluShape& s) {
  if (s.kept == 0) return {0, 0};
  const size_t d = partial_floats<T>(s.K, s.B, s.kept, 2, 1), w = partial_floats<T>(s.kept, s.K, s.B, 1, 2);
  return {al256(static_cast<size_t>(2) * s.kept * s.ldd * sizeof(T)), al256(4 * std::max(d, w))};
}

int check_ws(const Space& sp, const void* ws, size_t ws_bytes) {
  if (sp.bytes() == 0) return ARD_OK;
  if (!ws || ws_bytes < sp.bytes())
    return fail(ARD_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", sp.bytes(), ws ? ws_bytes : 0);
  if (!aligned16(ws)) return fail(ARD_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return ARD_OK;
}

// The kept rows of both projections, W[2][N][K], one after the other `stride` apart.
GemmOperand kept_weights(const GluShape& s, const void* W) {
  GemmOperand o = {};
  o.p = static_cast<const char*>(W) + static_cast<size_t>(s.offset) * s.K * s.es;
  o.ld = static_cast<int64_t>(s.K) * s.period;
  o.bstride = o.kbstride = static_cast<int64_t>(s.N) * s.K;
  return o;
}
GemmOperand plain(const void* p, int64_t ld, int64_t stride) {
  GemmOperand o = {};
  o.p = p;
  o.ld = ld;
  o.bstride = o.kbstride = stride;
  return o;
}

// A product of strided views, on the fast kernels or, past their load offsets, the general one.
template <typename T, bool AMC, bool BMC, typename OutT>
hipError_t product(const GemmArgs& g, int batch, hipStream_t stream, float* partial, size_t floats) {
  if (any_ok<AMC, BMC>(g, sizeof(T)))
    return run_strided_gemm<T, AMC, BMC, OutT, EPI_STORE>(g, batch, stream, floats ? partial : nullptr,
                                                          static_cast<int64_t>(floats));
  constexpr int A = AMC ? MC_ELEM : KC_ELEM, B = BMC ? MC_ELEM : KC_ELEM;
  return run_gemm<T, OutT, A, A, B, B, false, false, EPI_STORE>(g, batch, false, false, stream,
                                                                floats ? partial : nullptr);
}

template <typename T>
int fwd_impl(const ard_glu_desc* d, const GluShape& s, const void* Xt, const void* W, const float* bias, void* Zt,
             void* Ht, char* ws, hipStream_t stream) {
  const Space sp = fwd_space<T>(s);
  float* zf = reinterpret_cast<float*>(ws);
  if (s.kept > 0) {
    GemmArgs g = {};
    g.M = s.kept, g.N = s.B, g.K = s.K;
    g.a = kept_weights(s, W);
    g.b = plain(Xt, s.B, 0);
    g.c.p = zf, g.c.ld = s.B, g.c.bstride = static_cast<int64_t>(s.kept) * s.B;
    ARD_HIP_CHECK((product<T, false, true, float>(g, 2, stream, reinterpret_cast<float*>(ws + sp.head), sp.part / 4)));
  }
  hipLaunchKernelGGL(glu_join_kernel<T>, dim3(s.N), dim3(256), 0, stream, s, zf, bias, d->act, d->scale,
                     static_cast<T*>(Zt), static_cast<T*>(Ht));
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T, typename G>
int bwd_impl(const ard_glu_desc* d, const GluShape& s, const void* Xt, const void* W, const void* Zt, const void* dHt,
             void* dXt, void* dW, float* dbias, char* ws, hipStream_t stream) {
  const Space sp = bwd_space<T>(s);
  float* part = reinterpret_cast<float*>(ws + sp.head);
  const int64_t half = static_cast<int64_t>(s.kept) * s.ldd;
  if (s.kept == 0) {  // nothing is kept: nothing depends on the input
    if (dXt) ARD_HIP_CHECK(fill_zero(dXt, static_cast<size_t>(s.K) * s.B * s.es, stream));
  } else {
    hipLaunchKernelGGL(glu_derive_kernel<T>, dim3(s.kept), dim3(256), 0, stream, s, static_cast<const T*>(Zt),
                       static_cast<const T*>(dHt), d->act, d->scale, reinterpret_cast<T*>(ws), dbias);
    ARD_LAUNCH_CHECK();
    GemmArgs g = {};
    if (dXt) {
      g.M = s.K, g.N = s.B, g.K = s.kept, g.kbatch = 2;
      g.a = kept_weights(s, W);
      g.b = plain(ws, s.ldd, half);
      g.c.p = dXt, g.c.ld = s.B;
      ARD_HIP_CHECK((product<T, true, true, T>(g, 1, stream, part, sp.part / 4)));
    }
    if (dW) {
      g = {};
      g.M = s.kept, g.N = s.K, g.K = s.B;
      g.a = plain(ws, s.ldd, half);
      g.b = plain(Xt, s.B, 0);
      g.c.p = static_cast<G*>(dW) + static_cast<int64_t>(s.offset) * s.K;
      g.c.ld = static_cast<int64_t>(s.K) * s.period;
      g.c.bstride = static_cast<int64_t>(s.N) * s.K;
      ARD_HIP_CHECK((product<T, false, false, G>(g, 2, stream, part, sp.part / 4)));
    }
  }
  if (s.zero && s.period > 1 && (dW || dbias)) {
    hipLaunchKernelGGL(glu_clear_kernel<G>, dim3(2 * s.N), dim3(256), 0, stream, s, static_cast<G*>(dW), dbias);
    ARD_LAUNCH_CHECK();
  }
  return ARD_OK;
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

size_t ard_glu_workspace_bytes(const ard_glu_desc* desc) {
  GluShape s;
  if (check_desc(desc, &s) != ARD_OK) return 0;
  return desc->dtype == ARD_BF16 ? std::max(fwd_space<bf16>(s).bytes(), bwd_space<bf16>(s).bytes())
                                 : std::max(fwd_space<float>(s).bytes(), bwd_space<float>(s).bytes());
}

int ard_glu_fwd(const ard_glu_desc* desc, const void* Xt, const void* W, const float* bias, void* Zt, void* Ht,
                void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  GluShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Xt, "Xt")) || (st = need_ptr(W, "W")) || (st = may_ptr(bias, "bias")) ||
      (st = may_ptr(Zt, "Zt")) || (st = need_ptr(Ht, "Ht")) ||
      (st = check_ws(desc->dtype == ARD_BF16 ? fwd_space<bf16>(s) : fwd_space<float>(s), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? fwd_impl<bf16>(desc, s, Xt, W, bias, Zt, Ht, w, sm)
                                 : fwd_impl<float>(desc, s, Xt, W, bias, Zt, Ht, w, sm);
}

int ard_glu_bwd(const ard_glu_desc* desc, const void* Xt, const void* W, const void* Zt, const void* dHt, void* dXt,
                void* dW, float* dbias, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  GluShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Xt, "Xt")) || (st = need_ptr(W, "W")) || (st = need_ptr(Zt, "Zt")) ||
      (st = need_ptr(dHt, "dHt")) || (st = may_ptr(dXt, "dXt")) || (st = may_ptr(dW, "dW")) ||
      (st = may_ptr(dbias, "dbias")) ||
      (st = check_ws(desc->dtype == ARD_BF16 ? bwd_space<bf16>(s) : bwd_space<float>(s), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  if (desc->dtype == ARD_F32) return bwd_impl<float, float>(desc, s, Xt, W, Zt, dHt, dXt, dW, dbias, w, sm);
  return desc->grad_dtype == ARD_BF16 ? bwd_impl<bf16, bf16>(desc, s, Xt, W, Zt, dHt, dXt, dW, dbias, w, sm)
                                      : bwd_impl<bf16, float>(desc, s, Xt, W, Zt, dHt, dXt, dW, dbias, w, sm);
}

}  // extern "C"
