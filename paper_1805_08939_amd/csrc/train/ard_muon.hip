// Momentum update of a layer's kept weights by the orthogonalised momentum:
//   V = mu V + dW,  U = dW + mu V (Nesterov) or V,  X = U / (|U| + eps)
//   iterations times, with A = X X^T (or X^T X, whichever is smaller):
//     X = (a + b A + c A^2) X
//   W = (1 - lr decay) W - lr sqrt(max(1, outputs / inputs)) X
// Each iteration applies the odd polynomial a s + b s^3 + c s^5 to the singular values of X
// and leaves its singular vectors; |U| is the Frobenius norm, so that they start within 1.
// Method, default coefficients and the step's scale: Jordan et al., "Muon: an optimizer for
// hidden layers in neural networks", 2024.
//
// X, A and the polynomial are kept in bf16 parts (ard_parts_gemm.hpp): three for fp32 weights,
// 2^-24 of a value; two for bf16 ones, 2^-16, where a step is then 2.5e-5 off and the weight
// that takes it is rounded to 2^-8 of itself. Momentum, norm and the last X are fp32 and 64 bits.
//
// The kept block is gathered once, into a dense matrix. A and A^2 are symmetric, the third
// product has the shape of the block. Bound by the matrix cores, for small blocks by the
// latency of three products after one another.

#include "ard_parts_gemm.hpp"

namespace ard {
namespace {

// The kept block as it is stored: rows row_offset + row_period * i of W and V (rows of ld
// elements), columns likewise; the gradient in the same places or (ldg > 0) dense.
struct Block {
  int32_t R, C;                       // kept rows and columns
  int32_t row_period, row_offset, col_period, col_offset;
  int64_t ld, ldg;
  int64_t ldx;                        // rows of the dense copies
  int32_t width, row_pieces;          // of the passes over the block: threads on a row, pieces of a row
};
__device__ __forceinline__ int64_t place(const Block& b, int64_t i, int64_t j) {
  return (b.row_offset + i * b.row_period) * b.ld + b.col_offset + j * b.col_period;
}

constexpr int kNormBlocks = 1024;  // workgroups of the first pass, at most: one sum of squares each

// The workgroups take pieces in turn: some columns of a row, or of several rows where a row
// has fewer than 256. f(row, the thread's first column, its columns, their distance): up to four
// of them, to be in flight together (64 x 8192 fp32, the whole update: 164 us with a row to a
// workgroup and one place of a thread after the other, 150).
template <class F>
__device__ __forceinline__ void each_piece(const Block& b, F f) {
  const int32_t len = ((b.C + b.row_pieces - 1) / b.row_pieces + b.width - 1) / b.width * b.width;
  const int32_t t = static_cast<int32_t>(threadIdx.x), rows = 256 / b.width;
  const int64_t pieces = static_cast<int64_t>(b.row_pieces) * ((b.R + rows - 1) / rows);
  for (int64_t p = blockIdx.x; p < pieces; p += gridDim.x) {
    const int64_t q = b.row_pieces == 1 ? p : p / b.row_pieces, i = q * rows + t / b.width;
    const int32_t first = static_cast<int32_t>(p - q * b.row_pieces) * len, j0 = first + t % b.width;
    const int32_t end = min(b.C, first + len);
    if (i < b.R && j0 < end) f(i, j0, (end - j0 + b.width - 1) / b.width, b.width);
  }
}
void plan_pieces(Block* b) {
  b->width = 32;
  while (b->width < 256 && b->width < b->C) b->width *= 2;
  b->row_pieces = std::max(1, (b->C + 1023) / 1024);
}
unsigned piece_groups(const Block& b) {
  const int64_t rows = 256 / b.width;
  return static_cast<unsigned>(std::min<int64_t>((b.R + rows - 1) / rows * b.row_pieces, kNormBlocks));
}

// V and U, and the sum of U's squares of each workgroup, in 64 bits (momenta far below 1
// have squares below the smallest fp32 number).
__global__ void __launch_bounds__(256) muon_momentum_kernel(Block b, float* __restrict__ V, const float* __restrict__ dW,
                                                            float mu, bool nesterov, float* __restrict__ U,
                                                            double* __restrict__ sums) {
  double sum = 0.0;
  each_piece(b, [&](int64_t i, int32_t j0, int n, int32_t step_j) {
    float g[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) {
        const int64_t at = place(b, i, j0 + step_j * e);
        g[e] = b.ldg > 0 ? dW[i * b.ldg + j0 + step_j * e] : dW[at];
        v[e] = V[at];
      }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) {
        const float w = mu * v[e] + g[e], u = nesterov ? g[e] + mu * w : w;
        V[place(b, i, j0 + step_j * e)] = w;
        U[i * b.ldx + j0 + step_j * e] = u;
        sum += static_cast<double>(u) * u;
      }
  });
  __shared__ double red[4];
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_down(sum, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// 1 / (|U| + eps) from the workgroups' sums, in their order; every thread has it.
__device__ __forceinline__ double inverse_norm(const double* sums, int blocks, float eps) {
  __shared__ double red[256];
  double v = 0.0;
  for (int q = threadIdx.x; q < blocks; q += 256) v += sums[q];
  red[threadIdx.x] = v;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (static_cast<int>(threadIdx.x) < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  return 1.0 / (sqrt(red[0]) + static_cast<double>(eps));
}

// X = U / (|U| + eps), in parts.
template <int P>
__global__ void __launch_bounds__(256) muon_scale_kernel(Block b, const float* __restrict__ U, const double* __restrict__ sums,
                                                         int blocks, float eps, bf16* __restrict__ X, int64_t plane) {
  const double inv = inverse_norm(sums, blocks, eps);
  const int64_t per = b.ldx / 8, total = per * b.R, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < total; at += step) {
    const f32x4 lo = *reinterpret_cast<const f32x4*>(U + at * 8), hi = *reinterpret_cast<const f32x4*>(U + at * 8 + 4);
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(lo[e] * inv), v[4 + e] = static_cast<float>(hi[e] * inv);
    store_parts<P>(X + at * 8, plane, v);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) muon_update_kernel(Block b, const float* __restrict__ X, T* __restrict__ W, float keep,
                                                          float step) {
  each_piece(b, [&](int64_t i, int32_t j0, int n, int32_t step_j) {
    float w[4], x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) {
        w[e] = to_f32(W[place(b, i, j0 + step_j * e)]);
        x[e] = X[i * b.ldx + j0 + step_j * e];
      }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) W[place(b, i, j0 + step_j * e)] = from_f32<T>(keep * w[e] - step * x[e]);
  });
}

// Momentum SGD of the kept outputs' bias.
__global__ void __launch_bounds__(256) muon_bias_kernel(Kept out, float* __restrict__ bias, float* __restrict__ Vb,
                                                        const float* __restrict__ db, float lr, float mu) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= out.kept) return;
  const int64_t n = out.offset + i * out.period;
  const float v = mu * Vb[n] + db[n];
  Vb[n] = v;
  bias[n] -= lr * v;
}

// ------------------------------------------------------------------ host
struct MuonShape {
  Block b;
  Kept out;
  int32_t m, l;   // smaller and larger side
  int64_t lda;
  double stretch;  // sqrt(max(1, kept outputs / kept inputs))
};

int check_desc(const ard_fc_desc* d, MuonShape* s) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->in_features < 1 || d->out_features < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (in %d, out %d)", d->in_features, d->out_features);
  if (d->weight_layout < ARD_WEIGHTS_FULL || d->weight_layout > ARD_WEIGHTS_INPUT_MAJOR)
    return fail(ARD_ERR_INVALID_ARG, "unknown weight layout %d", d->weight_layout);
  int st = check_row_plan(d->in_plan, d->in_features, "in_plan", false);
  if (st != ARD_OK) return st;
  st = check_row_plan(d->out_plan, d->out_features, "out_plan", false);
  if (st != ARD_OK) return st;
  const Kept in = kept_of(d->in_plan, d->in_features), out = kept_of(d->out_plan, d->out_features);
  const bool input_major = d->weight_layout == ARD_WEIGHTS_INPUT_MAJOR;
  if (input_major && out.period != 1)
    return fail(ARD_ERR_UNSUPPORTED, "input-major weights need every output kept (out_plan NULL or period 1)");
  const Kept &r = input_major ? in : out, &c = input_major ? out : in;
  s->b = {r.kept, c.kept, r.period, r.offset, c.period, c.offset, c.n,
          d->weight_layout == ARD_WEIGHTS_COMPACT_GRAD ? up8(c.kept) : 0, up8(c.kept), 0, 0};
  plan_pieces(&s->b);
  s->out = out;
  s->m = std::min(r.kept, c.kept);
  s->l = std::max(r.kept, c.kept);
  s->lda = up8(s->m);
  if (s->l >= 1 << 22)  // offsets within a tile have 32 bits
    return fail(ARD_ERR_UNSUPPORTED, "%d x %d kept weights: sides must be below 2^22", r.kept, c.kept);
  s->stretch = in.kept > 0 ? std::sqrt(std::max(1.0, static_cast<double>(out.kept) / in.kept)) : 1.0;
  return ARD_OK;
}

int check_opts(const ard_muon_opts* o) {
  const float all[] = {o->lr, o->momentum, o->weight_decay, o->bias_lr, o->eps, o->a, o->b, o->c};
  for (float x : all)
    if (!std::isfinite(x)) return fail(ARD_ERR_INVALID_ARG, "every option must be finite");
  if (!(o->eps > 0.0f)) return fail(ARD_ERR_INVALID_ARG, "eps must be > 0");
  if (o->iterations < 1 || o->iterations > 64)
    return fail(ARD_ERR_INVALID_ARG, "iterations %d: 1 to 64", o->iterations);
  return ARD_OK;
}

// The workspace: the block in fp32 (U, at the end X), X twice and A and the polynomial in
// parts, the sums of squares, the products' partial sums.
struct Space {
  size_t u, x, a, sums, part;
  size_t bytes() const { return u + 2 * x + 2 * a + sums + part; }
};
template <int P>
Space space_of(const MuonShape& s) {
  if (s.m == 0) return {0, 0, 0, 0, 0};
  const size_t part = std::max({plan_parts<P>(s.m, s.m, s.l, true).floats, plan_parts<P>(s.m, s.m, s.m, true).floats,
                                plan_parts<P>(s.b.R, s.b.C, s.m, false).floats});
  const size_t x = static_cast<size_t>(s.b.R) * s.b.ldx, a = static_cast<size_t>(s.m) * s.lda;
  return {al256(x * 4), al256(x * 2 * P), al256(a * 2 * P), kNormBlocks * 8, al256(4 * part)};
}
size_t space_bytes(const ard_fc_desc* d, const MuonShape& s) {
  return d->dtype == ARD_BF16 ? space_of<2>(s).bytes() : space_of<3>(s).bytes();
}

template <int P, typename T>
int muon_impl(const MuonShape& s, const ard_muon_opts& o, void* W, float* V, const float* dW, char* ws, hipStream_t stream) {
  const Space sp = space_of<P>(s);
  const Block& b = s.b;
  const int64_t xp = static_cast<int64_t>(b.R) * b.ldx, ap = static_cast<int64_t>(s.m) * s.lda;  // planes
  float* Uf = reinterpret_cast<float*>(ws);
  bf16 *X = reinterpret_cast<bf16*>(ws + sp.u), *Y = reinterpret_cast<bf16*>(ws + sp.u + sp.x);
  bf16 *A = reinterpret_cast<bf16*>(ws + sp.u + 2 * sp.x), *Q = reinterpret_cast<bf16*>(ws + sp.u + 2 * sp.x + sp.a);
  char* rest = ws + sp.u + 2 * sp.x + 2 * sp.a;
  double* sums = reinterpret_cast<double*>(rest);
  float* part = reinterpret_cast<float*>(rest + sp.sums);
  const unsigned groups = piece_groups(b);
  hipLaunchKernelGGL(muon_momentum_kernel, dim3(groups), dim3(256), 0, stream, b, V, dW, o.momentum, o.nesterov != 0, Uf, sums);
  ARD_LAUNCH_CHECK();
  const unsigned chunks = static_cast<unsigned>(std::min<int64_t>(2048, (xp / 8 + 255) / 256));
  hipLaunchKernelGGL(muon_scale_kernel<P>, dim3(chunks), dim3(256), 0, stream, b, Uf, sums, static_cast<int>(groups), o.eps, X, xp);
  ARD_LAUNCH_CHECK();
  const bool wide = b.R <= b.C;
  for (int it = 0; it < o.iterations; ++it) {
    const bool last = it + 1 == o.iterations;
    PartsArgs g = {};
    g.M = g.N = s.m, g.K = s.l;
    g.a = g.b = PartsView{X, xp, b.ldx};
    g.symmetric = true;
    g.epi = PARTS_STORE;
    g.out = A, g.plane = ap, g.ldo = s.lda;
    ARD_HIP_CHECK((wide ? run_parts_gemm<P, false, false>(g, part, stream) : run_parts_gemm<P, true, true>(g, part, stream)));
    g.K = s.m;
    g.a = g.b = g.poly = PartsView{A, ap, s.lda};  // A is its own transpose
    g.epi = PARTS_POLY;
    g.out = Q;
    g.pa = o.a, g.pb = o.b, g.pc = o.c;
    ARD_HIP_CHECK((run_parts_gemm<P, false, false>(g, part, stream)));
    g = {};
    g.M = b.R, g.N = b.C, g.K = s.m;
    g.epi = last ? PARTS_FLOAT : PARTS_STORE;
    g.out = Y, g.plane = xp, g.ldo = b.ldx;
    g.fout = Uf, g.fstep = 1;
    const PartsView x{X, xp, b.ldx}, q{Q, ap, s.lda};
    if (wide) {
      g.a = q, g.b = x;
      ARD_HIP_CHECK((run_parts_gemm<P, false, true>(g, part, stream)));
    } else {
      g.a = x, g.b = q;
      ARD_HIP_CHECK((run_parts_gemm<P, false, false>(g, part, stream)));
    }
    std::swap(X, Y);
  }
  hipLaunchKernelGGL(muon_update_kernel<T>, dim3(groups), dim3(256), 0, stream, b, Uf, static_cast<T*>(W),
                     static_cast<float>(1.0 - static_cast<double>(o.lr) * o.weight_decay),
                     static_cast<float>(o.lr * s.stretch));
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

void ard_muon_opts_default(ard_muon_opts* opts) {
  if (!opts) return;
  *opts = ard_muon_opts{0.02f, 0.95f, 0.0f, 0.02f, 1e-7f, 3.4445f, -4.7750f, 2.0315f, 5, 1};
}

size_t ard_fc_muon_workspace_bytes(const ard_fc_desc* desc) {
  MuonShape s;
  if (check_desc(desc, &s) != ARD_OK) return 0;
  return space_bytes(desc, s);
}

int ard_fc_muon(const ard_fc_desc* desc, const ard_muon_opts* opts, void* W, float* V, const float* dW, float* bias, float* Vb,
                const float* dbias, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  MuonShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  ard_muon_opts o;
  ard_muon_opts_default(&o);
  if (opts) o = *opts;
  if ((st = check_opts(&o)) != ARD_OK) return st;
  if (!W || !V || !dW) return fail(ARD_ERR_INVALID_ARG, "W, V or dW is NULL");
  if ((bias == nullptr) != (Vb == nullptr) || (bias == nullptr) != (dbias == nullptr))
    return fail(ARD_ERR_INVALID_ARG, "bias, Vb and dbias must be all given or all NULL");
  if (reinterpret_cast<uintptr_t>(W) % (desc->dtype == ARD_BF16 ? 2 : 4) || reinterpret_cast<uintptr_t>(V) % 4 ||
      reinterpret_cast<uintptr_t>(dW) % 4 || reinterpret_cast<uintptr_t>(bias) % 4 || reinterpret_cast<uintptr_t>(Vb) % 4 ||
      reinterpret_cast<uintptr_t>(dbias) % 4)
    return fail(ARD_ERR_INVALID_ARG, "W, V, dW or the bias is not aligned to its element size");
  if ((st = check_space(space_bytes(desc, s), ws, ws_bytes)) != ARD_OK) return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  if (bias && s.out.kept > 0) {
    hipLaunchKernelGGL(muon_bias_kernel, dim3((s.out.kept + 255) / 256), dim3(256), 0, sm, s.out, bias, Vb, dbias, o.bias_lr,
                       o.momentum);
    ARD_LAUNCH_CHECK();
  }
  if (s.m == 0) return ARD_OK;
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? muon_impl<2, bf16>(s, o, W, V, dW, w, sm) : muon_impl<3, float>(s, o, W, V, dW, w, sm);
}

}  // extern "C"
