// Root-mean-square norm of a sum, forward and backward, on feature-major columns:
//   s = x + r,  inv = 1 / sqrt(mean_k s^2 + eps),  y = gain s inv
//   backward with xh = s inv, u = gain dY:  dX = dS + inv (u - xh mean_k(u xh)),
//   dgain_k = sum_b dY xh
//
// A norm runs down a column, and a column's values lie a row apart, so a workgroup takes a
// block of neighbouring columns (whole 128-byte lines of each row) and a range of rows. Two
// passes over the inputs: sums of the columns, then the results. Where one workgroup can
// take every row of its columns both passes are one launch and the second reads what the
// first left in the cache; else the ranges of rows meet in the workspace, added in their
// order, between two launches. Sums over a column are held in 64 bits: a square of a
// feature of 2^70 is infinite in 32, and the matrix of a norm has the memory for it anyway.
// Where the second pass is a launch of its own its results go past the caches (NT), which
// keeps the inputs there (bf16 8192 x 2048: forward 47.6 to 41.4 us, backward 57.4 to 54.2),
// and runs from its last row to the first (52.9). The sums that the ranges leave are joined
// with eight loads in flight (35.6 and 41.8).
// Bound by HBM.

#include "ard_train.hpp"

namespace ard {
namespace {

struct NormShape {
  int32_t B, K;
  float eps;
  int32_t lanes;      // threads side by side on a row
  int32_t blocks;     // blocks of columns
  int32_t ranges;     // ranges of rows
  int32_t rows;       // rows of a range
};

// Workgroups of a block of columns each: in rows of 2^20, since the threads along x have to stay below 2^32.
constexpr int32_t kGridRow = 1 << 20;
dim3 block_grid(int32_t blocks) { return dim3(std::min(blocks, kGridRow), (blocks - 1) / kGridRow + 1); }
__device__ __forceinline__ int32_t column_block() { return static_cast<int32_t>(blockIdx.y * gridDim.x + blockIdx.x); }

// The columns and rows of a thread (lanes divides the workgroup).
template <int VE>
struct Place {
  int32_t lane, row, step;  // lane: place in the block of columns; rows row, row + step, ...
  int64_t col;
  int n;                    // columns, <= 0: none
};
template <int VE>
__device__ __forceinline__ Place<VE> place_of(const NormShape& s, int32_t block) {
  const int nt = static_cast<int>(blockDim.x), t = static_cast<int>(threadIdx.x);
  Place<VE> p;
  p.step = nt / s.lanes;
  p.lane = t % s.lanes;
  p.row = t / s.lanes;
  p.col = (static_cast<int64_t>(block) * s.lanes + p.lane) * VE;
  p.n = static_cast<int>(min<int64_t>(VE, s.B - p.col));
  return p;
}

// Rows of a thread from r0 to r1.
template <int VE>
__device__ __forceinline__ int64_t rows_of(const Place<VE>& p, int64_t r0, int64_t r1) {
  const int64_t n = r1 - r0 - p.row;
  return n > 0 ? (n + p.step - 1) / p.step : 0;
}

// The sum over `lanes` neighbouring threads (1 to 16, a power of two), in a fixed order:
// exchanges within 16 lanes, without LDS.
__device__ __forceinline__ float row_sum(float v, int lanes) {
  auto add = [&](auto ctrl) {
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (lanes > 1) add(std::integral_constant<int, 0xb1>{});    // neighbours
  if (lanes > 2) add(std::integral_constant<int, 0x4e>{});    // pairs
  if (lanes > 4) add(std::integral_constant<int, 0x141>{});   // halves of 8
  if (lanes > 8) add(std::integral_constant<int, 0x140>{});   // halves of 16
  return v;
}

// Sums of the workgroup's columns over its threads, in a fixed order: v[e] of every thread
// -> red[lane * VE + e]. Two steps through LDS, so that no thread adds a long row alone.
template <int VE, int NT>
__device__ __forceinline__ void column_sums(const NormShape& s, const Place<VE>& p, const double (&v)[VE], double* red) {
  const int cols = s.lanes * VE, t = static_cast<int>(threadIdx.x);
#pragma unroll
  for (int e = 0; e < VE; ++e) red[p.row * cols + p.lane * VE + e] = v[e];
  __syncthreads();
  const int parts = min(min(NT / cols, p.step), 32), part = t / cols, c = t % cols;
  double sum = 0.0;
  if (part < parts)
    for (int r = part; r < p.step; r += parts) sum += red[r * cols + c];
  __syncthreads();
  if (part < parts) red[part * cols + c] = sum;
  __syncthreads();
  if (t < cols) {
    sum = red[t];
    for (int q = 1; q < parts; ++q) sum += red[q * cols + t];
  }
  __syncthreads();
  if (t < cols) red[t] = sum;
  __syncthreads();
}

// ------------------------------------------------------------------ forward
template <typename T>
struct FwdArgs {
  NormShape s;
  const T* X;
  const T* R;
  const float* gain;
  T* S;
  T* Y;
  float* inv;
  double* part;  // [ranges][B]
};

template <typename T, int VE, int U>
__device__ __forceinline__ void fwd_sums(const FwdArgs<T>& a, const Place<VE>& p, int64_t r0, int64_t r1,
                                         double (&sum)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) sum[e] = 0.0;
  if (p.n <= 0) return;
  auto add = [&](const Chunk<T, VE>& x, const Chunk<T, VE>& r) {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const double v = a.R ? x.at(e) + r.at(e) : x.at(e);
      sum[e] += v * v;
    }
  };
  int64_t k = r0 + p.row;
  for (; k + (U - 1) * p.step < r1; k += U * p.step) {
    Chunk<T, VE> x[U], r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (k + u * p.step) * a.s.B + p.col;
      x[u].load(a.X + at, p.n);
      if (a.R) r[u].load(a.R + at, p.n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) add(x[u], r[u]);
  }
  for (; k < r1; k += p.step) {
    Chunk<T, VE> x, r;
    x.load(a.X + k * a.s.B + p.col, p.n);
    if (a.R) r.load(a.R + k * a.s.B + p.col, p.n);
    add(x, r);
  }
}

template <typename T, int VE, int U, bool NT>
__device__ __forceinline__ void fwd_rows(const FwdArgs<T>& a, const Place<VE>& p, int64_t r0, int64_t r1,
                                         const float (&inv)[VE]) {
  if (p.n <= 0) return;
  auto put = [&](const Chunk<T, VE>& x, const Chunk<T, VE>& r, float g, int64_t at) {
    float v[VE], y[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      v[e] = a.R ? x.at(e) + r.at(e) : x.at(e);
      y[e] = g * (v[e] * inv[e]);
    }
    if (a.S) store_chunk<T, VE, NT>(a.S + at, v, p.n);
    store_chunk<T, VE, NT>(a.Y + at, y, p.n);
  };
  // from the last row to the first: the sums' pass has left the last ones in the L2
  int64_t left = rows_of(p, r0, r1);
  for (; left >= U; left -= U) {
    const int64_t k = r0 + p.row + (left - U) * p.step;
    Chunk<T, VE> x[U], r[U];
    float g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (k + u * p.step) * a.s.B + p.col;
      x[u].load(a.X + at, p.n);
      if (a.R) r[u].load(a.R + at, p.n);
      g[u] = a.gain ? a.gain[k + u * p.step] : 1.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) put(x[u], r[u], g[u], (k + u * p.step) * a.s.B + p.col);
  }
  for (; left > 0; --left) {
    const int64_t k = r0 + p.row + (left - 1) * p.step, at = k * a.s.B + p.col;
    Chunk<T, VE> x, r;
    x.load(a.X + at, p.n);
    if (a.R) r.load(a.R + at, p.n);
    put(x, r, a.gain ? a.gain[k] : 1.0f, at);
  }
}

// 1 / sqrt(mean + eps) of the block's columns from their sums of squares.
template <int VE>
__device__ __forceinline__ void inverse_roots(const NormShape& s, const Place<VE>& p, const double* sums,
                                              float (&inv)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e)
    inv[e] = static_cast<float>(1.0 / sqrt(sums[p.lane * VE + e] / s.K + static_cast<double>(s.eps)));
}

constexpr int kWhole = 1024;  // threads of a workgroup that takes every row
constexpr int kRange = 256;   // of one that takes a range

template <typename T, int VE>
__global__ void __launch_bounds__(kWhole) norm_fwd_whole_kernel(FwdArgs<T> a) {
  __shared__ double red[kWhole * VE];
  const int32_t block = column_block();
  if (block >= a.s.blocks) return;
  const Place<VE> p = place_of<VE>(a.s, block);
  double sum[VE];
  fwd_sums<T, VE, 4>(a, p, 0, a.s.K, sum);
  column_sums<VE, kWhole>(a.s, p, sum, red);
  float inv[VE];
  inverse_roots<VE>(a.s, p, red, inv);
  if (a.inv && p.row == 0) {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < p.n) a.inv[p.col + e] = inv[e];
  }
  fwd_rows<T, VE, 4, false>(a, p, 0, a.s.K, inv);
}

template <typename T, int VE>
__global__ void __launch_bounds__(kRange) norm_fwd_sums_kernel(FwdArgs<T> a) {
  __shared__ double red[kRange * VE];
  const int32_t block = blockIdx.x % a.s.blocks, range = blockIdx.x / a.s.blocks;
  const Place<VE> p = place_of<VE>(a.s, block);
  const int64_t r0 = static_cast<int64_t>(range) * a.s.rows;
  double sum[VE];
  fwd_sums<T, VE, 4>(a, p, r0, min<int64_t>(r0 + a.s.rows, a.s.K), sum);
  column_sums<VE, kRange>(a.s, p, sum, red);
  const int t = threadIdx.x;
  const int64_t col = static_cast<int64_t>(block) * a.s.lanes * VE + t;
  if (t < a.s.lanes * VE && col < a.s.B) a.part[static_cast<int64_t>(range) * a.s.B + col] = red[t];
}

// The sum of n values `step` apart, of the last index of which this thread's is `part` of
// `parts`: eight loads in flight, the threads' shares added in their order by the first of them.
// In 64 bits: a norm of heads has millions of blocks of columns, and a chain of equal ones in 32
// was up to 1.5e-3 off. red: parts x cols values of the workgroup; every thread of it calls.
template <typename V>
__device__ __forceinline__ double share_sum(const V* from, bool on, int n, int64_t step, int col, int cols, int part, int parts,
                                            double* red) {
  double v = 0.0;
  if (on && part < parts) {
#pragma unroll 8
    for (int q = part; q < n; q += parts) v += from[q * step];
  }
  if (part < parts) red[part * cols + col] = v;
  __syncthreads();
  if (part == 0)
    for (int u = 1; u < parts; ++u) v += red[u * cols + col];
  return v;
}

// The sums of the ranges of the block's columns.
__device__ __forceinline__ void join_ranges(const NormShape& s, const double* part, int32_t block, int cols, double* sums) {
  __shared__ double red[kRange];
  const int t = threadIdx.x, c = t % cols;
  const int64_t col = static_cast<int64_t>(block) * cols + c;
  const double v = share_sum(part + col, col < s.B, s.ranges, s.B, c, cols, t / cols, kRange / cols, red);
  if (t < cols) sums[t] = v;
  __syncthreads();
}

template <typename T, int VE>
__global__ void __launch_bounds__(kRange) norm_fwd_rows_kernel(FwdArgs<T> a) {
  __shared__ double sums[64];
  const int32_t block = blockIdx.x % a.s.blocks, range = blockIdx.x / a.s.blocks;
  const Place<VE> p = place_of<VE>(a.s, block);
  join_ranges(a.s, a.part, block, a.s.lanes * VE, sums);
  float inv[VE];
  inverse_roots<VE>(a.s, p, sums, inv);
  if (a.inv && range == 0 && p.row == 0) {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < p.n) a.inv[p.col + e] = inv[e];
  }
  const int64_t r0 = static_cast<int64_t>(range) * a.s.rows;
  fwd_rows<T, VE, 4, true>(a, p, r0, min<int64_t>(r0 + a.s.rows, a.s.K), inv);
}

// ------------------------------------------------------------------ backward
template <typename T>
struct BwdArgs {
  NormShape s;
  const T* S;
  const float* gain;
  const float* inv;
  const T* dY;
  const T* dS;
  T* dX;
  float* dgain;
  double* part;  // [ranges][B] sums of u xh
  float* gpart;  // [blocks][K] sums of dY xh over a block's columns
};

// The sums of u xh down the columns and, if asked, of dY xh along the rows of the block
// (row_out[k]). A row's threads are neighbours of one wave where lanes is a power of two.
template <typename T, int VE, int U>
__device__ __forceinline__ void bwd_sums(const BwdArgs<T>& a, const Place<VE>& p, int64_t r0, int64_t r1,
                                         const float (&inv)[VE], float* row_out, double (&sum)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) sum[e] = 0.0;
  const int lanes = a.s.lanes;
  auto add = [&](const Chunk<T, VE>& x, const Chunk<T, VE>& d, float g, int64_t k, bool on) {
    float along = 0.0f;
    if (on) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float w = d.at(e) * (x.at(e) * inv[e]);
        if (e < p.n) along += w;
        sum[e] += static_cast<double>(g) * w;
      }
    }
    if (row_out) {  // uniform
      along = row_sum(along, lanes);
      if (p.lane == 0 && on) row_out[k] = along;
    }
  };
  for (int64_t k0 = r0; k0 < r1; k0 += U * p.step) {
    Chunk<T, VE> x[U], d[U];
    float g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + p.row + u * p.step;
      x[u] = Chunk<T, VE>{};
      d[u] = Chunk<T, VE>{};
      g[u] = 0.0f;
      if (k < r1 && p.n > 0) {
        x[u].load(a.S + k * a.s.B + p.col, p.n);
        d[u].load(a.dY + k * a.s.B + p.col, p.n);
        g[u] = a.gain ? a.gain[k] : 1.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = k0 + p.row + u * p.step;
      add(x[u], d[u], g[u], k, k < r1);
    }
  }
}

template <typename T, int VE, int U, bool NT>
__device__ __forceinline__ void bwd_rows(const BwdArgs<T>& a, const Place<VE>& p, int64_t r0, int64_t r1,
                                         const float (&inv)[VE], const float (&mean)[VE]) {
  if (p.n <= 0) return;
  auto put = [&](const Chunk<T, VE>& x, const Chunk<T, VE>& d, const Chunk<T, VE>& r, float g, int64_t at) {
    float v[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      v[e] = inv[e] * (g * d.at(e) - (x.at(e) * inv[e]) * mean[e]);
      if (a.dS) v[e] += r.at(e);
    }
    store_chunk<T, VE, NT>(a.dX + at, v, p.n);
  };
  int64_t left = rows_of(p, r0, r1);  // as in fwd_rows
  for (; left >= U; left -= U) {
    const int64_t k = r0 + p.row + (left - U) * p.step;
    Chunk<T, VE> x[U], d[U], r[U];
    float g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (k + u * p.step) * a.s.B + p.col;
      x[u].load(a.S + at, p.n);
      d[u].load(a.dY + at, p.n);
      if (a.dS) r[u].load(a.dS + at, p.n);
      g[u] = a.gain ? a.gain[k + u * p.step] : 1.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) put(x[u], d[u], r[u], g[u], (k + u * p.step) * a.s.B + p.col);
  }
  for (; left > 0; --left) {
    const int64_t k = r0 + p.row + (left - 1) * p.step, at = k * a.s.B + p.col;
    Chunk<T, VE> x, d, r;
    x.load(a.S + at, p.n);
    d.load(a.dY + at, p.n);
    if (a.dS) r.load(a.dS + at, p.n);
    put(x, d, r, a.gain ? a.gain[k] : 1.0f, at);
  }
}

template <int VE>
__device__ __forceinline__ void load_inv(const float* inv, const Place<VE>& p, float (&v)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = e < p.n ? inv[p.col + e] : 0.0f;
}
template <int VE>
__device__ __forceinline__ void means(const NormShape& s, const Place<VE>& p, const double* sums, float (&mean)[VE]) {
#pragma unroll
  for (int e = 0; e < VE; ++e) mean[e] = static_cast<float>(sums[p.lane * VE + e] / s.K);
}

template <typename T, int VE>
__global__ void __launch_bounds__(kWhole) norm_bwd_whole_kernel(BwdArgs<T> a) {
  __shared__ double red[kWhole * VE];
  const int32_t block = column_block();
  if (block >= a.s.blocks) return;
  const Place<VE> p = place_of<VE>(a.s, block);
  float inv[VE], mean[VE];
  load_inv<VE>(a.inv, p, inv);
  double sum[VE];
  float* rows = a.dgain ? (a.gpart ? a.gpart + static_cast<int64_t>(block) * a.s.K : a.dgain) : nullptr;
  bwd_sums<T, VE, 2>(a, p, 0, a.s.K, inv, rows, sum);
  column_sums<VE, kWhole>(a.s, p, sum, red);
  means<VE>(a.s, p, red, mean);
  if (a.dX) bwd_rows<T, VE, 2, false>(a, p, 0, a.s.K, inv, mean);
}

template <typename T, int VE>
__global__ void __launch_bounds__(kRange) norm_bwd_sums_kernel(BwdArgs<T> a) {
  __shared__ double red[kRange * VE];
  const int32_t block = blockIdx.x % a.s.blocks, range = blockIdx.x / a.s.blocks;
  const Place<VE> p = place_of<VE>(a.s, block);
  const int64_t r0 = static_cast<int64_t>(range) * a.s.rows;
  float inv[VE];
  load_inv<VE>(a.inv, p, inv);
  double sum[VE];
  float* rows = a.dgain ? (a.gpart ? a.gpart + static_cast<int64_t>(block) * a.s.K : a.dgain) : nullptr;
  bwd_sums<T, VE, 4>(a, p, r0, min<int64_t>(r0 + a.s.rows, a.s.K), inv, rows, sum);
  column_sums<VE, kRange>(a.s, p, sum, red);
  const int t = threadIdx.x;
  const int64_t col = static_cast<int64_t>(block) * a.s.lanes * VE + t;
  if (t < a.s.lanes * VE && col < a.s.B) a.part[static_cast<int64_t>(range) * a.s.B + col] = red[t];
}

// dgain of 64 features from the blocks' sums (fp32 960 x 6111, 96 blocks, backward: 62 us with
// a thread for a feature, 48).
constexpr int kGain = 64;
template <typename T>
__device__ __forceinline__ void join_gain(const BwdArgs<T>& a, int64_t group) {
  __shared__ double red[kRange];
  const int t = threadIdx.x, c = t % kGain;
  const int64_t k = group * kGain + c;
  const double v = share_sum(a.gpart + k, k < a.s.K, a.s.blocks, a.s.K, c, kGain, t / kGain, kRange / kGain, red);
  if (t < kGain && k < a.s.K) a.dgain[k] = static_cast<float>(v);
}

// The workgroups behind those of the rows join dgain.
template <typename T, int VE>
__global__ void __launch_bounds__(kRange) norm_bwd_rows_kernel(BwdArgs<T> a, int32_t groups) {
  __shared__ double sums[64];
  if (static_cast<int32_t>(blockIdx.x) >= groups) {
    join_gain(a, static_cast<int64_t>(blockIdx.x) - groups);
    return;
  }
  const int32_t block = blockIdx.x % a.s.blocks, range = blockIdx.x / a.s.blocks;
  const Place<VE> p = place_of<VE>(a.s, block);
  join_ranges(a.s, a.part, block, a.s.lanes * VE, sums);
  float inv[VE], mean[VE];
  load_inv<VE>(a.inv, p, inv);
  means<VE>(a.s, p, sums, mean);
  const int64_t r0 = static_cast<int64_t>(range) * a.s.rows;
  bwd_rows<T, VE, 4, true>(a, p, r0, min<int64_t>(r0 + a.s.rows, a.s.K), inv, mean);
}

template <typename T>
__global__ void __launch_bounds__(kRange) norm_gain_kernel(BwdArgs<T> a) {
  join_gain(a, blockIdx.x);
}

// ------------------------------------------------------------------ host
struct NormPlan {
  NormShape s;
  bool vec;    // 16 bytes of a row a thread, else one element
  bool whole;  // one workgroup takes every row of its columns
};

int plan_norm(const ard_rmsnorm_desc* d, NormPlan* p) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->batch < 1 || d->features < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (batch %d, features %d)", d->batch, d->features);
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return fail(ARD_ERR_INVALID_ARG, "eps must be finite and >= 0");
  const int ve = d->dtype == ARD_BF16 ? 8 : 4;
  NormShape& s = p->s;
  s.B = d->batch;
  s.K = d->features;
  s.eps = d->eps;
  p->vec = s.B >= ve;
  // 64 columns of a block; a power of two of threads on a row, so that a wave holds whole rows
  const int per = p->vec ? ve : 1, most = 64 / per;
  s.lanes = 1;
  while (s.lanes < most && s.lanes * per < s.B) s.lanes *= 2;
  s.blocks = static_cast<int32_t>((static_cast<int64_t>(s.B) + s.lanes * per - 1) / (s.lanes * per));
  const int64_t bytes = static_cast<int64_t>(s.K) * std::min<int64_t>(s.B, 64) * (d->dtype == ARD_BF16 ? 2 : 4);
  // Measured on MI355X, forward, up to 128 and 32 KB of a block in one workgroup: bf16 4544 x 9 36.6, 18.5 us, 1024 x 64
  // 15.5, 9.8, fp32 126 x 1632 7.2, 7.1; ranges of at least four and two rows of a thread: bf16 4544 x 9 18.5, 10.9, 631 x
  // 433 18.7, 11.6, 8192 x 2048 35.3, 34.9.
  // More than 32704 columns always go to one workgroup a block: one launch whose threads stay below 2^32 whatever the
  // batch. Against ranges, forward and backward: fp32 256 x 262144 256, 339 us, ranges 316, 368; 1024 x 65536 279, 292 and
  // 299, 311; 1024 x 32768 151, 151 and 132, 146; bf16 512 x 131072 170, 201 and 157, 202; 1024 x 65536 168, 179 and 144,
  // 172; 512 x 32768 42.0, 49.0 and 36.4, 44.2: fp32 0.81 to 1.14 times ranges' time, bf16 0.98 to 1.17.
  p->whole = bytes <= 32 << 10 || s.blocks >= 2 * kTargetBlocks;
  s.ranges = 1;
  s.rows = s.K;
  if (!p->whole) {
    const int64_t step = kRange / s.lanes;
    const int64_t most_ranges = (s.K + 2 * step - 1) / (2 * step), want = (4 * kTargetBlocks + s.blocks - 1) / s.blocks;
    s.ranges = static_cast<int32_t>(std::max<int64_t>(1, std::min(most_ranges, want)));
    const int64_t rows = s.K;
    s.rows = static_cast<int32_t>((rows + s.ranges - 1) / s.ranges);
    s.ranges = static_cast<int32_t>((rows + s.rows - 1) / s.rows);
  }
  return ARD_OK;
}

struct NormSpace {
  size_t part, gain;
};
NormSpace norm_space(const NormPlan& p) {
  return {p.whole ? 0 : al256(static_cast<size_t>(p.s.ranges) * p.s.B * 8),
          p.s.blocks > 1 ? al256(static_cast<size_t>(p.s.blocks) * p.s.K * 4) : 0};
}

template <typename T, int VE>
int run_fwd(const NormPlan& p, const FwdArgs<T>& a, hipStream_t stream) {
  if (p.whole) {
    hipLaunchKernelGGL((norm_fwd_whole_kernel<T, VE>), block_grid(p.s.blocks), dim3(kWhole), 0, stream, a);
  } else {
    const dim3 grid(static_cast<unsigned>(p.s.blocks) * p.s.ranges);
    hipLaunchKernelGGL((norm_fwd_sums_kernel<T, VE>), grid, dim3(kRange), 0, stream, a);
    ARD_LAUNCH_CHECK();
    hipLaunchKernelGGL((norm_fwd_rows_kernel<T, VE>), grid, dim3(kRange), 0, stream, a);
  }
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T>
int fwd_impl(const NormPlan& p, const void* X, const void* R, const float* gain, void* S, void* Y, float* inv, char* ws,
             hipStream_t stream) {
  const FwdArgs<T> a{p.s, static_cast<const T*>(X), static_cast<const T*>(R), gain, static_cast<T*>(S),
                     static_cast<T*>(Y), inv, reinterpret_cast<double*>(ws)};
  return p.vec ? run_fwd<T, 16 / sizeof(T)>(p, a, stream) : run_fwd<T, 1>(p, a, stream);
}

// Workgroups that join dgain from several blocks of columns.
int64_t join_groups(const NormPlan& p) { return p.s.blocks > 1 ? (static_cast<int64_t>(p.s.K) + kGain - 1) / kGain : 0; }

template <typename T, int VE>
int run_bwd(const NormPlan& p, const BwdArgs<T>& a, hipStream_t stream) {
  const unsigned join = a.dgain ? static_cast<unsigned>(join_groups(p)) : 0;
  if (p.whole) {
    hipLaunchKernelGGL((norm_bwd_whole_kernel<T, VE>), block_grid(p.s.blocks), dim3(kWhole), 0, stream, a);
    ARD_LAUNCH_CHECK();
    if (join) hipLaunchKernelGGL(norm_gain_kernel<T>, dim3(join), dim3(kRange), 0, stream, a);
  } else {
    const unsigned grid = static_cast<unsigned>(p.s.blocks) * p.s.ranges, rows = a.dX ? grid : 0;
    hipLaunchKernelGGL((norm_bwd_sums_kernel<T, VE>), dim3(grid), dim3(kRange), 0, stream, a);
    ARD_LAUNCH_CHECK();
    if (rows + join)
      hipLaunchKernelGGL((norm_bwd_rows_kernel<T, VE>), dim3(rows + join), dim3(kRange), 0, stream, a,
                         static_cast<int32_t>(rows));
  }
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T>
int bwd_impl(const NormPlan& p, const void* S, const float* gain, const float* inv, const void* dY, const void* dS,
             void* dX, float* dgain, char* ws, hipStream_t stream) {
  const NormSpace sp = norm_space(p);
  const BwdArgs<T> a{p.s, static_cast<const T*>(S), gain, inv, static_cast<const T*>(dY), static_cast<const T*>(dS),
                     static_cast<T*>(dX), dgain, reinterpret_cast<double*>(ws),
                     sp.gain ? reinterpret_cast<float*>(ws + sp.part) : nullptr};
  return p.vec ? run_bwd<T, 16 / sizeof(T)>(p, a, stream) : run_bwd<T, 1>(p, a, stream);
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

size_t ard_rmsnorm_workspace_bytes(const ard_rmsnorm_desc* desc) {
  NormPlan p;
  if (plan_norm(desc, &p) != ARD_OK) return 0;
  const NormSpace sp = norm_space(p);
  return sp.part + sp.gain;
}

int ard_rmsnorm_fwd(const ard_rmsnorm_desc* desc, const void* Xt, const void* Rt, const float* gain, void* St, void* Yt,
                    float* inv_rms, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  NormPlan p;
  int st = plan_norm(desc, &p);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Xt, "Xt")) || (st = may_ptr(Rt, "Rt")) || (st = may_ptr(gain, "gain")) || (st = may_ptr(St, "St")) ||
      (st = need_ptr(Yt, "Yt")) || (st = may_ptr(inv_rms, "inv_rms")) ||
      (st = check_space(norm_space(p).part, ws, ws_bytes)))
    return st;
  if (St == Yt) return fail(ARD_ERR_INVALID_ARG, "St and Yt are the same buffer");
  // written by one workgroup while others read what they normalise and the gain
  if (same_buffer(inv_rms, {Xt, Rt, gain, St, Yt}))
    return fail(ARD_ERR_INVALID_ARG, "inv_rms is in the buffer of another argument");
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? fwd_impl<bf16>(p, Xt, Rt, gain, St, Yt, inv_rms, w, sm)
                                 : fwd_impl<float>(p, Xt, Rt, gain, St, Yt, inv_rms, w, sm);
}

int ard_rmsnorm_bwd(const ard_rmsnorm_desc* desc, const void* St, const float* gain, const float* inv_rms,
                    const void* dYt, const void* dSt, void* dXt, float* dgain, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  NormPlan p;
  int st = plan_norm(desc, &p);
  if (st != ARD_OK) return st;
  const NormSpace sp = norm_space(p);
  if ((st = need_ptr(St, "St")) || (st = may_ptr(gain, "gain")) || (st = need_ptr(inv_rms, "inv_rms")) ||
      (st = need_ptr(dYt, "dYt")) || (st = may_ptr(dSt, "dSt")) || (st = may_ptr(dXt, "dXt")) ||
      (st = may_ptr(dgain, "dgain")) || (st = check_space(sp.part + sp.gain, ws, ws_bytes)))
    return st;
  // the threads of a launch stay below 2^32
  if (dgain && (join_groups(p) + (p.whole ? 0 : static_cast<int64_t>(p.s.blocks) * p.s.ranges)) * kRange >= int64_t{1} << 32)
    return fail(ARD_ERR_UNSUPPORTED, "dgain of %d features in %d columns: too many features", p.s.K, p.s.B);
  // written by the sums' pass, in front of the one that reads the other arrays again
  if (same_buffer(dgain, {St, gain, inv_rms, dYt, dSt, dXt}))
    return fail(ARD_ERR_INVALID_ARG, "dgain is in the buffer of another argument");
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? bwd_impl<bf16>(p, St, gain, inv_rms, dYt, dSt, dXt, dgain, w, sm)
                                 : bwd_impl<float>(p, St, gain, inv_rms, dYt, dSt, dXt, dgain, w, sm);
}

}  // extern "C"
