// Distillation from a teacher's top logits, forward and backward, on
// feature-major logits Zt[V][B] (as ard_fc_fwd leaves them).
//
// Per column, with T the temperature and a the weight of the soft term:
//   p_j  = softmax over the column's valid teacher entries of t_j / T
//   q(T) = softmax over all V classes of z / T
//   loss = a T^2 sum_j p_j (log p_j - log q(T)[idx_j]) - (1 - a) log q(1)[label]
//   dZ   = dloss (a T (q(T) - p scattered to its classes) + (1 - a) (q(1) - onehot))
//
// Forward: one pass over the logits. A thread owns 16 bytes of neighbouring
// columns and walks down its rows with a running maximum and two running sums
// (one at temperature 1, one at T; T = 1 needs one); the row ranges of a column
// meet in LDS and, across workgroups, in the workspace, added in a fixed order.
// A second, small kernel joins them and does the teacher's entries, of which a
// column has few. Backward: the dense part of the gradient in one pass from the
// saved maximum and sums, then the few entries that a teacher's or a label's
// class touches once more, each with its whole value, so that nothing is rounded
// twice and no order of additions is left to chance.
//
// Bound by reading the logits (and writing the gradient).

#include <hip/hip_runtime.h>

#include <cmath>

#include "../ard_gemm_fast.hpp"
#include "../ard_internal.hpp"

namespace ard {
namespace {

// exp of a value <= 0. bf16 logits: the hardware's power of two; its argument's
// rounding costs at most 2^-24 |x| of relative error, which is far below what
// the logits themselves are rounded by. fp32 logits: the library function.
template <typename T>
__device__ __forceinline__ float exp_neg(float x) {
  if constexpr (sizeof(T) == 2)
    return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
  else
    return expf(x);
}

// VE consecutive columns of a row as loaded, and as fp32. Rows start at any element.
template <typename T, int VE>
struct Cols {
  typename std::conditional<VE == 1, T, u32x4>::type raw;
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VE == 1) raw = *p;
    else raw = load16_any<sizeof(T)>(reinterpret_cast<const char*>(p));
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (VE == 1)
      return to_f32(raw);
    else if constexpr (sizeof(T) == 2)
      return __uint_as_float((e & 1) ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
    else
      return __uint_as_float(raw[e]);
  }
};
template <typename T, int VE>
__device__ __forceinline__ void store_cols(T* p, const float (&v)[VE]) {
  if constexpr (VE == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    typedef u32x4 u32x4_a2 __attribute__((aligned(2), may_alias));
    T w[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) w[e] = from_f32<T>(v[e]);
    *reinterpret_cast<u32x4_a2*>(p) = *reinterpret_cast<const u32x4*>(w);
  }
}

// Launches of a workgroup for each group of columns, y such rows of workgroups: the groups
// in layers of 2^20 along z, since the threads along x have to stay below 2^32.
constexpr int32_t kGridRow = 1 << 20;
dim3 column_grid(int32_t groups, int32_t y) {
  return dim3(groups < kGridRow ? groups : kGridRow, y, (groups - 1) / kGridRow + 1);
}
__device__ __forceinline__ int64_t column_group() { return static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x; }

// How a launch lays its threads over the logits: tx threads side by side along
// a row (a power of two), 256 / tx rows at a time, `splits` ranges of rows.
struct Grid {
  int32_t tx, blocks, splits;
  int64_t rows;  // rows of a range
};

struct Columns {
  int64_t col;  // first column of the thread
  bool on;
};

// The thread's columns: chunk after chunk of VE, the last one moved back to end
// at the last column (its columns are then computed twice, alike).
template <int VE>
__device__ __forceinline__ Columns columns_of(int32_t B, int32_t tx) {
  const int64_t c = (column_group() * tx + (threadIdx.x & (tx - 1))) * VE;
  return {c + VE <= B ? c : static_cast<int64_t>(B) - VE, c < B};
}

// A running maximum m and the sums of exp(z - m) and exp((z - m) / T).
struct Run {
  float m, s1, sT;
};

// The reference of a maximum: 0 where there is no finite logit yet, so that
// exp(-inf - ref) is 0 and not NaN.
__device__ __forceinline__ float ref_of(float m) { return m == -__builtin_inff() ? 0.0f : m; }

template <typename T, bool TWO>
__device__ __forceinline__ void join(Run& a, const Run& b, float inv_t) {
  const float m = fmaxf(a.m, b.m), r = ref_of(m);
  a.s1 = a.s1 * exp_neg<T>(a.m - r) + b.s1 * exp_neg<T>(b.m - r);
  if constexpr (TWO) a.sT = a.sT * exp_neg<T>((a.m - r) * inv_t) + b.sT * exp_neg<T>((b.m - r) * inv_t);
  a.m = m;
}

// What the teacher's entries and the label add to a column's sums: its loss and the
// values kept for the backward. NY threads for each of NX columns (neighbouring
// threads neighbouring columns), `a` the column's joined sums; entries four at a time,
// so that their loads run together.
template <typename T, bool TWO>
__device__ __forceinline__ void finish_column(Run a, int64_t col, bool on, int tx, int ty, int NX, int NY,
                                              const T* __restrict__ Z, int32_t V, int32_t B, int32_t top,
                                              const int32_t* __restrict__ idx, const float* __restrict__ tl,
                                              const int32_t* __restrict__ labels, float temp, float weight,
                                              float* __restrict__ loss, float* __restrict__ stats, float* red) {
  constexpr int U = 4;
  const float inv_t = 1.0f / temp;
  if (!TWO) a.sT = a.s1;
  const float ref = ref_of(a.m);
  const bool read = on && weight > 0.0f;
  // the teacher's maximum over the valid entries
  float tm = -__builtin_inff();
  if (read)
    for (int64_t j = ty; j < top; j += U * NY) {
      int32_t v[U];
      float t[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t q = j + u * NY < top ? j + u * NY : j;
        v[u] = idx[q * B + col], t[u] = tl[q * B + col];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v[u] >= 0 && v[u] < V) tm = fmaxf(tm, t[u]);
    }
  red[ty * NX + tx] = tm;
  __syncthreads();
  for (int y = 0; y < NY; ++y) tm = fmaxf(tm, red[y * NX + tx]);
  __syncthreads();
  const float tref = ref_of(tm);
  // sums of e_j = exp((t_j - tm) / T) and of e_j ((t_j - tm) - (z_j - m)) / T
  float es = 0.0f, ds = 0.0f;
  if (read)
    for (int64_t j = ty; j < top; j += U * NY) {
      int32_t v[U];
      float t[U], z[U];
      bool ok[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t q = j + u * NY < top ? j + u * NY : j;
        v[u] = idx[q * B + col], t[u] = tl[q * B + col];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ok[u] = v[u] >= 0 && v[u] < V && j + u * NY < top;
        z[u] = to_f32(Z[static_cast<int64_t>(ok[u] ? v[u] : 0) * B + col]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float x = (t[u] - tref) * inv_t, e = ok[u] ? expf(x) : 0.0f;
        es += e;
        if (!(e == 0.0f)) ds += e * (x - (z[u] - ref) * inv_t);
      }
    }
  red[ty * NX + tx] = es;
  __syncthreads();
  es = 0.0f;
  for (int y = 0; y < NY; ++y) es += red[y * NX + tx];
  __syncthreads();
  red[ty * NX + tx] = ds;
  __syncthreads();
  if (ty != 0 || !on) return;
  ds = 0.0f;
  for (int y = 0; y < NY; ++y) ds += red[y * NX + tx];
  float out = 0.0f;
  // a column without a logit above -inf has s1 = 0 and no loss
  if (weight > 0.0f && !(es == 0.0f) && !(a.sT == 0.0f)) out += weight * temp * temp * (ds / es + logf(a.sT / es));
  const int32_t label = labels ? labels[col] : -1;
  if (weight < 1.0f && label >= 0 && label < V && !(a.s1 == 0.0f))
    out += (1.0f - weight) * (logf(a.s1) - (to_f32(Z[static_cast<int64_t>(label) * B + col]) - ref));
  loss[col] = out;
  const int64_t b = B;
  stats[col] = ref;
  stats[b + col] = a.s1;
  stats[2 * b + col] = a.sT;
  stats[3 * b + col] = tref;
  stats[4 * b + col] = es;
}

// The running sums of a range of rows; ONE: of all rows, and with them the loss. Bound by
// reading the logits: 32000 x 4096 bf16 (262 MB) 75 us, 3.5 TB/s; large reductions read at
// 4.0 to 4.5 TB/s here. Without its exponentials the kernel took 71 us; eight rows in
// flight, more workgroups or another order of them changed nothing.
template <typename T, int VE, bool TWO, bool ONE>
__global__ void __launch_bounds__(256) distill_sums_kernel(const T* __restrict__ Z, int32_t V, int32_t B, Grid g,
                                                           int32_t top, const int32_t* __restrict__ idx,
                                                           const float* __restrict__ tl,
                                                           const int32_t* __restrict__ labels, float temp,
                                                           float weight, float* __restrict__ part,
                                                           float* __restrict__ loss, float* __restrict__ stats) {
  constexpr int U = 4;  // rows in flight
  const float inv_t = 1.0f / temp;
  const Columns c = columns_of<VE>(B, g.tx);
  const int tx = threadIdx.x & (g.tx - 1), ty = threadIdx.x / g.tx, ny = 256 / g.tx;
  const int64_t r0 = blockIdx.y * g.rows;
  const int64_t r1 = r0 + g.rows < V ? r0 + g.rows : V;
  Run run[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) run[e] = {-__builtin_inff(), 0.0f, 0.0f};
  if (c.on) {
    const T* z = Z + c.col;
    auto take = [&](const Cols<T, VE>(&x)[U], int n) {  // n of the U rows
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        float m = run[e].m;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u < n) m = fmaxf(m, x[u].at(e));
        const float r = ref_of(m), old = run[e].m - r;
        float s1 = run[e].s1 * exp_neg<T>(old), sT = TWO ? run[e].sT * exp_neg<T>(old * inv_t) : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u < n) {
            s1 += exp_neg<T>(x[u].at(e) - r);
            if constexpr (TWO) sT += exp_neg<T>((x[u].at(e) - r) * inv_t);
          }
        }
        run[e] = {m, s1, sT};
      }
    };
    // the next rows are on their way while these are added
    const int64_t step = static_cast<int64_t>(U) * ny;
    Cols<T, VE> x[2][U];
    auto load = [&](int64_t r, Cols<T, VE>(&to)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) to[u].load(z + (r + static_cast<int64_t>(u) * ny) * B);
    };
    int64_t r = r0 + ty;
    const int64_t whole = r1 - (U - 1) * static_cast<int64_t>(ny);  // first rows below it have all U
    if (r < whole) load(r, x[0]);
    for (; r < whole; r += 2 * step) {
      if (r + step < whole) load(r + step, x[1]);
      take(x[0], U);
      if (r + step >= whole) {
        r += step;
        break;
      }
      if (r + 2 * step < whole) load(r + 2 * step, x[0]);
      take(x[1], U);
    }
    for (; r < r1; r += ny) {
      x[0][0].load(z + r * B);
      take(x[0], 1);
    }
  }
  // the rows' threads of a column, halved step by step
  __shared__ Run red[256];
  __shared__ float fin[256];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    __syncthreads();
    red[threadIdx.x] = run[e];
    for (int h = ny / 2; h > 0; h >>= 1) {
      __syncthreads();
      if (ty < h) join<T, TWO>(red[threadIdx.x], red[threadIdx.x + h * g.tx], inv_t);
    }
    if constexpr (ONE) {
      __syncthreads();
      finish_column<T, TWO>(red[tx], c.col + e, c.on, tx, ty, g.tx, ny, Z, V, B, top, idx, tl, labels, temp, weight,
                            loss, stats, fin);
    } else if (ty == 0 && c.on) {
      float* p = part + static_cast<int64_t>(blockIdx.y) * 3 * B + c.col + e;
      const Run& s = red[threadIdx.x];
      p[0] = s.m;
      p[B] = s.s1;
      p[2 * static_cast<int64_t>(B)] = TWO ? s.sT : s.s1;
    }
  }
}

// Joins a column's ranges, then the teacher's entries and the label: 16 columns
// of a workgroup, sixteen threads each. Bound by the latency of entry, then logit: 64
// entries of 4096 columns 10 us.
template <typename T, bool TWO>
__global__ void __launch_bounds__(256) distill_loss_kernel(const T* __restrict__ Z, int32_t V, int32_t B, int32_t top,
                                                           const int32_t* __restrict__ idx,
                                                           const float* __restrict__ tl,
                                                           const int32_t* __restrict__ labels, float temp,
                                                           float weight, int32_t splits,
                                                           const float* __restrict__ part, float* __restrict__ loss,
                                                           float* __restrict__ stats) {
  constexpr int NX = 16, NY = 16, U = 4;
  __shared__ Run red[256];
  __shared__ float fin[256];
  const int tx = threadIdx.x % NX, ty = threadIdx.x / NX;
  const int64_t col = column_group() * NX + tx;
  const bool on = col < B;
  const float inv_t = 1.0f / temp;
  Run a = {-__builtin_inff(), 0.0f, 0.0f};
  if (on) {
    for (int s = ty; s < splits; s += U * NY) {
      Run b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float* p = part + static_cast<int64_t>(s + u * NY < splits ? s + u * NY : s) * 3 * B + col;
        b[u] = {p[0], p[B], TWO ? p[2 * static_cast<int64_t>(B)] : 0.0f};
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s + u * NY < splits) join<T, TWO>(a, b[u], inv_t);
    }
  }
  red[threadIdx.x] = a;
  for (int h = NY / 2; h > 0; h >>= 1) {
    __syncthreads();
    if (ty < h) join<T, TWO>(red[threadIdx.x], red[threadIdx.x + h * NX], inv_t);
  }
  __syncthreads();
  finish_column<T, TWO>(red[tx], col, on, tx, ty, NX, NY, Z, V, B, top, idx, tl, labels, temp, weight, loss, stats, fin);
}

// A column's factors of the gradient: dz = fT exp((z - m) / T) + f1 exp(z - m),
// less cs p_j at the teacher's classes and ch at the label.
struct Factors {
  float m, fT, f1, cs, ch;
};
__device__ __forceinline__ Factors factors_of(int64_t col, int32_t V, int32_t B, const float* stats,
                                              const int32_t* labels, const float* dloss, float temp, float weight) {
  const int64_t b = B;
  const float s1 = stats[b + col], sT = stats[2 * b + col], es = stats[4 * b + col];
  const float dl = dloss ? dloss[col] : 1.0f;
  const int32_t label = labels ? labels[col] : -1;
  const bool soft = weight > 0.0f && !(es == 0.0f) && !(sT == 0.0f);
  const bool hard = weight < 1.0f && label >= 0 && label < V && !(s1 == 0.0f);
  Factors f;
  f.m = stats[col];
  f.cs = soft ? dl * weight * temp : 0.0f;
  f.ch = hard ? dl * (1.0f - weight) : 0.0f;
  f.fT = soft ? f.cs / sT : 0.0f;
  f.f1 = hard ? f.ch / s1 : 0.0f;
  return f;
}

template <typename T, bool TWO>
__device__ __forceinline__ float dense_grad(float z, float m, float fT, float f1, float inv_t) {
  const float x = z - m;
  if constexpr (TWO) {
    float g = 0.0f;
    if (!(fT == 0.0f)) g += fT * exp_neg<T>(x * inv_t);
    if (!(f1 == 0.0f)) g += f1 * exp_neg<T>(x);
    return g;
  } else {
    const float f = fT + f1;
    return f == 0.0f ? 0.0f : f * exp_neg<T>(x);
  }
}

// An entry at a teacher's class or the label, written whole (entry `top` is the
// label). A class that several entries name gets every one's share from each of
// their threads, the same value in the same order.
template <typename T, bool TWO>
__device__ __forceinline__ void sparse_entry(int64_t j, int64_t col, const Factors& f, const T* __restrict__ Z,
                                             int32_t V, int32_t B, int32_t top, const int32_t* __restrict__ idx,
                                             const float* __restrict__ tl, int32_t label, float tref, float es,
                                             float inv_t, T* dZ) {
  const int32_t v = j < top ? idx[j * B + col] : label;
  if (v < 0 || v >= V) return;
  const int64_t at = static_cast<int64_t>(v) * B + col;
  const float z = to_f32(Z[at]);
  float p = 0.0f;
  if (!(f.cs == 0.0f)) {
    constexpr int U = 8;  // entries in flight
    for (int64_t i = 0; i < top; i += U) {
      int32_t w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = idx[(i + u < top ? i + u : i) * B + col];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (w[u] == v && i + u < top) p += expf((tl[(i + u) * B + col] - tref) * inv_t);
    }
  }
  float g = dense_grad<T, TWO>(z, f.m, f.fT, f.f1, inv_t);
  if (!(f.cs == 0.0f)) g -= f.cs * (p / es);
  if (v == label) g -= f.ch;
  dZ[at] = from_f32<T>(g);
}

// The dense part of a range of rows; ONE: of all rows, and the entries after it. Bound by
// reading the logits and writing as much: 32000 x 4096 bf16 (524 MB) 93 us, 5.6 TB/s,
// which is what a copy reaches.
template <typename T, int VE, bool TWO, bool ONE>
__global__ void __launch_bounds__(256) distill_dense_kernel(const T* __restrict__ Z, int32_t V, int32_t B, Grid g,
                                                            int32_t top, const int32_t* __restrict__ idx,
                                                            const float* __restrict__ tl,
                                                            const int32_t* __restrict__ labels,
                                                            const float* __restrict__ stats,
                                                            const float* __restrict__ dloss, float temp, float weight,
                                                            T* dZ) {
  constexpr int U = 4;
  const Columns c = columns_of<VE>(B, g.tx);
  const int ty = threadIdx.x / g.tx, ny = 256 / g.tx;
  const float inv_t = 1.0f / temp;
  if (c.on) {
    float m[VE], fT[VE], f1[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const Factors f = factors_of(c.col + e, V, B, stats, labels, dloss, temp, weight);
      m[e] = f.m, fT[e] = f.fT, f1[e] = f.f1;
    }
    const int64_t r0 = blockIdx.y * g.rows;
    const int64_t r1 = r0 + g.rows < V ? r0 + g.rows : V;
    auto put = [&](int64_t r, const Cols<T, VE>& x) {
      float d[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) d[e] = dense_grad<T, TWO>(x.at(e), m[e], fT[e], f1[e], inv_t);
      store_cols<T, VE>(dZ + r * B + c.col, d);
    };
    int64_t r = r0 + ty;
    for (; r + static_cast<int64_t>(U - 1) * ny < r1; r += static_cast<int64_t>(U) * ny) {
      Cols<T, VE> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u].load(Z + (r + static_cast<int64_t>(u) * ny) * B + c.col);
#pragma unroll
      for (int u = 0; u < U; ++u) put(r + static_cast<int64_t>(u) * ny, x[u]);
    }
    for (; r < r1; r += ny) {
      Cols<T, VE> x;
      x.load(Z + r * B + c.col);
      put(r, x);
    }
  }
  if constexpr (ONE) {
    __syncthreads();  // waits for the stores above
    for (int e = 0; e < VE && c.on; ++e) {
      const int64_t col = c.col + e, b = B;
      const Factors f = factors_of(col, V, B, stats, labels, dloss, temp, weight);
      for (int64_t j = ty; j <= top; j += ny)
        sparse_entry<T, TWO>(j, col, f, Z, V, B, top, idx, tl, labels ? labels[col] : -1, stats[3 * b + col],
                             stats[4 * b + col], inv_t, dZ);
    }
  }
}

// The entries after a dense launch: 16 columns of a workgroup, 16 threads of each, OWN
// entries in a thread's registers. The column's entries pass through LDS, 16 OWN at a time,
// so that each is read and raised to its power once for all that compare with it. Bound by
// scattered reads and writes of single logits: 64 entries of 4096 columns (262144 of them)
// of 32000 bf16 classes 18.6 us, and the whole backward of 1024 entries of 1024 columns
// 170 us (each entry read again from memory for every other: 22.3 and 540).
template <typename T, bool TWO, int OWN>
__global__ void __launch_bounds__(256) distill_sparse_kernel(const T* __restrict__ Z, int32_t V, int32_t B,
                                                             int32_t top, const int32_t* __restrict__ idx,
                                                             const float* __restrict__ tl,
                                                             const int32_t* __restrict__ labels,
                                                             const float* __restrict__ stats,
                                                             const float* __restrict__ dloss, float temp,
                                                             float weight, T* dZ) {
  constexpr int NX = 16, NY = 16, PASSED = NY * OWN;  // entries in LDS at a time
  __shared__ int32_t si[PASSED][NX];
  __shared__ float se[PASSED][NX];
  const int tx = threadIdx.x % NX, ty = threadIdx.x / NX;
  const int64_t b = B, at = column_group() * NX + tx;
  const bool on = at < b;
  const int64_t col = on ? at : b - 1;  // past the last: read again, nothing written
  const int64_t j0 = static_cast<int64_t>(blockIdx.y) * NY * OWN + ty;
  const float inv_t = 1.0f / temp;
  const int32_t passed = weight > 0.0f ? top : 0;
  int32_t ci[OWN];
  float ct[OWN];
  auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < OWN; ++u) {
      const int64_t i = i0 + ty + u * NY < passed ? i0 + ty + u * NY : i0;
      ci[u] = idx[i * b + col], ct[u] = tl[i * b + col];
    }
  };
  if (passed > 0) fetch(0);
  const int32_t label = labels ? labels[col] : -1;
  int32_t v[OWN];
  float z[OWN], p[OWN];
#pragma unroll
  for (int q = 0; q < OWN; ++q) {  // entry `top` is the label
    const int64_t j = j0 + q * NY;
    const int32_t w = j < top ? idx[j * b + col] : j == top ? label : -1;
    v[q] = on && w >= 0 && w < V ? w : -1;
    p[q] = 0.0f;
  }
#pragma unroll
  for (int q = 0; q < OWN; ++q) z[q] = to_f32(Z[(v[q] < 0 ? 0 : v[q]) * b + col]);
  const Factors f = factors_of(col, V, B, stats, labels, dloss, temp, weight);
  const float tref = stats[3 * b + col], es = stats[4 * b + col];
  for (int64_t i0 = 0; i0 < passed; i0 += PASSED) {
    const int n = static_cast<int>(passed - i0 < PASSED ? passed - i0 : PASSED);
    if (i0 > 0) __syncthreads();
#pragma unroll
    for (int u = 0; u < OWN; ++u) si[ty + u * NY][tx] = ci[u], se[ty + u * NY][tx] = expf((ct[u] - tref) * inv_t);
    __syncthreads();
    if (i0 + PASSED < passed) fetch(i0 + PASSED);
    for (int i = 0; i < n; ++i) {
      const int32_t w = si[i][tx];
      const float e = se[i][tx];
#pragma unroll
      for (int q = 0; q < OWN; ++q) p[q] = w == v[q] ? p[q] + e : p[q];
    }
  }
#pragma unroll
  for (int q = 0; q < OWN; ++q) {
    if (v[q] < 0) continue;
    float g = dense_grad<T, TWO>(z[q], f.m, f.fT, f.f1, inv_t);
    if (!(f.cs == 0.0f)) g -= f.cs * (p[q] / es);
    if (v[q] == label) g -= f.ch;
    dZ[v[q] * b + col] = from_f32<T>(g);
  }
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

int check_desc(const ard_distill_desc* d) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->batch < 1 || d->classes < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (batch %d, classes %d)", d->batch, d->classes);
  if (d->top < 0 || d->top > 65536) return fail(ARD_ERR_INVALID_ARG, "top %d outside 0..65536", d->top);
  if (!(d->temperature > 0.0f) || !std::isfinite(d->temperature) || !std::isfinite(1.0f / d->temperature))
    return fail(ARD_ERR_INVALID_ARG, "temperature must be positive and finite");
  if (!(d->soft_weight >= 0.0f && d->soft_weight <= 1.0f))
    return fail(ARD_ERR_INVALID_ARG, "soft_weight must be in [0, 1]");
  return ARD_OK;
}

constexpr int kBlocks = 512;  // workgroups that fill the chip: two on a compute unit

// Few classes: one column per thread and 16 threads down its rows, the whole pass in
// one launch. A launch costs what the reading of some hundred rows does (10 classes,
// 128 columns, fp32, forward and backward: 11.6 us, in four launches of wide rows 18.5).
// 256 classes, bf16, 5 entries, forward and backward, calls with their host's part: 1024
// columns 16.1 us in two launches, 24.2 in four; 8192 16.7 and 25.9. Only at 65536 columns
// do the single elements cost more than the launches: 73.2 and 65.7 (64 classes 32.8 and 43.5).
constexpr int kOneLaunch = 256;
bool one_launch(const ard_distill_desc* d) { return d->classes <= kOneLaunch; }
// The backward's one launch compares every entry with every other from memory: 16 entries
// of 238 classes 8.2 us, with a launch for the entries 11; but 32 14 to 10 and 64 36 to 12.
constexpr int kInside = 16;
bool one_launch_bwd(const ard_distill_desc* d) { return one_launch(d) && d->top <= kInside; }

int vector_of(const ard_distill_desc* d) {
  const int ve = d->dtype == ARD_BF16 ? 8 : 4;
  return d->batch >= ve && !one_launch(d) ? ve : 1;
}

// At least 8 rows for each thread, so that a range's sums outweigh joining them.
Grid grid_of(const ard_distill_desc* d) {
  const int64_t chunks = (static_cast<int64_t>(d->batch) + vector_of(d) - 1) / vector_of(d);
  if (one_launch(d)) return {16, static_cast<int32_t>((chunks + 15) / 16), 1, d->classes};
  Grid g = {1, 0, 0, 0};
  while (g.tx < 64 && g.tx < chunks) g.tx *= 2;
  g.blocks = static_cast<int32_t>((chunks + g.tx - 1) / g.tx);
  const int64_t least = 8 * (256 / g.tx);
  int64_t splits = (kBlocks + g.blocks - 1) / g.blocks;
  const int64_t most = (static_cast<int64_t>(d->classes) + least - 1) / least;
  if (splits > most) splits = most;
  g.rows = (static_cast<int64_t>(d->classes) + splits - 1) / splits;
  g.splits = static_cast<int32_t>((static_cast<int64_t>(d->classes) + g.rows - 1) / g.rows);
  return g;
}

size_t workspace_bytes(const ard_distill_desc* d) {
  return one_launch(d) ? 0 : static_cast<size_t>(grid_of(d).splits) * 3 * static_cast<size_t>(d->batch) * 4;
}

int check_teacher(const ard_distill_desc* d, const int32_t* idx, const float* tl, const int32_t* labels) {
  int st;
  if (d->top > 0 && ((st = need_ptr(idx, "top_idx")) || (st = need_ptr(tl, "top_logits")))) return st;
  return may_ptr(labels, "labels");
}

template <typename T, int VE, bool TWO, bool ONE>
int fwd_impl(const ard_distill_desc* d, const void* Zt, const int32_t* idx, const float* tl, const int32_t* labels,
             float* loss, float* stats, float* part, hipStream_t stream) {
  const Grid g = grid_of(d);
  const T* Z = static_cast<const T*>(Zt);
  hipLaunchKernelGGL((distill_sums_kernel<T, VE, TWO, ONE>), column_grid(g.blocks, g.splits), dim3(256), 0, stream, Z,
                     d->classes, d->batch, g, d->top, idx, tl, labels, d->temperature, d->soft_weight, part, loss,
                     stats);
  ARD_LAUNCH_CHECK();
  if (ONE) return ARD_OK;
  hipLaunchKernelGGL((distill_loss_kernel<T, TWO>), column_grid((d->batch - 1) / 16 + 1, 1), dim3(256), 0, stream, Z,
                     d->classes, d->batch, d->top, idx, tl, labels, d->temperature, d->soft_weight, g.splits, part,
                     loss, stats);
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T, int VE, bool TWO, bool ONE>
int bwd_impl(const ard_distill_desc* d, const void* Zt, const int32_t* idx, const float* tl, const int32_t* labels,
             const float* stats, const float* dloss, void* dZt, hipStream_t stream) {
  const Grid g = grid_of(d);
  const T* Z = static_cast<const T*>(Zt);
  T* dZ = static_cast<T*>(dZt);
  hipLaunchKernelGGL((distill_dense_kernel<T, VE, TWO, ONE>), column_grid(g.blocks, g.splits), dim3(256), 0, stream, Z,
                     d->classes, d->batch, g, d->top, idx, tl, labels, stats, dloss, d->temperature, d->soft_weight,
                     dZ);
  ARD_LAUNCH_CHECK();
  if (!ONE && (d->top > 0 || labels)) {
    // few entries: fewer for each thread (20 of 700 columns, 8800 classes: backward 22.7 us, with 8 24.5)
    auto entries = [&](auto own) {
      constexpr int OWN = decltype(own)::value;
      const dim3 grid = column_grid((d->batch - 1) / 16 + 1, d->top / (16 * OWN) + 1);
      hipLaunchKernelGGL((distill_sparse_kernel<T, TWO, OWN>), grid, dim3(256), 0, stream, Z, d->classes, d->batch,
                         d->top, idx, tl, labels, stats, dloss, d->temperature, d->soft_weight, dZ);
    };
    if (d->top < 32) entries(std::integral_constant<int, 2>{});
    else entries(std::integral_constant<int, 8>{});
    ARD_LAUNCH_CHECK();
  }
  return ARD_OK;
}

// Calls f with a value of the element type, the columns per thread, whether the two
// softmaxes differ and whether one launch does it all.
template <class F>
int dispatch(const ard_distill_desc* d, bool one, F f) {
  using std::integral_constant;
  const bool two = d->temperature != 1.0f;
  auto with = [&](auto t, auto ve, auto single) {
    return two ? f(t, ve, std::true_type{}, single) : f(t, ve, std::false_type{}, single);
  };
  auto typed = [&](auto t, auto wide) {
    if (one) return with(t, integral_constant<int, 1>{}, std::true_type{});
    if (vector_of(d) == 1) return with(t, integral_constant<int, 1>{}, std::false_type{});
    return with(t, wide, std::false_type{});
  };
  return d->dtype == ARD_BF16 ? typed(bf16{}, integral_constant<int, 8>{}) : typed(float{}, integral_constant<int, 4>{});
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

size_t ard_distill_workspace_bytes(const ard_distill_desc* desc) {
  if (check_desc(desc) != ARD_OK) return 0;
  return workspace_bytes(desc);
}

int ard_distill_fwd(const ard_distill_desc* desc, const void* Zt, const int32_t* top_idx, const float* top_logits,
                    const int32_t* labels, float* loss, float* stats, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  int st = check_desc(desc);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Zt, "Zt")) || (st = need_ptr(loss, "loss")) || (st = need_ptr(stats, "stats")) ||
      (st = check_teacher(desc, top_idx, top_logits, labels)))
    return st;
  if (workspace_bytes(desc) > 0 && (!ws || ws_bytes < workspace_bytes(desc)))
    return fail(ARD_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", workspace_bytes(desc), ws ? ws_bytes : 0);
  if ((st = may_ptr(ws, "workspace"))) return st;
  return dispatch(desc, one_launch(desc), [&](auto t, auto ve, auto two, auto one) {
    return fwd_impl<decltype(t), decltype(ve)::value, decltype(two)::value, decltype(one)::value>(
        desc, Zt, top_idx, top_logits, labels, loss, stats, static_cast<float*>(ws), static_cast<hipStream_t>(stream));
  });
}

int ard_distill_bwd(const ard_distill_desc* desc, const void* Zt, const int32_t* top_idx, const float* top_logits,
                    const int32_t* labels, const float* stats, const float* dloss, void* dZt, void* stream) {
  clear_error();
  int st = check_desc(desc);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Zt, "Zt")) || (st = need_ptr(stats, "stats")) || (st = need_ptr(dZt, "dZt")) ||
      (st = may_ptr(dloss, "dloss")) || (st = check_teacher(desc, top_idx, top_logits, labels)))
    return st;
  if (dZt == Zt) return fail(ARD_ERR_INVALID_ARG, "dZt must not be Zt: the logits are read again after the first pass");
  return dispatch(desc, one_launch_bwd(desc), [&](auto t, auto ve, auto two, auto one) {
    return bwd_impl<decltype(t), decltype(ve)::value, decltype(two)::value, decltype(one)::value>(
        desc, Zt, top_idx, top_logits, labels, stats, dloss, dZt, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
