// Gated feed-forward layer under a row pattern on its hidden units:
//   g = W0 x + b0,  u = W1 x + b1,  h = scale act(g) u  on the kept units.
//
// Forward: one kernel, for a few columns bound by reading the weights once, for many by
// the matrix cores; grids too small for its tiles (and weights past 2^31 bytes) run both
// projections as a batched product and join them. Backward: one pass writes the derivatives
//   dg = scale dh u act'(g),  du = scale dh act(g)
// of the kept rows and their row sums, the bias gradients; then dX = W0^T dg + W1^T du as one
// product over both halves, and dW as a batch of two. The derivatives are rounded to the
// element type once, as operands of those products (the row sums are not): with bf16 the
// gradients' error is 1.4 times that of fp32 derivatives, whose products would run at 1/7
// of the rate. A pattern's kept rows are an arithmetic progression, so every gather is a
// row stride.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../ard_gemm_fast.hpp"
#include "../ard_internal.hpp"

namespace ard {
namespace {

// The activation and its derivative, in fp32. With bf16 data the exponential and the
// reciprocal are the hardware's, to a few 2^-24: far below what the results are
// rounded by, and a tenth of the library functions' instructions, which the epilogue
// of a product does not hide.
struct Act {
  float f, d;
};
template <typename T>
__device__ __forceinline__ Act act_of(int act, float g) {
  if (act == ARD_GLU_RELU) return {g > 0.0f ? g : (g == g ? 0.0f : g), g > 0.0f ? 1.0f : 0.0f};
  if (act == ARD_GLU_GELU) {
    const float cdf = 0.5f * erfcf(g * -0.70710678118654752440f);  // to its own last bits where it is small
    return {g * cdf, cdf + g * 0.39894228040143267794f * expf(-0.5f * g * g)};
  }
  float s;
  if constexpr (sizeof(T) == 2)
    s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504088896340736f));
  else
    s = 1.0f / (1.0f + expf(-g));
  if (act == ARD_GLU_SIGMOID) return {s, s * (1.0f - s)};
  return {g * s, s * (1.0f + g * (1.0f - s))};
}

// Launches of a workgroup for each hidden unit (or block of units): in rows of 2^20
// workgroups, since the threads along x have to stay below 2^32.
constexpr int32_t kGridRow = 1 << 20;
dim3 unit_grid(int32_t groups) { return dim3(std::min(groups, kGridRow), (groups - 1) / kGridRow + 1); }
__device__ __forceinline__ int32_t unit_group() { return static_cast<int32_t>(blockIdx.y * gridDim.x + blockIdx.x); }

struct GluShape {
  int32_t B, K, N, kept, period, offset;
  int64_t ldd;   // row length of the derivatives in the workspace, and of X's copy
  int64_t ldk;   // row length of the kept weights' copy
  size_t es;
  bool zero;     // dropped rows are written 0
};

// ------------------------------------------------------------------ rows off 16 bytes
// Products of rows that do not start on 16 bytes run at a third to a half of the rate of
// those that do (register loads in place of direct ones, smaller tiles), while a copy whose
// rows are a multiple of 16 bytes costs its bytes once: kept weights [2][kept][ldk], X
// [K][ldd]. bf16, every other of 8191 units kept, batch 2047: forward 945 to 311 us,
// backward (where the derivatives' launch makes the copies) 2866 to 679; 407 x 5687 -> 517
// forward 142 to 36.

// A row of n elements to one that starts on 16 bytes, 0 in the rest of its last 16; LANES threads.
template <int LANES, typename T>
__device__ __forceinline__ void copy_row(const T* __restrict__ from, T* __restrict__ to, int32_t n) {
  constexpr int E = 16 / static_cast<int>(sizeof(T)), U = 4;
  const int lane = threadIdx.x & (LANES - 1), whole = n / E;
  int c = lane;
  for (; c + (U - 1) * LANES < whole; c += U * LANES) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load16_any<sizeof(T)>(reinterpret_cast<const char*>(from + (c + u * LANES) * E));
#pragma unroll
    for (int u = 0; u < U; ++u) reinterpret_cast<u32x4*>(to)[c + u * LANES] = v[u];
  }
  for (; c < whole; c += LANES)
    reinterpret_cast<u32x4*>(to)[c] = load16_any<sizeof(T)>(reinterpret_cast<const char*>(from + c * E));
  if (c == whole && n % E) {
    T e[E];
#pragma unroll
    for (int q = 0; q < E; ++q) e[q] = whole * E + q < n ? from[whole * E + q] : from_f32<T>(0.0f);
    reinterpret_cast<u32x4*>(to)[whole] = *reinterpret_cast<const u32x4*>(e);
  }
}

// The forward's copies (Wc, Xc: NULL = not wanted), a row a wave.
template <typename T>
__global__ void __launch_bounds__(256) glu_copy_kernel(GluShape s, const T* __restrict__ X, const T* __restrict__ W,
                                                       T* __restrict__ Xc, T* __restrict__ Wc) {
  const int64_t rw = Wc ? 2 * static_cast<int64_t>(s.kept) : 0, rows = rw + (Xc ? s.K : 0);
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4ll) {
    if (r < rw) {
      const int64_t h = r >= s.kept, i = r - h * s.kept;
      copy_row<64>(W + (h * s.N + s.offset + i * s.period) * s.K, Wc + r * s.ldk, s.K);
    } else {
      copy_row<64>(X + (r - rw) * s.B, Xc + (r - rw) * s.ldd, s.B);
    }
  }
}

// Joins the projections zf[2][kept][B] (fp32): a workgroup per hidden unit, a
// dropped one's row cleared if asked. 2000 units of 700 columns, fp32: 10 us.
template <typename T>
__global__ void __launch_bounds__(256) glu_join_kernel(GluShape s, const float* __restrict__ zf,
                                                       const float* __restrict__ bias, int act, float scale,
                                                       T* __restrict__ Z, T* __restrict__ H) {
  const int64_t n = unit_group();
  if (n >= s.N) return;
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
    h[b] = from_f32<T>(scale * act_of<T>(act, g).f * u);
    if (Z) {
      Z[n * s.B + b] = from_f32<T>(g);
      Z[(s.N + n) * s.B + b] = from_f32<T>(u);
    }
  }
}

// ------------------------------------------------------------------ few columns
// Up to 64 columns (single tokens of as many sequences): bound by reading the kept
// weights once. A workgroup takes PAIRS hidden units (16, or 8 so that a small layer
// still reaches every compute unit: both projections then share one block of 16
// rows); its eight waves split the inputs and read the weights straight into MFMA
// operands, 16 bytes of a lane, nothing shared through LDS. The columns' part is read
// as it lies, [k][batch], and turned in wave-private LDS (bf16; fp32 operands are
// single elements). The waves' sums meet in LDS, where the layer is finished.
// bf16, 16 columns, 4096 -> 8192 (134 MB of weights): 31.7 us, 4.2 TB/s; one column,
// 1024 -> 2048: 4.0 us, most of it the launch and the latency of the loads.
// NB: blocks of 16 columns; 0: one column, whose inputs are contiguous already.
constexpr int kSmallWaves = 8;

template <typename T, int PAIRS, int NB>
struct Small {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int NC = NB == 0 ? 1 : NB;         // blocks of columns
  static constexpr int FR = PAIRS == 16 ? 2 : 1;      // blocks of weight rows
  static constexpr int STEP = BF ? 32 : 16;           // k of one step
  static constexpr int U = NC >= 4 ? 2 : 4;           // steps in flight
  static constexpr int XB = BF && NB > 0 ? STEP * NB * 32 : 0;  // bytes of a step's columns in LDS
  static constexpr int RED = kSmallWaves * FR * NC * 1024;
  static constexpr int LDS = kSmallWaves * U * XB > RED ? kSmallWaves * U * XB : RED;
};

template <typename T, int PAIRS, int NB>
__global__ void __launch_bounds__(64 * kSmallWaves) glu_small_kernel(GluShape s, const T* __restrict__ X,
                                                                     const T* __restrict__ W,
                                                                     const float* __restrict__ bias, int act,
                                                                     float scale, T* __restrict__ Z,
                                                                     T* __restrict__ H) {
  using C = Small<T, PAIRS, NB>;
  constexpr int ES = sizeof(T), VE = 16 / ES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = lane & 15, grp = lane >> 4;
  const int i0 = xcd_position(unit_group(), static_cast<int>(gridDim.x * gridDim.y)) * PAIRS;
  if (i0 >= s.kept) return;
  const int64_t K = s.K, B = s.B;

  // the lane's weight rows: gate and other projection, or (8 units) one of them
  const T* wp[C::FR];
#pragma unroll
  for (int f = 0; f < C::FR; ++f) {
    const int half = PAIRS == 16 ? f : row >> 3;
    const int i = min(i0 + (PAIRS == 16 ? row : row & 7), s.kept - 1);  // past the last: its results are discarded
    wp[f] = W + (half * static_cast<int64_t>(s.N) + s.offset + static_cast<int64_t>(i) * s.period) * K + VE * grp;
  }
  f32x4 acc[C::FR][C::NC];
#pragma unroll
  for (int f = 0; f < C::FR; ++f)
#pragma unroll
    for (int c = 0; c < C::NC; ++c) acc[f][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // a step's products: a = 16 bytes of each weight row, x = the columns' operand
  auto mma = [&](const u32x4 a, const u32x4 x, f32x4& to) {
    if constexpr (C::BF) {
      to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, x), to, 0, 0, 0);
    } else {
      const f32x4 af = __builtin_bit_cast(f32x4, a), xf = __builtin_bit_cast(f32x4, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) to = __builtin_amdgcn_mfma_f32_16x16x4f32(af[e], xf[e], to, 0, 0, 0);
    }
  };
  // Steps of this wave. A whole step reads 16 bytes at a time and stays inside the
  // operands: the columns' reads reach up to 16 NB - B elements past the last row read.
  const int steps = static_cast<int>((K + C::STEP - 1) / C::STEP);
  const int q0 = steps * wv / kSmallWaves, q1 = steps * (wv + 1) / kSmallWaves;
  int64_t whole = K / C::STEP;
  if (C::BF && NB > 0)
    while (whole > 0 && (whole * C::STEP - 1) * B + 16 * NB > K * B) --whole;
  const int qw = min(q1, static_cast<int>(whole));
  char* xl = smem + wv * C::U * C::XB;
  for (int q = q0; q < qw; q += C::U) {
    u32x4 a[C::U][C::FR], x[C::U][C::NC];
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
      const int64_t k = static_cast<int64_t>(min(q + u, qw - 1)) * C::STEP;  // past the last: read again, not used
#pragma unroll
      for (int f = 0; f < C::FR; ++f) a[u][f] = load16_any<ES>(reinterpret_cast<const char*>(wp[f] + k));
      if constexpr (NB == 0) {
        x[u][0] = load16_any<ES>(reinterpret_cast<const char*>(X + k + VE * grp));
      } else if constexpr (C::BF) {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const int at = c * 64 + lane, r = at / (2 * NB), ch = at % (2 * NB);
          x[u][c] = load16_any<ES>(reinterpret_cast<const char*>(X + (k + r) * B + 8 * ch));
        }
      } else {
#pragma unroll
        for (int c = 0; c < NB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[u][c][e] = __float_as_uint(X[(k + 4 * grp + e) * B + min(static_cast<int64_t>(16 * c + row), B - 1)]);
      }
    }
    if constexpr (C::XB > 0) {
#pragma unroll
      for (int u = 0; u < C::U; ++u)
#pragma unroll
        for (int c = 0; c < NB; ++c) *reinterpret_cast<u32x4*>(xl + u * C::XB + (c * 64 + lane) * 16) = x[u][c];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < C::U; ++u)
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          // 8 k of one column: two transposed reads of 4 k by 16 columns
          const char* p = xl + u * C::XB + (8 * grp + (row >> 2)) * (NB * 32) + c * 32 + (row & 3) * 8;
          const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
          const i16x4 hi =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + 4 * NB * 32));
          typedef short i16x8 __attribute__((ext_vector_type(8)));
          x[u][c] = __builtin_bit_cast(u32x4, static_cast<i16x8>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
        }
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
      if (q + u >= qw) break;
#pragma unroll
      for (int f = 0; f < C::FR; ++f)
#pragma unroll
        for (int c = 0; c < C::NC; ++c) mma(a[u][f], x[u][c], acc[f][c]);
    }
  }
  // the last steps, element by element
#pragma unroll 1
  for (int q = max(q0, qw); q < q1; ++q) {
    const int64_t k = static_cast<int64_t>(q) * C::STEP + VE * grp;
    u32x4 a[C::FR], x[C::NC];
    auto gather = [&](const T* p, int64_t stride) {  // VE elements from p (element k), 0 past K
      T e[VE];
      u32x4 v;
#pragma unroll
      for (int j = 0; j < VE; ++j) e[j] = p[(k + j < K ? j : 0) * stride];
#pragma unroll
      for (int j = 0; j < VE; ++j) reinterpret_cast<T*>(&v)[j] = k + j < K ? e[j] : from_f32<T>(0.0f);
      return v;
    };
    const int64_t kc = k < K ? k : K - 1;
#pragma unroll
    for (int f = 0; f < C::FR; ++f) a[f] = gather(wp[f] + (kc - VE * grp), 1);
#pragma unroll
    for (int c = 0; c < C::NC; ++c) {
      const int64_t col = NB == 0 ? 0 : min(static_cast<int64_t>(16 * c + row), B - 1);
      x[c] = gather(X + kc * B + col, B);
    }
#pragma unroll
    for (int f = 0; f < C::FR; ++f)
#pragma unroll
      for (int c = 0; c < C::NC; ++c) mma(a[f], x[c], acc[f][c]);
  }

  // the waves' sums, and the layer: output block rows 4 grp + r, column lane % 16
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(smem);
#pragma unroll
  for (int f = 0; f < C::FR; ++f)
#pragma unroll
    for (int c = 0; c < C::NC; ++c) red[((wv * C::FR + f) * C::NC + c) * 64 + lane] = acc[f][c];
  __syncthreads();
  auto sum = [&](int f, int m, int b) {  // row m of block f, column b
    const float* p = reinterpret_cast<const float*>(red + (f * C::NC + b / 16) * 64 + (m >> 2) * 16 + b % 16) + (m & 3);
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) v += p[w * C::FR * C::NC * 256];
    return v;
  };
  for (int64_t e = threadIdx.x; e < PAIRS * B; e += 64 * kSmallWaves) {
    const int m = static_cast<int>(e / B), b = static_cast<int>(e % B);
    if (i0 + m >= s.kept) break;
    const int64_t n = s.offset + static_cast<int64_t>(i0 + m) * s.period;
    float g = sum(0, m, b), u = PAIRS == 16 ? sum(C::FR - 1, m, b) : sum(0, m + 8, b);
    if (bias) g += bias[n], u += bias[s.N + n];
    H[n * B + b] = from_f32<T>(scale * act_of<T>(act, g).f * u);
    if (Z) {
      Z[n * B + b] = from_f32<T>(g);
      Z[(s.N + n) * B + b] = from_f32<T>(u);
    }
  }
  // the dropped rows behind each kept one (and those in front of the first)
  if (s.zero && s.period > 1) {
    const int64_t first = i0 == 0 ? 0 : s.offset + static_cast<int64_t>(i0) * s.period;
    const int64_t end = i0 + PAIRS >= s.kept ? s.N : s.offset + static_cast<int64_t>(i0 + PAIRS) * s.period;
    for (int64_t e = first * B + threadIdx.x; e < end * B; e += 64 * kSmallWaves)
      if (static_cast<int32_t>(e / B % s.period) != s.offset) H[e] = from_f32<T>(0.0f);
  }
}

// ------------------------------------------------------------------ one product
// Both projections in one product of the fast kernel's tiles: a tile's rows are blocks
// of 32 kept gate rows and the same 32 units' other rows in turn, so that a wave holds
// g and u of the same places in neighbouring accumulators, and activation and product
// are the epilogue: nothing of the 2 x kept x batch sums passes through memory in fp32.
// Bound by the matrix cores: 8192 -> 8192 (every other unit kept, 275 GFLOP), batch 2048:
// 242 us, 1136 TFLOP/s; a square product of 8192 by the library runs at 1111.
struct GluTileArgs {
  GluShape s;
  const void* X;     // rows of ldx
  const void* W;     // a projection's first kept row; rows of ldw, those kept w_step apart
  int64_t ldx, ldw;
  int32_t w_step, w_half;  // rows between kept ones, and between the projections
  const float* bias;
  void* Z;
  void* H;
  int32_t act;
  float scale;
};

// LDS: the stages, then the outputs of each wave on their way out (g, u, h: 32 rows
// each, and the biases of its units).
template <class Cfg>
struct GluLds {
  static constexpr int ROW = Cfg::TN * 2 + 16, PART = 32 * ROW, PAIRS = Cfg::TM / 2;
  static constexpr int WAVE = 3 * PART + 2 * PAIRS * 4;
  static constexpr int BYTES = Cfg::NW * WAVE > Cfg::LDS ? Cfg::NW * WAVE : Cfg::LDS;
};

template <class Cfg>
__global__ void __launch_bounds__(Cfg::NT) glu_tile_kernel(GluTileArgs g) {
  static_assert(Cfg::TM % 64 == 0 && Cfg::KSPLIT == 1 && Cfg::ES == 2, "whole pairs of 32 rows in a wave");
  constexpr int ES = Cfg::ES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const GluShape& s = g.s;
  int tile_row, tile_col;
  grouped_tile(blockIdx.x, (s.B + Cfg::BN - 1) / Cfg::BN, (s.kept + Cfg::BM / 2 - 1) / (Cfg::BM / 2), tile_row, tile_col);
  const int p0 = tile_row * (Cfg::BM / 2), n0 = tile_col * Cfg::BN;  // first pair, first column
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wv / Cfg::WGN, wn = wv % Cfg::WGN;
  f32x16 acc[Cfg::FM][Cfg::FN];
#pragma unroll
  for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  const int nslab = (s.K + Cfg::BK - 1) / Cfg::BK;
  auto row_of = [&](int r) {  // tile row -> row of W; past the last pair: the last one, discarded
    return ((r >> 5) & 1) * g.w_half + min(p0 + (r >> 6) * 32 + (r & 31), s.kept - 1) * g.w_step;
  };
  SlabLoader<Cfg, false, true> ld;
  ld.wv = wv;
  ld.da.init_rows(g.ldw, row_of, wv);
  ld.db.init(g.ldx, n0, s.B, wv);
  ld.K = s.K;
  ld.ik = 0;
  ld.a_step = static_cast<int64_t>(Cfg::BK) * ES;
  ld.b_step = g.ldx * Cfg::BK * ES;
  ld.a_wrap = ld.b_wrap = 0;
  ld.na = uniform_ptr(static_cast<const char*>(g.W));
  ld.nb = uniform_ptr(static_cast<const char*>(g.X));
  ld.lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem));
  ld.is = 0;
  ld.left = nslab - 1;
  run_slabs<Cfg, false, true, true, false>(ld, nslab, s.K, 0, acc, wm, wn, 0, smem);

  // Each block of 32 units passes through the wave's own LDS, g, u and h side by side,
  // and is written 16 bytes of a row at a time. The units' biases come first, every
  // load in flight together.
  using L = GluLds<Cfg>;
  constexpr int ROW = L::ROW, PART = L::PART, CPRW = Cfg::TN / 8, RPI = 64 / CPRW, PAIRS = L::PAIRS;
  lds_barrier();  // every wave is done with the stages
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  char* region = smem + wv * L::WAVE;
  float* bl = reinterpret_cast<float*>(region + 3 * PART);
  const int pw = p0 + wm * PAIRS;  // the wave's first pair
  auto unit = [&](int p) { return s.offset + static_cast<int64_t>(pw + p) * s.period; };
  if (g.bias) {
#pragma unroll
    for (int e = 0; e < 2 * PAIRS; e += 64)
      if (e + lane < 2 * PAIRS) {
        const int p = (e + lane) % PAIRS;
        bl[e + lane] = g.bias[(e + lane) / PAIRS * static_cast<int64_t>(s.N) + unit(min(pw + p, s.kept - 1) - pw)];
      }
  }
#pragma unroll
  for (int i = 0; i < Cfg::FM; i += 2) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int rl = 8 * (r >> 2) + 4 * lh + (r & 3);
      const float b0 = g.bias ? bl[16 * i + rl] : 0.0f, b1 = g.bias ? bl[PAIRS + 16 * i + rl] : 0.0f;
#pragma unroll
      for (int j = 0; j < Cfg::FN; ++j) {
        const float x = acc[i][j][r] + b0, u = acc[i + 1][j][r] + b1;
        bf16* at = reinterpret_cast<bf16*>(region + rl * ROW) + 32 * j + lr;
        if (g.Z) {
          at[0] = static_cast<bf16>(x);
          at[PART / 2] = static_cast<bf16>(u);
        }
        at[PART] = static_cast<bf16>(g.scale * act_of<bf16>(g.act, x).f * u);
      }
    }
    for (int part = g.Z ? 0 : 2; part < 3; ++part) {
      bf16* out = part == 2 ? static_cast<bf16*>(g.H)
                            : static_cast<bf16*>(g.Z) + (part == 1 ? static_cast<int64_t>(s.N) * s.B : 0);
#pragma unroll
      for (int t = 0; t < 32 / RPI; ++t) {
        const int rl = lane / CPRW + RPI * t, n = n0 + wn * Cfg::TN + 8 * (lane % CPRW);
        const char* from = region + part * PART + rl * ROW + (lane % CPRW) * 16;
        if (pw + 16 * i + rl >= s.kept || n >= s.B) continue;
        bf16* o = out + unit(16 * i + rl) * s.B + n;
        typedef u32x4 u32x4_a2 __attribute__((aligned(2), may_alias));
        if (n + 8 <= s.B) {
          *reinterpret_cast<u32x4_a2*>(o) = *reinterpret_cast<const u32x4*>(from);
        } else {
          for (int e = 0; n + e < s.B; ++e) o[e] = reinterpret_cast<const bf16*>(from)[e];
        }
      }
    }
  }
}

// Clears the dropped rows of H.
template <typename T>
__global__ void __launch_bounds__(256) glu_clear_kernel(GluShape s, T* __restrict__ H) {
  const int64_t n = unit_group();
  if (n >= s.N || static_cast<int32_t>(n % s.period) == s.offset) return;
  T* h = H + n * s.B;
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  if (s.B % E == 0) {
    for (int b = threadIdx.x; b < s.B / E; b += 256) reinterpret_cast<u32x4*>(h)[b] = u32x4{0u, 0u, 0u, 0u};
  } else {
    for (int b = threadIdx.x; b < s.B; b += 256) h[b] = from_f32<T>(0.0f);
  }
}

// The derivatives D[2][kept][ldd] and their row sums, a workgroup per hidden unit; that
// of a dropped one clears its rows of dW and entries of dbias, if asked. Bound by
// reading g, u and dH and writing both derivatives (16 bytes of a lane at a time), and the
// products' copies where rows are off 16 bytes: 4096 of 8192 units kept, batch 2048, dW[2][8192][8192] bf16 (84 MB
// and 134 MB cleared) 35.6 us, 6.1 TB/s.
template <typename T, typename G>
__global__ void __launch_bounds__(256) glu_derive_kernel(GluShape s, const T* __restrict__ Z,
                                                         const T* __restrict__ dH, const T* __restrict__ X,
                                                         const T* __restrict__ W, int act, float scale,
                                                         T* __restrict__ D, G* __restrict__ dW,
                                                         float* __restrict__ dbias, T* __restrict__ Xc,
                                                         T* __restrict__ Wc) {
  const int64_t n = unit_group();
  if (n >= s.N) return;
  if (static_cast<int32_t>(n % s.period) != s.offset) {
    if (!s.zero) return;
    if (dW) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        G* row = dW + (h * static_cast<int64_t>(s.N) + n) * s.K;
        constexpr int E = 16 / static_cast<int>(sizeof(G));
        if (static_cast<int64_t>(s.K) * sizeof(G) % 16 == 0) {
          for (int64_t k = threadIdx.x; k < s.K / E; k += 256)
            reinterpret_cast<u32x4*>(row)[k] = u32x4{0u, 0u, 0u, 0u};
        } else {
          for (int64_t k = threadIdx.x; k < s.K; k += 256) row[k] = from_f32<G>(0.0f);
        }
      }
    }
    if (dbias && threadIdx.x < 2) dbias[threadIdx.x * static_cast<int64_t>(s.N) + n] = 0.0f;
    return;
  }
  const int64_t i = (n - s.offset) / s.period;
  const T *gp = Z + n * s.B, *up = Z + (s.N + n) * s.B, *hp = dH + n * s.B;
  T *dg = D + i * s.ldd, *du = D + (s.kept + i) * s.ldd;
  float sg = 0.0f, su = 0.0f;
  auto one = [&](float z, float u, float h, float& og, float& ou) {
    const Act a = act_of<T>(act, z);
    const float d = scale * h;
    og = d * u * a.d;
    ou = d * a.f;
    sg += og;
    su += ou;
  };
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  for (int b = threadIdx.x * E; b < s.B; b += 256 * E) {
    u32x4 r[3], og, ou;  // g, u and dH
    const T* from[3] = {gp + b, up + b, hp + b};
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      if (b + E <= s.B) {
        r[q] = load16_any<sizeof(T)>(reinterpret_cast<const char*>(from[q]));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) reinterpret_cast<T*>(&r[q])[e] = b + e < s.B ? from[q][e] : from_f32<T>(0.0f);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x = 0.0f, y = 0.0f;
      if (b + e < s.B)
        one(to_f32(reinterpret_cast<const T*>(&r[0])[e]), to_f32(reinterpret_cast<const T*>(&r[1])[e]),
            to_f32(reinterpret_cast<const T*>(&r[2])[e]), x, y);
      reinterpret_cast<T*>(&og)[e] = from_f32<T>(x);
      reinterpret_cast<T*>(&ou)[e] = from_f32<T>(y);
    }
    *reinterpret_cast<u32x4*>(dg + b) = og;
    *reinterpret_cast<u32x4*>(du + b) = ou;
  }
  // the products' copies: this unit's weights, and X's rows i, i + kept, ...
  if (Wc) {
    const int64_t h = threadIdx.x >> 7;
    copy_row<128>(W + (h * s.N + n) * s.K, Wc + (h * s.kept + i) * s.ldk, s.K);
  }
  for (int64_t r = i + (threadIdx.x >> 6) * static_cast<int64_t>(s.kept); Xc && r < s.K; r += 4 * static_cast<int64_t>(s.kept))
    copy_row<64>(X + r * s.B, Xc + r * s.ldd, s.B);
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
  s->ldk = (static_cast<int64_t>(s->K) + 7) / 8 * 8;
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

// Whether the forward runs on glu_small_kernel. Measured against the products and the
// join (4096 -> 8192 / 1024 -> 2048, us): bf16 batch 1 30.7 to 92.0 / 9 to 16, 16 32.9 to
// 42.6 / 9 to 12.5, 64 43.5 to 46.0 / 9 to 12.5; fp32 batch 1 57 to 77 / 9 to 17, 16 67 to
// 66 / 9 to 17, but 32 81 to 66 and 64 137 to 96 / 14 to 14.
bool small_batch(const GluShape& s) { return s.B <= (s.es == 2 ? 64 : 16) && s.kept > 0; }

// The tile of glu_tile_kernel with the least modelled time: rounds of the chip times a
// tile's work over the rate that it reaches with the chip full (FastKind; -1: none). bf16
// only: fp32 products are planned by the layers' cost model, split contractions and
// 64 x 64 tiles included, and what a fused epilogue saved there (1 to 5 us) the tiles
// with 64 rows in a wave lost several times over (700 x 1500 -> 2000 units 113 to 94 us).
int plan_tile(const GluShape& s) {
  if (s.es != 2 || int64_t{4} * s.N * s.ldk + 4096 >= int64_t{1} << 31 || 514 * s.ldd >= int64_t{1} << 31)
    return -1;
  struct Tile {
    int kind, bm, bn;
    double rate;  // flop/s of a compute unit
  };
  static constexpr Tile tiles[] = {
      {FAST_HUGE, 256, 256, 4.2e12}, {FAST_WIDE, 128, 256, 3.5e12}, {FAST_TALL, 256, 128, 3.4e12}, {FAST_BIG, 128, 128, 2.7e12}};
  int best = -1;
  double best_t = 1e300;
  for (const Tile& c : tiles) {
    const int64_t n = (static_cast<int64_t>(s.kept) + c.bm / 2 - 1) / (c.bm / 2) * ((s.B + c.bn - 1) / c.bn);
    if (n < kTargetBlocks * 5 / 8) continue;
    const double t = static_cast<double>((n + kTargetBlocks - 1) / kTargetBlocks) * 2.0 * c.bm * c.bn * s.K / c.rate;
    if (t < best_t) best_t = t, best = c.kind;
  }
  return best;
}
bool one_product(const GluShape& s) { return s.kept > 0 && !small_batch(s) && plan_tile(s) >= 0; }

// The workspace: what the products read or write first, their partial sums behind it.
struct Space {
  size_t head, part, wc, xc;
  size_t bytes() const { return head + part + wc + xc; }
  template <typename T>
  T* weights(char* ws) const { return wc ? reinterpret_cast<T*>(ws + head + part) : nullptr; }
  template <typename T>
  T* inputs(char* ws) const { return xc ? reinterpret_cast<T*>(ws + head + part + wc) : nullptr; }
};
size_t copy_w(const GluShape& s) {
  return s.K * s.es % 16 ? al256(static_cast<size_t>(2) * s.kept * s.ldk * s.es) : 0;
}
size_t copy_x(const GluShape& s) { return s.B * s.es % 16 ? al256(static_cast<size_t>(s.K) * s.ldd * s.es) : 0; }
double work_of(const GluShape& s) { return static_cast<double>(s.kept) * s.K * s.B; }
// The forward's copies are a launch of their own, 2 to 4 us: for the tiles, which take no
// other rows, and for products that gain more: bf16 100 x 1023 -> 512 kept 18.0 to 15.8 us,
// but 70 x 301 -> 500 12.1 to 13.8; fp32 594 x 735 -> 1804 73 to 64, 474 x 719 -> 1220 47 to
// 47, 100 x 1023 -> 512 17.8 to 19.8.
bool fwd_copies(const GluShape& s) { return one_product(s) || work_of(s) >= (s.es == 2 ? 32e6 : 400e6); }
// The backward copies beside the derivatives: the weights always (bf16 70 x 301 -> 500 24 to
// 19, 1681 x 1194 -> 1330 190 to 84), X for dW from 1e8 multiply-adds of a projection on,
// where both types gain. us without and with the copy of X, dW in fp32: bf16 133 x 512 -> 512
// (3.5e7) 17.8 to 20.4, 255 x 512 -> 512 (6.7e7) 18.4 to 17.5, 101 x 1024 -> 1024 (1.1e8) 29.0
// to 27.1, 255 x 2048 -> 2048 (1.1e9) 49.3 to 43.9; fp32 22.0 to 23.1, 24.2 to 24.6, 30.0 to
// 28.6, 103.5 to 91.1. Smaller ones lie between a gain of 4 us and a loss of 3.
bool bwd_copies_x(const GluShape& s) { return work_of(s) >= 100e6; }
template <typename T>
Space fwd_space(const GluShape& s) {
  if (s.kept == 0 || small_batch(s)) return {0, 0, 0, 0};
  const bool c = fwd_copies(s);
  const size_t w = c ? copy_w(s) : 0, x = c ? copy_x(s) : 0;
  if (one_product(s)) return {0, 0, w, x};
  return {al256(static_cast<size_t>(2) * s.kept * s.B * 4), al256(4 * partial_floats<T>(s.kept, s.B, s.K, 1, 2)), w, x};
}
template <typename T>
Space bwd_space(const GluShape& s) {
  if (s.kept == 0) return {0, 0, 0, 0};
  const size_t d = partial_floats<T>(s.K, s.B, s.kept, 2, 1), w = partial_floats<T>(s.kept, s.K, s.B, 1, 2);
  return {al256(static_cast<size_t>(2) * s.kept * s.ldd * sizeof(T)), al256(4 * std::max(d, w)), copy_w(s),
          bwd_copies_x(s) ? copy_x(s) : 0};
}

int check_ws(const Space& sp, const void* ws, size_t ws_bytes) {
  if (sp.bytes() == 0) return ARD_OK;
  if (!ws || ws_bytes < sp.bytes())
    return fail(ARD_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", sp.bytes(), ws ? ws_bytes : 0);
  if (!aligned16(ws)) return fail(ARD_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return ARD_OK;
}

// The kept rows of both projections, in W[2][N][K] or in their copy.
GemmOperand kept_weights(const GluShape& s, const void* W, const void* copy) {
  GemmOperand o = {};
  if (copy) {
    o.p = copy;
    o.ld = s.ldk;
    o.bstride = o.kbstride = s.kept * s.ldk;
    return o;
  }
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

template <typename T, int PAIRS, int NB>
hipError_t launch_small_pairs(const ard_glu_desc* d, const GluShape& s, const void* X, const void* W, const float* bias,
                              void* Z, void* H, hipStream_t stream) {
  using C = Small<T, PAIRS, NB>;
  auto kern = glu_small_kernel<T, PAIRS, NB>;
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, unit_grid((s.kept + PAIRS - 1) / PAIRS), dim3(64 * kSmallWaves), C::LDS, stream, s,
                     static_cast<const T*>(X), static_cast<const T*>(W), bias, d->act, d->scale, static_cast<T*>(Z),
                     static_cast<T*>(H));
  return hipGetLastError();
}
template <typename T>
hipError_t launch_small_fwd(const ard_glu_desc* d, const GluShape& s, const void* X, const void* W, const float* bias,
                            void* Z, void* H, hipStream_t stream) {
  const bool eight = s.kept < 4096;  // 16 units of each would leave compute units without work
  auto with = [&](auto nb) {
    constexpr int NB = decltype(nb)::value;
    return eight ? launch_small_pairs<T, 8, NB>(d, s, X, W, bias, Z, H, stream)
                 : launch_small_pairs<T, 16, NB>(d, s, X, W, bias, Z, H, stream);
  };
  using std::integral_constant;
  if (s.B == 1) return with(integral_constant<int, 0>{});
  if constexpr (sizeof(T) == 2) {
    if (s.B > 32) return with(integral_constant<int, 4>{});
    if (s.B > 16) return with(integral_constant<int, 2>{});
  }
  return with(integral_constant<int, 1>{});
}

template <class Cfg>
hipError_t launch_tile(const GluTileArgs& g, hipStream_t stream) {
  auto kern = glu_tile_kernel<Cfg>;
  constexpr int LDS = GluLds<Cfg>::BYTES;
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return attr;
  const unsigned tiles = static_cast<unsigned>((g.s.kept + Cfg::BM / 2 - 1) / (Cfg::BM / 2)) *
                         static_cast<unsigned>((g.s.B + Cfg::BN - 1) / Cfg::BN);
  hipLaunchKernelGGL(kern, dim3(tiles), dim3(Cfg::NT), LDS, stream, g);
  return hipGetLastError();
}
hipError_t run_tile(const GluTileArgs& g, hipStream_t stream) {
  using C = FastCfgs<bf16>;
  switch (plan_tile(g.s)) {
    case FAST_HUGE: return launch_tile<C::Huge>(g, stream);
    case FAST_WIDE: return launch_tile<C::Wide>(g, stream);
    case FAST_TALL: return launch_tile<C::Tall>(g, stream);
    default: return launch_tile<C::Big>(g, stream);
  }
}

template <typename T>
int fwd_impl(const ard_glu_desc* d, const GluShape& s, const void* Xt, const void* W, const float* bias, void* Zt,
             void* Ht, char* ws, hipStream_t stream) {
  if (small_batch(s)) {
    ARD_HIP_CHECK(launch_small_fwd<T>(d, s, Xt, W, bias, Zt, Ht, stream));
    return ARD_OK;
  }
  const Space sp = fwd_space<T>(s);
  T *wc = sp.weights<T>(ws), *xc = sp.inputs<T>(ws);
  if (wc || xc) {
    const int64_t rows = (wc ? 2 * static_cast<int64_t>(s.kept) : 0) + (xc ? s.K : 0);
    hipLaunchKernelGGL(glu_copy_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>((rows + 3) / 4, 65536))),
                       dim3(256), 0, stream, s, static_cast<const T*>(Xt), static_cast<const T*>(W), xc, wc);
    ARD_LAUNCH_CHECK();
  }
  const void* x = xc ? xc : Xt;
  const int64_t ldx = xc ? s.ldd : s.B;
  if (one_product(s)) {
    const T* w = wc ? wc : static_cast<const T*>(W) + static_cast<int64_t>(s.offset) * s.K;
    ARD_HIP_CHECK(run_tile(GluTileArgs{s, x, w, ldx, wc ? s.ldk : s.K, wc ? 1 : s.period, wc ? s.kept : s.N, bias, Zt, Ht,
                                       d->act, d->scale},
                           stream));
    if (s.zero && s.period > 1) {
      hipLaunchKernelGGL(glu_clear_kernel<T>, unit_grid(s.N), dim3(256), 0, stream, s, static_cast<T*>(Ht));
      ARD_LAUNCH_CHECK();
    }
    return ARD_OK;
  }
  float* zf = reinterpret_cast<float*>(ws);
  if (s.kept > 0) {
    GemmArgs g = {};
    g.M = s.kept, g.N = s.B, g.K = s.K;
    g.a = kept_weights(s, W, wc);
    g.b = plain(x, ldx, 0);
    g.c.p = zf, g.c.ld = s.B, g.c.bstride = static_cast<int64_t>(s.kept) * s.B;
    ARD_HIP_CHECK((product<T, false, true, float>(g, 2, stream, reinterpret_cast<float*>(ws + sp.head), sp.part / 4)));
  }
  hipLaunchKernelGGL(glu_join_kernel<T>, unit_grid(s.N), dim3(256), 0, stream, s, zf, bias, d->act, d->scale,
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
  T *wc = dXt ? sp.weights<T>(ws) : nullptr, *xc = dW ? sp.inputs<T>(ws) : nullptr;
  hipLaunchKernelGGL((glu_derive_kernel<T, G>), unit_grid(s.N), dim3(256), 0, stream, s, static_cast<const T*>(Zt),
                     static_cast<const T*>(dHt), static_cast<const T*>(Xt), static_cast<const T*>(W), d->act, d->scale,
                     reinterpret_cast<T*>(ws), static_cast<G*>(dW), dbias, xc, wc);
  ARD_LAUNCH_CHECK();
  if (s.kept == 0) {  // nothing is kept: nothing depends on the input
    if (dXt) ARD_HIP_CHECK(fill_zero(dXt, static_cast<size_t>(s.K) * s.B * s.es, stream));
  } else {
    GemmArgs g = {};
    if (dXt) {
      g.M = s.K, g.N = s.B, g.K = s.kept, g.kbatch = 2;
      g.a = kept_weights(s, W, wc);
      g.b = plain(ws, s.ldd, half);
      g.c.p = dXt, g.c.ld = s.B;
      ARD_HIP_CHECK((product<T, true, true, T>(g, 1, stream, part, sp.part / 4)));
    }
    if (dW) {
      g = {};
      g.M = s.kept, g.N = s.K, g.K = s.B;
      g.a = plain(ws, s.ldd, half);
      g.b = xc ? plain(xc, s.ldd, 0) : plain(Xt, s.B, 0);
      g.c.p = static_cast<G*>(dW) + static_cast<int64_t>(s.offset) * s.K;
      g.c.ld = static_cast<int64_t>(s.K) * s.period;
      g.c.bstride = static_cast<int64_t>(s.N) * s.K;
      ARD_HIP_CHECK((product<T, false, false, G>(g, 2, stream, part, sp.part / 4)));
    }
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
