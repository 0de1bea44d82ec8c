// Softmax cross entropy of a head layer whose logits are never kept:
//   z = W x + b,  loss = log sum_v exp z_v - z_label
//   dz = (exp z / sum - onehot) dloss,  dX = W^T dz,  dW = dz X^T,  db = sum_b dz
//
// Forward: a product whose epilogue reduces each tile's logits to a maximum and a sum of
// exponentials a column; the tiles' pairs are joined by a second, small kernel. Backward:
// the classes in pieces; the same product with an epilogue that writes dz of a piece
// (rounded once, the operand of two products; its row sums, the bias gradient, are taken
// before that), then dX and dW from it. A piece's dz is a few ten MB, so that the products
// find it in the memory-side cache. Logits are fp32 throughout.
//
// Columns without a label contribute nothing: their loss and dz are 0, and the inputs that
// meet their dz in dW are 0 too, whatever they hold.
//
// Bound by the matrix cores for many columns, by reading W for few.

#include "ard_train.hpp"

namespace ard {
namespace {

// exp of a value <= 0; see the forward's roundings: bf16 logits are sums of products of
// values with 8 bits, for which the hardware's power of two is exact enough by far.
template <typename T>
__device__ __forceinline__ float exp_neg(float x) {
  if constexpr (sizeof(T) == 2)
    return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
  else
    return expf(x);
}

constexpr float kInf = __builtin_inff();

// A maximum and the sum of exp(z - maximum), the maximum taken as 0 while it is -inf. NaN
// stays in the sum.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ float safe(float m) { return m == -kInf ? 0.0f : m; }
template <typename T>
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m), t = safe(m);
  return {m, a.s * exp_neg<T>(a.m - t) + b.s * exp_neg<T>(b.m - t)};
}

struct HeadShape {
  int32_t B, V;
  Kept in;
  int64_t ldp;       // row length of dz and of X's copy
  int64_t ldc;       // row length of W's copy
  size_t es;
  bool input_major;  // W^T[K][V]
  bool zero;         // gradients of dropped inputs are written 0
  bool copy_w;       // output-major weights of kept inputs, or with rows off 16 bytes, are copied
  bool copy_x;       // so is X with rows off 16 bytes in the forward (always in the backward)
};

struct TileArgs {
  int64_t M;             // classes of the launch, the first of them is class0
  int64_t class0;
  int32_t B, K;
  const void* W;         // the launch's first class; rows of ldw
  const void* X;         // rows of ldx
  int64_t ldw, ldx;
  const float* bias;     // of the launch's first class, or NULL
  const int32_t* labels;
  int32_t classes;
  // forward
  float2* part;          // [tile rows][B] maxima and sums
  float* zlabel;         // [B]
  // backward
  const float* stats;    // [2][B]: maximum, 1 / sum
  const float* dloss;    // [B] or NULL
  void* P;               // [M][ldp]
  int64_t ldp;
  float* dbias;          // [parts][classes] row sums from the launch's first class on, or NULL
};

enum Way { WAY_LOSS, WAY_GRAD };

template <class Cfg>
struct HeadLds {
  // the epilogue's staging: bias of the rows and four values of the columns, then the maxima and sums of the
  // waves, or 32 rows of dz of each wave
  static constexpr int HEAD = (Cfg::BM + 4 * Cfg::BN) * 4;
  static constexpr int ROW = Cfg::TN * 4 + 32;
  static constexpr int SUMS = Cfg::WGM * Cfg::BN * 8, STAGE = Cfg::NW * 32 * ROW;
  // waves that split k: their accumulators, then the tile's logits
  static constexpr int RED = Cfg::KSPLIT > 1 ? Cfg::NW * Cfg::FM * Cfg::FN * 16 * 64 * 4 : 0;
  static constexpr int ZT = Cfg::KSPLIT > 1 ? Cfg::BM * (Cfg::BN + 1) * 4 + Cfg::NT * 8 : 0;
  static constexpr int one(int way) {
    return Cfg::KSPLIT > 1 ? HEAD + (RED > ZT ? RED : ZT) + ZT : HEAD + (way == WAY_LOSS ? SUMS : STAGE);
  }
  static constexpr int bytes(int way, int ld) {
    const int main = ld == LOAD_ANY ? 2 * Cfg::STAGE : Cfg::LDS;
    return one(way) > main ? one(way) : main;
  }
};

template <class Cfg, bool AMC, int LD, int WAY>
__global__ void __launch_bounds__(Cfg::NT) head_tile_kernel(TileArgs g) {
  using T = typename Cfg::T;
  constexpr int ES = Cfg::ES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int nx = (g.B + Cfg::BN - 1) / Cfg::BN;
  const int ny = static_cast<int>((g.M + Cfg::BM - 1) / Cfg::BM);
  const int64_t bid = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
  if (bid >= static_cast<int64_t>(nx) * ny) return;
  int tile_row, tile_col;
  grouped_tile(static_cast<int>(bid), nx, ny, tile_row, tile_col);
  const int64_t m0 = static_cast<int64_t>(tile_row) * Cfg::BM, n0 = static_cast<int64_t>(tile_col) * Cfg::BN;
  const int rows = static_cast<int>(min<int64_t>(g.M - m0, Cfg::BM)), cols = static_cast<int>(min<int64_t>(g.B - n0, Cfg::BN));
  const int wave = threadIdx.x >> 6, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ks = wave / (Cfg::WGM * Cfg::WGN), wmn = wave % (Cfg::WGM * Cfg::WGN);
  const int wm = wmn / Cfg::WGN, wn = wmn % Cfg::WGN;
  f32x16 acc[Cfg::FM][Cfg::FN];
#pragma unroll
  for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  // the tile's first class and column go into the 64-bit bases, so that offsets stay within the tile
  const int nslab = (g.K + Cfg::BK - 1) / Cfg::BK;
  const char* wp = static_cast<const char*>(g.W) + (AMC ? m0 : m0 * g.ldw) * ES;
  const char* xp = static_cast<const char*>(g.X) + n0 * ES;
  {
    using Loader = typename std::conditional<LD == LOAD_ANY, RegLoader<Cfg, AMC, true>, SlabLoader<Cfg, AMC, true>>::type;
    Loader ld;
    ld.wv = wv;
    ld.da.init(g.ldw, 0, rows, wv);
    ld.db.init(g.ldx, 0, cols, wv);
    ld.K = g.K;
    ld.ik = 0;
    ld.a_step = (AMC ? g.ldw : 1) * Cfg::BK * ES;
    ld.b_step = g.ldx * Cfg::BK * ES;
    ld.a_wrap = ld.b_wrap = 0;
    ld.na = uniform_ptr(wp);
    ld.nb = uniform_ptr(xp);
    if constexpr (LD == LOAD_ANY) {
      run_slabs_reg<Cfg, AMC, true, false>(ld, nslab, acc, wm, wn, ks * Cfg::KW, smem, nullptr);
    } else {
      ld.lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem));
      ld.is = 0;
      ld.left = nslab - 1;
      run_slabs<Cfg, AMC, true, true, false>(ld, nslab, g.K, 0, acc, wm, wn, ks * Cfg::KW, smem);
    }
  }

  // what the epilogue knows of its rows and columns
  using L = HeadLds<Cfg>;
  const int t = static_cast<int>(threadIdx.x), lane = t & 63, lr = lane & 31, lh = lane >> 5;
  float* bl = reinterpret_cast<float*>(smem);
  int* label = reinterpret_cast<int*>(bl + Cfg::BM);   // the label's row of the tile; -1: in another tile; -2: no label
  float* cm = reinterpret_cast<float*>(label + Cfg::BN);
  float* cg = cm + Cfg::BN;
  float* cd = cg + Cfg::BN;
  char* stage = smem + L::HEAD;
  __syncthreads();  // every wave is done with the stages
  for (int e = t; e < Cfg::BM; e += Cfg::NT) bl[e] = g.bias && e < rows ? g.bias[m0 + e] : 0.0f;
  for (int e = t; e < Cfg::BN; e += Cfg::NT) {
    int l = -2;
    if (e < cols) {
      const int64_t n = n0 + e, at = g.labels ? g.labels[n] : -1;
      if (at >= 0 && at < g.classes) l = at >= g.class0 + m0 && at < g.class0 + m0 + rows ? static_cast<int>(at - g.class0 - m0) : -1;
      if constexpr (WAY == WAY_GRAD) {
        const float inv = g.stats[g.B + n], d = g.dloss ? g.dloss[n] : 1.0f;
        if (inv == 0.0f) l = -2;  // every class masked
        cm[e] = g.stats[n];
        cg[e] = inv * d;
        cd[e] = d;
      }
    }
    label[e] = l;
  }

  // dz of a logit
  auto dz = [&](float z, int row, int col) {
    const int l = label[col];
    float p = exp_neg<T>(z - cm[col]) * cg[col];
    if (row == l) p -= cd[col];
    return l == -2 ? 0.0f : p;
  };

  if constexpr (Cfg::KSPLIT == 1) {
    __syncthreads();
    auto row_of = [&](int i, int r) { return wm * Cfg::TM + 32 * i + 8 * (r >> 2) + 4 * lh + (r & 3); };
    if constexpr (WAY == WAY_LOSS) {
      MaxSum* sums = reinterpret_cast<MaxSum*>(stage);
#pragma unroll
      for (int j = 0; j < Cfg::FN; ++j) {
        const int col = wn * Cfg::TN + 32 * j + lr, l = label[col];
        float m = -kInf, zl = 0.0f, s = 0.0f;
#pragma unroll
        for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = row_of(i, r);
            const float z = row < rows ? acc[i][j][r] + bl[row] : -kInf;
            acc[i][j][r] = z;
            m = fmaxf(m, z);
            zl = row == l ? z : zl;
          }
        const float mm = safe(m);
#pragma unroll
        for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) s += exp_neg<T>(acc[i][j][r] - mm);
        // the lane whose rows hold the label
        const int lw = l - wm * Cfg::TM;
        if (l >= 0 && lw >= 0 && lw < Cfg::TM && ((lw >> 2) & 1) == lh) g.zlabel[n0 + col] = zl;
        const MaxSum both = merge<T>({m, s}, {__shfl_xor(m, 32), __shfl_xor(s, 32)});
        if (lh == 0) sums[wm * Cfg::BN + col] = both;
      }
      __syncthreads();
      for (int c = t; c < cols; c += Cfg::NT) {
        MaxSum v = sums[c];
#pragma unroll
        for (int w = 1; w < Cfg::WGM; ++w) v = merge<T>(v, sums[w * Cfg::BN + c]);
        g.part[tile_row * static_cast<int64_t>(g.B) + n0 + c] = float2{v.m, v.s};
      }
    } else {
      // 32 rows of a wave at a time through its own LDS, then 16 bytes of a row a lane
      constexpr int VE = 16 / ES, CPRW = Cfg::TN / VE, RPI = 64 / CPRW;
      char* region = stage + wave * 32 * L::ROW;
#pragma unroll
      for (int i = 0; i < Cfg::FM; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = row_of(i, r), rl = row - wm * Cfg::TM - 32 * i;
          const float b = bl[row];
#pragma unroll
          for (int j = 0; j < Cfg::FN; ++j)
            *reinterpret_cast<float*>(region + rl * L::ROW + (32 * j + lr) * 4) =
                dz(acc[i][j][r] + b, row, wn * Cfg::TN + 32 * j + lr);
        }
#pragma unroll
        for (int q = 0; q < 32 / RPI; ++q) {
          const int rl = lane / CPRW + RPI * q, ch = lane % CPRW, row = wm * Cfg::TM + 32 * i + rl;
          const float* from = reinterpret_cast<const float*>(region + rl * L::ROW) + ch * VE;
          float v[VE], sum = 0.0f;
#pragma unroll
          for (int e = 0; e < VE; ++e) v[e] = from[e], sum += v[e];
#pragma unroll
          for (int o = CPRW / 2; o > 0; o >>= 1) sum += __shfl_down(sum, o, CPRW);
          if (row >= rows) continue;
          const int c = wn * Cfg::TN + ch * VE;
          if (n0 + c < g.ldp) {
            T w[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) w[e] = from_f32<T>(v[e]);
            *reinterpret_cast<u32x4_any*>(static_cast<T*>(g.P) + (m0 + row) * g.ldp + n0 + c) =
                *reinterpret_cast<const u32x4_any*>(w);
          }
          if (g.dbias && ch == 0)
            g.dbias[(static_cast<int64_t>(tile_col) * Cfg::WGN + wn) * g.classes + m0 + row] = sum;
        }
      }
    }
  } else {
    // the waves' shares of k meet in LDS, then the tile's logits lie there
    constexpr int NREG = Cfg::FM * Cfg::FN * 16, ZLD = Cfg::BN + 1;
    float* red = reinterpret_cast<float*>(stage);
    float* zt = reinterpret_cast<float*>(stage + (L::RED > L::ZT ? L::RED : L::ZT));
#pragma unroll
    for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
      for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) red[(wave * NREG + (i * Cfg::FN + j) * 16 + r) * 64 + lane] = acc[i][j][r];
    __syncthreads();
#pragma unroll
    for (int q = ks; q < NREG; q += Cfg::KSPLIT) {
      const int i = q / (Cfg::FN * 16), j = (q / 16) % Cfg::FN, r = q % 16;
      float v = 0.0f;
#pragma unroll
      for (int u = 0; u < Cfg::KSPLIT; ++u) v += red[((u * Cfg::WGM * Cfg::WGN + wmn) * NREG + q) * 64 + lane];
      const int row = wm * Cfg::TM + 32 * i + 8 * (r >> 2) + 4 * lh + (r & 3);
      zt[row * ZLD + wn * Cfg::TN + 32 * j + lr] = v + bl[row];
    }
    __syncthreads();
    constexpr int PARTS = Cfg::NT / Cfg::BN;
    const int col = t % Cfg::BN, part = t / Cfg::BN;
    if constexpr (WAY == WAY_LOSS) {
      MaxSum* sums = reinterpret_cast<MaxSum*>(red);
      float m = -kInf, s = 0.0f;
      for (int row = part; row < rows; row += PARTS) m = fmaxf(m, zt[row * ZLD + col]);
      const float mm = safe(m);
      for (int row = part; row < rows; row += PARTS) s += exp_neg<T>(zt[row * ZLD + col] - mm);
      sums[part * Cfg::BN + col] = {m, s};
      __syncthreads();
      if (t < cols) {
        MaxSum v = sums[t];
        for (int q = 1; q < PARTS; ++q) v = merge<T>(v, sums[q * Cfg::BN + t]);
        g.part[tile_row * static_cast<int64_t>(g.B) + n0 + t] = float2{v.m, v.s};
        if (label[t] >= 0) g.zlabel[n0 + t] = zt[label[t] * ZLD + t];
      }
    } else {
      for (int row = part; row < rows; row += PARTS) {
        const float p = dz(zt[row * ZLD + col], row, col);
        zt[row * ZLD + col] = p;
        if (n0 + col < g.ldp) static_cast<T*>(g.P)[(m0 + row) * g.ldp + n0 + col] = from_f32<T>(p);
      }
      __syncthreads();
      if (g.dbias && t < rows) {
        float sum = 0.0f;
        for (int c = 0; c < Cfg::BN; ++c) sum += zt[t * ZLD + c];
        g.dbias[static_cast<int64_t>(tile_col) * g.classes + m0 + t] = sum;
      }
    }
  }
}

// The tiles' pairs of a column, joined: 16 columns of a workgroup, 16 runs of tile rows each.
template <typename T>
__global__ void __launch_bounds__(256) head_join_kernel(const float2* __restrict__ part, const float* __restrict__ zlabel,
                                                        const int32_t* __restrict__ labels, int32_t B, int32_t classes,
                                                        int64_t tile_rows, float* __restrict__ loss,
                                                        float* __restrict__ stats) {
  __shared__ MaxSum sums[16][17];
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4;
  const int64_t n = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 16 + c;
  MaxSum v = {-kInf, 0.0f};
  if (n < B)
    for (int64_t r = q; r < tile_rows; r += 16) {
      const float2 p = part[r * B + n];
      v = merge<T>(v, {p.x, p.y});
    }
  sums[q][c] = v;
  __syncthreads();
  if (q != 0 || n >= B) return;
  for (int w = 1; w < 16; ++w) v = merge<T>(v, sums[w][c]);
  const int32_t l = labels ? labels[n] : -1;
  const bool on = l >= 0 && l < classes && v.s != 0.0f;  // a sum of 0: every class is masked
  loss[n] = on ? logf(v.s) - (zlabel[n] - safe(v.m)) : 0.0f;
  if (stats) {
    stats[n] = safe(v.m);
    stats[B + n] = v.s != 0.0f ? 1.0f / v.s : 0.0f;
  }
}

// The kept rows of X with rows of ldp; columns without a label are 0 where they meet dz.
template <typename T>
__global__ void __launch_bounds__(256) head_columns_kernel(const T* __restrict__ X, const int32_t* __restrict__ labels,
                                                           int32_t classes, int32_t B, Kept in, int64_t ldp,
                                                           T* __restrict__ Xc) {
  constexpr int E = 16 / static_cast<int>(sizeof(T));
  const int64_t per = ldp / E, total = per * in.kept, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < total; at += step) {
    const int64_t i = at / per, b = (at - i * per) * E;
    const T* from = X + (in.offset + i * in.period) * B + b;
    const int n = static_cast<int>(min<int64_t>(E, B - b));
    u32x4 v = {0u, 0u, 0u, 0u};
    if (n > 0) {
      Chunk<T, E> c;
      c.load(from, n);
      v = c.raw;
      if (classes > 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int32_t l = e < n && labels ? labels[b + e] : -1;
          if (l >= 0 && l < classes) continue;
          if constexpr (sizeof(T) == 2)
            v[e / 2] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
          else
            v[e] = 0u;
        }
      }
    }
    *reinterpret_cast<u32x4_any*>(Xc + i * ldp + b) = v;
  }
}

// dbias from the parts of the tile columns, in their order.
__global__ void __launch_bounds__(256) head_bias_kernel(const float* __restrict__ part, int32_t parts, int32_t classes,
                                                        float* __restrict__ dbias) {
  const int64_t v = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (v >= classes) return;
  float sum = 0.0f;
  for (int q = 0; q < parts; ++q) sum += part[static_cast<int64_t>(q) * classes + v];
  dbias[v] = sum;
}

// dX of the pieces: the first is kept in fp32, the next are added, the last is written out.
template <typename T>
__global__ void __launch_bounds__(256) head_add_kernel(float* __restrict__ all, const float* __restrict__ piece, int32_t B,
                                                       Kept in, T* __restrict__ dX) {
  const int64_t total = static_cast<int64_t>(in.kept) * B, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < total; at += step) {
    const float v = all[at] + piece[at];
    if (dX) {
      const int64_t i = at / B;
      dX[(in.offset + i * in.period) * B + (at - i * B)] = from_f32<T>(v);
    } else {
      all[at] = v;
    }
  }
}

// Zeros in the rows (by columns: the columns) of dropped inputs of an array of rows x cols.
template <typename T>
__global__ void __launch_bounds__(256) head_clear_kernel(T* __restrict__ p, int64_t rows, int64_t cols, Kept in,
                                                         bool by_columns) {
  const int64_t total = rows * cols, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < total; at += step) {
    const int64_t r = at / cols, x = by_columns ? at - r * cols : r;
    if (static_cast<int32_t>(x % in.period) != in.offset) p[at] = from_f32<T>(0.0f);
  }
}

unsigned sweep(int64_t n) { return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(4096, (n + 255) / 256))); }

// ------------------------------------------------------------------ host
int check_desc(const ard_headloss_desc* d, HeadShape* s) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->batch < 1 || d->in_features < 1 || d->classes < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (batch %d, in %d, classes %d)", d->batch, d->in_features, d->classes);
  if (d->weight_layout != ARD_WEIGHTS_FULL && d->weight_layout != ARD_WEIGHTS_INPUT_MAJOR)
    return fail(ARD_ERR_INVALID_ARG, "weight layout %d: ARD_WEIGHTS_FULL or ARD_WEIGHTS_INPUT_MAJOR", d->weight_layout);
  if (d->dropped != ARD_DROPPED_ZERO && d->dropped != ARD_DROPPED_SKIP)
    return fail(ARD_ERR_INVALID_ARG, "unknown dropped-input mode %d", d->dropped);
  if (d->grad_dtype != ARD_F32 && d->grad_dtype != d->dtype)
    return fail(ARD_ERR_INVALID_ARG, "grad_dtype must be ARD_F32 or dtype");
  const int st = check_row_plan(d->in_plan, d->in_features, "in_plan", false);
  if (st != ARD_OK) return st;
  s->B = d->batch;
  s->V = d->classes;
  s->in = kept_of(d->in_plan, d->in_features);
  s->ldp = up8(s->B);
  s->ldc = up8(s->in.kept);
  s->es = d->dtype == ARD_BF16 ? 2 : 4;
  s->input_major = d->weight_layout == ARD_WEIGHTS_INPUT_MAJOR;
  s->zero = d->dropped == ARD_DROPPED_ZERO;
  s->copy_w = s->in.kept > 0 && !s->input_major && (s->in.period > 1 || s->in.n * s->es % 16);
  s->copy_x = s->in.kept > 0 && s->B * s->es % 16;
  return ARD_OK;
}

// The strides of the tile kernel's operands: offsets within a slab and a tile have 32 bits.
constexpr int64_t kMostStride = int64_t{1} << 22;
int check_strides(const HeadShape& s) {
  const int64_t x = s.copy_x ? s.ldp : static_cast<int64_t>(s.B) * s.in.period;
  const int64_t w = s.input_major ? static_cast<int64_t>(s.V) * s.in.period : s.copy_w ? s.ldc : s.in.n;
  if (x >= kMostStride || w >= kMostStride || s.ldp >= kMostStride)
    return fail(ARD_ERR_UNSUPPORTED, "rows of the inputs (%lld) and of the weights (%lld elements apart) must be below 2^22",
                static_cast<long long>(x), static_cast<long long>(w));
  if ((s.V / 32 + int64_t{1}) * (s.B / 32 + int64_t{1}) >= int64_t{1} << 31)  // tiles are counted in 32 bits
    return fail(ARD_ERR_UNSUPPORTED, "%d classes of %d columns are too many tiles", s.V, s.B);
  return ARD_OK;
}

bool any_rows(const HeadShape& s) { return s.input_major && s.V * s.es % 16; }  // weights off 16 bytes in place

// The tile with the least modelled time: rounds of the chip times a tile's work over the
// rate that it reaches with the chip full (bf16), or the layers' cost model (fp32).
template <typename T>
int plan_tile(const HeadShape& s, int64_t M) {
  const int64_t K = s.in.kept;
  int best = FAST_SMALL;
  double best_t = 1e300;
  if constexpr (sizeof(T) == 2) {
    using C = FastCfgs<bf16>;
    struct Tile {
      int kind, bm, bn, bk;
      double rate;
    };
    static constexpr Tile tiles[] = {{FAST_HUGE, 256, 256, C::Huge::BK, 4.2e12}, {FAST_WIDE, 128, 256, C::Wide::BK, 3.5e12},
                                     {FAST_TALL, 256, 128, C::Tall::BK, 3.4e12}, {FAST_BIG, 128, 128, C::Big::BK, 2.7e12},
                                     {FAST_SMALL, 32, 32, C::Small::BK, 0.5e12}};
    for (const Tile& c : tiles) {
      if (any_rows(s) && c.kind != FAST_BIG && c.kind != FAST_SMALL) continue;
      const int64_t n = (M + c.bm - 1) / c.bm * ((s.B + c.bn - 1) / c.bn), slabs = (K + c.bk - 1) / c.bk;
      const double occ = n < kTargetBlocks ? static_cast<double>(n) / kTargetBlocks : 1.0;
      const double t = static_cast<double>((n + kTargetBlocks - 1) / kTargetBlocks) * 2.0 * c.bm * c.bn * c.bk * slabs /
                       (c.rate * (1.0 + 0.3 * (1.0 - occ)));
      if (t < best_t) best_t = t, best = c.kind;
    }
  } else {
    for (const CostF32& c : any_rows(s) ? kCostRegF32[1] : kCostF32) {
      if (c.kind != FAST_HUGE && c.kind != FAST_MID && c.kind != FAST_SMALL) continue;
      if (any_rows(s) && c.kind == FAST_HUGE) continue;
      const double t = time_f32(c, tile_f32(c.kind), static_cast<int>(M), s.B, static_cast<int>(K), 1, 1, 1);
      if (t < best_t) best_t = t, best = c.kind;
    }
  }
  return best;
}

struct TileDims {
  int bm, bn, wgn;
};
template <typename T>
TileDims dims_of(int kind) {
  auto of = [](auto cfg) {
    using C = decltype(cfg);
    return TileDims{C::BM, C::BN, C::KSPLIT == 1 ? C::WGN : 1};
  };
  using C = FastCfgs<T>;
  if (kind == FAST_HUGE) return of(typename C::Huge{});
  if constexpr (sizeof(T) == 2) {
    if (kind == FAST_WIDE) return of(typename C::Wide{});
    if (kind == FAST_TALL) return of(typename C::Tall{});
    if (kind == FAST_BIG) return of(typename C::Big{});
  } else {
    if (kind == FAST_MID) return of(typename C::Mid{});
  }
  return of(typename C::Small{});
}

template <class Cfg, bool AMC, int LD, int WAY>
hipError_t launch_tile(const TileArgs& g, hipStream_t stream) {
  auto kern = head_tile_kernel<Cfg, AMC, LD, WAY>;
  constexpr int LDS = HeadLds<Cfg>::bytes(WAY, LD);
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return attr;
  const int64_t tiles = (g.M + Cfg::BM - 1) / Cfg::BM * ((g.B + Cfg::BN - 1) / Cfg::BN);
  constexpr int64_t kRow = 1 << 20;  // workgroups of a grid row: the threads along x have to stay below 2^32
  const dim3 grid(static_cast<unsigned>(std::min(tiles, kRow)), static_cast<unsigned>((tiles - 1) / kRow + 1));
  hipLaunchKernelGGL(kern, grid, dim3(Cfg::NT), LDS, stream, g);
  return hipGetLastError();
}

template <typename T, int WAY>
hipError_t run_tile(const HeadShape& s, int kind, const TileArgs& g, hipStream_t stream) {
  using C = FastCfgs<T>;
  auto go = [&](auto cfg) {
    using Cfg = decltype(cfg);
    return s.input_major ? launch_tile<Cfg, true, LOAD_DMA, WAY>(g, stream) : launch_tile<Cfg, false, LOAD_DMA, WAY>(g, stream);
  };
  if (any_rows(s)) {
    if constexpr (sizeof(T) == 2) {
      if (kind == FAST_BIG) return launch_tile<typename C::Big, true, LOAD_ANY, WAY>(g, stream);
    } else {
      if (kind == FAST_MID) return launch_tile<typename C::Mid, true, LOAD_ANY, WAY>(g, stream);
    }
    return launch_tile<typename C::Small, true, LOAD_ANY, WAY>(g, stream);
  }
  if (kind == FAST_HUGE) return go(typename C::Huge{});
  if constexpr (sizeof(T) == 2) {
    if (kind == FAST_WIDE) return go(typename C::Wide{});
    if (kind == FAST_TALL) return go(typename C::Tall{});
    if (kind == FAST_BIG) return go(typename C::Big{});
  } else {
    if (kind == FAST_MID) return go(typename C::Mid{});
  }
  return go(typename C::Small{});
}

// Classes of a piece of the backward: dz of at most 128 MB, whole tiles.
int64_t piece_of(const HeadShape& s) {
  const int64_t most = std::max<int64_t>(256, (int64_t{128} << 20) / (s.ldp * static_cast<int64_t>(s.es)) / 256 * 256);
  const int64_t pieces = (s.V + most - 1) / most;
  return std::min<int64_t>(s.V, ((s.V + pieces - 1) / pieces + 255) / 256 * 256);
}

// The workspace. fwd: copies, the tiles' pairs, the labels' logits. bwd: copies, dz of a piece, row sums, dX of the
// pieces, the products' partial sums.
struct FwdSpace {
  size_t wc, xc, part, zl;
  size_t bytes() const { return wc + xc + part + zl; }
};
struct BwdSpace {
  size_t wc, xc, p, db, dx, part;
  size_t bytes() const { return wc + xc + p + db + 2 * dx + part; }
};
template <typename T>
FwdSpace fwd_space(const HeadShape& s) {
  const TileDims t = dims_of<T>(plan_tile<T>(s, s.V));
  return {s.copy_w ? al256(static_cast<size_t>(s.V) * s.ldc * s.es) : 0,
          s.copy_x ? al256(static_cast<size_t>(s.in.kept) * s.ldp * s.es) : 0,
          al256(static_cast<size_t>((s.V + t.bm - 1) / t.bm) * s.B * 8), al256(static_cast<size_t>(s.B) * 4)};
}
template <typename T>
BwdSpace bwd_space(const HeadShape& s) {
  const int64_t piece = piece_of(s);
  const TileDims t = dims_of<T>(plan_tile<T>(s, piece));
  const int m = static_cast<int>(piece), last = static_cast<int>(s.V - (s.V - 1) / piece * piece), k = s.in.kept;
  size_t part = 0;
  if (k > 0)
    for (int v : {m, last}) {
      part = std::max(part, partial_floats<T>(k, s.B, v));
      part = std::max(part, s.input_major ? partial_floats<T>(k, v, s.B) : partial_floats<T>(v, k, s.B));
    }
  return {s.copy_w ? al256(static_cast<size_t>(s.V) * s.ldc * s.es) : 0, al256(static_cast<size_t>(k) * s.ldp * s.es),
          al256(static_cast<size_t>(piece) * s.ldp * s.es),
          al256(static_cast<size_t>((s.B + t.bn - 1) / t.bn) * t.wgn * s.V * 4),
          piece < s.V ? al256(static_cast<size_t>(k) * s.B * 4) : 0, al256(4 * part)};
}

// The operands of the tile kernel from class v on.
template <typename T>
void tile_operands(const HeadShape& s, const void* W, const char* wc, const void* X, const char* xc, TileArgs* g) {
  g->B = s.B;
  g->K = s.in.kept;
  g->classes = s.V;
  if (s.input_major) {
    g->W = static_cast<const T*>(W) + static_cast<int64_t>(s.in.offset) * s.V;
    g->ldw = static_cast<int64_t>(s.V) * s.in.period;
  } else {
    g->W = s.copy_w ? static_cast<const void*>(wc) : W;
    g->ldw = s.copy_w ? s.ldc : s.in.n;
  }
  g->X = xc ? static_cast<const void*>(xc) : static_cast<const T*>(X) + static_cast<int64_t>(s.in.offset) * s.B;
  g->ldx = xc ? s.ldp : static_cast<int64_t>(s.B) * s.in.period;
}

int copy_weights(const ard_headloss_desc* d, const HeadShape& s, const void* W, char* wc, void* stream) {
  if (!s.copy_w) return ARD_OK;
  ard_fc_desc fc = {};
  fc.dtype = d->dtype;
  fc.batch = 1;
  fc.in_features = s.in.n;
  fc.out_features = s.V;
  fc.in_plan = d->in_plan;
  fc.scale = 1.0f;
  return ard_fc_compact_weights(&fc, W, wc, stream);
}

template <typename T>
int copy_columns(const HeadShape& s, const void* X, const int32_t* labels, bool mask, char* xc, hipStream_t stream) {
  if (s.in.kept == 0) return ARD_OK;
  hipLaunchKernelGGL(head_columns_kernel<T>, dim3(sweep(s.in.kept * (s.ldp * static_cast<int64_t>(s.es) / 16))), dim3(256), 0,
                     stream, static_cast<const T*>(X), labels, mask ? s.V : 0, s.B, s.in, s.ldp, reinterpret_cast<T*>(xc));
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T>
int fwd_impl(const ard_headloss_desc* d, const HeadShape& s, const void* Xt, const void* W, const float* bias,
             const int32_t* labels, float* loss, float* stats, char* ws, hipStream_t stream) {
  const FwdSpace sp = fwd_space<T>(s);
  char *wc = ws, *xc = wc + sp.wc, *part = xc + sp.xc, *zl = part + sp.part;
  int st = copy_weights(d, s, W, wc, stream);
  if (st != ARD_OK) return st;
  if (s.copy_x && (st = copy_columns<T>(s, Xt, labels, false, xc, stream)) != ARD_OK) return st;
  TileArgs g = {};
  tile_operands<T>(s, W, wc, Xt, s.copy_x ? xc : nullptr, &g);
  g.M = s.V;
  g.bias = bias;
  g.labels = labels;
  g.part = reinterpret_cast<float2*>(part);
  g.zlabel = reinterpret_cast<float*>(zl);
  const int kind = plan_tile<T>(s, s.V);
  ARD_HIP_CHECK((run_tile<T, WAY_LOSS>(s, kind, g, stream)));
  const int64_t groups = (static_cast<int64_t>(s.B) + 15) / 16;
  const int bm = dims_of<T>(kind).bm;
  hipLaunchKernelGGL(head_join_kernel<T>, dim3(static_cast<unsigned>(groups)), dim3(256), 0, stream, g.part, g.zlabel, labels,
                     s.B, s.V, (static_cast<int64_t>(s.V) + bm - 1) / bm, loss, stats);
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

template <typename T, typename G>
int bwd_impl(const ard_headloss_desc* d, const HeadShape& s, const void* Xt, const void* W, const float* bias,
             const int32_t* labels, const float* stats, const float* dloss, void* dXt, void* dW, float* dbias, char* ws,
             hipStream_t stream) {
  const BwdSpace sp = bwd_space<T>(s);
  char *wc = ws, *xc = wc + sp.wc, *p = xc + sp.xc, *db = p + sp.p, *all = db + sp.db, *one = all + sp.dx, *pt = one + sp.dx;
  float* partial = reinterpret_cast<float*>(pt);
  int st = copy_weights(d, s, W, wc, stream);
  if (st != ARD_OK) return st;
  if ((st = copy_columns<T>(s, Xt, labels, true, xc, stream)) != ARD_OK) return st;
  const int64_t piece = piece_of(s), K = s.in.n, kin = s.in.kept;
  const int kind = plan_tile<T>(s, piece);
  const TileDims td = dims_of<T>(kind);
  TileArgs base = {};
  tile_operands<T>(s, W, wc, Xt, xc, &base);
  base.labels = labels;
  base.stats = stats;
  base.dloss = dloss;
  base.P = p;
  base.ldp = s.ldp;
  for (int64_t v = 0; v < s.V; v += piece) {
    TileArgs g = base;
    g.M = std::min<int64_t>(piece, s.V - v);
    g.class0 = v;
    g.W = static_cast<const T*>(base.W) + (s.input_major ? v : v * base.ldw);
    g.bias = bias ? bias + v : nullptr;
    g.dbias = dbias ? reinterpret_cast<float*>(db) + v : nullptr;
    ARD_HIP_CHECK((run_tile<T, WAY_GRAD>(s, kind, g, stream)));
    if (dXt && kin > 0) {
      GemmArgs q = {};
      q.M = static_cast<int>(kin), q.N = s.B, q.K = static_cast<int>(g.M);
      q.a = view(g.W, g.ldw);
      q.b = view(p, s.ldp);
      const bool whole = piece >= s.V;
      if (whole) {
        q.c.p = static_cast<T*>(dXt) + static_cast<int64_t>(s.in.offset) * s.B;
        q.c.ld = static_cast<int64_t>(s.B) * s.in.period;
        ARD_HIP_CHECK((s.input_major ? product<T, false, true, T>(q, stream, partial, sp.part / 4)
                                     : product<T, true, true, T>(q, stream, partial, sp.part / 4)));
      } else {
        q.c.p = v == 0 ? all : one;
        q.c.ld = s.B;
        ARD_HIP_CHECK((s.input_major ? product<T, false, true, float>(q, stream, partial, sp.part / 4)
                                     : product<T, true, true, float>(q, stream, partial, sp.part / 4)));
        if (v > 0) {
          hipLaunchKernelGGL(head_add_kernel<T>, dim3(sweep(kin * s.B)), dim3(256), 0, stream, reinterpret_cast<float*>(all),
                             reinterpret_cast<const float*>(one), s.B, s.in, v + piece >= s.V ? static_cast<T*>(dXt) : nullptr);
          ARD_LAUNCH_CHECK();
        }
      }
    }
    if (dW && kin > 0) {
      GemmArgs q = {};
      const GemmOperand dz = view(p, s.ldp), x = view(xc, s.ldp);
      if (s.input_major) {
        q.M = static_cast<int>(kin), q.N = static_cast<int>(g.M), q.K = s.B;
        q.a = x, q.b = dz;
        q.c.p = static_cast<G*>(dW) + static_cast<int64_t>(s.in.offset) * s.V + v;
        q.c.ld = static_cast<int64_t>(s.V) * s.in.period;
      } else {
        q.M = static_cast<int>(g.M), q.N = static_cast<int>(kin), q.K = s.B;
        q.a = dz, q.b = x;
        q.c.p = static_cast<G*>(dW) + v * K + s.in.offset;
        q.c.ld = K;
        q.c.col_stride = s.in.period;
      }
      ARD_HIP_CHECK((product<T, false, false, G>(q, stream, partial, sp.part / 4)));
    }
  }
  if (dbias) {
    const int parts = static_cast<int>((s.B + td.bn - 1) / td.bn) * td.wgn;
    hipLaunchKernelGGL(head_bias_kernel, dim3(static_cast<unsigned>((static_cast<int64_t>(s.V) + 255) / 256)), dim3(256), 0, stream,
                       reinterpret_cast<const float*>(db), parts, s.V, dbias);
    ARD_LAUNCH_CHECK();
  }
  if (s.in.period > 1 && s.zero) {
    if (dXt) {
      hipLaunchKernelGGL(head_clear_kernel<T>, dim3(sweep(K * s.B)), dim3(256), 0, stream, static_cast<T*>(dXt), K,
                         static_cast<int64_t>(s.B), s.in, false);
      ARD_LAUNCH_CHECK();
    }
    if (dW) {
      hipLaunchKernelGGL(head_clear_kernel<G>, dim3(sweep(K * s.V)), dim3(256), 0, stream, static_cast<G*>(dW),
                         s.input_major ? K : s.V, s.input_major ? s.V : K, s.in, !s.input_major);
      ARD_LAUNCH_CHECK();
    }
  }
  return ARD_OK;
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

size_t ard_headloss_workspace_bytes(const ard_headloss_desc* desc) {
  HeadShape s;
  if (check_desc(desc, &s) != ARD_OK || check_strides(s) != ARD_OK) return 0;
  return desc->dtype == ARD_BF16 ? std::max(fwd_space<bf16>(s).bytes(), bwd_space<bf16>(s).bytes())
                                 : std::max(fwd_space<float>(s).bytes(), bwd_space<float>(s).bytes());
}

int ard_headloss_fwd(const ard_headloss_desc* desc, const void* Xt, const void* W, const float* bias, const int32_t* labels,
                     float* loss, float* stats, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HeadShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  if ((st = check_strides(s)) || (st = need_ptr(Xt, "Xt")) || (st = need_ptr(W, "W")) || (st = may_ptr(bias, "bias")) ||
      (st = need_ptr(labels, "labels")) || (st = need_ptr(loss, "loss")) || (st = may_ptr(stats, "stats")) ||
      (st = check_space(desc->dtype == ARD_BF16 ? fwd_space<bf16>(s).bytes() : fwd_space<float>(s).bytes(), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? fwd_impl<bf16>(desc, s, Xt, W, bias, labels, loss, stats, w, sm)
                                 : fwd_impl<float>(desc, s, Xt, W, bias, labels, loss, stats, w, sm);
}

int ard_headloss_bwd(const ard_headloss_desc* desc, const void* Xt, const void* W, const float* bias, const int32_t* labels,
                     const float* stats, const float* dloss, void* dXt, void* dW, float* dbias, void* ws, size_t ws_bytes,
                     void* stream) {
  clear_error();
  HeadShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  if ((st = check_strides(s)) || (st = need_ptr(Xt, "Xt")) || (st = need_ptr(W, "W")) || (st = may_ptr(bias, "bias")) ||
      (st = need_ptr(labels, "labels")) || (st = need_ptr(stats, "stats")) || (st = may_ptr(dloss, "dloss")) ||
      (st = may_ptr(dXt, "dXt")) || (st = may_ptr(dW, "dW")) || (st = may_ptr(dbias, "dbias")) ||
      (st = check_space(desc->dtype == ARD_BF16 ? bwd_space<bf16>(s).bytes() : bwd_space<float>(s).bytes(), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  if (desc->dtype == ARD_F32)
    return bwd_impl<float, float>(desc, s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm);
  return desc->grad_dtype == ARD_BF16 ? bwd_impl<bf16, bf16>(desc, s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm)
                                      : bwd_impl<bf16, float>(desc, s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm);
}

}  // extern "C"
