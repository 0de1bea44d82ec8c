// Softmax cross entropy of a head layer whose logits are never kept:
//   z = W x + b,  loss = log sum_v exp z_v - z_label
//   dz = (exp z / sum - onehot) dloss,  dX = W^T dz,  dW = dz X^T,  db = sum_b dz
//
// Forward: a product whose epilogue reduces each tile's logits to a maximum and a sum of
// exponentials a column; the tiles' pairs are joined by a second, small kernel. Backward:
// the classes in pieces; the same product with an epilogue that writes dz of a piece (the
// operand of two products; its row sums, the bias gradient, are taken before it is rounded
// for that), then dX and dW from it. Logits are fp32 throughout.
//
// bf16 operands are read in place where their rows start on 16 bytes, else from copies.
// fp32 operands, dz among them, are copied into three bf16 parts (ard_parts_gemm.hpp):
// exact to 2^-24 and, with six bf16 products for one, still faster than fp32 products (8800
// classes of 750 inputs, batch 700, forward and backward: 418 to 287 us). The rest of an
// infinite value is NaN: an infinite W or X makes NaN in its sums.
// A few classes take a kernel of their own (head_few_kernel) without any copy.
//
// Columns without a label contribute nothing: their loss and dz are 0, and the inputs that
// meet their dz in dW are 0 too, whatever they hold.
//
// Bound by the matrix cores for many columns, by reading W for few.

#include "ard_parts_gemm.hpp"

namespace ard {
namespace {

// exp of a value <= 0. With bf16 operands the hardware's power of two, one rounding off, of an
// argument that is off by 2^-24 of itself: no more than the logits' own sums are.
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
  int64_t wrows;     // its rows
  size_t es;
  bool input_major;  // W^T[K][V]
  bool zero;         // gradients of dropped inputs are written 0
  bool few;          // head_few_kernel
  bool parts;        // operands in parts
  bool copy_w, copy_x;  // the forward reads a copy of W, of X (the backward's X is always one)
};

struct TileArgs {
  int64_t M;             // classes of the launch, the first of them is class0
  int64_t class0;
  int32_t B, K;
  const void* W;         // the launch's first class; rows of ldw
  const void* X;         // rows of ldx
  int64_t ldw, ldx;
  int64_t wplane, xplane;  // elements from a part to the next
  const float* bias;     // of the launch's first class, or NULL
  const int32_t* labels;
  int32_t classes;
  // forward
  float2* part;          // [tile rows][B] maxima and sums
  float* zlabel;         // [B]
  // backward
  const float* stats;    // [2][B]: maximum, 1 / sum
  const float* dloss;    // [B] or NULL
  void* P;               // [M][ldp], in parts as W and X are
  int64_t ldp, pplane;
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
  static constexpr int bytes(int way) { return one(way) > Cfg::LDS ? one(way) : Cfg::LDS; }
};

// P parts of each operand, or (0) the operands themselves.
template <class Cfg, int P, bool AMC, int WAY>
__global__ void __launch_bounds__(Cfg::NT) head_tile_kernel(TileArgs g) {
  using T = typename std::conditional<P == 0, typename Cfg::T, float>::type;
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
    using Loader = typename std::conditional<P == 0, SlabLoader<Cfg, AMC, true>, PartsLoader<Cfg, AMC, true>>::type;
    Loader ld;
    ld.wv = wv;
    ld.da.init(g.ldw, 0, rows, wv);
    ld.db.init(g.ldx, 0, cols, wv);
    ld.K = g.K;
    ld.ik = 0;
    ld.a_step = (AMC ? g.ldw : 1) * Cfg::BK * ES;
    ld.b_step = g.ldx * Cfg::BK * ES;
    ld.na = uniform_ptr(wp);
    ld.nb = uniform_ptr(xp);
    ld.lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem));
    ld.is = 0;
    ld.left = nslab - 1;
    if constexpr (P == 0) {
      ld.a_wrap = ld.b_wrap = 0;
      run_slabs<Cfg, AMC, true, true, false>(ld, nslab, g.K, 0, acc, wm, wn, ks * Cfg::KW, smem);
    } else {
      ld.a_plane = g.wplane * ES;
      ld.b_plane = g.xplane * ES;
      run_parts<Cfg, AMC, true>(ld, nslab, g.K, 0, acc, wm, wn, ks * Cfg::KW, smem);
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
      constexpr int CPRW = Cfg::TN / 8, RPI = 64 / CPRW;
      char* region = stage + wave * 32 * L::ROW;
      auto put_sum = [&](int row, float sum) {
        g.dbias[(static_cast<int64_t>(tile_col) * Cfg::WGN + wn) * g.classes + m0 + row] = sum;
      };
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
        if constexpr (P == 0) {
#pragma unroll
          for (int q = 0; q < 32 / RPI; ++q) {
            const int rl = lane / CPRW + RPI * q, ch = lane % CPRW, row = wm * Cfg::TM + 32 * i + rl;
            const float* from = reinterpret_cast<const float*>(region + rl * L::ROW) + ch * 8;
            float v[8], sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = from[e], sum += v[e];
#pragma unroll
            for (int o = CPRW / 2; o > 0; o >>= 1) sum += __shfl_down(sum, o, CPRW);
            if (row >= rows) continue;
            const int64_t n = n0 + wn * Cfg::TN + ch * 8;
            if (n < g.ldp) store_parts<1>(static_cast<bf16*>(g.P) + (m0 + row) * g.ldp + n, 0, v);
            if (g.dbias && ch == 0) put_sum(row, sum);
          }
        } else {
          // a row's chunks are no power of two
#pragma unroll
          for (int e0 = 0; e0 < 32 * CPRW; e0 += 64) {
            const int rl = (e0 + lane) / CPRW, ch = (e0 + lane) % CPRW, row = wm * Cfg::TM + 32 * i + rl;
            const float* from = reinterpret_cast<const float*>(region + rl * L::ROW) + ch * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = from[e];
            const int64_t n = n0 + wn * Cfg::TN + ch * 8;
            if (row < rows && n < g.ldp) store_parts<P, true>(static_cast<bf16*>(g.P) + (m0 + row) * g.ldp + n, g.pplane, v);
          }
          const float* half = reinterpret_cast<const float*>(region + lr * L::ROW) + lh * (Cfg::TN / 2);
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < Cfg::TN / 2; ++e) sum += half[e];
          sum += __shfl_xor(sum, 32);
          const int row = wm * Cfg::TM + 32 * i + lr;
          if (g.dbias && lh == 0 && row < rows) put_sum(row, sum);
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
        if (n0 + col < g.ldp) {
          bf16 part[P > 0 ? P : 1];
          split_parts<(P > 0 ? P : 1), true>(p, part);
#pragma unroll
          for (int u = 0; u < (P > 0 ? P : 1); ++u)
            static_cast<bf16*>(g.P)[u * g.pplane + (m0 + row) * g.ldp + n0 + col] = part[u];
        }
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

// A matrix copied into dense rows of ld elements (a multiple of 8; zeros behind cols), as it
// is or in parts.
struct PackJob {
  const void* src;
  int64_t row_step, col_step;  // elements
  int32_t rows, cols;
  int64_t ld, plane;
  void* out;
  const int32_t* labels;       // columns without a label are zeros
  int32_t classes;             // 0: no labels are looked at
  uint32_t groups;
};
// A chunk value by value: of rows shorter than one, and of the kept columns of output-major weights, which lie apart.
template <typename T, int P>
__device__ __forceinline__ void pack_one(const PackJob& j, int64_t r, int64_t c) {
  const T* from = static_cast<const T*>(j.src) + r * j.row_step + c * j.col_step;
  const int n = static_cast<int>(min<int64_t>(8, j.cols - c));
  T x[8];
  int32_t l[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = from[min(e, n - 1) * j.col_step];
#pragma unroll
  for (int e = 0; e < 8; ++e) l[e] = j.classes > 0 ? j.labels[c + min(e, n - 1)] : 0;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = e >= n || (j.classes > 0 && (l[e] < 0 || l[e] >= j.classes)) ? 0.0f : to_f32(x[e]);
  store_parts<P, true>(static_cast<bf16*>(j.out) + r * j.ld + c, j.plane, v);
}
// Whole rows: chunks of a thread are in flight together, without a branch between them; a
// row's last, partial one is read as the row's last eight values and moved down (bf16 4096 x
// 4096 with labels: 42 us one chunk after the other, 19). Columns that lie apart are taken chunk
// after chunk (pack_one): with every other of 1500 inputs kept, 8800 classes and batch 700 in
// bf16 the loss takes 39.4 us, input-major, without a copy of the weights, 26.5.
template <typename T, int P>
__device__ __forceinline__ void pack_rows(const PackJob& j, int64_t block) {
  constexpr int U = P == 1 ? 4 : 2, E = 16 / static_cast<int>(sizeof(T)), H = 8 / E;
  typedef u32x4 u32x4_a4 __attribute__((aligned(4), may_alias));
  const int64_t per = j.ld / 8, total = per * j.rows, step = static_cast<int64_t>(j.groups) * 256;
  const bool vec = j.col_step == 1 && j.cols >= 8;
  for (int64_t at = block * 256 + threadIdx.x; at < total; at += U * step) {
    int64_t r[U], c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t q = min(at + u * step, total - 1);
      r[u] = total < int64_t{1} << 31 ? static_cast<uint32_t>(q) / static_cast<uint32_t>(per) : q / per;
      c[u] = (q - r[u] * per) * 8;
    }
    if (!vec) {
      for (int u = 0; u < U; ++u)
        if (at + u * step < total) pack_one<T, P>(j, r[u], c[u]);
      continue;
    }
    Chunk<T, E> x[U][H];
    u32x4 l[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t first = min<int64_t>(c[u], j.cols - 8);
#pragma unroll
      for (int h = 0; h < H; ++h)
        x[u][h].raw = load16_any<sizeof(T)>(
            reinterpret_cast<const char*>(static_cast<const T*>(j.src) + r[u] * j.row_step + first + h * E));
      if (j.classes > 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) l[u][h] = *reinterpret_cast<const u32x4_a4*>(j.labels + first + 4 * h);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = x[u][e / E].at(e % E);
        // as unsigned numbers labels below 0 are past the last class
        if (j.classes > 0 && l[u][e / 4][e % 4] >= static_cast<uint32_t>(j.classes)) v[e] = 0.0f;
      }
      const int down = static_cast<int>(max<int64_t>(0, c[u] + 8 - j.cols));
#pragma unroll
      for (int by = 4; by > 0; by /= 2)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = down & by ? (e + by < 8 ? v[e + by] : 0.0f) : v[e];
      if (at + u * step < total) store_parts<P, true>(static_cast<bf16*>(j.out) + r[u] * j.ld + c[u], j.plane, v);
    }
  }
}
template <typename T, int P>
__global__ void __launch_bounds__(256) head_pack_kernel(PackJob a, PackJob b) {
  if (blockIdx.x < a.groups)
    pack_rows<T, P>(a, blockIdx.x);
  else
    pack_rows<T, P>(b, blockIdx.x - a.groups);
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

// What is left behind the products: dbias from the parts of the tile columns, in their
// order, and zeros in the rows of dropped inputs. The parts are added in 64 bits: 2^21 equal
// columns make up to 2^17 of them, whose chain in 32 was 1.4e-3 off.
struct ClearJob {
  char* p;
  int64_t row_bytes;  // a multiple of 2
  int64_t pieces;     // of 4 KB, of all dropped rows
  Kept in;
  uint32_t groups;
};
struct FinishArgs {
  const float* part;
  int32_t parts, classes;
  float* dbias;
  uint32_t bias_groups;
  ClearJob a, b;
};
__device__ __forceinline__ void clear_rows(const ClearJob& j, int64_t block) {
  typedef uint16_t u16_any __attribute__((may_alias));
  const int64_t per = (j.row_bytes + 4095) / 4096;
  for (int64_t at = block; at < j.pieces; at += j.groups) {
    // dropped row d: one of the period - 1 residues but the kept one
    const int64_t d = at / per, q = d / (j.in.period - 1);
    const int32_t rem = static_cast<int32_t>(d - q * (j.in.period - 1));
    const int64_t x = q * j.in.period + (rem < j.in.offset ? rem : rem + 1);
    if (x >= j.in.n) continue;
    const int64_t o = (at - d * per) * 4096 + threadIdx.x * 16, left = j.row_bytes - o;
    char* p = j.p + x * j.row_bytes + o;
    if (left >= 16) {
      *reinterpret_cast<u32x4_any2*>(p) = u32x4{0u, 0u, 0u, 0u};
    } else {
      for (int e = 0; e < left; e += 2) *reinterpret_cast<u16_any*>(p + e) = 0;
    }
  }
}
__global__ void __launch_bounds__(256) head_finish_kernel(FinishArgs g) {
  uint32_t block = blockIdx.x;
  if (block < g.bias_groups) {
    const int64_t v = static_cast<int64_t>(block) * 256 + threadIdx.x;
    if (v >= g.classes) return;
    double sum = 0.0;
#pragma unroll 8
    for (int q = 0; q < g.parts; ++q) sum += g.part[static_cast<int64_t>(q) * g.classes + v];
    g.dbias[v] = static_cast<float>(sum);
    return;
  }
  block -= g.bias_groups;
  if (block < g.a.groups)
    clear_rows(g.a, block);
  else
    clear_rows(g.b, block - g.a.groups);
}

// Rows of all inputs from those of the kept ones (rows of ldk): zeros in between. Whole rows
// are written once; the product writing its columns period elements apart and a pass for
// the zeros behind it write every line twice in pieces.
template <typename G>
__global__ void __launch_bounds__(256) head_expand_kernel(const G* __restrict__ from, int64_t ldk, int64_t rows, Kept in,
                                                          G* __restrict__ to) {
  const int64_t per = (static_cast<int64_t>(in.n) + 7) / 8, total = per * rows, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < total; at += step) {
    const int64_t r = total < int64_t{1} << 31 ? static_cast<uint32_t>(at) / static_cast<uint32_t>(per) : at / per;
    const int32_t c = static_cast<int32_t>(at - r * per) * 8, n = min(8, in.n - c);
    uint32_t q = static_cast<uint32_t>(c) / static_cast<uint32_t>(in.period);
    int32_t rem = c - static_cast<int32_t>(q) * in.period;
    const G* f = from + r * ldk;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = e < n && rem == in.offset ? to_f32(f[q]) : 0.0f;
      if (++rem == in.period) rem = 0, ++q;
    }
    G* o = to + r * in.n + c;
    constexpr int E = 16 / static_cast<int>(sizeof(G));
#pragma unroll
    for (int h = 0; h < 8 / E; ++h) {
      float w[E];
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = v[h * E + e];
      if (n > h * E) store_chunk<G, E>(o + h * E, w, n - h * E);
    }
  }
}

// ------------------------------------------------------------------ few classes
// A workgroup takes 16 columns and every class and input: its waves share the inputs, their
// sums meet in LDS, and what follows from a column's logits (loss, dz) is at hand in the same
// workgroup, dX as well. Products on the fp32 matrix instructions of 16 x 16 x 4, whose lanes
// hold single values, so that weights and inputs of any layout and alignment are loaded as
// they lie. fp32 with up to 32 classes; measured on MI355X against tiles on copies in parts,
// loss alone, and with gradients: 10 classes, 1024 of 2048 inputs, input-major, batch 128:
// 8.7, 25.7 us, tiles 20.8, 53.7; 32 classes, 4096 inputs, batch 4096: 28.6, 164, tiles 70,
// 224; 32 classes, 784 inputs, batch 128: 8.9, 29.9, tiles 19.7, 49.2.
// bf16, whose tiles need no copies, loses with it (10 classes, 4096 inputs, batch 4096: 29.8
// us, tiles 15.8).
constexpr int kFewClasses = 32, kFewCols = 16, kFewWaves = 16;
struct FewArgs {
  int32_t B, V;
  Kept in;
  bool zero;
  int32_t shares;      // workgroups of 16 columns: each takes a share of dX's rows (the sums are taken by all)
  const float* X;      // the first kept row
  const float* W;      // the first kept input
  int64_t wv, wk;      // elements from a class, from a kept input to the next
  bool whole;          // four inputs of a class lie together, on 16 bytes
  const float* bias;
  const int32_t* labels;
  float* loss;         // forward
  float* stats;
  const float* dloss;  // backward
  float* dX;           // or NULL
  float* P;            // dz [V][ldp] and the inputs of the columns with a label [kept][ldp], for dW; or NULL
  float* Xc;
  int64_t ldp;
  float* dbias;        // [workgroups][V], or NULL
};

template <int VB, int WAY>
__global__ void __launch_bounds__(64 * kFewWaves) head_few_kernel(FewArgs g) {
  __shared__ float red[kFewWaves * VB * 256];
  __shared__ float zs[VB * 16 * 17], es[VB * 16 * 17];
  constexpr int U = VB == 2 && WAY == WAY_GRAD ? 3 : 4;  // 16 inputs each in flight, as the registers allow
  const int t = static_cast<int>(threadIdx.x), lane = t & 63, wave = t >> 6, lc = lane & 15, lg = lane >> 4;
  const int at = xcd_position(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
  const int block = at / g.shares, share = at - block * g.shares;
  const int64_t n = static_cast<int64_t>(block) * kFewCols + lc;
  const int64_t nc = n < g.B ? n : g.B - 1;
  const float* X = g.X + nc;
  const float* W = g.W;
  const int64_t xk = static_cast<int64_t>(g.B) * g.in.period;
  const int K = g.in.kept, chunks = (K + 15) / 16;
  const int32_t label = n < g.B ? g.labels[n] : -1;
  const bool on = label >= 0 && label < g.V;
  f32x4 acc[VB];
#pragma unroll
  for (int b = 0; b < VB; ++b) acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int c0 = wave; c0 < chunks; c0 += kFewWaves * U) {
    float a[U][VB][4], x[U][4];  // of inputs past the last one: the last one's, and 0 below
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t k = min(16 * (c0 + kFewWaves * u) + 4 * lg + j, K - 1);
        x[u][j] = X[k * xk];
        if (g.whole) continue;
#pragma unroll
        for (int b = 0; b < VB; ++b) a[u][b][j] = W[min(16 * b + lc, g.V - 1) * g.wv + k * g.wk];
      }
    if (g.whole) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < VB; ++b) {
          const int64_t k = min(16 * (c0 + kFewWaves * u) + 4 * lg, K - 4);
          const f32x4 w = *reinterpret_cast<const f32x4*>(W + min(16 * b + lc, g.V - 1) * g.wv + k);
#pragma unroll
          for (int j = 0; j < 4; ++j) a[u][b][j] = w[j];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool mine = WAY == WAY_GRAD && (c0 + kFewWaves * u) / kFewWaves % g.shares == share;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t k = 16 * (c0 + kFewWaves * u) + 4 * lg + j;
        const float xv = k < K ? x[u][j] : 0.0f;
        if constexpr (WAY == WAY_GRAD) {
          if (g.Xc && mine && k < K && n < g.ldp) g.Xc[k * g.ldp + n] = on ? x[u][j] : 0.0f;
        }
#pragma unroll
        for (int b = 0; b < VB; ++b)
          acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k < K ? a[u][b][j] : 0.0f, xv, acc[b], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int b = 0; b < VB; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) red[(wave * VB + b) * 256 + r * 64 + lane] = acc[b][r];
  __syncthreads();
  if (t < VB * 256) {
    const int b = t >> 8, r = (t >> 6) & 3, v = 16 * b + 4 * lg + r;
    float z = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) z += red[w * VB * 256 + t];
    zs[v * 17 + lc] = v < g.V ? z + (g.bias ? g.bias[v] : 0.0f) : -kInf;
  }
  __syncthreads();
  const int q = t >> 4;  // of the columns' threads: classes q and q + 16
  if constexpr (WAY == WAY_LOSS) {
    float m = -kInf;
    if (t < 256) {
      for (int v = 0; v < g.V; ++v) m = fmaxf(m, zs[v * 17 + lc]);
      m = safe(m);
#pragma unroll
      for (int b = 0; b < VB; ++b) es[(16 * b + q) * 17 + lc] = expf(zs[(16 * b + q) * 17 + lc] - m);
    }
    __syncthreads();
    if (t < 16 && n < g.B) {
      float s = 0.0f;
      for (int v = 0; v < g.V; ++v) s += es[v * 17 + lc];
      g.loss[n] = on && s != 0.0f ? logf(s) - (zs[label * 17 + lc] - m) : 0.0f;
      if (g.stats) {
        g.stats[n] = m;
        g.stats[g.B + n] = s != 0.0f ? 1.0f / s : 0.0f;
      }
    }
  } else {
    if (t < 256) {
      float cm = 0.0f, inv = 0.0f, d = 0.0f;
      if (on) {
        cm = g.stats[n];
        inv = g.stats[g.B + n];
        d = g.dloss ? g.dloss[n] : 1.0f;
      }
#pragma unroll
      for (int b = 0; b < VB; ++b) {
        const int v = 16 * b + q;
        float p = 0.0f;
        if (inv != 0.0f && v < g.V) {  // 0: no label, or every class masked
          p = expf(zs[v * 17 + lc] - cm) * (inv * d);
          if (v == label) p -= d;
        }
        es[v * 17 + lc] = p;
        if (g.P && share == 0 && v < g.V && n < g.ldp) g.P[v * g.ldp + n] = p;
      }
    }
    __syncthreads();
    if (g.dbias && share == 0 && t < g.V) {
      float sum = 0.0f;
      for (int c = 0; c < 16; ++c) sum += es[t * 17 + c];
      g.dbias[static_cast<int64_t>(block) * g.V + t] = sum;
    }
    if (!g.dX) return;
    float* dX = g.dX + n;
    float dz[VB * 4];
#pragma unroll
    for (int s = 0; s < VB * 4; ++s) dz[s] = es[(4 * s + lg) * 17 + lc];
    for (int c0 = share + g.shares * wave; c0 < chunks; c0 += g.shares * kFewWaves * U) {
      float w[U][VB * 4];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < VB * 4; ++s)
          w[u][s] = W[min(4 * s + lg, g.V - 1) * g.wv + min(16 * (c0 + g.shares * kFewWaves * u) + lc, K - 1) * g.wk];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f32x4 out = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < VB * 4; ++s)
          out = __builtin_amdgcn_mfma_f32_16x16x4f32(4 * s + lg < g.V ? w[u][s] : 0.0f, dz[s], out, 0, 0, 0);
        const int k0 = 16 * (c0 + g.shares * kFewWaves * u) + 4 * lg;
        if (n >= g.B) continue;
        float* at = dX + (g.in.offset + static_cast<int64_t>(k0) * g.in.period) * g.B;
#pragma unroll
        for (int r = 0; r < 4; ++r, at += xk) {
          if (k0 + r >= K) continue;
          *at = out[r];
          if (g.zero) {
            const int zeros = min(g.in.period, g.in.n - g.in.offset - (k0 + r) * g.in.period);
            float* z = at;
            for (int e = 1; e < zeros; ++e) *(z += g.B) = 0.0f;
          }
        }
      }
    }
    if (g.zero && n < g.B && share == 0)
      for (int64_t e = q; e < min(g.in.offset, g.in.n); e += 4 * kFewWaves) dX[e * g.B] = 0.0f;
  }
}

template <int WAY>
hipError_t run_few(FewArgs g, hipStream_t stream) {
  const int64_t blocks = (static_cast<int64_t>(g.B) + kFewCols - 1) / kFewCols, rows = g.in.kept / (16 * kFewWaves);
  g.shares = g.dX ? static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>({4, rows, kTargetBlocks / blocks}))) : 1;
  const dim3 grid(static_cast<unsigned>(blocks * g.shares)), threads(64 * kFewWaves);
  if (g.V <= 16)
    hipLaunchKernelGGL((head_few_kernel<1, WAY>), grid, threads, 0, stream, g);
  else
    hipLaunchKernelGGL((head_few_kernel<2, WAY>), grid, threads, 0, stream, g);
  return hipGetLastError();
}

unsigned sweep(int64_t n) { return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(4096, (n + 255) / 256))); }

// ------------------------------------------------------------------ host
// Elements between the rows of the tile kernel's operands: offsets within a slab and a tile have 32 bits.
constexpr int64_t kMostStride = int64_t{1} << 22;
// Kept inputs: counted in 32 bits, rounded up to a tile or a slab (256) or to what the waves of head_few_kernel
// take in a turn and load ahead (16 inputs, 4 shares, 16 waves, 7 turns: 7168).
constexpr int32_t kMostKept = INT32_MAX - (1 << 16) + 1;

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
  s->es = d->dtype == ARD_BF16 ? 2 : 4;
  s->input_major = d->weight_layout == ARD_WEIGHTS_INPUT_MAJOR;
  s->zero = d->dropped == ARD_DROPPED_ZERO;
  s->few = s->es == 4 && s->V <= kFewClasses;
  s->parts = !s->few && s->es == 4;
  s->ldp = up8(s->B);
  s->wrows = s->input_major ? s->in.kept : s->V;
  s->ldc = up8(s->input_major ? s->V : s->in.kept);
  const bool any = s->in.kept > 0 && !s->few;
  auto in_place = [&](int64_t row) { return !s->parts && row % 8 == 0 && row * s->in.period < kMostStride; };
  s->copy_w = any && !(s->input_major ? in_place(s->V) : s->in.period == 1 && in_place(s->in.n));
  s->copy_x = any && !in_place(s->B);
  return ARD_OK;
}

int check_strides(const HeadShape& s) {
  if (s.in.kept > kMostKept)
    return fail(ARD_ERR_UNSUPPORTED, "%d kept inputs: at most 2^31 - 2^16", s.in.kept);
  if (s.ldp >= kMostStride || s.ldc >= kMostStride)
    return fail(ARD_ERR_UNSUPPORTED, "%d columns and rows of %lld weights must be below 2^22", s.B, static_cast<long long>(s.ldc));
  if ((s.V / 32 + int64_t{1}) * (s.B / 32 + int64_t{1}) >= int64_t{1} << 31)  // tiles are counted in 32 bits
    return fail(ARD_ERR_UNSUPPORTED, "%d classes of %d columns are too many tiles", s.V, s.B);
  return ARD_OK;
}

// The tiles of the kernel, with their rates: flop/us of a compute unit (parts: of bf16 products) with as many
// workgroups on it as it holds. Measured on MI355X over 12 sizes of each type, forward, batch 8 to 4096, 256 to 4096
// inputs, 100 to 32000 classes: the pick takes at most 1.07 of the best tile's time (bf16 2048 x 256 to 2000: 12.9 and
// 12.1 us), one tile for all up to 5 times (256 x 256 for 64 x 4096 to 1000: 76 us, 32 x 32 15; that for 512 x 1024 to
// 32000: 199 us, 256 x 256 42).
struct HeadTile {
  int bm, bn, bk, wgn, per;
  double rate;
};
template <class Cfg>
constexpr HeadTile head_tile(int per, double rate) {
  return {Cfg::BM, Cfg::BN, Cfg::BK, Cfg::KSPLIT == 1 ? Cfg::WGN : 1, per, rate};
}
using HeadMid = FastCfg<bf16, 64, 128, 64, 3, 2, 2, 1>;  // 72 KB, 4 waves
constexpr HeadTile kTiles[] = {
    head_tile<FastCfgs<bf16>::Huge>(1, 4.2e6), head_tile<FastCfgs<bf16>::Wide>(1, 3.5e6),
    head_tile<FastCfgs<bf16>::Tall>(1, 3.4e6), head_tile<FastCfgs<bf16>::Big>(1, 2.7e6),
    head_tile<HeadMid>(2, 2.4e6),              head_tile<FastCfgs<bf16>::Small>(2, 0.7e6),
    head_tile<PartsCfgs<3>::C256>(1, 4.9e6),   head_tile<PartsCfgs<3>::C192>(1, 4.6e6),
    head_tile<PartsCfgs<3>::C128>(1, 3.8e6),   head_tile<PartsCfgs<3>::C64>(1, 3.2e6)};
constexpr int kFirstParts = 6, kAllTiles = 10;
template <class F>
hipError_t with_tile(int kind, F f) {
  using std::integral_constant;
  switch (kind) {
    case 0: return f(FastCfgs<bf16>::Huge{}, integral_constant<int, 0>{});
    case 1: return f(FastCfgs<bf16>::Wide{}, integral_constant<int, 0>{});
    case 2: return f(FastCfgs<bf16>::Tall{}, integral_constant<int, 0>{});
    case 3: return f(FastCfgs<bf16>::Big{}, integral_constant<int, 0>{});
    case 4: return f(HeadMid{}, integral_constant<int, 0>{});
    case 5: return f(FastCfgs<bf16>::Small{}, integral_constant<int, 0>{});
    case 6: return f(PartsCfgs<3>::C256{}, integral_constant<int, 3>{});
    case 7: return f(PartsCfgs<3>::C192{}, integral_constant<int, 3>{});
    case 8: return f(PartsCfgs<3>::C128{}, integral_constant<int, 3>{});
    default: return f(PartsCfgs<3>::C64{}, integral_constant<int, 3>{});
  }
}

// The tile with the least modelled time: rounds of the chip times a workgroup's slabs.
int plan_tile(const HeadShape& s, int64_t M) {
  const int64_t K = s.in.kept;
  int best = 0;
  double best_t = 1e300;
  for (int kind = s.parts ? kFirstParts : 0; kind < (s.parts ? kAllTiles : kFirstParts); ++kind) {
    const HeadTile& c = kTiles[kind];
    const int64_t n = (M + c.bm - 1) / c.bm * ((s.B + c.bn - 1) / c.bn), slabs = (K + c.bk - 1) / c.bk;
    const int64_t rounds = (n + kTargetBlocks * c.per - 1) / (kTargetBlocks * c.per);
    // workgroups that share a compute unit take its rate between them
    const double share = n >= kTargetBlocks * c.per ? c.per : std::max(1.0, static_cast<double>(n) / kTargetBlocks);
    const double t = rounds * (2.0 + share * 2.0 * c.bm * c.bn * c.bk * slabs * (s.parts ? 6 : 1) / c.rate);
    if (t < best_t) best_t = t, best = kind;
  }
  return best;
}

template <class Cfg, int P, bool AMC, int WAY>
hipError_t launch_tile(const TileArgs& g, hipStream_t stream) {
  auto kern = head_tile_kernel<Cfg, P, AMC, WAY>;
  constexpr int LDS = HeadLds<Cfg>::bytes(WAY);
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return attr;
  const int64_t tiles = (g.M + Cfg::BM - 1) / Cfg::BM * ((g.B + Cfg::BN - 1) / Cfg::BN);
  constexpr int64_t kRow = 1 << 20;  // workgroups of a grid row: the threads along x have to stay below 2^32
  const dim3 grid(static_cast<unsigned>(std::min(tiles, kRow)), static_cast<unsigned>((tiles - 1) / kRow + 1));
  hipLaunchKernelGGL(kern, grid, dim3(Cfg::NT), LDS, stream, g);
  return hipGetLastError();
}
template <int WAY>
hipError_t run_tile(const HeadShape& s, int kind, const TileArgs& g, hipStream_t stream) {
  return with_tile(kind, [&](auto cfg, auto parts) {
    using Cfg = decltype(cfg);
    constexpr int P = decltype(parts)::value;
    return s.input_major ? launch_tile<Cfg, P, true, WAY>(g, stream) : launch_tile<Cfg, P, false, WAY>(g, stream);
  });
}

// Classes of a piece of the backward, whole tiles: dz of at most 512 MB in bf16, 192 in parts. Measured on MI355X,
// forward and backward, 128, 512 MB of bf16: 4096 x 4096 to 32000 3455, 3417 us, 16384 x 1024 to 32000 4481, 4206 (2 GB:
// 4052); of parts for 128, 512 MB of fp32: 4096 x 1024 to 32000 5097, 5255.
int64_t piece_of(const HeadShape& s) {
  const int64_t most = std::max<int64_t>(256, (int64_t{s.parts ? 128 : 512} << 20) / (s.ldp * static_cast<int64_t>(s.es)) / 256 * 256);
  const int64_t pieces = (s.V + most - 1) / most;
  return std::min<int64_t>(s.V, ((s.V + pieces - 1) / pieces + 255) / 256 * 256);
}

// Bytes of a copy of rows x ld: in three bf16 parts, or as it is.
size_t copy_bytes(const HeadShape& s, int64_t rows, int64_t ld) {
  return al256(static_cast<size_t>(rows) * ld * (s.parts ? 6 : s.es));
}
bool expands(const HeadShape& s) { return s.zero && !s.input_major && s.in.period > 1; }

// The workspace. fwd: copies, the tiles' pairs, the labels' logits. bwd: copies, dz of a piece, row sums, dX of the
// pieces, dW of the kept inputs of a piece, the products' partial sums.
struct FwdSpace {
  size_t wc, xc, part, zl;
  size_t bytes() const { return wc + xc + part + zl; }
};
struct BwdSpace {
  size_t wc, xc, p, db, dx, dw, part;
  size_t bytes() const { return wc + xc + p + db + 2 * dx + dw + part; }
};
FwdSpace fwd_space(const HeadShape& s) {
  if (s.few) return {0, 0, 0, 0};
  const HeadTile& t = kTiles[plan_tile(s, s.V)];
  return {s.copy_w ? copy_bytes(s, s.wrows, s.ldc) : 0, s.copy_x ? copy_bytes(s, s.in.kept, s.ldp) : 0,
          al256(static_cast<size_t>((s.V + t.bm - 1) / t.bm) * s.B * 8), al256(static_cast<size_t>(s.B) * 4)};
}
size_t product_floats(const HeadShape& s, int M, int N, int K) {
  return s.parts ? plan_parts<3>(M, N, K, false).floats : s.es == 2 ? partial_floats<bf16>(M, N, K) : partial_floats<float>(M, N, K);
}
int bias_parts(const HeadShape& s, int64_t piece) {
  if (s.few) return static_cast<int>((static_cast<int64_t>(s.B) + kFewCols - 1) / kFewCols);
  const HeadTile& t = kTiles[plan_tile(s, piece)];
  return static_cast<int>((static_cast<int64_t>(s.B) + t.bn - 1) / t.bn * t.wgn);
}
BwdSpace bwd_space(const HeadShape& s, size_t gs) {
  const int64_t piece = s.few ? s.V : piece_of(s);
  const int m = static_cast<int>(piece), last = static_cast<int>(s.V - (s.V - 1) / piece * piece), k = s.in.kept;
  size_t part = 0;
  if (k > 0)
    for (int v : {m, last}) {
      if (!s.few) part = std::max(part, product_floats(s, k, s.B, v));
      part = std::max(part, s.input_major ? product_floats(s, k, v, s.B) : product_floats(s, v, k, s.B));
    }
  return {s.copy_w ? copy_bytes(s, s.wrows, s.ldc) : 0, copy_bytes(s, k, s.ldp), copy_bytes(s, piece, s.ldp),
          al256(static_cast<size_t>(bias_parts(s, piece)) * s.V * 4), piece < s.V ? al256(static_cast<size_t>(k) * s.B * 4) : 0,
          expands(s) ? al256(static_cast<size_t>(piece) * up8(k) * gs) : 0, al256(4 * part)};
}

size_t space_bytes(const ard_headloss_desc* d, const HeadShape& s) {
  return std::max(fwd_space(s).bytes(), bwd_space(s, d->grad_dtype == ARD_BF16 ? 2 : 4).bytes());
}

// The copies that the tile kernel reads: of W, of X (labels: for the backward).
template <typename T>
int pack(const HeadShape& s, const void* W, char* wc, const void* X, char* xc, const int32_t* labels, hipStream_t stream) {
  constexpr int P = sizeof(T) == 4 ? 3 : 1;
  auto groups = [](const PackJob& j) {
    return static_cast<uint32_t>(std::max<int64_t>(1, std::min<int64_t>(4096, (j.rows * (j.ld / 8) - 1) / (P == 1 ? 1024 : 512) + 1)));
  };
  PackJob w = {}, x = {};
  if (s.copy_w) {
    const int64_t p = s.in.period, o = s.in.offset;
    w.src = static_cast<const T*>(W) + (s.input_major ? o * s.V : o);
    w.row_step = s.input_major ? s.V * p : s.in.n;
    w.col_step = s.input_major ? 1 : p;
    w.rows = static_cast<int32_t>(s.wrows), w.cols = s.input_major ? s.V : s.in.kept;
    w.ld = s.ldc, w.plane = s.wrows * s.ldc;
    w.out = wc;
    w.groups = groups(w);
  }
  if (xc && s.in.kept > 0) {
    x.src = static_cast<const T*>(X) + static_cast<int64_t>(s.in.offset) * s.B;
    x.row_step = static_cast<int64_t>(s.B) * s.in.period, x.col_step = 1;
    x.rows = s.in.kept, x.cols = s.B;
    x.ld = s.ldp, x.plane = s.in.kept * s.ldp;
    x.out = xc;
    x.labels = labels, x.classes = labels ? s.V : 0;
    x.groups = groups(x);
  }
  if (w.groups + x.groups == 0) return ARD_OK;
  hipLaunchKernelGGL((head_pack_kernel<T, P>), dim3(w.groups + x.groups), dim3(256), 0, stream, w, x);
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

// The operands of the tile kernel from class 0 on.
template <typename T>
TileArgs tile_operands(const HeadShape& s, const void* W, const char* wc, const void* X, const char* xc) {
  TileArgs g = {};
  g.B = s.B;
  g.K = s.in.kept;
  g.classes = s.V;
  if (s.copy_w) {
    g.W = wc, g.ldw = s.ldc, g.wplane = s.wrows * s.ldc;
  } else if (s.input_major) {
    g.W = static_cast<const T*>(W) + static_cast<int64_t>(s.in.offset) * s.V;
    g.ldw = static_cast<int64_t>(s.V) * s.in.period;
  } else {
    g.W = W, g.ldw = s.in.n;
  }
  if (xc) {
    g.X = xc, g.ldx = s.ldp, g.xplane = s.in.kept * s.ldp;
  } else {
    g.X = static_cast<const T*>(X) + static_cast<int64_t>(s.in.offset) * s.B;
    g.ldx = static_cast<int64_t>(s.B) * s.in.period;
  }
  return g;
}

FewArgs few_args(const HeadShape& s, const void* X, const void* W, const float* bias, const int32_t* labels) {
  FewArgs g = {};
  g.B = s.B, g.V = s.V, g.in = s.in, g.zero = s.zero;
  g.X = static_cast<const float*>(X) + static_cast<int64_t>(s.in.offset) * s.B;
  g.W = static_cast<const float*>(W) + static_cast<int64_t>(s.in.offset) * (s.input_major ? s.V : 1);
  g.wv = s.input_major ? 1 : s.in.n;
  g.wk = static_cast<int64_t>(s.in.period) * (s.input_major ? s.V : 1);
  g.whole = !s.input_major && s.in.period == 1 && s.in.n % 4 == 0;
  g.bias = bias;
  g.labels = labels;
  g.ldp = s.ldp;
  return g;
}

template <typename T>
int fwd_impl(const HeadShape& s, const void* Xt, const void* W, const float* bias, const int32_t* labels, float* loss,
             float* stats, char* ws, hipStream_t stream) {
  if (s.few) {
    FewArgs g = few_args(s, Xt, W, bias, labels);
    g.loss = loss, g.stats = stats;
    ARD_HIP_CHECK((run_few<WAY_LOSS>(g, stream)));
    return ARD_OK;
  }
  const FwdSpace sp = fwd_space(s);
  char *wc = ws, *xc = wc + sp.wc, *part = xc + sp.xc, *zl = part + sp.part;
  const int st = pack<T>(s, W, wc, Xt, s.copy_x ? xc : nullptr, nullptr, stream);
  if (st != ARD_OK) return st;
  TileArgs g = tile_operands<T>(s, W, wc, Xt, s.copy_x ? xc : nullptr);
  g.M = s.V;
  g.bias = bias;
  g.labels = labels;
  g.part = reinterpret_cast<float2*>(part);
  g.zlabel = reinterpret_cast<float*>(zl);
  const int kind = plan_tile(s, s.V);
  ARD_HIP_CHECK(run_tile<WAY_LOSS>(s, kind, g, stream));
  const int64_t groups = (static_cast<int64_t>(s.B) + 15) / 16;
  const int bm = kTiles[kind].bm;
  hipLaunchKernelGGL(head_join_kernel<T>, dim3(static_cast<unsigned>(groups)), dim3(256), 0, stream, g.part, g.zlabel, labels,
                     s.B, s.V, (static_cast<int64_t>(s.V) + bm - 1) / bm, loss, stats);
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

// A product of A[M][K] (a_across: stored [K][M]) and B[K][N] (b_along: stored [N][K]), both as
// bf16 matrices of rows lda, ldb, fp32 ones, or in parts, to rows of ldc with values cstep apart.
struct Operand {
  const void* p;
  int64_t ld, plane;
};
template <typename T, bool AMC, bool BMC, typename OutT>
hipError_t head_product(const HeadShape& s, int64_t M, int64_t N, int64_t K, Operand a, Operand b, OutT* c, int64_t ldc,
                        int32_t cstep, float* partial, size_t floats, hipStream_t stream) {
  if constexpr (sizeof(T) == 4) {
    if (s.parts) {
      PartsArgs g = {};
      g.M = static_cast<int>(M), g.N = static_cast<int>(N), g.K = static_cast<int>(K);
      g.a = {static_cast<const bf16*>(a.p), a.plane, a.ld};
      g.b = {static_cast<const bf16*>(b.p), b.plane, b.ld};
      g.epi = PARTS_FLOAT;
      g.fout = c, g.ldo = ldc, g.fstep = cstep;
      return run_parts_gemm<3, AMC, BMC>(g, partial, stream);
    }
  }
  if constexpr (sizeof(T) == 4 && (AMC || BMC)) {
    return hipErrorNotSupported;  // of a few classes dW alone is a product
  } else {
    GemmArgs q = {};
    q.M = static_cast<int>(M), q.N = static_cast<int>(N), q.K = static_cast<int>(K);
    q.a = view(a.p, a.ld), q.b = view(b.p, b.ld);
    q.c.p = c, q.c.ld = ldc, q.c.col_stride = cstep;
    return product<T, AMC, BMC, OutT>(q, stream, partial, floats);
  }
}

template <typename T, typename G>
int bwd_impl(const HeadShape& s, const void* Xt, const void* W, const float* bias, const int32_t* labels, const float* stats,
             const float* dloss, void* dXt, void* dW, float* dbias, char* ws, hipStream_t stream) {
  const BwdSpace sp = bwd_space(s, sizeof(G));
  char *wc = ws, *xc = wc + sp.wc, *p = xc + sp.xc, *db = p + sp.p, *all = db + sp.db, *one = all + sp.dx, *dwk = one + sp.dx,
       *pt = dwk + sp.dw;
  float* partial = reinterpret_cast<float*>(pt);
  const size_t floats = sp.part / 4;
  const int64_t piece = s.few ? s.V : piece_of(s), K = s.in.n, kin = s.in.kept, xplane = kin * s.ldp;
  const int parts = bias_parts(s, piece);
  float* sums = !dbias ? nullptr : parts == 1 ? dbias : reinterpret_cast<float*>(db);
  TileArgs base = {};
  int kind = 0;
  if (s.few) {
    FewArgs g = few_args(s, Xt, W, bias, labels);
    g.stats = const_cast<float*>(stats), g.dloss = dloss;
    g.dX = static_cast<float*>(dXt);
    if (dW) g.P = reinterpret_cast<float*>(p), g.Xc = reinterpret_cast<float*>(xc);
    g.dbias = sums;
    ARD_HIP_CHECK((run_few<WAY_GRAD>(g, stream)));
  } else {
    const int st = pack<T>(s, W, wc, Xt, xc, labels, stream);
    if (st != ARD_OK) return st;
    base = tile_operands<T>(s, W, wc, Xt, xc);
    base.labels = labels;
    base.stats = stats;
    base.dloss = dloss;
    base.P = p;
    base.ldp = s.ldp;
    kind = plan_tile(s, piece);
  }
  const size_t ws_es = s.parts ? 2 : s.es;  // of the copies
  for (int64_t v = 0; v < s.V; v += piece) {
    const int64_t M = std::min<int64_t>(piece, s.V - v), pplane = M * s.ldp;
    TileArgs g = base;
    if (!s.few) {
      g.M = M;
      g.class0 = v;
      g.W = static_cast<const char*>(base.W) + (s.input_major ? v : v * base.ldw) * ws_es;
      g.bias = bias ? bias + v : nullptr;
      g.dbias = sums ? sums + v : nullptr;
      g.pplane = pplane;
      ARD_HIP_CHECK(run_tile<WAY_GRAD>(s, kind, g, stream));
    }
    const Operand dz = {p, s.ldp, pplane}, x = {xc, s.ldp, xplane}, w = {g.W, g.ldw, g.wplane};
    if (dXt && kin > 0 && !s.few) {
      auto to = [&](auto* c, int64_t ld) {
        return s.input_major ? head_product<T, false, true>(s, kin, s.B, M, w, dz, c, ld, 1, partial, floats, stream)
                             : head_product<T, true, true>(s, kin, s.B, M, w, dz, c, ld, 1, partial, floats, stream);
      };
      if (piece >= s.V) {
        ARD_HIP_CHECK(to(static_cast<T*>(dXt) + static_cast<int64_t>(s.in.offset) * s.B, static_cast<int64_t>(s.B) * s.in.period));
      } else {
        ARD_HIP_CHECK(to(reinterpret_cast<float*>(v == 0 ? all : one), s.B));
        if (v > 0) {
          hipLaunchKernelGGL(head_add_kernel<T>, dim3(sweep(kin * s.B)), dim3(256), 0, stream, reinterpret_cast<float*>(all),
                             reinterpret_cast<const float*>(one), s.B, s.in, v + piece >= s.V ? static_cast<T*>(dXt) : nullptr);
          ARD_LAUNCH_CHECK();
        }
      }
    }
    if (dW && kin > 0) {
      G* out = static_cast<G*>(dW);
      if (s.input_major) {
        ARD_HIP_CHECK((head_product<T, false, false>(s, kin, M, s.B, x, dz, out + static_cast<int64_t>(s.in.offset) * s.V + v,
                                                     static_cast<int64_t>(s.V) * s.in.period, 1, partial, floats, stream)));
      } else if (!expands(s)) {
        ARD_HIP_CHECK((head_product<T, false, false>(s, M, kin, s.B, dz, x, out + v * K + s.in.offset, K, s.in.period, partial,
                                                     floats, stream)));
      } else {
        G* kept = reinterpret_cast<G*>(dwk);
        ARD_HIP_CHECK((head_product<T, false, false>(s, M, kin, s.B, dz, x, kept, up8(kin), 1, partial, floats, stream)));
        hipLaunchKernelGGL(head_expand_kernel<G>, dim3(sweep(M * ((K + 7) / 8))), dim3(256), 0, stream, kept, up8(kin), M, s.in,
                           out + v * K);
        ARD_LAUNCH_CHECK();
      }
    }
  }
  FinishArgs f = {};
  if (dbias && parts > 1) {
    f.part = sums, f.parts = parts, f.classes = s.V, f.dbias = dbias;
    f.bias_groups = static_cast<uint32_t>((static_cast<int64_t>(s.V) + 255) / 256);
  }
  auto clear = [&](void* q, int64_t row_bytes) {
    ClearJob j = {static_cast<char*>(q), row_bytes, 0, s.in, 0};
    j.pieces = (static_cast<int64_t>(s.in.n) + s.in.period - 1) / s.in.period * (s.in.period - 1) * ((row_bytes + 4095) / 4096);
    j.groups = static_cast<uint32_t>(std::min<int64_t>(j.pieces, 4096));
    return j;
  };
  if (s.in.period > 1 && s.zero) {
    if (dXt && !s.few) f.a = clear(dXt, s.B * static_cast<int64_t>(s.es));
    if (dW && (s.input_major || kin == 0)) f.b = clear(dW, s.V * static_cast<int64_t>(sizeof(G)));
  }
  const uint32_t groups = f.bias_groups + f.a.groups + f.b.groups;
  if (groups > 0) {
    hipLaunchKernelGGL(head_finish_kernel, dim3(groups), dim3(256), 0, stream, f);
    ARD_LAUNCH_CHECK();
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
  return space_bytes(desc, s);
}

int ard_headloss_fwd(const ard_headloss_desc* desc, const void* Xt, const void* W, const float* bias, const int32_t* labels,
                     float* loss, float* stats, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  HeadShape s;
  int st = check_desc(desc, &s);
  if (st != ARD_OK) return st;
  if ((st = check_strides(s)) || (st = need_ptr(Xt, "Xt")) || (st = need_ptr(W, "W")) || (st = may_ptr(bias, "bias")) ||
      (st = need_ptr(labels, "labels")) || (st = need_ptr(loss, "loss")) || (st = may_ptr(stats, "stats")) ||
      (st = check_space(space_bytes(desc, s), ws, ws_bytes)))
    return st;
  // written by one workgroup while others read the inputs
  if (same_buffer(loss, {Xt, W, bias, labels, stats}) || same_buffer(stats, {Xt, W, bias, labels}))
    return fail(ARD_ERR_INVALID_ARG, "loss or stats is in the buffer of another argument");
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16 ? fwd_impl<bf16>(s, Xt, W, bias, labels, loss, stats, w, sm)
                                 : fwd_impl<float>(s, Xt, W, bias, labels, loss, stats, w, sm);
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
      (st = check_space(space_bytes(desc, s), ws, ws_bytes)))
    return st;
  if (same_buffer(dXt, {Xt, W, bias, labels, stats, dloss, dW, dbias}) || same_buffer(dW, {Xt, W, bias, labels, stats, dloss, dbias}) ||
      same_buffer(dbias, {Xt, W, bias, labels, stats, dloss}))
    return fail(ARD_ERR_INVALID_ARG, "a gradient is in the buffer of another argument");
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  if (desc->dtype == ARD_F32)
    return bwd_impl<float, float>(s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm);
  return desc->grad_dtype == ARD_BF16 ? bwd_impl<bf16, bf16>(s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm)
                                      : bwd_impl<bf16, float>(s, Xt, W, bias, labels, stats, dloss, dXt, dW, dbias, w, sm);
}

}  // extern "C"
