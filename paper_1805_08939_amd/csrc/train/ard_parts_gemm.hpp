// Products of matrices held as sums of bf16 parts, on the bf16 matrix cores.
//
// A fp32 value is kept as 2 or 3 bf16 parts, each the rounded rest of those before it: 16
// or 24 significant bits, in planes of the same shape. A product of two such matrices is
// the sum of the parts' products down to the precision of the parts,
//   2 parts: hh + hl + lh        (operands to 2^-16, three matrix instructions)
//   3 parts: + mm + hl' + l'h    (operands to 2^-24, six)
// accumulated in fp32. The bf16 matrix cores run at 16 times the fp32 ones' rate, so that
// three or six instructions for one still gain, and a slab's loads serve three or six
// instructions instead of one.
//
// Tiles, direct loads, LDS layout and fragments are those of the layers' products
// (ard_gemm_fast.hpp); a slab holds every part of both operands.
#pragma once

#include "ard_train.hpp"

namespace ard {

struct PartsView {
  const bf16* p;   // first part
  int64_t plane;   // elements from a part to the next
  int64_t ld;
};

// What becomes of a product's values.
enum PartsEpi {
  PARTS_STORE = 0,  // split into parts
  PARTS_POLY = 1,   // a I + b A + c v, split into parts
  PARTS_FLOAT = 2   // fp32
};

struct PartsArgs {
  int32_t M, N, K;
  PartsView a, b;
  bool symmetric;   // M == N and the result its own transpose: tiles above the diagonal are mirrored, not computed
  int32_t epi;
  bf16* out;        // PARTS_STORE, PARTS_POLY
  int64_t plane, ldo;
  float* fout;      // PARTS_FLOAT, rows of ldo at any element, values of a row fstep apart
  int32_t fstep;
  PartsView poly;   // PARTS_POLY: A
  float pa, pb, pc;
  int32_t splits;   // of the slabs, each writing its sums to partial
  float* partial;   // [splits][tiles][wave][block][16][64]
};

template <int PARTS_, int BM_, int BN_, int WGM_, int WGN_, int STAGES_, int BK_ = 32, int KSPLIT_ = 1>
struct PartsCfg : FastCfg<bf16, BM_, BN_, BK_, STAGES_, WGM_, WGN_, KSPLIT_> {
  using Base = FastCfg<bf16, BM_, BN_, BK_, STAGES_, WGM_, WGN_, KSPLIT_>;
  static constexpr int PARTS = PARTS_;
  static constexpr int STAGE = PARTS * Base::STAGE;            // A's parts, then B's
  static constexpr int AREGION = PARTS * Base::ABYTES;
  static constexpr int LPW = PARTS * Base::LPW;
  static constexpr int OUTS = Base::WGM * Base::WGN;           // waves with outputs (the others share their k)
  static constexpr int SUMS = Base::FM * Base::FN * 16 * 64;   // a wave's sums
  static constexpr int ROW = Base::TN * 4 + 32;                // of the epilogue's staging: 32 rows of a wave
  static constexpr int RED = (Base::KSPLIT - 1) * OUTS * SUMS * 4;
  static constexpr int MAIN = STAGES_ * STAGE, ENDS = RED + OUTS * 32 * ROW;
  static constexpr int LDS = MAIN > ENDS ? MAIN : ENDS;
};

// The parts of a value. ANY: of any finite one in three parts; where the first would round to
// infinity it is the largest bf16 number, and the others hold the rest. (An iterate's values are
// about 1 at most; the comparison would cost 512 x 784 in three parts 188 us for 186.)
template <int PARTS, bool ANY = false>
__device__ __forceinline__ void split_parts(float v, bf16 (&p)[PARTS]) {
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    p[q] = static_cast<bf16>(v);
    if (ANY && PARTS == 3 && q == 0 && fabsf(v) >= 0x1.ffp127f)  // an infinite one stays infinite
      p[0] = __builtin_bit_cast(bf16, static_cast<uint16_t>(__float_as_uint(v) >> 16));
    if (q + 1 < PARTS) v -= static_cast<float>(p[q]);
  }
}

// Tile t of the lower triangle, row by row.
__device__ __forceinline__ void triangle_tile(int t, int& row, int& col) {
  int r = static_cast<int>((sqrtf(8.0f * static_cast<float>(t) + 1.0f) - 1.0f) * 0.5f);
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  while (r * (r + 1) / 2 > t) --r;
  row = r;
  col = t - r * (r + 1) / 2;
}

// Splits eight values and writes a chunk of each part.
template <int PARTS, bool ANY = false>
__device__ __forceinline__ void store_parts(bf16* out, int64_t plane, const float (&v)[8]) {
  bf16 w[PARTS][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bf16 p[PARTS];
    split_parts<PARTS, ANY>(v[e], p);
#pragma unroll
    for (int q = 0; q < PARTS; ++q) w[q][e] = p[q];
  }
#pragma unroll
  for (int q = 0; q < PARTS; ++q)
    *reinterpret_cast<u32x4_any*>(out + q * plane) = *reinterpret_cast<const u32x4_any*>(w[q]);
}
template <int PARTS>
__device__ __forceinline__ void load_parts(const bf16* p, int64_t plane, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.0f;
#pragma unroll
  for (int q = PARTS - 1; q >= 0; --q) {
    Chunk<bf16, 8> c;
    c.raw = *reinterpret_cast<const u32x4_any*>(p + q * plane);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += c.at(e);
  }
}

// The results of 32 rows x TN columns, from row m0 and column n0 on, through the wave's LDS:
// eight columns of a row a lane, and for a mirrored tile eight rows of a column. Rows of parts
// hold whole chunks (ldo is a multiple of 8), so that a chunk is written whole.
template <class Cfg>
__device__ __forceinline__ void parts_block(const PartsArgs& g, const f32x16 (&acc)[Cfg::FN], int m0, int n0, bool mirror,
                                            char* region) {
  constexpr int TN = Cfg::TN, CH = TN / 8, ROW = Cfg::ROW;
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
      *reinterpret_cast<float*>(region + (8 * (r >> 2) + 4 * lh + (r & 3)) * ROW + (32 * j + lr) * 4) = acc[j][r];
#pragma unroll
  for (int e0 = 0; e0 < 32 * CH; e0 += 64) {
    const int e = e0 + lane, rl = e / CH, ch = e % CH;
    const int m = m0 + rl, n = n0 + 8 * ch;
    float* at = reinterpret_cast<float*>(region + rl * ROW) + 8 * ch;
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = at[x];
    if (m >= g.M || n >= g.N) continue;
    if (g.epi == PARTS_FLOAT) {
      float* o = g.fout + m * g.ldo + static_cast<int64_t>(n) * g.fstep;
      if (g.fstep == 1 && n + 8 <= g.N) {
        const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
        store_chunk<float, 4>(o, lo, 4);
        store_chunk<float, 4>(o + 4, hi, 4);
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (n + x < g.N) o[static_cast<int64_t>(x) * g.fstep] = v[x];
      }
      continue;
    }
    if (g.epi == PARTS_POLY) {
      float a[8];
      load_parts<Cfg::PARTS>(g.poly.p + m * g.poly.ld + n, g.poly.plane, a);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        v[x] = g.pc * v[x] + g.pb * a[x] + (m == n + x ? g.pa : 0.0f);
        if (mirror) at[x] = v[x];
      }
    }
    store_parts<Cfg::PARTS>(g.out + m * g.ldo + n, g.plane, v);
  }
  if (!mirror) return;
#pragma unroll
  for (int e0 = 0; e0 < TN * 4; e0 += 64) {
    const int e = e0 + lane, c = e >> 2, ch = e & 3;
    const int m = n0 + c, n = m0 + 8 * ch;  // of the transpose
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const float*>(region + (8 * ch + x) * ROW + c * 4);
    if (m >= g.N || n >= g.M) continue;
    store_parts<Cfg::PARTS>(g.out + m * g.ldo + n, g.plane, v);
  }
}

// The direct loads of a slab: every part of A, then of B.
template <class Cfg, bool AMC, bool BMC>
struct PartsLoader {
  DmaSrc<typename Cfg::Base, Cfg::BM, AMC> da;
  DmaSrc<typename Cfg::Base, Cfg::BN, BMC> db;
  const char* na;
  const char* nb;
  int64_t a_step, b_step, a_plane, b_plane;
  int K, ik, is, left, wv;
  uint32_t lds0;

  __device__ __forceinline__ void issue_a() {
#pragma unroll
    for (int q = 0; q < Cfg::PARTS; ++q)
      da.issue(na + q * a_plane, K - ik, lds0 + static_cast<uint32_t>(is * Cfg::STAGE + q * Cfg::ABYTES), wv);
  }
  __device__ __forceinline__ void issue_b() {
#pragma unroll
    for (int q = 0; q < Cfg::PARTS; ++q)
      db.issue(nb + q * b_plane, K - ik, lds0 + static_cast<uint32_t>(is * Cfg::STAGE + Cfg::AREGION + q * Cfg::BBYTES), wv);
    is = is + 1 == Cfg::STAGES ? 0 : is + 1;
    if (left > 0) {
      --left;
      na += a_step;
      nb += b_step;
      ik += Cfg::BK;
    }
  }
};

// Fragments of one part of a k step.
template <class Cfg, bool AMC, bool BMC>
struct PartFrags {
  bf16x8 a[Cfg::FM], b[Cfg::FN];
  __device__ __forceinline__ void load(const char* st, int part, int wm, int wn, int kk) {
#pragma unroll
    for (int i = 0; i < Cfg::FM; ++i)
      a[i] = frag_bf16<typename Cfg::Base, Cfg::BM, AMC>(st + part * Cfg::ABYTES, wm * Cfg::TM + 32 * i, kk);
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
      b[j] = frag_bf16<typename Cfg::Base, Cfg::BN, BMC>(st + Cfg::AREGION + part * Cfg::BBYTES, wn * Cfg::TN + 32 * j, kk);
  }
};
template <class Cfg>
__device__ __forceinline__ void parts_mma(const bf16x8 (&a)[Cfg::FM], const bf16x8 (&b)[Cfg::FN], f32x16 (&acc)[Cfg::FM][Cfg::FN]) {
#pragma unroll
  for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
}

// The slab pipeline. A k step's instructions run in the order in which its fragments come:
// first parts (loaded during the step before), then with each further part while the
// instructions before them run. The barrier to the next slab lies behind the last
// fragments' reads and in front of the last instructions.
template <class Cfg, bool AMC, bool BMC>
__device__ __forceinline__ void run_parts(PartsLoader<Cfg, AMC, BMC>& ld, int nslab, int K, int k0,
                                          f32x16 (&acc)[Cfg::FM][Cfg::FN], int wm, int wn, int kw0, char* smem) {
  using Frags = PartFrags<Cfg, AMC, BMC>;
  using Base = typename Cfg::Base;
  using Acc = f32x16[Cfg::FM][Cfg::FN];
  // A wave with one block of outputs would wait for each instruction's result before the
  // next one: its further products go to sums of their own.
  constexpr bool CHAINS = Cfg::FM * Cfg::FN == 1;
  f32x16 more[CHAINS ? 2 : 1][Cfg::FM][Cfg::FN];
  if constexpr (CHAINS) {
#pragma unroll
    for (int r = 0; r < 16; ++r) more[0][0][0][r] = more[1][0][0][r] = 0.0f;
  }
  auto chain = [&](int c) -> Acc& { return CHAINS && c > 0 ? more[c - 1] : acc; };
  constexpr int STEPS = Cfg::KW / 16, AHEAD = Cfg::STAGES - 1;
  static_assert(STEPS == 2, "two k steps of a slab for each wave");
  if (nslab <= 0) return;
  auto tail = [&](char* st, int ck) {
    if (K - ck >= Cfg::BK) return;
#pragma unroll
    for (int q = 0; q < Cfg::PARTS; ++q) {
      fast_zero_tail<Base, Cfg::BM, AMC>(st + q * Cfg::ABYTES, K - ck);
      fast_zero_tail<Base, Cfg::BN, BMC>(st + Cfg::AREGION + q * Cfg::BBYTES, K - ck);
    }
    lds_barrier();
  };
  Frags h[2];
  int cs = 0, ck = k0;
  char* st = smem;
#pragma unroll
  for (int s = 0; s < AHEAD; ++s) ld.issue_a(), ld.issue_b();
  wait_vm<(AHEAD - 1) * Cfg::LPW>();
  lds_barrier();
  tail(st, ck);
  ld.issue_a();
  h[0].load(st, 0, wm, wn, kw0);
  for (int q = 0; q < nslab; ++q) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int kk = kw0 + 16 * s;
      Frags& f = h[s & 1];
      Frags lo, mid;
      lo.load(st, Cfg::PARTS - 1, wm, wn, kk);
      if constexpr (Cfg::PARTS == 3) mid.load(st, 1, wm, wn, kk);
      parts_mma<Cfg>(f.a, f.b, acc);
      if (s == 0) ld.issue_b();
      if constexpr (Cfg::PARTS == 3) {
        parts_mma<Cfg>(f.a, mid.b, chain(1));
        parts_mma<Cfg>(mid.a, f.b, chain(2));
        parts_mma<Cfg>(mid.a, mid.b, acc);
      }
      if (s + 1 < STEPS) {
        h[(s + 1) & 1].load(st, 0, wm, wn, kk + 16);
      } else if (q + 1 < nslab) {
        cs = cs + 1 == Cfg::STAGES ? 0 : cs + 1;
        ck += Cfg::BK;
        st = smem + cs * Cfg::STAGE;
        wait_vm<(AHEAD - 1) * Cfg::LPW>();
        lds_barrier();  // the next slab is visible; this one's fragments have been read by every wave
        tail(st, ck);
        ld.issue_a();
        h[0].load(st, 0, wm, wn, kw0);
      }
      parts_mma<Cfg>(f.a, lo.b, chain(1));
      parts_mma<Cfg>(lo.a, f.b, chain(2));
    }
  }
  if constexpr (CHAINS) acc[0][0] += more[0][0][0] + more[1][0][0];
  wait_vm<0>();  // no direct load may still write LDS past this point
}

struct PartsTiles {
  int nx, ny, tiles;
};
template <class Cfg>
__host__ __device__ inline PartsTiles parts_tiles(int M, int N, bool symmetric) {
  const int nx = (N + Cfg::BN - 1) / Cfg::BN, ny = (M + Cfg::BM - 1) / Cfg::BM;
  return {nx, ny, symmetric ? ny * (ny + 1) / 2 : nx * ny};
}

template <class Cfg, bool AMC, bool BMC>
__global__ void __launch_bounds__(Cfg::NT) parts_gemm_kernel(PartsArgs g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const PartsTiles n = parts_tiles<Cfg>(g.M, g.N, g.symmetric);
  const int pos = xcd_position(blockIdx.x, gridDim.x), split = pos / n.tiles, tile = pos - split * n.tiles;
  int row, col;
  if (g.symmetric)
    triangle_tile(tile, row, col);
  else
    grouped_order(tile, n.nx, n.ny, row, col);
  const int64_t m0 = static_cast<int64_t>(row) * Cfg::BM, n0 = static_cast<int64_t>(col) * Cfg::BN;
  const int lane = threadIdx.x & 63, ks = (threadIdx.x >> 6) / Cfg::OUTS, wave = (threadIdx.x >> 6) % Cfg::OUTS;
  const int wm = wave / Cfg::WGN, wn = wave % Cfg::WGN;
  f32x16 acc[Cfg::FM][Cfg::FN];
#pragma unroll
  for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  const int slabs = (g.K + Cfg::BK - 1) / Cfg::BK;
  const int q0 = static_cast<int>(static_cast<int64_t>(slabs) * split / g.splits);
  const int q1 = static_cast<int>(static_cast<int64_t>(slabs) * (split + 1) / g.splits);
  {
    PartsLoader<Cfg, AMC, BMC> ld;
    ld.wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the tile's first row and column go into the 64-bit bases
    ld.da.init(g.a.ld, 0, static_cast<int>(min<int64_t>(g.M - m0, Cfg::BM)), ld.wv);
    ld.db.init(g.b.ld, 0, static_cast<int>(min<int64_t>(g.N - n0, Cfg::BN)), ld.wv);
    ld.K = g.K;
    ld.ik = q0 * Cfg::BK;
    ld.a_step = (AMC ? g.a.ld : 1) * Cfg::BK * 2;
    ld.b_step = (BMC ? g.b.ld : 1) * Cfg::BK * 2;
    ld.a_plane = g.a.plane * 2;
    ld.b_plane = g.b.plane * 2;
    ld.na = uniform_ptr(reinterpret_cast<const char*>(g.a.p + (AMC ? m0 : m0 * g.a.ld)) + q0 * ld.a_step);
    ld.nb = uniform_ptr(reinterpret_cast<const char*>(g.b.p + (BMC ? n0 : n0 * g.b.ld)) + q0 * ld.b_step);
    ld.lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem));
    ld.is = 0;
    ld.left = q1 - q0 - 1;
    run_parts<Cfg, AMC, BMC>(ld, q1 - q0, g.K, q0 * Cfg::BK, acc, wm, wn, ks * Cfg::KW, smem);
  }
  // sums[4 (i, j, r / 4) + r % 4] of a lane, in pieces of four
  auto each4 = [&](float* sums, auto f) {
#pragma unroll
    for (int i = 0; i < Cfg::FM; ++i)
#pragma unroll
      for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; r += 4) f(*reinterpret_cast<f32x4*>(sums + (((i * Cfg::FN + j) * 4 + r / 4) * 64 + lane) * 4), acc[i][j], r);
  };
  auto put = [](f32x4& to, f32x16& a, int r) { to = f32x4{a[r], a[r + 1], a[r + 2], a[r + 3]}; };
  lds_barrier();  // every wave is done with the stages
  if constexpr (Cfg::KSPLIT > 1) {
    float* red = reinterpret_cast<float*>(smem);
    if (ks > 0) each4(red + ((ks - 1) * Cfg::OUTS + wave) * Cfg::SUMS, put);
    lds_barrier();
    if (ks > 0) return;
#pragma unroll
    for (int u = 0; u < Cfg::KSPLIT - 1; ++u)
      each4(red + (u * Cfg::OUTS + wave) * Cfg::SUMS, [](f32x4& from, f32x16& a, int r) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[r + e] += from[e];
      });
  }
  if (g.splits > 1) {
    each4(g.partial + ((static_cast<int64_t>(split) * n.tiles + tile) * Cfg::OUTS + wave) * Cfg::SUMS, put);
    return;
  }
  char* region = smem + Cfg::RED + wave * 32 * Cfg::ROW;
#pragma unroll
  for (int i = 0; i < Cfg::FM; ++i)
    parts_block<Cfg>(g, acc[i], static_cast<int>(m0) + wm * Cfg::TM + 32 * i, static_cast<int>(n0) + wn * Cfg::TN,
                     g.symmetric && row != col, region);
}

// Joins the splits' sums, in their order: a wave for 32 rows of a wave's part of a tile.
template <class Cfg>
__global__ void __launch_bounds__(64) parts_join_kernel(PartsArgs g) {
  __shared__ __attribute__((aligned(16))) char region[32 * Cfg::ROW];
  const PartsTiles n = parts_tiles<Cfg>(g.M, g.N, g.symmetric);
  const int i = blockIdx.x % Cfg::FM, wave = blockIdx.x / Cfg::FM % Cfg::OUTS, tile = blockIdx.x / (Cfg::FM * Cfg::OUTS);
  int row, col;
  if (g.symmetric)
    triangle_tile(tile, row, col);
  else
    grouped_order(tile, n.nx, n.ny, row, col);
  const int wm = wave / Cfg::WGN, wn = wave % Cfg::WGN;
  f32x16 acc[Cfg::FN];
#pragma unroll
  for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
  for (int split = 0; split < g.splits; ++split) {
    const float* from = g.partial + ((static_cast<int64_t>(split) * n.tiles + tile) * Cfg::OUTS + wave) * Cfg::SUMS;
#pragma unroll
    for (int j = 0; j < Cfg::FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(from + (((i * Cfg::FN + j) * 4 + r / 4) * 64 + threadIdx.x) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][r + e] += v[e];
      }
  }
  parts_block<Cfg>(g, acc, row * Cfg::BM + wm * Cfg::TM + 32 * i, col * Cfg::BN + wn * Cfg::TN, g.symmetric && row != col, region);
}

// ------------------------------------------------------------------ plans
enum PartsKind { PARTS_256, PARTS_192, PARTS_128, PARTS_64 };

// The 64 x 64 tile, for few tiles: two groups of waves share a slab's k, so that twice the
// waves hide its loads (512 x 784 in three parts, five iterations: 204 us with one, 184).
template <int P>
struct PartsCfgs {
  // two stages of 256 x 256 hold two parts only
  using C256 = typename std::conditional<P == 2, PartsCfg<P, 256, 256, 2, 4, 2>, PartsCfg<P, 256, 128, 4, 2, 2>>::type;
  using C192 = PartsCfg<P, 192, 192, 2, 2, P == 2 ? 3 : 2>;
  using C128 = PartsCfg<P, 128, 128, 2, 2, P == 2 ? 2 : 3>;
  using C64 = PartsCfg<P, 64, 64, 2, 2, P == 2 ? 4 : 3, 64, 2>;
};

struct PartsPlan {
  int kind, splits;
  size_t floats;  // of partial sums
};

constexpr int kPartsSplits = 16;

// The tile and split with the least modelled time, in us: rounds of the chip times a tile's
// instructions over the rate that a compute unit reaches with it, the partial sums' bytes
// twice and the launch that joins them. Measured on MI355X over 11 blocks of each type (64 x
// 64 to 1500 x 6000, five iterations): the pick takes at most 1.06 of the time of the best
// single tile (2048 x 2048 in two parts: 753 and 713 us), one tile for all up to 4.7 times
// (192 x 192 without splits on 512 x 512 in three: 764 us, the pick 173).
template <int P>
PartsPlan plan_parts(int M, int N, int K, bool symmetric) {
  struct Tile {
    int kind, bm, bn, bk, per;  // per: workgroups of a compute unit
    double one, full;           // flop/us of a compute unit on bf16 products, with one of them and with all
  };
  static constexpr Tile two[] = {{PARTS_256, 256, 256, 32, 1, 5.1e6, 5.1e6}, {PARTS_192, 192, 192, 32, 1, 4.3e6, 4.3e6},
                                 {PARTS_128, 128, 128, 32, 2, 2.9e6, 4.4e6}, {PARTS_64, 64, 64, 64, 1, 2.4e6, 2.4e6}};
  static constexpr Tile three[] = {{PARTS_256, 256, 128, 32, 1, 4.9e6, 4.9e6}, {PARTS_192, 192, 192, 32, 1, 4.6e6, 4.6e6},
                                   {PARTS_128, 128, 128, 32, 1, 3.8e6, 3.8e6}, {PARTS_64, 64, 64, 64, 1, 3.2e6, 3.2e6}};
  PartsPlan best = {PARTS_64, 1, 0};
  double best_t = 1e300;
  const int products = P == 2 ? 3 : 6;
  for (const Tile& c : P == 2 ? two : three) {
    if (symmetric && c.bm != c.bn) continue;  // the triangle is one of square tiles
    const int64_t ny = (M + c.bm - 1) / c.bm, nx = (N + c.bn - 1) / c.bn, n = symmetric ? ny * (ny + 1) / 2 : nx * ny;
    const int64_t slabs = (K + c.bk - 1) / c.bk;
    for (int s = 1; s <= kPartsSplits && (s == 1 || slabs / s >= 4); ++s) {
      const int64_t wgs = n * s, rounds = (wgs + kTargetBlocks * c.per - 1) / (kTargetBlocks * c.per);
      const double share = wgs >= kTargetBlocks * c.per ? c.per : static_cast<double>(wgs) / kTargetBlocks;
      const double work = 2.0 * c.bm * c.bn * c.bk * products * ((slabs + s - 1) / s);
      double t = 4.5 + 2.0 * (rounds - 1) + rounds * work * std::max(1.0 / c.one, share / c.full);
      const double bytes = 4.0 * c.bm * c.bn * wgs;
      if (s > 1) t += 4.0 + 2.0 * bytes / 5e6;
      if (t < best_t) best_t = t, best = {c.kind, s, s > 1 ? static_cast<size_t>(bytes / 4) : 0};
    }
  }
  return best;
}

template <class Cfg, bool AMC, bool BMC>
hipError_t launch_parts(const PartsArgs& g, hipStream_t stream) {
  auto kern = parts_gemm_kernel<Cfg, AMC, BMC>;
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, Cfg::LDS);
  if (attr != hipSuccess) return attr;
  const unsigned tiles = static_cast<unsigned>(parts_tiles<Cfg>(g.M, g.N, g.symmetric).tiles);
  hipLaunchKernelGGL(kern, dim3(tiles * g.splits), dim3(Cfg::NT), Cfg::LDS, stream, g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.splits == 1) return e;
  hipLaunchKernelGGL(parts_join_kernel<Cfg>, dim3(tiles * Cfg::FM * Cfg::OUTS), dim3(64), 0, stream, g);
  return hipGetLastError();
}

// g but for splits; partial holds the plan's floats.
template <int P, bool AMC, bool BMC>
hipError_t run_parts_gemm(PartsArgs g, float* partial, hipStream_t stream) {
  if (g.M <= 0 || g.N <= 0) return hipSuccess;
  const PartsPlan p = plan_parts<P>(g.M, g.N, g.K, g.symmetric);
  g.splits = p.splits;
  g.partial = partial;
  using C = PartsCfgs<P>;
  switch (p.kind) {
    case PARTS_256: return launch_parts<typename C::C256, AMC, BMC>(g, stream);
    case PARTS_192: return launch_parts<typename C::C192, AMC, BMC>(g, stream);
    case PARTS_128: return launch_parts<typename C::C128, AMC, BMC>(g, stream);
    default: return launch_parts<typename C::C64, AMC, BMC>(g, stream);
  }
}

}  // namespace ard
