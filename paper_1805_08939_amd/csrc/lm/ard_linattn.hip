// Linear attention with a decay for each head: prompts, their gradients, and
// single tokens.
//
// With a = exp(log_decay) of the head, for every sequence
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t.
// One operator does the forward pass and every gradient. For three inputs x, y, w
// of the tokens it computes, running forward or backward in time,
//   forward:  out_i = sum_{j <= i} a^{i-j} (x_i . y_j) w_j + a^{i+1} x_i R
//   backward: out_i = sum_{j >= i} a^{j-i} (x_i . y_j) w_j + a^{n-1-i} x_i R
// with R the state given at the start (or the end) of the sequence, and
//   forward pass: (x, y, w) = (q, k, v)      dQ: forward,  (dO, v, k), R = S0^T
//   dK: backward, (v, dO, q), R = dST^T      dV: backward, (k, q, dO), R = dST
// whose last state is dS0 (the backward run carries a R_{i+1} from token to token).
//
// Chunks of 64 tokens: with y' the weighted y, per chunk of L tokens
//   out = ((x y^T) . weights) w + weights' (x R),   R <- a^L R + y'^T w.
// All matrix products are MFMA (16 x 16 blocks) on tiles in LDS, [row][token] as
// in memory. The inner products of a chunk stay in registers: a lane of the
// product y^T x holds, of one token i, the four j that it must hold as an operand
// of the product with w. R is kept in fp32 accumulators from chunk to chunk.
//
// Roundings with bf16 inputs: the weighted inner products, and R as an operand of
// x R (once per chunk, never in the running state): each adds an error of the size
// of the output's own rounding to one of the two terms (measured: 1.4 times the error of
// a pass in fp32 throughout), for products at 7 times the rate of fp32 operands. y' is
// split into three bf16 parts (its 24 bits), so the state is exact to fp32; into two
// where a state goes into outputs only, which round it to 8 bits. fp32 inputs use fp32
// MFMA throughout.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "../ard_gemm_fast.hpp"
#include "../ard_internal.hpp"

namespace ard {
namespace {

constexpr int kChunk = 64;

struct MixArgs {
  const void* x;
  const void* y;
  const void* w;
  void* out;             // of the element type, or fp32 (Mix::PART)
  const float* decay;    // [heads]
  const float* s0;       // given states, or NULL
  float* sT;             // last states, or NULL
  float* seg;            // states of the segments, or NULL (one segment)
  const int32_t* offsets;
  int32_t n_seqs, max_len, tokens, heads, group;
  int32_t ydim, wdim;    // rows of x and y, of w and out
  int32_t x_shared, y_shared, w_shared;  // read by head / group
  int32_t s_trans;       // states are stored [wdim][ydim]
  int32_t nseg, seg_len; // segments of a sequence; tokens of one, whole chunks
  int32_t wtiles;        // tiles of w rows
  float cp, cy, cx;      // factors of the inner products, of y' and of x R
};

// Columns [first, first + len) of sequence s, within the row.
struct Span {
  int32_t first, len;
};
__device__ __forceinline__ Span span_of(const MixArgs& g, int s) {
  if (!g.offsets) return {s * g.max_len, g.max_len};
  const int32_t a = min(max(g.offsets[s], 0), g.tokens), b = min(max(g.offsets[s + 1], 0), g.tokens);
  return {a, min(max(b - a, 0), g.max_len)};
}

// a^n as 2^(n log2 a); a decay of -inf gives a^0 = 1 and 0 beyond.
struct Decay {
  float l2;
  __device__ __forceinline__ explicit Decay(float g) : l2((g < -1e30f ? -1e30f : g) * 1.44269504088896340736f) {}
  __device__ __forceinline__ float pow(int n) const { return pow(static_cast<float>(n)); }
  __device__ __forceinline__ float pow(float n) const { return __builtin_amdgcn_exp2f(l2 * n); }
  // Of an inner product that is no masked one: not 0, which mul_masked would take for the
  // mask (what the smallest normal number adds is below every rounding).
  __device__ __forceinline__ float weight(int n) const {
    const float w = pow(n);
    return w < 1.17549435e-38f ? 1.17549435e-38f : w;
  }
};

// ------------------------------------------------------------------ LDS tiles
// [rows][COLS] of 16-byte chunks, chunk c of row r at position c ^ swz(r): free of bank
// conflicts for 16 rows at one chunk (operands along the contraction; a pass of the
// 16-byte reads takes rows 0-3 and 12-15 of one chunk with rows 4-11 of the next), for
// rows {0, 1, 4, 5} + 8 g at two neighbouring chunks (transposed reads) and for four
// neighbouring rows at four chunks (fp32 elements). swz depends on r % 16 only.
template <int ES, int COLS>
__device__ __forceinline__ int swz(int r) {
  if constexpr (COLS * ES / 16 == 8)
    return (r >> 1) & 7;
  else if constexpr (ES == 4)
    return ((r & 3) << 2) | (((r >> 2) & 3) ^ ((r >> 1) & 2));
  else
    return ((r & 1) << 1) | (r & 12) | ((r >> 1) & 1);
}
template <int ES, int COLS>
__device__ __forceinline__ int tile_off(int r, int c) {
  return r * COLS * ES + ((c ^ swz<ES, COLS>(r)) << 4);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// MFMA operands of 16 x 16 blocks. Along: 16 rows of a tile, the contraction along
// its columns (16 bytes of a lane). Across: 16 columns, the contraction along its
// rows. bf16: a step of 32; fp32: Along 16 (four MFMAs, slot g holding 4 g + e),
// Across 4. A lane's address is computed once per kind of read (base_*) for row and
// column 0; constant columns enter by exclusive or, constant rows by addition, so
// that a read costs no arithmetic and no register of its own.
template <typename T>
struct Ops;
template <>
struct Ops<bf16> {
  using Along = bf16x8;
  using Across = bf16x8;
  static constexpr int ALONG = 32, ACROSS = 32;
  template <int COLS>
  static __device__ __forceinline__ int base_along() {
    return tile_off<2, COLS>(threadIdx.x & 15, (threadIdx.x >> 4) & 3);
  }
  template <int COLS>
  static __device__ __forceinline__ Along along(const char* t, int base, int row, int col) {
    return *reinterpret_cast<const bf16x8*>(t + row * COLS * 2 + (base ^ (col * 2)));
  }
  struct Base {
    int lo, hi;  // rows 8 g + {0, 1, 4, 5} and + {2, 3, 6, 7}
  };
  template <int COLS>
  static __device__ __forceinline__ Base base_across() {
    const int lane = threadIdx.x & 63, s = lane & 15, c = 4 * (s & 3);
    const int r = 8 * (lane >> 4) + ((s >> 2) & 1) + 4 * (s >> 3);
    return {tile_off<2, COLS>(r, c >> 3) + (c & 7) * 2, tile_off<2, COLS>(r + 2, c >> 3) + (c & 7) * 2};
  }
  template <int COLS>
  static __device__ __forceinline__ Across across(const char* t, Base base, int row, int col) {
    const char* p0 = t + row * COLS * 2 + (base.lo ^ (col * 2));
    const char* p1 = t + row * COLS * 2 + (base.hi ^ (col * 2));
    const bf16x4 lo = __builtin_bit_cast(
        bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p0)));
    const bf16x4 hi = __builtin_bit_cast(
        bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p1)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // The four columns 4 g .. of a row, 16 rows: how a lane holds a product's block.
  template <int COLS>
  static __device__ __forceinline__ int base_block() {
    const int g = (threadIdx.x >> 4) & 3;
    return tile_off<2, COLS>(threadIdx.x & 15, g >> 1) + (g & 1) * 8;
  }
  template <int COLS>
  static __device__ __forceinline__ bf16x4* block(char* t, int base, int row, int col) {
    return reinterpret_cast<bf16x4*>(t + row * COLS * 2 + (base ^ (col * 2)));
  }
  static __device__ __forceinline__ bf16x4 round(f32x4 v) { return __builtin_convertvector(v, bf16x4); }
  static __device__ __forceinline__ f32x4 mma(Across a, Across b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Ops<float> {
  using Along = f32x4;
  using Across = float;
  static constexpr int ALONG = 16, ACROSS = 4;
  template <int COLS>
  static __device__ __forceinline__ int base_along() {
    return tile_off<4, COLS>(threadIdx.x & 15, (threadIdx.x >> 4) & 3);
  }
  template <int COLS>
  static __device__ __forceinline__ Along along(const char* t, int base, int row, int col) {
    return *reinterpret_cast<const f32x4*>(t + row * COLS * 4 + (base ^ (col * 4)));
  }
  using Base = int;
  template <int COLS>
  static __device__ __forceinline__ Base base_across() {
    const int lane = threadIdx.x & 63;
    return tile_off<4, COLS>(lane >> 4, (lane & 15) >> 2) + (lane & 3) * 4;
  }
  template <int COLS>
  static __device__ __forceinline__ Across across(const char* t, Base base, int row, int col) {
    return *reinterpret_cast<const float*>(t + row * COLS * 4 + (base ^ (col * 4) ^ ((((row >> 2) & 3) ^ ((row >> 1) & 2)) << 4)));
  }
  template <int COLS>
  static __device__ __forceinline__ int base_block() {
    return base_along<COLS>();
  }
  template <int COLS>
  static __device__ __forceinline__ f32x4* block(char* t, int base, int row, int col) {
    return reinterpret_cast<f32x4*>(t + row * COLS * 4 + (base ^ (col * 4)));
  }
  static __device__ __forceinline__ f32x4 round(f32x4 v) { return v; }
  static __device__ __forceinline__ f32x4 mma(Across a, Across b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

// A thread's share of a [D][64] tile on its way from memory. Rows past the operand's
// and tokens past L are zero in LDS; every load is made all the same, of the last
// row or, in a partial chunk, of whatever follows (branches around the loads would
// keep them from running together). The 16 bytes that would reach past the tensor
// itself (of its last rows only) are read again, token by token.
template <typename T, int D, int NT>
struct TileRegs {
  static constexpr int ES = sizeof(T), EPC = 16 / ES, CPR = kChunk * ES / 16, PER = D * CPR / NT, RPI = NT / CPR;
  static_assert(D * CPR % NT == 0, "whole rounds");
  u32x4 v[PER];
  const char* last;  // where 16 bytes of the tensor may start at the latest
  const T* base;     // row 0 at the sequence's first token
  const T* end;
  int64_t ld;
  int rows;
  int tid;  // threadIdx.x, by name: a kernel may keep what follows from it out of its registers

  // base: row 0 at the sequence's first token; first, end: the tensor (of a tensor
  // below 16 bytes, which starts on 16, the 16 that it starts are read)
  __device__ __forceinline__ void init(const T* base_, int64_t ld_, int rows_, const T* first, const T* end_) {
    base = base_, ld = ld_, rows = rows_, end = end_, tid = threadIdx.x;
    last = reinterpret_cast<const char*>(end - first < EPC ? first : end - EPC);
  }
  __device__ __forceinline__ const char* at(int i, int t) const {  // the thread's bytes i of the chunk at t
    const int r = tid / CPR, c = tid % CPR;
    return reinterpret_cast<const char*>(base + t + static_cast<int64_t>(min(r + i * RPI, rows - 1)) * ld + c * EPC);
  }
  __device__ __forceinline__ void load(int t) {  // a whole chunk
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = load16_any<ES>(at(i, t));
  }
  __device__ __forceinline__ void load_part(int t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const char* q = at(i, t);
      v[i] = load16_any<ES>(q < last ? q : last);
    }
  }
  __device__ __forceinline__ void store(char* lds, int t, int L) {
    const int r = tid / CPR, c = tid % CPR, n = L - c * EPC;
    if (L < kChunk || rows < D) {  // uniform
      u32x4 keep;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int m = (n - q * (EPC / 4)) * ES * 8;  // valid bits of the word
        keep[q] = m >= 32 ? ~0u : m <= 0 ? 0u : 0xffffu;
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) v[i] &= r + i * RPI < rows ? keep : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = i * NT + tid;
      *reinterpret_cast<u32x4*>(lds + tile_off<ES, kChunk>(at / CPR, at % CPR)) = v[i];
    }
    if (L < kChunk && base + t + (rows - 1) * ld + (L + EPC - 1) / EPC * EPC > end) {  // uniform
#pragma unroll 1
      for (int i = 0; i < PER; ++i) {
        const int row = r + i * RPI;
        if (row >= rows || n <= 0) continue;
        const T* q = base + t + row * ld + c * EPC;
        T e[EPC];
#pragma unroll
        for (int u = 0; u < EPC; ++u) e[u] = q[u < n ? u : n - 1];
        T* to = reinterpret_cast<T*>(lds + tile_off<ES, kChunk>(row, c));
#pragma unroll
        for (int u = 0; u < EPC; ++u) to[u] = u < n ? e[u] : from_f32<T>(0.0f);
      }
    }
  }
};

// Eight fp32 as N bf16 each that add up to it (N = 3: to its 24 bits; 2: to 17).
template <int N>
__device__ __forceinline__ void split(const float (&f)[8], bf16x8 (&s)[N]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    f32x2 v = {f[e], f[e + 1]};
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const bf16x2 h = __builtin_convertvector(v, bf16x2);
      s[q][e] = h[0], s[q][e + 1] = h[1];
      if (q + 1 < N) v[0] -= static_cast<float>(h[0]), v[1] -= static_cast<float>(h[1]);
    }
  }
}

// Tokens behind the mask that are not finite. As an operand y they are kept from the
// inner products by mul_masked (0 times anything is 0). As an operand w they make NaN of
// the outputs in front of them, 0 times not finite in the matrix product: a wave that has
// an output that is not finite computes its outputs again (mend_outputs).
//
// v_mul_legacy_f32 by the name of its intrinsic, which the compiler has no builtin for (one
// that lacks the intrinsic fails to link). A comparison and a choice in its place cost 2 to 8%:
// 9 sequences, 16411 tokens in all, 16 heads of 64, bf16: 83.5 to 89.4 us, gradients 259 to 275.
extern "C" __device__ __attribute__((const)) float mul_masked(float p, float weight) __asm("llvm.amdgcn.fmul.legacy");

// Four values that w holds of a row: 0 in place of those that are not finite, and 1 for
// each of those.
template <typename V>
__device__ __forceinline__ void sort_out(V& w, V& bad) {
  constexpr int N = sizeof(V) / sizeof(w[0]);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float f = static_cast<float>(w[e]);
    const bool fin = fabsf(f) <= 3.4028234663852886e38f;
    w[e] = fin ? w[e] : static_cast<decltype(f)>(0.0f);
    bad[e] = fin ? static_cast<decltype(f)>(0.0f) : static_cast<decltype(f)>(1.0f);
  }
}

// The outputs of 16 tokens again (whole waves), from the tiles in LDS and in the order of
// the first computation, with 0 in place of the values of w that are not finite. A second
// product of the mask and the places of those values tells which outputs the formula has
// one of them in; the others are written over what Out holds. Blocks b0 .. b0 + blocks - 1
// of 16 rows; SROW: the state is read along its rows, S[row][k], else across, S[k][row].
// A chunk that needs it costs a second computation of its outputs, whatever the values: 4 x
// 4096 tokens, 16 heads of 128, bf16: 128 us forward and 300 backward, with a token that is
// not finite in every chunk 190 and 470; fp32 472 and 1470, then 940 and 2890. Finite inputs
// pay for the check of the outputs, 128 x 128 3 to 4%, 64 x 64 1%.
template <typename T, typename OutT, int XD, int SCOLS, bool SROW, bool REV>
__device__ __forceinline__ void mend_outputs(const char* X, const char* Y, char* W, const char* S, char* Out, int ib,
                                             int b0, int blocks, int L, const Decay& a, float cp, float cx) {
  using O = Ops<T>;
  using OutOps = Ops<OutT>;
  // nothing of this is computed ahead of the chunks and kept in registers for them
  int lane = threadIdx.x & 63, at_block = O::template base_block<kChunk>();
  auto at_cols = O::template base_across<kChunk>();
  asm volatile("" : "+v"(lane), "+v"(at_block));
  if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(at_cols.lo), "+v"(at_cols.hi));
  else asm volatile("" : "+v"(at_cols));
  const int grp = lane >> 4;
  f32x4 p[4], in[4];  // weighted inner products, and the mask
#pragma unroll
  for (int jb = 0; jb < 4; ++jb) p[jb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
  for (int k = 0; k < XD; k += O::ACROSS) {
    const auto xf = O::template across<kChunk>(X, at_cols, k, 16 * ib);
#pragma unroll
    for (int jb = 0; jb < 4; ++jb) p[jb] = O::mma(O::template across<kChunk>(Y, at_cols, k, 16 * jb), xf, p[jb]);
  }
#pragma unroll
  for (int jb = 0; jb < 4; ++jb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = (REV ? -1 : 1) * (16 * (ib - jb) + (lane & 15) - 4 * grp - r);
      p[jb][r] = mul_masked(p[jb][r], n >= 0 ? cp * a.weight(max(n, 0)) : 0.0f);
      in[jb][r] = n >= 0 ? 1.0f : 0.0f;
    }
  bf16x8 pf[2], inf[2];  // of 32 tokens j each
#pragma unroll
  for (int h = 0; h < 2 && sizeof(T) == 2; ++h) {
    pf[h] = __builtin_shufflevector(Ops<bf16>::round(p[2 * h]), Ops<bf16>::round(p[2 * h + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
    inf[h] = __builtin_shufflevector(Ops<bf16>::round(in[2 * h]), Ops<bf16>::round(in[2 * h + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
  }
#pragma unroll 1
  for (int b = b0; b < b0 + blocks; ++b) {
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f}, q = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int k = 0; k < XD; k += O::ACROSS) {
      auto xf = O::template across<kChunk>(X, at_cols, k, 16 * ib);
      if constexpr (SROW) {  // its rows in order (bf16)
        xf = __builtin_shufflevector(xf, xf, 0, 1, 4, 5, 2, 3, 6, 7);
        acc = O::mma(xf, O::template along<SCOLS>(S, O::template base_along<SCOLS>(), 16 * b, k), acc);
      } else {
        acc = O::mma(xf, O::template across<SCOLS>(S, O::template base_across<SCOLS>(), k, 16 * b), acc);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * ib + 4 * grp + r;
      acc[r] *= cx * a.pow(max(REV ? L - 1 - i : i + 1, 0));
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x4 lo = *O::template block<kChunk>(W, at_block, 16 * b, 32 * h), lob;
        bf16x4 hi = *O::template block<kChunk>(W, at_block, 16 * b, 32 * h + 16), hib;
        sort_out(lo, lob);
        sort_out(hi, hib);
        acc = O::mma(pf[h], __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), acc);
        q = O::mma(inf[h], __builtin_shufflevector(lob, hib, 0, 1, 2, 3, 4, 5, 6, 7), q);
      }
    } else {
#pragma unroll
      for (int jb = 0; jb < 4; ++jb) {
        if ((REV ? jb < ib : jb > ib) || 16 * jb >= L) continue;
        f32x4 w = O::template along<kChunk>(W, at_block, 16 * b, 16 * jb), bad;
        sort_out(w, bad);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          acc = O::mma(p[jb][r], w[r], acc);
          q = O::mma(in[jb][r], bad[r], q);
        }
      }
    }
    auto* to = OutOps::template block<kChunk>(Out, OutOps::template base_block<kChunk>(), 16 * b, 16 * ib);
    auto v = *to;
    const auto clean = OutOps::round(acc);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = q[r] == 0.0f ? clean[r] : v[r];
    *to = v;
  }
}

template <typename T_, int YD_, int WD_, bool REV_, bool OUT_, bool PART_, int PARTS_ = 3>
struct Mix {
  using T = T_;
  static constexpr int YD = YD_, WD = WD_;  // rows of x and y, of w, as padded
  static constexpr bool REV = REV_;
  static constexpr bool OUT = OUT_;    // outputs (else the states of segments only)
  static constexpr bool PART = PART_;  // outputs in fp32, to be added over the heads that share a row
  static constexpr int PARTS = PARTS_;  // bf16 parts of y': 3, or 2 where the state ends in outputs only
  static constexpr int ES = sizeof(T), OS = PART ? 4 : ES;
  // a wave for each 16 rows of y (its part of the state); for the outputs, of which
  // there are four blocks of 16 tokens, eight waves share the rows of w by halves
  static constexpr int NW = YD / 16, NT = 64 * NW, HALVES = NW / 4;
  static constexpr int WB = WD / 16, OB = WB / HALVES;  // 16-blocks of w rows: all, and a wave's
  static constexpr int XT = YD * kChunk * ES, WT = WD * kChunk * ES;
  static constexpr int ST = YD * WD * ES, OT = WD * kChunk * OS;
  static constexpr int MINW = 2;
  static constexpr int LDS = OUT ? 2 * XT + WT + ST + OT : XT + WT;
};

// The state's accumulators of a wave: its 16 rows of y (lane % 16) by blocks of 16
// rows of w (4 (lane / 16) + r).
template <class M>
struct State {
  f32x4 a[M::WB];
  __device__ __forceinline__ int y(int wv) const { return wv * 16 + (threadIdx.x & 15); }
  __device__ __forceinline__ int w(int b) const { return b * 16 + 4 * ((threadIdx.x >> 4) & 3); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < M::WB; ++i) a[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // a state of the caller's: [ydim][wdim] or its transpose; w0: first row of w of this tile
  template <bool STORE>
  __device__ __forceinline__ void given(float* p, const MixArgs& g, int wv, int w0) {
    const int yr = y(wv);
    if (yr >= g.ydim) return;
    if (!g.s_trans && g.wdim % 4 == 0) {  // 16 bytes of a row (states are 16-byte aligned)
#pragma unroll
      for (int i = 0; i < M::WB; ++i) {
        const int wr = w0 + w(i);
        f32x4* at = reinterpret_cast<f32x4*>(p + yr * g.wdim + wr);
        if (wr < g.wdim) {
          if constexpr (STORE) *at = a[i];
          else a[i] = *at;
        }
      }
      return;
    }
    const int ys = g.s_trans ? 1 : g.wdim, ws = g.s_trans ? g.ydim : 1;
#pragma unroll
    for (int i = 0; i < M::WB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int wr = w0 + w(i) + r;
        float* at = p + yr * ys + wr * ws;
        if (wr < g.wdim) {
          if constexpr (STORE) *at = a[i][r];
          else a[i][r] = *at;
        }
      }
  }
  // a segment's, in the accumulators' own order
  __device__ __forceinline__ f32x4* place(float* p, int wv, int i) const {
    return reinterpret_cast<f32x4*>(p) + (wv * M::WB + i) * 64 + (threadIdx.x & 63);
  }
};

// A workgroup per segment of a sequence, head and tile of w rows: with OUT the outputs from
// the state in front of the segment, else only what the segment adds to the state. Long
// sequences of few heads are split so, as one workgroup on each would leave the chip empty;
// y and w are then read twice. A chunk is a chain of waits (loads, LDS, matrix products,
// LDS, store) on one or two workgroups of a compute unit, which is what bounds it: 4 x 4096
// tokens, 16 heads of 128, bf16: states 41 us, outputs 84 us, matrix cores 26% and 20% busy;
// where one segment is enough (32 x 1024, heads of 64) the whole call is 57 us, 5.0 TB/s of
// inputs and outputs. fp32 is bound by its matrix products (1/16 of the bf16 rate): the
// same 4 x 4096 466 us forward.
template <class M>
__global__ void __launch_bounds__(M::NT, M::MINW) mix_kernel(MixArgs g) {
  using T = typename M::T;
  using O = Ops<T>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* Y = smem;
  char* W = Y + M::XT;
  char* X = W + M::WT;
  char* S = X + M::XT;   // the state as an operand
  char* Out = S + M::ST;  // the outputs on their way out

  // workgroup -> segment, tile of w, head, sequence (neighbours on one XCD)
  int id = xcd_position(blockIdx.x, gridDim.x);
  const int seg = id % g.nseg;
  id /= g.nseg;
  const int wt = id % g.wtiles;
  id /= g.wtiles;
  const int head = id % g.heads, seq = id / g.heads;
  const Span sp = span_of(g, seq);
  const int t0 = seg * g.seg_len, t1 = t0 + min(sp.len - t0, g.seg_len);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w0 = wt * M::WD, wrows = min(g.wdim - w0, M::WD);
  const int64_t hs = static_cast<int64_t>(seq) * g.heads + head;
  const int64_t sdim = static_cast<int64_t>(g.ydim) * g.wdim;
  float* segp = g.seg ? g.seg + ((hs * g.wtiles + wt) * g.nseg + seg) * M::YD * M::WD : nullptr;
  if (g.nseg > 1 && t0 >= t1) return;  // whole workgroups

  const Decay a(g.decay[head]);
  State<M> st;
  st.clear();
  if (M::OUT) {
    if (g.nseg > 1) {
#pragma unroll
      for (int i = 0; i < M::WB; ++i) st.a[i] = *st.place(segp, wv, i);
    } else if (g.s0) {
      st.template given<false>(const_cast<float*>(g.s0) + hs * sdim, g, wv, w0);
    }
  }

  const int64_t ld = g.tokens;
  auto rows = [&](const void* p, int shared, int dim) {
    return static_cast<const T*>(p) + (static_cast<int64_t>(shared ? head / g.group : head) * dim) * ld + sp.first;
  };
  auto end = [&](const void* p, int shared, int dim) {
    const int64_t n = static_cast<int64_t>(shared ? g.heads / g.group : g.heads) * dim * ld;
    return static_cast<const T*>(p) + n;
  };
  TileRegs<T, M::YD, M::NT> xr, yr;
  TileRegs<T, M::WD, M::NT> wr;
  if (M::OUT)
    xr.init(rows(g.x, g.x_shared, g.ydim), ld, g.ydim, static_cast<const T*>(g.x), end(g.x, g.x_shared, g.ydim));
  yr.init(rows(g.y, g.y_shared, g.ydim), ld, g.ydim, static_cast<const T*>(g.y), end(g.y, g.y_shared, g.ydim));
  wr.init(rows(g.w, g.w_shared, g.wdim) + w0 * ld, ld, wrows, static_cast<const T*>(g.w),
          end(g.w, g.w_shared, g.wdim));
  int at_along = O::template base_along<kChunk>(), at_block = O::template base_block<kChunk>();
  const int at_state = O::template base_block<M::WD>();
  auto at_cols = O::template base_across<kChunk>();
  auto at_scols = O::template base_across<M::WD>();
  // the wave's 16 columns: part of the lane's address, since they differ by wave
  using OutT = typename std::conditional<M::PART, float, T>::type;
  using OutOps = Ops<OutT>;
  auto at_icols = at_cols;
  const int ic = (wv & 3) * 16 * M::ES, sc = M::HALVES > 1 ? (wv >> 2) * (M::WD / 2) * M::ES : 0;
  if constexpr (M::ES == 2) at_icols.lo ^= ic, at_icols.hi ^= ic, at_scols.lo ^= sc, at_scols.hi ^= sc;
  else at_icols ^= ic, at_scols ^= sc;
  const int at_out = OutOps::template base_block<kChunk>() ^ ((wv & 3) * 16 * M::OS);

  const int nchunk = static_cast<int>((static_cast<uint32_t>(t1 - t0) + kChunk - 1) / kChunk);
  auto first_of = [&](int c) { return t0 + (M::REV ? nchunk - 1 - c : c) * kChunk; };
  auto fetch = [&](int c) {
    const int t = first_of(c);
    if (t1 - t >= kChunk) {
      if (M::OUT) xr.load(t);
      yr.load(t);
      wr.load(t);
    } else {
      if (M::OUT) xr.load_part(t);
      yr.load_part(t);
      wr.load_part(t);
    }
  };
  // The weights, of a lane: those of the inner products (its token i, the tokens j =
  // 16 jb + 4 grp + r), of x R (tokens 16 ib + 4 grp + r) and of y' (of each step's
  // tokens). Only the last two know the chunk's length: they change for a partial one.
  constexpr int NA = 16 / M::ES;  // tokens of a lane in a step of the state's product
  const int ib = wv & 3, grp = lane >> 4;
  f32x4 pw[M::OUT ? 4 : 1], wx;
  float fy[kChunk / O::ALONG][NA];
  if constexpr (M::OUT) {
#pragma unroll
    for (int jb = 0; jb < 4; ++jb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = (M::REV ? -1 : 1) * (16 * (ib - jb) + (lane & 15) - 4 * grp - r);
        pw[jb][r] = n >= 0 ? g.cp * a.weight(n) : 0.0f;
      }
  }
  auto weigh = [&](int L) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * ib + 4 * grp + r;
      wx[r] = g.cx * a.pow(max(M::REV ? L - 1 - i : i + 1, 0));
    }
#pragma unroll
    for (int k = 0; k < kChunk / O::ALONG; ++k)
#pragma unroll
      for (int e = 0; e < NA; ++e) {
        const int tok = k * O::ALONG + NA * grp + e;
        fy[k][e] = g.cy * a.pow(M::REV ? tok + 1 : max(L - 1 - tok, 0));
      }
  };
  int weighed = -1;

  // The barriers order LDS only: the next chunk's loads and this one's stores stay in flight.
  if (nchunk > 0) fetch(0);
  for (int c = 0; c < nchunk; ++c) {
    const int t = first_of(c), L = min(kChunk, t1 - t);
    // fp32 reads across rows have 16 addresses for each base (bf16: 4): computed in each
    // chunk, as they do not fit the registers if they are kept from one to the next
    if constexpr (M::OUT && M::ES == 4)
      asm volatile("" : "+v"(at_along), "+v"(at_block), "+v"(at_cols), "+v"(at_icols), "+v"(at_scols));
    if constexpr (M::OUT && M::ES == 2 && M::YD < M::WD)  // four waves hold the state that elsewhere eight do
      asm volatile("" : "+v"(at_along), "+v"(at_block), "+v"(at_cols.lo), "+v"(at_cols.hi));
    yr.store(Y, t, L);
    wr.store(W, t, L);
    if constexpr (M::OUT) {
      xr.store(X, t, L);
#pragma unroll
      for (int i = 0; i < M::WB; ++i)
        *O::template block<M::WD>(S + wv * 16 * M::WD * M::ES, at_state, 0, 16 * i) = O::round(st.a[i]);
    }
    lds_barrier();
    if (c + 1 < nchunk) fetch(c + 1);
    if (L != weighed) weigh(weighed = L);
    // The outputs read the state in LDS, the state's update the one in registers: neither
    // waits for the other.
    const int b0 = M::HALVES > 1 ? (wv >> 2) * M::OB : 0;
    float bad = 0.0f;  // NaN if an output of the lane is not finite
    auto outputs = [&]() {
      // outputs of 16 tokens i: out[i][w] = sum_y x[y][i] R[y][w], weighted, plus the chunk's own.
      // A lane of p holds token i = 16 ib + lane % 16 and tokens j = 16 jb + 4 grp + r; one of acc
      // tokens i = 16 ib + 4 grp + r and row w = 16 b + lane % 16.
      char* Wo = W + b0 * 16 * kChunk * M::ES;
      f32x4 acc[M::OB];
#pragma unroll
      for (int b = 0; b < M::OB; ++b) acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      f32x4 p[4];
#pragma unroll
      for (int jb = 0; jb < 4; ++jb) p[jb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < M::YD; k += O::ACROSS) {
        const auto xf = O::template across<kChunk>(X, at_icols, k, 0);
#pragma unroll
        for (int b = 0; b < M::OB; ++b) acc[b] = O::mma(xf, O::template across<M::WD>(S, at_scols, k, 16 * b), acc[b]);
        if constexpr (M::ES == 2) {  // every block of j: branches would cost more than the products
#pragma unroll
          for (int jb = 0; jb < 4; ++jb) p[jb] = O::mma(O::template across<kChunk>(Y, at_cols, k, 16 * jb), xf, p[jb]);
        }
      }
#pragma unroll
      for (int b = 0; b < M::OB; ++b) acc[b] *= wx;
      auto weighed_p = [&](int jb) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = mul_masked(p[jb][r], pw[jb][r]);
        return v;
      };
      if constexpr (M::ES == 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 32 tokens j
          const bf16x8 pf =
              __builtin_shufflevector(O::round(weighed_p(2 * h)), O::round(weighed_p(2 * h + 1)), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int b = 0; b < M::OB; ++b) {
            const bf16x4 lo = *O::template block<kChunk>(Wo, at_block, 16 * b, 32 * h);
            const bf16x4 hi = *O::template block<kChunk>(Wo, at_block, 16 * b, 32 * h + 16);
            acc[b] = O::mma(pf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), acc[b]);
          }
        }
      } else {
#pragma unroll
        for (int jb = 0; jb < 4; ++jb) {
          if ((M::REV ? jb < ib : jb > ib) || 16 * jb >= L) continue;
#pragma unroll
          for (int k = 0; k < M::YD; k += O::ACROSS)
            p[jb] = O::mma(O::template across<kChunk>(Y, at_cols, k, 16 * jb),
                           O::template across<kChunk>(X, at_icols, k, 0), p[jb]);
          p[jb] = weighed_p(jb);
#pragma unroll
          for (int b = 0; b < M::OB; ++b) {
            const auto wf = O::template along<kChunk>(Wo, at_along, 16 * b, 16 * jb);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[b] = O::mma(p[jb][r], wf[r], acc[b]);
          }
        }
      }
#pragma unroll
      for (int b = 0; b < M::OB; ++b)
        *OutOps::template block<kChunk>(Out + b0 * 16 * kChunk * M::OS, at_out, 16 * b, 0) = OutOps::round(acc[b]);
#pragma unroll
      for (int b = 0; b < M::OB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) bad = fmaf(acc[b][r], 0.0f, bad);
    };
    auto update = [&]() {  // the state past this chunk
      const float aL = a.pow(L);
#pragma unroll
      for (int i = 0; i < M::WB; ++i) st.a[i] *= aL;
      char* Yw = Y + wv * 16 * kChunk * M::ES;
#pragma unroll
      for (int k = 0; k < kChunk; k += O::ALONG) {
        if (M::ES == 4 && k >= L) break;
        const auto yf = O::template along<kChunk>(Yw, at_along, 0, k);
        float f[NA];
#pragma unroll
        for (int e = 0; e < NA; ++e) f[e] = static_cast<float>(yf[e]) * fy[k / O::ALONG][e];
        if constexpr (M::ES == 2) {
          bf16x8 ys[M::PARTS];
          split(f, ys);
#pragma unroll
          for (int i = 0; i < M::WB; ++i) {
            const bf16x8 wf = O::template along<kChunk>(W, at_along, 16 * i, k);
#pragma unroll
            for (int q = M::PARTS - 1; q >= 0; --q) st.a[i] = O::mma(wf, ys[q], st.a[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < M::WB; ++i) {
            const f32x4 wf = O::template along<kChunk>(W, at_along, 16 * i, k);
#pragma unroll
            for (int e = 0; e < NA; ++e) st.a[i] = O::mma(wf[e], f[e], st.a[i]);
          }
        }
      }
    };
    if constexpr (M::OUT) {
      // fp32 leaves out the blocks past a chunk's last token (1 x 3 tokens, 8 heads of 96: 17.6 to
      // 12.5 us; whole chunks 1% slower); bf16 products cost less than the branches
      if (M::ES == 2 || 16 * ib < L) outputs();
    }
    update();
    if constexpr (M::OUT) {
      if (__any(bad != bad))  // whole waves
        mend_outputs<T, OutT, M::YD, M::WD, false, M::REV>(X, Y, W, S, Out, ib, b0, M::OB, L, a, g.cp, g.cx);
    }
    lds_barrier();  // the outputs are whole; no wave reads the tiles or the state any more
    if (M::OUT && g.out) {
      constexpr int EPC = 16 / M::OS, CPR = kChunk * M::OS / 16;
      OutT* op = static_cast<OutT*>(g.out) + (static_cast<int64_t>(head) * g.wdim + w0) * ld + sp.first + t;
      typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));
#pragma unroll
      for (int q = 0; q < M::WD * CPR / M::NT; ++q) {
        const int at = q * M::NT + threadIdx.x, r = at / CPR, cc = at % CPR, n = L - cc * EPC;
        if (r >= wrows || n <= 0) continue;
        const u32x4 v = *reinterpret_cast<const u32x4*>(Out + tile_off<M::OS, kChunk>(r, cc));
        OutT* p = op + r * ld + cc * EPC;
        if (n >= EPC) {
          *reinterpret_cast<u32x4_any*>(p) = v;
        } else {
          int rc = r;  // addresses of their own: kept from chunk to chunk they would take the sums' registers
          asm volatile("" : "+v"(rc));
          OutT* o = op + rc * ld + cc * EPC;
          const OutT* e = reinterpret_cast<const OutT*>(Out + tile_off<M::OS, kChunk>(rc, cc));
#pragma unroll 1
          for (int u = 0; u < n; ++u) o[u] = e[u];
        }
      }
    }
  }
  if (!M::OUT) {
#pragma unroll
    for (int i = 0; i < M::WB; ++i) *st.place(segp, wv, i) = st.a[i];
  } else if (g.nseg == 1 && g.sT) {
    st.template given<true>(g.sT + hs * sdim, g, wv, w0);
  }
}

// dK and dV together (bf16). Both run backward from the same state G: with
// R = G,  dV_i = sum a^{j-i} (k_i . q_j) dO_j + a^{n-1-i} k_i R
// R^T:    dK_i = sum a^{j-i} (v_i . dO_j) q_j + a^{n-1-i} R v_i,   R <- a^L R + q'^T dO,
// so that the four inputs are read and the state is carried once. Of eight waves four
// compute 16 tokens of dV each and four the same of dK (the state in LDS is read across
// its rows or along them); all share the state's update. Against one run for each: 4
// sequences of 4096 tokens, 16 heads of 128, dK and dV 247 us one after the
// other (states and outputs), together 177 us (states 40, scan 8, this kernel 129).
// Bound as mix_kernel is, on one workgroup of a compute unit.
struct PairArgs {
  MixArgs m;  // y = q (ydim: key rows), w = dO (wdim: value rows), segments, states
  const void* k;
  const void* v;
  void* dk;  // of the element type, or fp32 to be added over the heads of a group
  void* dv;
};

template <int KD_, int VD_, bool PART_, int PARTS_>
struct Pair {
  using T = bf16;
  static constexpr int YD = KD_, WD = VD_;
  static constexpr bool PART = PART_;
  static constexpr int PARTS = PARTS_, NW = 8, NT = 512, ES = 2, OS = PART ? 4 : 2;
  // the state: a wave holds 16 rows of q by WBW blocks of 16 rows of dO
  static constexpr int YW = YD / 16, WBW = WD / 16 / (NW / YW);
  static constexpr int YT = YD * kChunk * ES, WT = WD * kChunk * ES, ST = YD * WD * ES;
  static constexpr int LDS = 2 * YT + 2 * WT + ST + (YD + WD) * kChunk * OS;
  // Addresses and weights computed in each chunk, where they are used: kept from one chunk
  // to the next, some 60 registers, they would push the accumulators of the larger tiles
  // into scratch memory. 64 by 64 has room for them (backward of 8 x 2048 tokens, 16 heads:
  // 154 us; computed in each chunk 163 us).
  static constexpr bool LEAN = KD_ + VD_ > 128;
};

template <class P>
__global__ void __launch_bounds__(P::NT, 2) pair_kernel(PairArgs pa) {
  using T = bf16;
  using O = Ops<bf16>;
  using OutT = typename std::conditional<P::PART, float, bf16>::type;
  using OutOps = Ops<OutT>;
  const MixArgs& g = pa.m;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* Q = smem;
  char* K = Q + P::YT;
  char* D = K + P::YT;
  char* V = D + P::WT;
  char* S = V + P::WT;
  char* OutV = S + P::ST;
  char* OutK = OutV + P::WD * kChunk * P::OS;

  int id = xcd_position(blockIdx.x, gridDim.x);
  const int seg = id % g.nseg;
  id /= g.nseg;
  const int head = id % g.heads, seq = id / g.heads;
  const Span sp = span_of(g, seq);
  const int t0 = seg * g.seg_len, t1 = t0 + min(sp.len - t0, g.seg_len);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t hs = static_cast<int64_t>(seq) * g.heads + head;
  const int64_t sdim = static_cast<int64_t>(g.ydim) * g.wdim;
  float* segp = g.seg ? g.seg + (hs * g.nseg + seg) * P::YD * P::WD : nullptr;
  if (g.nseg > 1 && t0 >= t1) return;  // whole workgroups

  const Decay a(g.decay[head]);
  const int yb = wv % P::YW, wb = wv / P::YW * P::WBW, grp = lane >> 4;
  const int srow = yb * 16 + (lane & 15);  // the lane's row of the state
  f32x4 st[P::WBW];
#pragma unroll
  for (int i = 0; i < P::WBW; ++i) st[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (g.nseg > 1) {
#pragma unroll
    for (int i = 0; i < P::WBW; ++i)
      st[i] = reinterpret_cast<const f32x4*>(segp)[(yb * (P::WD / 16) + wb + i) * 64 + lane];
  } else if (g.s0 && srow < g.ydim) {
#pragma unroll
    for (int i = 0; i < P::WBW; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int wr = (wb + i) * 16 + 4 * grp + r;
        if (wr < g.wdim) st[i][r] = g.s0[hs * sdim + srow * g.wdim + wr];
      }
  }

  const int64_t ld = g.tokens;
  const int kv = head / g.group, nkv = g.heads / g.group;
  auto start = [&](auto& regs, const void* p, int h, int heads, int dim) {
    const T* b = static_cast<const T*>(p);
    regs.init(b + static_cast<int64_t>(h) * dim * ld + sp.first, ld, dim, b, b + static_cast<int64_t>(heads) * dim * ld);
  };
  TileRegs<T, P::YD, P::NT> qr, kr;
  TileRegs<T, P::WD, P::NT> dr, vr;
  start(qr, g.y, head, g.heads, g.ydim);
  start(kr, pa.k, kv, nkv, g.ydim);
  start(dr, g.w, head, g.heads, g.wdim);
  start(vr, pa.v, kv, nkv, g.wdim);

  const int ib = wv & 3;
  int at_along = O::base_along<kChunk>(), at_block = O::base_block<kChunk>();
  int at_state = O::base_block<P::WD>() ^ (wb * 32), at_srow = O::base_along<P::WD>();
  auto at_cols = O::base_across<kChunk>();
  auto at_scols = O::base_across<P::WD>();
  auto at_icols = at_cols;
  at_icols.lo ^= ib * 32, at_icols.hi ^= ib * 32;
  const int at_out = OutOps::template base_block<kChunk>() ^ (ib * 16 * P::OS);

  const int nchunk = static_cast<int>((static_cast<uint32_t>(t1 - t0) + kChunk - 1) / kChunk);
  auto first_of = [&](int c) { return t0 + (nchunk - 1 - c) * kChunk; };
  auto fetch = [&](int c) {
    const int t = first_of(c);
    if (t1 - t >= kChunk) {
      qr.load(t), kr.load(t), dr.load(t), vr.load(t);
    } else {
      qr.load_part(t), kr.load_part(t), dr.load_part(t), vr.load_part(t);
    }
  };
  if (nchunk > 0) fetch(0);
  for (int c = 0; c < nchunk; ++c) {
    const int t = first_of(c), L = min(kChunk, t1 - t);
    int tid = threadIdx.x;
    if constexpr (P::LEAN) {
      asm volatile("" : "+v"(tid));
      qr.tid = kr.tid = dr.tid = vr.tid = tid;
      asm volatile("" : "+v"(at_along), "+v"(at_block), "+v"(at_state), "+v"(at_srow), "+v"(at_cols.lo),
                   "+v"(at_cols.hi), "+v"(at_scols.lo), "+v"(at_scols.hi));
    }
    qr.store(Q, t, L);
    kr.store(K, t, L);
    dr.store(D, t, L);
    vr.store(V, t, L);
#pragma unroll
    for (int i = 0; i < P::WBW; ++i)
      *O::block<P::WD>(S + yb * 16 * P::WD * P::ES, at_state, 0, 16 * i) = O::round(st[i]);
    lds_barrier();
    if (c + 1 < nchunk) fetch(c + 1);
    Decay here = a;
    if constexpr (P::LEAN) asm volatile("" : "+v"(here.l2));
    float bad = 0.0f;  // NaN if an output of the lane is not finite
    // 16 tokens of dV or dK: X and Y meet in the inner products, W follows them, OD rows out
    auto outputs = [&](auto of_v, char* X, char* Y, char* W, char* Out) {
      constexpr bool OFV = decltype(of_v)::value;
      constexpr int XD = OFV ? P::YD : P::WD, OB = (OFV ? P::WD : P::YD) / 16;
      f32x4 acc[OB], p[4];
#pragma unroll
      for (int b = 0; b < OB; ++b) acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int jb = 0; jb < 4; ++jb) p[jb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < XD; k += 32) {
        const bf16x8 xf = O::across<kChunk>(X, at_icols, k, 0);
        const bf16x8 xo = OFV ? xf : __builtin_shufflevector(xf, xf, 0, 1, 4, 5, 2, 3, 6, 7);  // its rows in order
#pragma unroll
        for (int b = 0; b < OB; ++b) {
          const bf16x8 sf = OFV ? O::across<P::WD>(S, at_scols, k, 16 * b) : O::along<P::WD>(S, at_srow, 16 * b, k);
          acc[b] = O::mma(xo, sf, acc[b]);
        }
#pragma unroll
        for (int jb = 0; jb < 4; ++jb) p[jb] = O::mma(O::across<kChunk>(Y, at_cols, k, 16 * jb), xf, p[jb]);
        if constexpr (P::LEAN) __builtin_amdgcn_sched_barrier(0);  // later reads would take the sums' registers
      }
      // weights as in mix_kernel, running backward
      f32x4 wx;
#pragma unroll
      for (int r = 0; r < 4; ++r) wx[r] = g.cx * here.pow(max(L - 1 - (16 * ib + 4 * grp + r), 0));
#pragma unroll
      for (int b = 0; b < OB; ++b) acc[b] *= wx;
#pragma unroll
      for (int jb = 0; jb < 4; ++jb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int n = 16 * (jb - ib) + 4 * grp + r - (lane & 15);
          p[jb][r] = mul_masked(p[jb][r], n >= 0 ? g.cp * here.weight(max(n, 0)) : 0.0f);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 pf = __builtin_shufflevector(O::round(p[2 * h]), O::round(p[2 * h + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int b = 0; b < OB; ++b) {
          const bf16x4 lo = *O::block<kChunk>(W, at_block, 16 * b, 32 * h);
          const bf16x4 hi = *O::block<kChunk>(W, at_block, 16 * b, 32 * h + 16);
          acc[b] = O::mma(pf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), acc[b]);
        }
        if constexpr (P::LEAN) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int b = 0; b < OB; ++b) *OutOps::template block<kChunk>(Out, at_out, 16 * b, 0) = OutOps::round(acc[b]);
#pragma unroll
      for (int b = 0; b < OB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) bad = fmaf(acc[b][r], 0.0f, bad);
    };
    if (wv < 4) outputs(std::true_type{}, K, Q, D, OutV);
    else outputs(std::false_type{}, V, D, Q, OutK);
    // the state in front of this chunk
    const float aL = a.pow(L);
#pragma unroll
    for (int i = 0; i < P::WBW; ++i) st[i] *= aL;
#pragma unroll
    for (int k = 0; k < kChunk; k += 32) {
      const bf16x8 yf = O::along<kChunk>(Q + yb * 16 * kChunk * P::ES, at_along, 0, k);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = static_cast<float>(yf[e]) * (g.cy * here.pow(k + 8 * grp + e + 1));
      bf16x8 ys[P::PARTS];
      split(f, ys);
#pragma unroll
      for (int i = 0; i < P::WBW; ++i) {
        const bf16x8 wf = O::along<kChunk>(D + wb * 16 * kChunk * P::ES, at_along, 16 * i, k);
#pragma unroll
        for (int q = P::PARTS - 1; q >= 0; --q) st[i] = O::mma(wf, ys[q], st[i]);
      }
    }
    if (__any(bad != bad)) {  // whole waves
      if (wv < 4) mend_outputs<T, OutT, P::YD, P::WD, false, true>(K, Q, D, S, OutV, ib, 0, P::WD / 16, L, a, g.cp, g.cx);
      else mend_outputs<T, OutT, P::WD, P::WD, true, true>(V, D, Q, S, OutK, ib, 0, P::YD / 16, L, a, g.cp, g.cx);
    }
    lds_barrier();  // the outputs are whole; no wave reads the tiles or the state any more
    auto put = [&](char* Out, void* to, int dim, auto rows_c) {
      constexpr int EPC = 16 / P::OS, CPR = kChunk * P::OS / 16, ROWS = decltype(rows_c)::value;
      if (!to) return;
      OutT* op = static_cast<OutT*>(to) + static_cast<int64_t>(head) * dim * ld + sp.first + t;
      typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));
#pragma unroll
      for (int q = 0; q < ROWS * CPR / P::NT; ++q) {
        const int at = q * P::NT + tid, r = at / CPR, cc = at % CPR, n = L - cc * EPC;
        if (r >= dim || n <= 0) continue;
        const char* from = Out + tile_off<P::OS, kChunk>(r, cc);
        OutT* o = op + r * ld + cc * EPC;
        if (n >= EPC) {
          *reinterpret_cast<u32x4_any*>(o) = *reinterpret_cast<const u32x4*>(from);
        } else {
#pragma unroll 1
          for (int u = 0; u < n; ++u) o[u] = reinterpret_cast<const OutT*>(from)[u];
        }
      }
    };
    put(OutV, pa.dv, g.wdim, std::integral_constant<int, P::WD>{});
    put(OutK, pa.dk, g.ydim, std::integral_constant<int, P::YD>{});
  }
  if (g.nseg == 1 && g.sT && srow < g.ydim) {
#pragma unroll
    for (int i = 0; i < P::WBW; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int wr = (wb + i) * 16 + 4 * grp + r;
        if (wr < g.wdim) g.sT[hs * sdim + srow * g.wdim + wr] = st[i][r];
      }
  }
}

// Segment states -> the state in front of each segment, in running order, and the
// last one. Four neighbouring accumulators of a thread, bound by the latency of segment
// after segment: 4 x 4096 tokens, 16 heads of 128: 7 us.
template <class M>
__global__ void __launch_bounds__(256) mix_scan_kernel(MixArgs g) {
  int id = blockIdx.x;
  const int wt = id % g.wtiles;
  id /= g.wtiles;
  const int head = id % g.heads, seq = id / g.heads;
  const Span sp = span_of(g, seq);
  const Decay a(g.decay[head]);
  const int at = blockIdx.y * 256 + threadIdx.x;  // of YD * WD / 4
  const int lane = at & 63, i = (at >> 6) % M::WB, wv = (at >> 6) / M::WB;
  const int yr = wv * 16 + (lane & 15), wr = wt * M::WD + i * 16 + 4 * (lane >> 4);
  const int64_t hs = static_cast<int64_t>(seq) * g.heads + head, sdim = static_cast<int64_t>(g.ydim) * g.wdim;
  auto given = [&](int r) {
    return hs * sdim + (g.s_trans ? static_cast<int64_t>(wr + r) * g.ydim + yr
                                  : static_cast<int64_t>(yr) * g.wdim + wr + r);
  };
  f32x4 run = {0.0f, 0.0f, 0.0f, 0.0f};
  if (g.s0) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (yr < g.ydim && wr + r < g.wdim) run[r] = g.s0[given(r)];
  }
  f32x4* p = reinterpret_cast<f32x4*>(g.seg) + (hs * g.wtiles + wt) * g.nseg * (M::YD * M::WD / 4) + at;
  constexpr int AHEAD = 4;  // segments read ahead: their states do not wait for each other
  for (int q0 = 0; q0 < g.nseg; q0 += AHEAD) {
    f32x4 u[AHEAD];
    auto seg_of = [&](int q) { return M::REV ? g.nseg - 1 - q : q; };
    auto len_of = [&](int q) { return q < g.nseg ? min(sp.len - seg_of(q) * g.seg_len, g.seg_len) : 0; };
    auto at_of = [&](int q) { return p + static_cast<int64_t>(seg_of(q)) * (M::YD * M::WD / 4); };
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
      if (len_of(q0 + q) > 0) u[q] = *at_of(q0 + q);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int len = len_of(q0 + q);
      if (len <= 0) continue;
      *at_of(q0 + q) = run;
      run = run * a.pow(len) + u[q];
    }
  }
  if (g.sT) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (yr < g.ydim && wr + r < g.wdim) g.sT[given(r)] = run[r];
  }
}

// out[head][row][token] = the sum over the heads of a group, for the tokens of the
// sequences.
template <typename T>
__global__ void __launch_bounds__(256) mix_group_kernel(MixArgs g, const float* __restrict__ part, int32_t dim,
                                                        T* __restrict__ out) {
  const int64_t head = blockIdx.y / dim, r = blockIdx.y % dim, row = blockIdx.y;
  const int per = (g.max_len - 1) / 256 + 1;  // blocks of a sequence
  for (int64_t id = blockIdx.x; id < static_cast<int64_t>(per) * g.n_seqs; id += gridDim.x) {
    const Span sp = span_of(g, static_cast<int>(id / per));
    const int t = static_cast<int>(id % per) * 256 + threadIdx.x;
    if (t >= sp.len) continue;
    const float* p = part + (head * g.group * dim + r) * g.tokens + sp.first + t;
    float s = 0.0f;
    for (int q = 0; q < g.group; ++q) s += p[static_cast<int64_t>(q) * dim * g.tokens];
    out[row * g.tokens + sp.first + t] = from_f32<T>(s);
  }
}

// ------------------------------------------------------------------ one token
// A workgroup per sequence and head: the state passes once through registers,
// VE columns of a row in a thread. Bound by reading and writing the state: 64 sequences,
// 16 heads of 128 x 128 (134 MB) 32 us, 4.2 TB/s.
template <typename T, int VE>
__global__ void __launch_bounds__(256) step_kernel(const T* __restrict__ Q, const T* __restrict__ K,
                                                   const T* __restrict__ V, const float* __restrict__ decay,
                                                   const float* S0, T* __restrict__ O, float* ST, int32_t n,
                                                   int32_t heads, int32_t group, int32_t kd, int32_t vd,
                                                   float scale) {
  __shared__ float q[128], k[128], v[128];
  __shared__ float red[256 * VE];
  const int id = xcd_position(blockIdx.x, gridDim.x);
  const int head = id % heads, seq = id / heads, tid = threadIdx.x;
  const int64_t hk = head / group;
  if (tid < kd) {
    q[tid] = to_f32(Q[(static_cast<int64_t>(head) * kd + tid) * n + seq]);
    k[tid] = to_f32(K[(hk * kd + tid) * n + seq]);
  } else if (tid >= 128 && tid - 128 < vd) {
    v[tid - 128] = to_f32(V[(hk * vd + tid - 128) * n + seq]);
  }
  const float a = Decay(decay[head]).pow(1);
  const int nx = (vd + VE - 1) / VE;  // threads along a row
  const int ny = 256 / nx, tx = tid % nx, ty = tid / nx;
  const int64_t base = (static_cast<int64_t>(seq) * heads + head) * kd * vd;
  float o[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) o[e] = 0.0f;
  __syncthreads();
  if (ty < ny) {
#pragma unroll 4
    for (int d = ty; d < kd; d += ny) {
      const int64_t at = base + static_cast<int64_t>(d) * vd + tx * VE;
      float s[VE];
      if constexpr (VE == 4)
        *reinterpret_cast<f32x4*>(s) = S0 ? *reinterpret_cast<const f32x4*>(S0 + at) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      else
        s[0] = S0 ? S0[at] : 0.0f;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        s[e] = a * s[e] + k[d] * v[tx * VE + e];
        o[e] += q[d] * s[e];
      }
      if constexpr (VE == 4)
        *reinterpret_cast<f32x4*>(ST + at) = *reinterpret_cast<const f32x4*>(s);
      else
        ST[at] = s[0];
    }
  }
#pragma unroll
  for (int e = 0; e < VE; ++e) red[(ty * nx + tx) * VE + e] = o[e];
  __syncthreads();
  if (tid < vd) {
    float s = 0.0f;
    for (int y = 0; y < ny; ++y) s += red[y * nx * VE + tid];
    O[(static_cast<int64_t>(head) * vd + tid) * n + seq] = from_f32<T>(scale * s);
  }
}

// ------------------------------------------------------------------ host
int need_ptr(const void* p, const char* name) {
  if (!p) return fail(ARD_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}
int may_ptr(const void* p, const char* name) {
  if (p && !aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}

int check_desc(const ard_linattn_desc* d) {
  if (!d) return fail(ARD_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != ARD_F32 && d->dtype != ARD_BF16) return fail(ARD_ERR_UNSUPPORTED, "dtype %d not supported", d->dtype);
  if (d->n_seqs < 1 || d->max_len < 1 || d->tokens < 1)
    return fail(ARD_ERR_INVALID_ARG, "sizes must be >= 1 (n_seqs %d, max_len %d, tokens %d)", d->n_seqs, d->max_len,
                d->tokens);
  if (d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads)
    return fail(ARD_ERR_INVALID_ARG, "%d query heads are no multiple of %d key heads", d->q_heads, d->kv_heads);
  if (d->key_dim < 1 || d->key_dim > 128 || d->value_dim < 1 || d->value_dim > 128)
    return fail(ARD_ERR_UNSUPPORTED, "head sizes must be 1..128 (key %d, value %d)", d->key_dim, d->value_dim);
  if (!std::isfinite(d->scale)) return fail(ARD_ERR_INVALID_ARG, "scale must be finite");
  if (!d->d_offsets && static_cast<int64_t>(d->n_seqs) * d->max_len > d->tokens)
    return fail(ARD_ERR_INVALID_ARG, "%d sequences of %d columns do not fit %d", d->n_seqs, d->max_len, d->tokens);
  if (reinterpret_cast<uintptr_t>(d->d_offsets) % 4) return fail(ARD_ERR_INVALID_ARG, "d_offsets is not 4-byte aligned");
  if (static_cast<int64_t>(d->kv_heads) * std::max(d->key_dim, d->value_dim) > 65535)
    return fail(ARD_ERR_UNSUPPORTED, "%d key heads: at most 65535 rows of keys or values", d->kv_heads);
  // a workgroup of up to 512 threads for each sequence, head, tile (two at most) and segment (plan_mix)
  if (static_cast<int64_t>(d->n_seqs) * d->q_heads >= (int64_t{1} << 22))
    return fail(ARD_ERR_UNSUPPORTED, "%d sequences of %d heads: at most 2^22 states", d->n_seqs, d->q_heads);
  return ARD_OK;
}

constexpr int kFill4 = 512, kFill8 = 256;  // workgroups of four or eight waves that fill the chip

int pad_dim(int d) { return d <= 64 ? 64 : 128; }

// The longest that a sequence can be: max_len may be any bound, and tokens are all there are.
int longest(const ard_linattn_desc* d) { return std::min(d->max_len, d->tokens); }

// How one run lays out its work: rows of a w tile, and segments.
struct MixPlan {
  int yd, wd, wtiles, nseg, seg_len;
};
MixPlan plan_mix(const ard_linattn_desc* d, int ydim, int wdim) {
  MixPlan p;
  p.yd = pad_dim(ydim);
  p.wd = d->dtype == ARD_BF16 ? pad_dim(wdim) : 64;
  p.wtiles = (wdim + p.wd - 1) / p.wd;
  // as many sequences as there can be of the longest length: of ragged ones, most are shorter
  const int64_t full = std::min<int64_t>(d->n_seqs, (d->tokens - 1) / longest(d) + 1);
  const int64_t base = full * d->q_heads * p.wtiles, fill = p.yd == 64 ? kFill4 : kFill8;
  // fp32 is bound by its products, which a second pass adds to, but not by as much as idle units
  const int64_t n = base >= (d->dtype == ARD_BF16 ? fill / 2 : fill) ? 1 : (fill + base - 1) / base;
  const int64_t chunks = (static_cast<int64_t>(longest(d)) + kChunk - 1) / kChunk;
  int64_t per = (chunks + n - 1) / n;
  if (n > 1) {
    // Segments, shorter than four chunks where it gains: the chunks that one workgroup goes
    // through (one of states is a third of one of outputs) against two more launches and the
    // states, written, read twice and scanned (of every sequence, though most be short). us:
    // bf16, 8 x 256 tokens, 8 heads of 64: 11.6 in one segment, 17.8 in four; 1 x 256, 8 of 128:
    // 22.7 and 17.8; 16 x 256, 4 of 128: 24.5 and 31.8. fp32, 3 x 781, 8 of 80: 87 with four
    // chunks to a segment, 63 with three; 5 x 303, 8 of 128: 64 in one segment, 37 in five.
    const bool wide = p.yd == 128, wider = p.wd == 128;
    const double tc = d->dtype == ARD_F32 ? (wide ? 15.0 : 7.5) : wide && wider ? 5.5 : wide || wider ? 4.0 : 2.4;
    const double state = 4.0 * static_cast<double>(d->n_seqs) * d->q_heads * p.wtiles * p.yd * p.wd * 4 / 5.2e6;
    double least = chunks * tc;
    int64_t best = chunks;
    const int64_t tiles = static_cast<int64_t>(d->n_seqs) * d->q_heads * p.wtiles;
    for (int64_t q = std::max(per, std::min<int64_t>(4, chunks - 1)); q >= per && q < chunks; --q) {
      if (tiles * ((chunks + q - 1) / q) >= int64_t{1} << 23) continue;  // threads of a launch below 2^32
      const double us = q * tc * 4 / 3 + 11.0 + (state + 0.25) * static_cast<double>((chunks + q - 1) / q);
      if (us < 0.97 * least) least = us, best = q;
    }
    per = best;
  }
  p.seg_len = static_cast<int>(std::min<int64_t>(per * kChunk, std::numeric_limits<int>::max()));
  p.nseg = static_cast<int>((chunks + per - 1) / per);
  return p;
}

size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

size_t seg_bytes(const ard_linattn_desc* d, int ydim, int wdim) {
  const MixPlan p = plan_mix(d, ydim, wdim);
  if (p.nseg == 1) return 0;
  return al256(static_cast<size_t>(d->n_seqs) * d->q_heads * p.wtiles * p.nseg * p.yd * p.wd * 4);
}
// Gradients of shared heads before they are added: bf16 both at once, fp32 one after the other.
size_t part_bytes(const ard_linattn_desc* d) {
  if (d->q_heads == d->kv_heads) return 0;
  const int rows = d->dtype == ARD_BF16 ? d->key_dim + d->value_dim : std::max(d->key_dim, d->value_dim);
  return al256(static_cast<size_t>(d->q_heads) * rows * d->tokens * 4);
}
size_t fwd_bytes(const ard_linattn_desc* d) { return seg_bytes(d, d->key_dim, d->value_dim); }
size_t bwd_bytes(const ard_linattn_desc* d) {
  return std::max(fwd_bytes(d), seg_bytes(d, d->value_dim, d->key_dim)) + part_bytes(d);
}

template <class M>
hipError_t launch_mix(const MixArgs& g, hipStream_t stream) {
  auto kern = mix_kernel<M>;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, M::LDS);
  if (attr != hipSuccess) return attr;
  const unsigned blocks = static_cast<unsigned>(g.n_seqs) * g.heads * g.wtiles * g.nseg;
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(M::NT), M::LDS, stream, g);
  return hipGetLastError();
}

// The states of the segments, and what lies in front of each.
template <typename T, int YD, int WD, bool REV>
hipError_t run_states(const MixArgs& g, hipStream_t stream) {
  using U = Mix<T, YD, WD, REV, false, false>;
  const hipError_t e = launch_mix<U>(g, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(mix_scan_kernel<U>, dim3(g.n_seqs * g.heads * g.wtiles, YD * WD / 1024), dim3(256), 0, stream, g);
  return hipGetLastError();
}

template <typename T, int YD, int WD, bool REV>
hipError_t run_mix(const MixArgs& g, bool part, hipStream_t stream) {
  if (g.nseg > 1) {
    const hipError_t e = run_states<T, YD, WD, REV>(g, stream);
    if (e != hipSuccess) return e;
  }
  // with more than one segment the last state came from the pass above, and a chunk's
  // own ends in outputs only
  if constexpr (sizeof(T) == 2) {
    return g.nseg > 1 ? launch_mix<Mix<T, YD, WD, REV, true, false, 2>>(g, stream)
                      : launch_mix<Mix<T, YD, WD, REV, true, false, 3>>(g, stream);
  } else {
    return part ? launch_mix<Mix<T, YD, WD, REV, true, true>>(g, stream)
                : launch_mix<Mix<T, YD, WD, REV, true, false>>(g, stream);
  }
}

void fill_args(const ard_linattn_desc* d, const MixPlan& p, MixArgs* g) {
  g->offsets = d->d_offsets;
  g->n_seqs = d->n_seqs;
  g->max_len = longest(d);
  g->tokens = d->tokens;
  g->heads = d->q_heads;
  g->group = d->q_heads / d->kv_heads;
  g->nseg = p.nseg;
  g->seg_len = p.seg_len;
  g->wtiles = p.wtiles;
  if (p.nseg == 1) g->seg = nullptr;
}

// Adds the fp32 gradients part[q_heads * dim][tokens] over the heads of a group.
template <typename T>
hipError_t add_group(const ard_linattn_desc* d, const MixArgs& g, const float* part, int dim, void* out,
                     hipStream_t stream) {
  const int64_t blocks = ((g.max_len - 1) / 256 + 1) * static_cast<int64_t>(g.n_seqs);
  hipLaunchKernelGGL(mix_group_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(blocks, 1 << 16)),
                                               d->kv_heads * dim),
                     dim3(256), 0, stream, g, part, dim, static_cast<T*>(out));
  return hipGetLastError();
}

// part: where a group's gradients go before they are added, or NULL (fp32 only).
template <typename T, bool REV>
hipError_t run_mix(const ard_linattn_desc* d, MixArgs g, void* out, float* part, hipStream_t stream) {
  const MixPlan p = plan_mix(d, g.ydim, g.wdim);
  fill_args(d, p, &g);
  if (!out) part = nullptr;  // the last state alone is asked for
  g.out = part ? part : out;
  hipError_t e;
  if constexpr (sizeof(T) == 2) {
    static_assert(!REV, "dK and dV are pair_kernel's");
    if (p.yd == 64 && p.wd == 64) e = run_mix<T, 64, 64, REV>(g, false, stream);
    else if (p.yd == 64) e = run_mix<T, 64, 128, REV>(g, false, stream);
    else if (p.wd == 64) e = run_mix<T, 128, 64, REV>(g, false, stream);
    else e = run_mix<T, 128, 128, REV>(g, false, stream);
  } else {
    const bool pt = part != nullptr;
    e = p.yd == 64 ? run_mix<T, 64, 64, REV>(g, pt, stream) : run_mix<T, 128, 64, REV>(g, pt, stream);
  }
  if (e != hipSuccess || !part) return e;
  return add_group<T>(d, g, part, g.wdim, out, stream);
}

template <int KD, int VD>
hipError_t run_pair(const PairArgs& a, bool part, hipStream_t stream) {
  auto go = [&](auto cfg) {
    using P = decltype(cfg);
    auto kern = pair_kernel<P>;
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
    if (attr != hipSuccess) return attr;
    const unsigned blocks = static_cast<unsigned>(a.m.n_seqs) * a.m.heads * a.m.nseg;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(P::NT), P::LDS, stream, a);
    return hipGetLastError();
  };
  if (a.m.nseg > 1) {
    const hipError_t e = run_states<bf16, KD, VD, true>(a.m, stream);
    if (e != hipSuccess) return e;
    return part ? go(Pair<KD, VD, true, 2>{}) : go(Pair<KD, VD, false, 2>{});
  }
  return part ? go(Pair<KD, VD, true, 3>{}) : go(Pair<KD, VD, false, 3>{});
}

template <typename T>
int fwd_impl(const ard_linattn_desc* d, const void* Q, const void* K, const void* V, const float* decay,
             const float* S0, void* O, float* ST, float* ws, hipStream_t stream) {
  MixArgs g = {};
  g.x = Q, g.y = K, g.w = V;
  g.y_shared = g.w_shared = 1;
  g.ydim = d->key_dim, g.wdim = d->value_dim;
  g.decay = decay, g.s0 = S0, g.sT = ST, g.seg = ws;
  g.cp = d->scale, g.cy = 1.0f, g.cx = d->scale;
  ARD_HIP_CHECK((run_mix<T, false>(d, g, O, nullptr, stream)));
  return ARD_OK;
}

template <typename T>
int bwd_impl(const ard_linattn_desc* d, const void* Q, const void* K, const void* V, const float* decay,
             const float* S0, const void* dO, const float* dST, void* dQ, void* dK, void* dV, float* dS0, char* ws,
             hipStream_t stream) {
  float* part = part_bytes(d) ? reinterpret_cast<float*>(ws) : nullptr;
  float* seg = reinterpret_cast<float*>(ws + part_bytes(d));
  MixArgs g = {};
  g.decay = decay, g.seg = seg;
  g.cp = d->scale;
  if (dQ) {
    MixArgs r = g;
    r.x = dO, r.y = V, r.w = K;
    r.y_shared = r.w_shared = 1;
    r.ydim = d->value_dim, r.wdim = d->key_dim;
    r.s0 = S0, r.s_trans = 1;
    r.cy = 1.0f, r.cx = d->scale;
    ARD_HIP_CHECK((run_mix<T, false>(d, r, dQ, nullptr, stream)));
  }
  MixArgs r = g;
  if constexpr (sizeof(T) == 2) {
    if (!dK && !dV && !dS0) return ARD_OK;
    r.y = Q, r.w = dO;
    r.ydim = d->key_dim, r.wdim = d->value_dim;
    r.s0 = dST, r.sT = dS0;
    r.cy = d->scale, r.cx = 1.0f;
    const MixPlan p = plan_mix(d, r.ydim, r.wdim);
    fill_args(d, p, &r);
    float* kp = part && dK ? part : nullptr;
    float* vp = part && dV ? part + static_cast<size_t>(d->q_heads) * d->key_dim * d->tokens : nullptr;
    const PairArgs a = {r, K, V, part ? kp : dK, part ? vp : dV};
    if (p.yd == 64 && p.wd == 64) ARD_HIP_CHECK((run_pair<64, 64>(a, part != nullptr, stream)));
    else if (p.yd == 64) ARD_HIP_CHECK((run_pair<64, 128>(a, part != nullptr, stream)));
    else if (p.wd == 64) ARD_HIP_CHECK((run_pair<128, 64>(a, part != nullptr, stream)));
    else ARD_HIP_CHECK((run_pair<128, 128>(a, part != nullptr, stream)));
    if (kp) ARD_HIP_CHECK(add_group<T>(d, r, kp, d->key_dim, dK, stream));
    if (vp) ARD_HIP_CHECK(add_group<T>(d, r, vp, d->value_dim, dV, stream));
  } else {
    if (dK) {
      r.x = V, r.y = dO, r.w = Q;
      r.x_shared = 1;
      r.ydim = d->value_dim, r.wdim = d->key_dim;
      r.s0 = dST, r.s_trans = 1;
      r.cy = d->scale, r.cx = 1.0f;
      ARD_HIP_CHECK((run_mix<T, true>(d, r, dK, part, stream)));
    }
    if (dV || dS0) {
      r = g;
      r.x = K, r.y = Q, r.w = dO;
      r.x_shared = 1;
      r.ydim = d->key_dim, r.wdim = d->value_dim;
      r.s0 = dST, r.sT = dS0;
      r.cy = d->scale, r.cx = 1.0f;
      ARD_HIP_CHECK((run_mix<T, true>(d, r, dV, part, stream)));
    }
  }
  return ARD_OK;
}

template <typename T>
int step_impl(const ard_linattn_desc* d, const void* Q, const void* K, const void* V, const float* decay,
              const float* S0, void* O, float* ST, hipStream_t stream) {
  const int group = d->q_heads / d->kv_heads;
  const dim3 grid(static_cast<unsigned>(d->n_seqs) * d->q_heads);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, static_cast<const T*>(Q), static_cast<const T*>(K),
                       static_cast<const T*>(V), decay, S0, static_cast<T*>(O), ST, d->n_seqs, d->q_heads, group,
                       d->key_dim, d->value_dim, d->scale);
  };
  if (d->value_dim % 4 == 0) go(step_kernel<T, 4>);
  else go(step_kernel<T, 1>);
  ARD_LAUNCH_CHECK();
  return ARD_OK;
}

int check_inputs(const ard_linattn_desc* d, const void* Q, const void* K, const void* V, const float* decay) {
  int st = check_desc(d);
  if (st != ARD_OK) return st;
  if ((st = need_ptr(Q, "Qt")) || (st = need_ptr(K, "Kt")) || (st = need_ptr(V, "Vt")) ||
      (st = need_ptr(decay, "log_decay")))
    return st;
  return ARD_OK;
}
int check_ws(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return ARD_OK;
  if (!ws || ws_bytes < need)
    return fail(ARD_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : 0);
  if (!aligned16(ws)) return fail(ARD_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return ARD_OK;
}

}  // namespace
}  // namespace ard

using namespace ard;

extern "C" {

size_t ard_linattn_workspace_bytes(const ard_linattn_desc* desc) {
  if (check_desc(desc) != ARD_OK) return 0;
  return bwd_bytes(desc);
}

int ard_linattn_fwd(const ard_linattn_desc* desc, const void* Qt, const void* Kt, const void* Vt,
                    const float* log_decay, const float* S0, void* Ot, float* ST, void* ws, size_t ws_bytes,
                    void* stream) {
  clear_error();
  int st = check_inputs(desc, Qt, Kt, Vt, log_decay);
  if (st != ARD_OK) return st;
  if ((st = may_ptr(S0, "S0")) || (st = need_ptr(Ot, "Ot")) || (st = may_ptr(ST, "ST")) ||
      (st = check_ws(fwd_bytes(desc), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  float* w = static_cast<float*>(ws);
  return desc->dtype == ARD_BF16 ? fwd_impl<bf16>(desc, Qt, Kt, Vt, log_decay, S0, Ot, ST, w, sm)
                                 : fwd_impl<float>(desc, Qt, Kt, Vt, log_decay, S0, Ot, ST, w, sm);
}

int ard_linattn_bwd(const ard_linattn_desc* desc, const void* Qt, const void* Kt, const void* Vt,
                    const float* log_decay, const float* S0, const void* dOt, const float* dST, void* dQt, void* dKt,
                    void* dVt, float* dS0, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  int st = check_inputs(desc, Qt, Kt, Vt, log_decay);
  if (st != ARD_OK) return st;
  if ((st = may_ptr(S0, "S0")) || (st = need_ptr(dOt, "dOt")) || (st = may_ptr(dST, "dST")) ||
      (st = may_ptr(dQt, "dQt")) || (st = may_ptr(dKt, "dKt")) || (st = may_ptr(dVt, "dVt")) ||
      (st = may_ptr(dS0, "dS0")) || (st = check_ws(bwd_bytes(desc), ws, ws_bytes)))
    return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  return desc->dtype == ARD_BF16
             ? bwd_impl<bf16>(desc, Qt, Kt, Vt, log_decay, S0, dOt, dST, dQt, dKt, dVt, dS0, w, sm)
             : bwd_impl<float>(desc, Qt, Kt, Vt, log_decay, S0, dOt, dST, dQt, dKt, dVt, dS0, w, sm);
}

int ard_linattn_step(const ard_linattn_desc* desc, const void* Qt, const void* Kt, const void* Vt,
                     const float* log_decay, const float* S0, void* Ot, float* ST, void* stream) {
  clear_error();
  int st = check_inputs(desc, Qt, Kt, Vt, log_decay);
  if (st != ARD_OK) return st;
  if (desc->max_len != 1 || desc->d_offsets || desc->tokens != desc->n_seqs)
    return fail(ARD_ERR_INVALID_ARG, "a step takes one token for each sequence: max_len 1, no d_offsets, tokens == n_seqs");
  if ((st = may_ptr(S0, "S0")) || (st = need_ptr(Ot, "Ot")) || (st = need_ptr(ST, "ST"))) return st;
  hipStream_t sm = static_cast<hipStream_t>(stream);
  return desc->dtype == ARD_BF16 ? step_impl<bf16>(desc, Qt, Kt, Vt, log_decay, S0, Ot, ST, sm)
                                 : step_impl<float>(desc, Qt, Kt, Vt, log_decay, S0, Ot, ST, sm);
}

}  // extern "C"
