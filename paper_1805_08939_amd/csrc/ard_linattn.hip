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
// of the output's own rounding to one of the two terms. y' is split into three
// bf16 parts (its 24 bits), so the state is exact to fp32. fp32 inputs use fp32
// MFMA throughout.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ard_gemm_fast.hpp"
#include "ard_internal.hpp"

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
  __device__ __forceinline__ float pow(int n) const { return __builtin_amdgcn_exp2f(l2 * static_cast<float>(n)); }
};

// ------------------------------------------------------------------ LDS tiles
// [rows][COLS] of 16-byte chunks, chunk c of row r at position c ^ swz(r), so that
// neither 16 rows at one chunk (operands contiguous along the contraction) nor
// rows r .. r + 3 and r + 8 .. r + 11 at neighbouring chunks (transposed reads, and
// fp32's element reads of four rows) meet in a bank.
template <int ES, int COLS>
__device__ __forceinline__ int tile_off(int r, int c) {
  constexpr int CPR = COLS * ES / 16;
  int s;
  if constexpr (CPR == 8) {
    const int h = (r >> 1) & 7;
    s = ((h & 1) << 1) | (h & 4) | ((h >> 1) & 1);
  } else if constexpr (ES == 4) {
    s = ((r & 3) << 2) | ((r >> 2) & 3);
  } else {
    s = ((r & 3) << 1) | (r & 8);
  }
  return (r * CPR + (c ^ s)) * 16;
}

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// MFMA operands of 16 x 16 blocks. Along: 16 rows of a tile, the contraction along
// its columns (16 bytes of a lane). Across: 16 columns, the contraction along its
// rows. bf16: a step of 32; fp32: Along 16 (four MFMAs, slot g holding 4 g + e),
// Across 4.
template <typename T>
struct Ops;
template <>
struct Ops<bf16> {
  using Along = bf16x8;
  using Across = bf16x8;
  static constexpr int ALONG = 32, ACROSS = 32;
  template <int COLS>
  static __device__ __forceinline__ Along along(const char* t, int row, int col) {
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const bf16x8*>(t + tile_off<2, COLS>(row + (lane & 15), (col >> 3) + (lane >> 4)));
  }
  template <int COLS>
  static __device__ __forceinline__ Across across(const char* t, int row, int col) {
    const int lane = threadIdx.x & 63, s = lane & 15;
    const int r = row + 8 * (lane >> 4) + (s >> 2), c = col + 4 * (s & 3);
    const char* p0 = t + tile_off<2, COLS>(r, c >> 3) + (c & 7) * 2;
    const char* p1 = t + tile_off<2, COLS>(r + 4, c >> 3) + (c & 7) * 2;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p0));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p1));
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = __builtin_bit_cast(bf16x4, lo)[e];
      o[e + 4] = __builtin_bit_cast(bf16x4, hi)[e];
    }
    return o;
  }
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
  static __device__ __forceinline__ Along along(const char* t, int row, int col) {
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const f32x4*>(t + tile_off<4, COLS>(row + (lane & 15), (col >> 2) + (lane >> 4)));
  }
  template <int COLS>
  static __device__ __forceinline__ Across across(const char* t, int row, int col) {
    const int lane = threadIdx.x & 63;
    const int r = row + (lane >> 4), c = col + (lane & 15);
    return *reinterpret_cast<const float*>(t + tile_off<4, COLS>(r, c >> 2) + (c & 3) * 4);
  }
  static __device__ __forceinline__ f32x4 mma(Across a, Across b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
};

// A thread's share of a [D][64] tile on its way from memory: rows past `rows` and
// tokens past L are zero, and nothing past them is read.
template <typename T, int D>
struct TileRegs {
  static constexpr int ES = sizeof(T), EPC = 16 / ES, CPR = kChunk * ES / 16, PER = D * CPR / 256;
  u32x4 v[PER];

  __device__ __forceinline__ void load(const T* base, int64_t ld, int rows, int L) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = i * 256 + threadIdx.x, r = at / CPR, c = at % CPR;
      const int n = r < rows ? L - c * EPC : 0;
      const char* p = reinterpret_cast<const char*>(base + r * ld + c * EPC);
      if (n >= EPC)
        v[i] = load16_any<ES>(p);
      else
        v[i] = load16_part<ES>(p, n);
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = i * 256 + threadIdx.x;
      *reinterpret_cast<u32x4*>(lds + tile_off<ES, kChunk>(at / CPR, at % CPR)) = v[i];
    }
  }
};

// fp32 as three bf16 that add up to it.
__device__ __forceinline__ void split3(float f, bf16& a, bf16& b, bf16& c) {
  a = static_cast<bf16>(f);
  const float r = f - static_cast<float>(a);
  b = static_cast<bf16>(r);
  c = static_cast<bf16>(r - static_cast<float>(b));
}

template <typename T_, int YD_, int WD_, bool REV_, bool OUT_, bool PART_>
struct Mix {
  using T = T_;
  static constexpr int YD = YD_, WD = WD_;  // rows of x and y, of w, as padded
  static constexpr bool REV = REV_;
  static constexpr bool OUT = OUT_;    // outputs (else the states of segments only)
  static constexpr bool PART = PART_;  // outputs in fp32, to be added over the heads that share a row
  static constexpr int ES = sizeof(T), OS = PART ? 4 : ES;
  static constexpr int YB = YD / 64, WB = WD / 16;  // 16-blocks: of a wave's part of y rows, of w rows
  static constexpr int XT = YD * kChunk * ES, WT = WD * kChunk * ES;
  static constexpr int ST = YD * WD * ES, OT = WD * kChunk * OS;
  static constexpr int LDS = OUT ? 2 * XT + WT + (ST > OT ? ST : OT) : XT + WT;
};

// The state's accumulators of a wave: 16 rows of y in a block (lane % 16), of which
// wave wv holds blocks wv * YB .., by 16 rows of w (4 (lane / 16) + r).
template <class M>
struct State {
  f32x4 a[M::WB][M::YB];
  __device__ __forceinline__ int y(int wv, int b) const { return (wv * M::YB + b) * 16 + (threadIdx.x & 15); }
  __device__ __forceinline__ int w(int b) const { return b * 16 + 4 * ((threadIdx.x >> 4) & 3); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < M::WB; ++i)
#pragma unroll
      for (int j = 0; j < M::YB; ++j) a[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // a state of the caller's: [ydim][wdim] or its transpose; w0: first row of w of this tile
  template <bool STORE>
  __device__ __forceinline__ void given(float* p, const MixArgs& g, int wv, int w0) {
#pragma unroll
    for (int i = 0; i < M::WB; ++i)
#pragma unroll
      for (int j = 0; j < M::YB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int yr = y(wv, j), wr = w0 + w(i) + r;
          if (yr < g.ydim && wr < g.wdim) {
            float* at = p + (g.s_trans ? wr * g.ydim + yr : yr * g.wdim + wr);
            if constexpr (STORE) *at = a[i][j][r];
            else a[i][j][r] = *at;
          }
        }
  }
  // a segment's, in the accumulators' own order
  __device__ __forceinline__ f32x4* place(float* p, int wv, int i, int j) const {
    return reinterpret_cast<f32x4*>(p) + ((wv * M::WB + i) * M::YB + j) * 64 + (threadIdx.x & 63);
  }
};

template <class M>
__global__ void __launch_bounds__(256) mix_kernel(MixArgs g) {
  using T = typename M::T;
  using O = Ops<T>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* Y = smem;
  char* W = Y + M::XT;
  char* X = W + M::WT;
  char* S = X + M::XT;  // the state as an operand, then the outputs on their way out

  // workgroup -> segment, tile of w, head, sequence (neighbours on one XCD)
  int id = xcd_position(blockIdx.x, gridDim.x);
  const int seg = id % g.nseg;
  id /= g.nseg;
  const int wt = id % g.wtiles;
  id /= g.wtiles;
  const int head = id % g.heads, seq = id / g.heads;
  const Span sp = span_of(g, seq);
  const int t0 = seg * g.seg_len, t1 = min(sp.len, t0 + g.seg_len);
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int w0 = wt * M::WD, wrows = min(g.wdim - w0, M::WD);
  const int64_t hs = static_cast<int64_t>(seq) * g.heads + head;
  const int64_t sdim = static_cast<int64_t>(g.ydim) * g.wdim;
  float* segp = g.seg ? g.seg + ((hs * g.wtiles + wt) * g.nseg + seg) * M::YD * M::WD : nullptr;
  if (g.nseg > 1 && t0 >= t1) return;  // whole workgroups

  const Decay a(g.decay[head]);
  State<M> st;
  st.clear();
  bool have = false;
  if (M::OUT) {
    if (g.nseg > 1) {
#pragma unroll
      for (int i = 0; i < M::WB; ++i)
#pragma unroll
        for (int j = 0; j < M::YB; ++j) st.a[i][j] = *st.place(segp, wv, i, j);
      have = true;
    } else if (g.s0) {
      st.template given<false>(const_cast<float*>(g.s0) + hs * sdim, g, wv, w0);
      have = true;
    }
  }

  const int64_t ld = g.tokens;
  auto rows = [&](const void* p, int shared, int dim) {
    return static_cast<const T*>(p) + (static_cast<int64_t>(shared ? head / g.group : head) * dim) * ld + sp.first;
  };
  const T* xp = M::OUT ? rows(g.x, g.x_shared, g.ydim) : nullptr;
  const T* yp = rows(g.y, g.y_shared, g.ydim);
  const T* wp = rows(g.w, g.w_shared, g.wdim) + w0 * ld;

  const int nchunk = (t1 - t0 + kChunk - 1) / kChunk;
  auto first_of = [&](int c) { return t0 + (M::REV ? nchunk - 1 - c : c) * kChunk; };
  TileRegs<T, M::YD> xr, yr;
  TileRegs<T, M::WD> wr;
  auto fetch = [&](int c) {
    const int t = first_of(c), L = min(kChunk, t1 - t);
    if (M::OUT) xr.load(xp + t, ld, g.ydim, L);
    yr.load(yp + t, ld, g.ydim, L);
    wr.load(wp + t, ld, wrows, L);
  };
  if (nchunk > 0) fetch(0);
  for (int c = 0; c < nchunk; ++c) {
    const int t = first_of(c), L = min(kChunk, t1 - t);
    yr.store(Y);
    wr.store(W);
    if constexpr (M::OUT) {
      xr.store(X);
      if (have) {
#pragma unroll
        for (int i = 0; i < M::WB; ++i)
#pragma unroll
          for (int j = 0; j < M::YB; ++j) {
            const int r = st.y(wv, j), cc = st.w(i);
            char* p = S + tile_off<M::ES, M::WD>(r, cc * M::ES / 16);
            if constexpr (M::ES == 4) {
              *reinterpret_cast<f32x4*>(p) = st.a[i][j];
            } else {
              bf16x4 b;
#pragma unroll
              for (int e = 0; e < 4; ++e) b[e] = static_cast<bf16>(st.a[i][j][e]);
              *reinterpret_cast<bf16x4*>(p + (cc & 7) * 2) = b;
            }
          }
      }
    }
    __syncthreads();
    if (c + 1 < nchunk) fetch(c + 1);
    if constexpr (M::OUT) {
      // outputs of 16 tokens i: out[w][i] = sum_y R[y][w] x[y][i], weighted, plus the chunk's own
      const int i0 = wv * 16, i = i0 + (lane & 15), grp = lane >> 4;
      f32x4 acc[M::WB];
#pragma unroll
      for (int b = 0; b < M::WB; ++b) acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      f32x4 p[4];
#pragma unroll
      for (int jb = 0; jb < 4; ++jb) p[jb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i0 < L) {
#pragma unroll 4
        for (int k = 0; k < M::YD; k += O::ACROSS) {
          const auto xf = O::template across<kChunk>(X, k, i0);
          if (have) {
#pragma unroll
            for (int b = 0; b < M::WB; ++b) acc[b] = O::mma(O::template across<M::WD>(S, k, 16 * b), xf, acc[b]);
          }
#pragma unroll
          for (int jb = 0; jb < 4; ++jb)
            if (M::REV ? jb >= wv : jb <= wv) p[jb] = O::mma(O::template across<kChunk>(Y, k, 16 * jb), xf, p[jb]);
        }
        const float wx = g.cx * a.pow(max(M::REV ? L - 1 - i : i + 1, 0));
#pragma unroll
        for (int b = 0; b < M::WB; ++b) acc[b] *= wx;
#pragma unroll
        for (int jb = 0; jb < 4; ++jb)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int n = M::REV ? jb * 16 + 4 * grp + r - i : i - (jb * 16 + 4 * grp + r);
            p[jb][r] = n >= 0 ? p[jb][r] * (g.cp * a.pow(max(n, 0))) : 0.0f;
          }
        if constexpr (M::ES == 2) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 32 tokens j
            if (M::REV ? 2 * h + 1 < wv : 2 * h > wv) continue;
            bf16x8 pf;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              pf[r] = static_cast<bf16>(p[2 * h][r]);
              pf[r + 4] = static_cast<bf16>(p[2 * h + 1][r]);
            }
#pragma unroll
            for (int b = 0; b < M::WB; ++b) {
              const int row = 16 * b + (lane & 15), col = 32 * h + 4 * grp;
              const bf16x4 lo = *reinterpret_cast<const bf16x4*>(W + tile_off<2, kChunk>(row, col >> 3) + (col & 7) * 2);
              const bf16x4 hi =
                  *reinterpret_cast<const bf16x4*>(W + tile_off<2, kChunk>(row, (col + 16) >> 3) + (col & 7) * 2);
              bf16x8 wf;
#pragma unroll
              for (int r = 0; r < 4; ++r) wf[r] = lo[r], wf[r + 4] = hi[r];
              acc[b] = O::mma(wf, pf, acc[b]);
            }
          }
        } else {
#pragma unroll
          for (int jb = 0; jb < 4; ++jb) {
            if (M::REV ? jb < wv : jb > wv) continue;
#pragma unroll
            for (int b = 0; b < M::WB; ++b) {
              const auto wf = O::template along<kChunk>(W, 16 * b, 16 * jb);
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[b] = O::mma(wf[r], p[jb][r], acc[b]);
            }
          }
        }
      }
      __syncthreads();  // no wave reads X or S any more
      using OutT = typename std::conditional<M::PART, float, T>::type;
#pragma unroll
      for (int b = 0; b < M::WB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * b + 4 * grp + r;
          *reinterpret_cast<OutT*>(S + tile_off<M::OS, kChunk>(row, i * M::OS / 16) + (i * M::OS & 15)) =
              from_f32<OutT>(acc[b][r]);
        }
    }
    // the state past this chunk
    {
      const float aL = a.pow(L);
#pragma unroll
      for (int i = 0; i < M::WB; ++i)
#pragma unroll
        for (int j = 0; j < M::YB; ++j) st.a[i][j] *= aL;
      const int grp = lane >> 4;
#pragma unroll
      for (int k = 0; k < kChunk; k += O::ALONG) {
        constexpr int N = 16 / M::ES;  // tokens of a lane
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int tok = k + N * grp + e;
          f[e] = g.cy * a.pow(M::REV ? tok + 1 : max(L - 1 - tok, 0));
        }
        if constexpr (M::ES == 2) {
          bf16x8 y3[M::YB][3];
#pragma unroll
          for (int j = 0; j < M::YB; ++j) {
            const bf16x8 yf = O::template along<kChunk>(Y, (wv * M::YB + j) * 16, k);
#pragma unroll
            for (int e = 0; e < N; ++e) {
              bf16 s0, s1, s2;
              split3(static_cast<float>(yf[e]) * f[e], s0, s1, s2);
              y3[j][0][e] = s0, y3[j][1][e] = s1, y3[j][2][e] = s2;
            }
          }
#pragma unroll
          for (int i = 0; i < M::WB; ++i) {
            const bf16x8 wf = O::template along<kChunk>(W, 16 * i, k);
#pragma unroll
            for (int j = 0; j < M::YB; ++j)
#pragma unroll
              for (int q = 2; q >= 0; --q) st.a[i][j] = O::mma(wf, y3[j][q], st.a[i][j]);
          }
        } else {
          f32x4 yf[M::YB];
#pragma unroll
          for (int j = 0; j < M::YB; ++j) {
            yf[j] = O::template along<kChunk>(Y, (wv * M::YB + j) * 16, k);
#pragma unroll
            for (int e = 0; e < N; ++e) yf[j][e] *= f[e];
          }
#pragma unroll
          for (int i = 0; i < M::WB; ++i) {
            const f32x4 wf = O::template along<kChunk>(W, 16 * i, k);
#pragma unroll
            for (int j = 0; j < M::YB; ++j)
#pragma unroll
              for (int e = 0; e < N; ++e) st.a[i][j] = O::mma(wf[e], yf[j][e], st.a[i][j]);
          }
        }
      }
      have = true;
    }
    __syncthreads();  // the outputs are whole; no wave reads Y or W any more
    if (M::OUT && g.out) {
      constexpr int EPC = 16 / M::OS, CPR = kChunk * M::OS / 16;
      using OutT = typename std::conditional<M::PART, float, T>::type;
      OutT* op = static_cast<OutT*>(g.out) + (static_cast<int64_t>(head) * g.wdim + w0) * ld + sp.first + t;
      typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));
#pragma unroll
      for (int q = 0; q < M::WD * CPR / 256; ++q) {
        const int at = q * 256 + threadIdx.x, r = at / CPR, cc = at % CPR, n = L - cc * EPC;
        if (r >= wrows || n <= 0) continue;
        const u32x4 v = *reinterpret_cast<const u32x4*>(S + tile_off<M::OS, kChunk>(r, cc));
        OutT* p = op + r * ld + cc * EPC;
        if (n >= EPC) {
          *reinterpret_cast<u32x4_any*>(p) = v;
        } else {
          const OutT* e = reinterpret_cast<const OutT*>(&v);
#pragma unroll
          for (int u = 0; u < EPC; ++u)
            if (u < n) p[u] = e[u];
        }
      }
    }
    if constexpr (M::OUT) {
      if (c + 1 < nchunk) __syncthreads();  // the next chunk's state goes where the outputs were
    }
  }
  if (!M::OUT) {
#pragma unroll
    for (int i = 0; i < M::WB; ++i)
#pragma unroll
      for (int j = 0; j < M::YB; ++j) *st.place(segp, wv, i, j) = st.a[i][j];
  } else if (g.nseg == 1 && g.sT) {
    st.template given<true>(g.sT + hs * sdim, g, wv, w0);
  }
}

// Segment states -> the state in front of each segment, in running order, and the
// last one. Four neighbouring accumulators of a thread.
template <class M>
__global__ void __launch_bounds__(256) mix_scan_kernel(MixArgs g) {
  int id = blockIdx.x;
  const int wt = id % g.wtiles;
  id /= g.wtiles;
  const int head = id % g.heads, seq = id / g.heads;
  const Span sp = span_of(g, seq);
  const Decay a(g.decay[head]);
  const int at = blockIdx.y * 256 + threadIdx.x;  // of YD * WD / 4
  const int lane = at & 63, j = (at >> 6) % M::YB, i = (at >> 6) / M::YB % M::WB, wv = (at >> 6) / M::YB / M::WB;
  const int yr = (wv * M::YB + j) * 16 + (lane & 15), wr = wt * M::WD + i * 16 + 4 * (lane >> 4);
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
  for (int q = 0; q < g.nseg; ++q) {
    const int seg = M::REV ? g.nseg - 1 - q : q;
    const int len = min(sp.len - seg * g.seg_len, g.seg_len);
    if (len <= 0) continue;
    f32x4* s = p + static_cast<int64_t>(seg) * (M::YD * M::WD / 4);
    const f32x4 u = *s;
    *s = run;
    run = run * a.pow(len) + u;
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
__global__ void __launch_bounds__(256) mix_group_kernel(MixArgs g, T* __restrict__ out) {
  const int64_t head = blockIdx.y / g.wdim, r = blockIdx.y % g.wdim, row = blockIdx.y;
  const int per = (g.max_len - 1) / 256 + 1;  // blocks of a sequence
  for (int64_t id = blockIdx.x; id < static_cast<int64_t>(per) * g.n_seqs; id += gridDim.x) {
    const Span sp = span_of(g, static_cast<int>(id / per));
    const int t = static_cast<int>(id % per) * 256 + threadIdx.x;
    if (t >= sp.len) continue;
    const float* p = static_cast<const float*>(g.out) + (head * g.group * g.wdim + r) * g.tokens + sp.first + t;
    float s = 0.0f;
    for (int q = 0; q < g.group; ++q) s += p[static_cast<int64_t>(q) * g.wdim * g.tokens];
    out[row * g.tokens + sp.first + t] = from_f32<T>(s);
  }
}

// ------------------------------------------------------------------ one token
// A workgroup per sequence and head: the state passes once through registers,
// VE columns of a row in a thread. Bound by reading and writing the state.
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
  // one workgroup per sequence, head, tile and segment, numbered in 31 bits
  if (static_cast<int64_t>(d->n_seqs) * d->q_heads >= (int64_t{1} << 22))
    return fail(ARD_ERR_UNSUPPORTED, "%d sequences of %d heads: at most 2^22 states", d->n_seqs, d->q_heads);
  return ARD_OK;
}

constexpr int kFill = 512;  // workgroups that fill the chip

int pad_dim(int d) { return d <= 64 ? 64 : 128; }

// How one run lays out its work: rows of a w tile, and segments.
struct MixPlan {
  int yd, wd, wtiles, nseg, seg_len;
};
MixPlan plan_mix(const ard_linattn_desc* d, int ydim, int wdim) {
  MixPlan p;
  p.yd = pad_dim(ydim);
  p.wd = d->dtype == ARD_BF16 ? pad_dim(wdim) : 64;
  p.wtiles = (wdim + p.wd - 1) / p.wd;
  const int64_t base = static_cast<int64_t>(d->n_seqs) * d->q_heads * p.wtiles;
  int64_t n = base >= kFill / 2 ? 1 : (kFill + base - 1) / base;
  const int64_t chunks = (static_cast<int64_t>(d->max_len) + kChunk - 1) / kChunk;
  n = std::max<int64_t>(1, std::min(n, chunks / 4));  // four chunks at least
  const int64_t per = (chunks + n - 1) / n;
  p.seg_len = static_cast<int>(per * kChunk);
  p.nseg = static_cast<int>((chunks + per - 1) / per);
  return p;
}

size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

size_t seg_bytes(const ard_linattn_desc* d, int ydim, int wdim) {
  const MixPlan p = plan_mix(d, ydim, wdim);
  if (p.nseg == 1) return 0;
  return al256(static_cast<size_t>(d->n_seqs) * d->q_heads * p.wtiles * p.nseg * p.yd * p.wd * 4);
}
size_t part_bytes(const ard_linattn_desc* d) {
  if (d->q_heads == d->kv_heads) return 0;
  return al256(static_cast<size_t>(d->q_heads) * std::max(d->key_dim, d->value_dim) * d->tokens * 4);
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
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), M::LDS, stream, g);
  return hipGetLastError();
}

template <typename T, int YD, int WD, bool REV>
hipError_t run_mix(const MixArgs& g, bool part, hipStream_t stream) {
  hipError_t e;
  if (g.nseg > 1) {
    using U = Mix<T, YD, WD, REV, false, false>;
    if ((e = launch_mix<U>(g, stream)) != hipSuccess) return e;
    hipLaunchKernelGGL(mix_scan_kernel<U>, dim3(g.n_seqs * g.heads * g.wtiles, YD * WD / 1024), dim3(256), 0, stream, g);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return part ? launch_mix<Mix<T, YD, WD, REV, true, true>>(g, stream)
              : launch_mix<Mix<T, YD, WD, REV, true, false>>(g, stream);
}

template <typename T, bool REV>
hipError_t run_mix(const ard_linattn_desc* d, MixArgs g, void* out, float* part, hipStream_t stream) {
  const MixPlan p = plan_mix(d, g.ydim, g.wdim);
  g.offsets = d->d_offsets;
  g.n_seqs = d->n_seqs;
  g.max_len = d->max_len;
  g.tokens = d->tokens;
  g.heads = d->q_heads;
  g.group = d->q_heads / d->kv_heads;
  g.nseg = p.nseg;
  g.seg_len = p.seg_len;
  g.wtiles = p.wtiles;
  if (p.nseg == 1) g.seg = nullptr;
  if (!out) part = nullptr;  // the last state alone is asked for
  g.out = part ? part : out;
  hipError_t e;
  const bool pt = part != nullptr;
  if constexpr (sizeof(T) == 2) {
    if (p.yd == 64 && p.wd == 64) e = run_mix<T, 64, 64, REV>(g, pt, stream);
    else if (p.yd == 64) e = run_mix<T, 64, 128, REV>(g, pt, stream);
    else if (p.wd == 64) e = run_mix<T, 128, 64, REV>(g, pt, stream);
    else e = run_mix<T, 128, 128, REV>(g, pt, stream);
  } else {
    e = p.yd == 64 ? run_mix<T, 64, 64, REV>(g, pt, stream) : run_mix<T, 128, 64, REV>(g, pt, stream);
  }
  if (e != hipSuccess || !part) return e;
  const int64_t blocks = ((g.max_len - 1) / 256 + 1) * static_cast<int64_t>(g.n_seqs);
  hipLaunchKernelGGL(mix_group_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(blocks, 1 << 16)),
                                               d->kv_heads * g.wdim),
                     dim3(256), 0, stream, g, static_cast<T*>(out));
  return hipGetLastError();
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
  if (dK) {
    MixArgs r = g;
    r.x = V, r.y = dO, r.w = Q;
    r.x_shared = 1;
    r.ydim = d->value_dim, r.wdim = d->key_dim;
    r.s0 = dST, r.s_trans = 1;
    r.cy = d->scale, r.cx = 1.0f;
    ARD_HIP_CHECK((run_mix<T, true>(d, r, dK, part, stream)));
  }
  if (dV || dS0) {
    MixArgs r = g;
    r.x = K, r.y = Q, r.w = dO;
    r.x_shared = 1;
    r.ydim = d->key_dim, r.wdim = d->value_dim;
    r.s0 = dST, r.sT = dS0;
    r.cy = d->scale, r.cx = 1.0f;
    ARD_HIP_CHECK((run_mix<T, true>(d, r, dV, part, stream)));
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
