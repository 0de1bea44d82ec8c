// Shared by the kernels of a training step's end: argument checks, strided views, copies of
// matrices whose rows do not start on 16 bytes, fills and products.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "../ard_gemm_fast.hpp"
#include "../ard_internal.hpp"

namespace ard {

inline int need_ptr(const void* p, const char* name) {
  if (!p) return fail(ARD_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}
inline int may_ptr(const void* p, const char* name) {
  if (p && !aligned16(p)) return fail(ARD_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return ARD_OK;
}
inline int check_space(size_t need, const void* ws, size_t ws_bytes) {
  if (need == 0) return ARD_OK;
  if (!ws || ws_bytes < need)
    return fail(ARD_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : 0);
  if (!aligned16(ws)) return fail(ARD_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  return ARD_OK;
}

// Whether an output starts where one of these arguments does.
inline bool same_buffer(const void* out, std::initializer_list<const void*> others) {
  return out && std::find(others.begin(), others.end(), out) != others.end();
}

inline size_t al256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

// The kept indices of a plan over n neurons (NULL or period 1: all of them).
struct Kept {
  int32_t n, kept, period, offset;
};
inline Kept kept_of(const ard_row_plan* plan, int32_t n) {
  if (!plan || plan->period == 1) return {n, n, 1, 0};
  return {n, plan->kept, plan->period, plan->offset};
}

inline GemmOperand view(const void* p, int64_t ld) {
  GemmOperand o = {};
  o.p = p;
  o.ld = ld;
  return o;
}

// Floats of partial sums of a product, whichever kernel takes it.
template <typename T>
size_t partial_floats(int M, int N, int K) {
  int64_t s = plan_gemm<T>(M, N, K, 1, 1).splits;
  if constexpr (sizeof(T) == 4) {
    s = std::max<int64_t>(s, plan_fast_f32(M, N, K, 1, 1, kAnyRoom).splits);
    for (const auto& costs : kCostRegF32)
      s = std::max<int64_t>(s, plan_fast_f32(M, N, K, 1, 1, kAnyRoom, false, costs).splits);
  } else {
    s = std::max<int64_t>(s, plan_fast_bf16(M, N, K, 1, 1).splits);
  }
  return s > 1 ? static_cast<size_t>(s) * M * N : 0;
}

// A product of strided views, on the fast kernels or, past their load offsets, the general one.
template <typename T, bool AMC, bool BMC, typename OutT>
hipError_t product(const GemmArgs& g, hipStream_t stream, float* partial, size_t floats) {
  if (any_ok<AMC, BMC>(g, sizeof(T)))
    return run_strided_gemm<T, AMC, BMC, OutT, EPI_STORE>(g, 1, stream, floats ? partial : nullptr,
                                                          static_cast<int64_t>(floats));
  constexpr int A = AMC ? MC_ELEM : KC_ELEM, B = BMC ? MC_ELEM : KC_ELEM;
  return run_gemm<T, OutT, A, A, B, B, false, false, EPI_STORE>(g, 1, false, false, stream, floats ? partial : nullptr);
}

// Sixteen bytes of an array of any type.
typedef u32x4 u32x4_any __attribute__((may_alias));
typedef u32x4 u32x4_any2 __attribute__((aligned(2), may_alias));

// Sixteen bytes of a row as loaded, and its elements in fp32; rows start at any element.
template <typename T, int VE>
struct Chunk {
  typename std::conditional<VE == 1, T, u32x4>::type raw;
  // the first n (>= 1) elements at p, 0 behind them
  __device__ __forceinline__ void load(const T* p, int n) {
    if constexpr (VE == 1)
      raw = *p;
    else if (n >= VE)
      raw = load16_any<sizeof(T)>(reinterpret_cast<const char*>(p));
    else
      raw = load16_part<sizeof(T)>(reinterpret_cast<const char*>(p), n);
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
// NT: past the caches, for what is not read again soon.
template <typename T, int VE, bool NT = false>
__device__ __forceinline__ void store_chunk(T* p, const float (&v)[VE], int n) {
  if constexpr (VE == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    T w[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) w[e] = from_f32<T>(v[e]);
    if (n >= VE) {
      if constexpr (NT)
        __builtin_nontemporal_store(*reinterpret_cast<const u32x4_any*>(w), reinterpret_cast<u32x4_any2*>(p));
      else
        *reinterpret_cast<u32x4_any2*>(p) = *reinterpret_cast<const u32x4_any*>(w);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (e < n) p[e] = w[e];
    }
  }
}

}  // namespace ard
