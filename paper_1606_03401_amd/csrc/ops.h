// What the operators of the selective state space block share: element types, vectors of eight, sums over a workgroup, checks of
// arguments.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "common.h"

namespace mebptt {
namespace ops {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x3 __attribute__((ext_vector_type(3)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVE = 64;
constexpr size_t ALIGN = 256;
inline size_t align_up(size_t v) { return (v + ALIGN - 1) / ALIGN * ALIGN; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- elements --------------------------------------------------------------------------------------

// V consecutive elements as floats; the address is a multiple of V elements' size, at most 16 bytes.
template <int V>
__device__ inline void load(const float* p, float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e + i] = x[i];
    }
  } else if constexpr (V == 2) {
    const f32x2 x = *reinterpret_cast<const f32x2*>(p);
    v[0] = x[0];
    v[1] = x[1];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = p[e];
  }
}
template <int V>
__device__ inline void load(const __bf16* p, float (&v)[V]) {
  if constexpr (V % 8 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 8) {
      const bf16x8 x = *reinterpret_cast<const bf16x8*>(p + e);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[e + i] = (float)x[i];
    }
  } else if constexpr (V == 4) {
    const bf16x4 x = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)x[i];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (float)p[e];
  }
}
// Rounds to nearest even where the type is narrower.
template <int V>
__device__ inline void store(float* p, const float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) *reinterpret_cast<f32x4*>(p + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
  } else if constexpr (V == 2) {
    *reinterpret_cast<f32x2*>(p) = f32x2{v[0], v[1]};
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = v[e];
  }
}
template <int V>
__device__ inline void store(__bf16* p, const float (&v)[V]) {
  if constexpr (V % 8 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 8) {
      bf16x8 x;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (__bf16)v[e + i];
      *reinterpret_cast<bf16x8*>(p + e) = x;
    }
  } else if constexpr (V == 4) {
    bf16x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x4*>(p) = x;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = (__bf16)v[e];
  }
}

// Off by at most 6 * 2^-24 of itself above zero and (6 + 1.5 |x|) 2^-24 below, where the rounding of x log2 e counts |x| times; zero below -88.
__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// ---- sums ------------------------------------------------------------------------------------------

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int m = WAVE / 2; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
// The larger one; NaN if either is.
__device__ inline float max_or_nan(float a, float b) { return (b > a || b != b) ? b : a; }
__device__ inline float wave_max_or_nan(float v) {
#pragma unroll
  for (int m = WAVE / 2; m; m >>= 1) v = max_or_nan(v, __shfl_xor(v, m));
  return v;
}

// ---- checks ----------------------------------------------------------------------------------------

inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t elem_bytes(int dtype) { return dtype == MEBPTT_FP32 ? 4 : dtype == MEBPTT_BF16 ? 2 : 1; }
inline bool float_dtype(int dtype) { return dtype == MEBPTT_FP32 || dtype == MEBPTT_BF16; }

// Rows of V elements at 16-byte (or the vector's own, if that is smaller) boundaries.
inline bool rows_aligned(const void* p, int64_t ld, int dtype, int V) {
  if (!p) return true;
  const size_t unit = std::min<size_t>(16, V * elem_bytes(dtype));
  return aligned(p, unit) && (ld * (int64_t)elem_bytes(dtype)) % (int64_t)unit == 0;
}
inline bool rows_aligned(const mebptt_seq& s, int dtype, int V) {
  return rows_aligned(s.data, s.stride_t, dtype, V) && rows_aligned(s.data, s.stride_b, dtype, V);
}

// Whether the t x B rows of C elements of an output lie apart from each other.
inline bool rows_apart(const mebptt_seq& s, int64_t t, int64_t B, int64_t C) {
  const int64_t st = s.stride_t < 0 ? -s.stride_t : s.stride_t, sb = s.stride_b < 0 ? -s.stride_b : s.stride_b;
  if (t <= 1 && B <= 1) return true;
  if (t <= 1) return sb >= C;
  if (B <= 1) return st >= C;
  return st >= sb ? sb >= C && st >= (B - 1) * sb + C : st >= C && sb >= (t - 1) * st + C;
}

inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MEBPTT_OK : set_error(MEBPTT_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline int check_workspace(const void* workspace, size_t bytes, size_t needed) {
  if (!needed) return MEBPTT_OK;
  if (!workspace) return set_error(MEBPTT_EWORKSPACE, "workspace is NULL");
  if (bytes < needed) return set_error(MEBPTT_EWORKSPACE, "workspace has %zu bytes, %zu needed", bytes, needed);
  if (!aligned(workspace, ALIGN)) return set_error(MEBPTT_EWORKSPACE, "workspace must be 256-byte aligned");
  return MEBPTT_OK;
}

// Sums of P partial rows in one fixed order, in a launch of their own: a row's first cols[0] floats go to outs[0], its next cols[1] to
// outs[1], and so on (NULL: nowhere), at most three.
int sum_parts(const float* parts, int64_t P, int n, const int64_t* cols, float* const* outs, hipStream_t stream);

}  // namespace ops
}  // namespace mebptt
