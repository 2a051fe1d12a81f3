// Root-mean-square norm of rows with the residual's addition, forward and backward:
//     r = x + residual,   y = r * rstd * weight,   rstd = rsqrt(mean(r^2) + eps)
//     dr = rstd (weight dy - n mean(weight dy n)) + dresidual_out,   n = r rstd,   dweight = sum over rows of dy n
// A row stays in the registers of the threads that read it from its first byte to its last: one pass over memory each way.
// Bound: HBM.  64000 x 1024, bf16 with an fp32 residual: forward 136 us, 5.8 TB/s (part of it never leaves the last cache), backward 199, 5.3 TB/s, and 6
// for the sum of its partial dweight; 8192 x 4096 to 8 bits 66 us, 5.6 TB/s; 4 x 1024 3.7 us.
// A row of up to 2048 values belongs to one wave, so that its sums need no barrier and four rows share a
// workgroup; wider ones to a workgroup of 4 or 16 waves.
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int MAX_WIDTH = 16384;
constexpr int V = 8;               // consecutive values a thread reads at once
constexpr int BACK_GROUPS = 1024;  // workgroups of a backward launch: four per compute unit, each with a partial dweight

struct Norm {
  const void *x, *residual;
  void *y, *residual_out;
  const float* weight;
  float *scale, *rstd;
  int64_t rows, ldx, ldr, ldy, ldo;
  int width;
  float eps;
};
struct NormBack {
  const void *r, *dy, *dout;
  void *dx, *dres;
  const float *weight, *rstd;
  float* parts;   // [workgroups][width], or NULL
  int64_t rows, ldr, lddy, lddo, lddx, lddr;
  int width;
};

// Sum (or maximum) over the waves of a row.  LDS: WAVES floats per call site, written before and read after a barrier.
template <int WAVES, bool MAX>
__device__ inline float row_reduce(float v, float* lds) {
  v = MAX ? wave_max_or_nan(v) : wave_sum(v);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = MAX ? max_or_nan(v, lds[w]) : v + lds[w];
  }
  return v;
}

// The columns of a thread's values: VEC, groups of V neighbours, TPR groups per chunk; otherwise single columns TPR apart, so that
// neighbouring threads read neighbouring columns of rows at any alignment.
template <int TPR, bool VEC>
__device__ inline int column(int chunk, int e, int lane) {
  return VEC ? (chunk * TPR + lane) * V + e : (chunk * V + e) * TPR + lane;
}
// A chunk's values as they came, and then as floats, zeros beyond the row: apart, so that all of a row's loads are on their way before the first one is
// waited for.  Columns beyond the row read its last ones again where that costs no more registers than there are (a VEC width is a multiple of V),
// which keeps branches out from between the loads: 20000 x 2047, forward and backward, 263 us instead of 610.  Wider rows at any alignment
// would need an address per value (1183 x 7931, forward: 70 us instead of 60), the largest workgroups' threads have 128 registers.
template <typename T, bool VEC>
struct Raw {
  typedef T Eight __attribute__((ext_vector_type(V), aligned(16)));
  std::conditional_t<VEC, Eight, T[V]> v;
};
template <int TPR, bool VEC, typename T>
__device__ inline void load_chunk(const T* row, int chunk, int lane, int width, Raw<T, VEC>& raw) {
  constexpr bool CLAMP = TPR == WAVE || (VEC && TPR < 16 * WAVE);
  if constexpr (VEC) {
    const int c = column<TPR, true>(chunk, 0, lane);
    if (!CLAMP) raw.v = {};
    if (CLAMP || c < width) raw.v = *reinterpret_cast<const typename Raw<T, VEC>::Eight*>(row + (unsigned)(CLAMP ? min(c, width - V) : c));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = column<TPR, false>(chunk, e, lane);
      if (!CLAMP) raw.v[e] = (T)0.0f;
      if (CLAMP || c < width) raw.v[e] = row[(unsigned)(CLAMP ? min(c, width - 1) : c)];
    }
  }
}
template <int TPR, bool VEC, typename T>
__device__ inline void widen(const Raw<T, VEC>& raw, int chunk, int lane, int width, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = column<TPR, VEC>(chunk, VEC ? 0 : e, lane) < width ? (float)raw.v[e] : 0.0f;
}

template <int TPR, bool VEC, typename T>
__device__ inline void store_chunk(T* row, int chunk, int lane, int width, const float (&v)[V]) {
  if constexpr (VEC) {
    const int c = column<TPR, true>(chunk, 0, lane);
    if (c < width) store<V>(row + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = column<TPR, false>(chunk, e, lane);
      if (c < width) row[c] = (T)v[e];
    }
  }
}
template <int TPR, bool VEC>
__device__ inline void store_chunk(int8_t* row, int chunk, int lane, int width, const float (&v)[V]) {
  if constexpr (VEC) {
    const int c = column<TPR, true>(chunk, 0, lane);
    union { int8_t b[V]; u32x2 u; } q;
#pragma unroll
    for (int e = 0; e < V; ++e) q.b[e] = (int8_t)(int)v[e];
    if (c < width) *reinterpret_cast<u32x2*>(row + c) = q.u;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = column<TPR, false>(chunk, e, lane);
      if (c < width) row[c] = (int8_t)(int)v[e];
    }
  }
}

template <int WAVES>
constexpr int threads_of() { return WAVES == 1 ? 4 * WAVE : WAVES * WAVE; }   // four rows of one wave each share a workgroup

// WAVES waves per row, NC chunks of V values per thread.  TX, TR, TY: x, residual, y.
template <typename TX, typename TR, typename TY, int WAVES, int NC, bool VEC>
__global__ __launch_bounds__(threads_of<WAVES>()) void norm_forward_kernel(Norm p) {
  constexpr int TPR = WAVES * WAVE, ROWS = WAVES == 1 ? 4 : 1;
  constexpr bool QUANT = sizeof(TY) == 1, AHEAD = WAVES < 16;   // (the largest workgroups have no registers for it)
  __shared__ float lds[2][WAVES];
  const int lane = threadIdx.x % TPR, sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);   // (uniform over a wave, and so are rows' addresses)
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < p.rows; row += (int64_t)gridDim.x * ROWS) {
    float r[NC][V];
    float sum = 0.0f;
    const TX* x = (const TX*)p.x + row * p.ldx;
    Raw<TX, VEC> xs[NC];
    Raw<TR, VEC> as[NC];
    Raw<float, VEC> ws[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(x, c, lane, p.width, xs[c]);
    if (p.residual) {
      const TR* res = (const TR*)p.residual + row * p.ldr;
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(res, c, lane, p.width, as[c]);
    }
    if (AHEAD && p.weight) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(p.weight, c, lane, p.width, ws[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) widen<TPR, VEC>(xs[c], c, lane, p.width, r[c]);
    if (p.residual) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float a[V];
        widen<TPR, VEC>(as[c], c, lane, p.width, a);
#pragma unroll
        for (int e = 0; e < V; ++e) r[c][e] += a[e];
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) sum += r[c][e] * r[c][e];
    // (the barriers inside also stand between the row's last load and its first store, where buffers are shared)
    sum = row_reduce<WAVES, false>(sum, lds[0]);
    const float rstd = rsqrtf(sum / (float)p.width + p.eps);
    // a row whose squares vanish is a row of zeros in 8 bits, without an eps too
    const float times = QUANT && rstd == __builtin_inff() ? 0.0f : rstd;
    if (p.residual_out) {
      TR* out = (TR*)p.residual_out + row * p.ldo;
#pragma unroll
      for (int c = 0; c < NC; ++c) store_chunk<TPR, VEC>(out, c, lane, p.width, r[c]);
    }
    if (p.rstd && lane == 0) p.rstd[row] = rstd;
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float w[V];
      if constexpr (!AHEAD) __builtin_amdgcn_sched_barrier(0);
      if (!AHEAD && p.weight) load_chunk<TPR, VEC>(p.weight, c, lane, p.width, ws[c]);
      if (p.weight) widen<TPR, VEC>(ws[c], c, lane, p.width, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        r[c][e] = r[c][e] * times * (p.weight ? w[e] : 1.0f);
        if constexpr (QUANT) top = max_or_nan(top, fabsf(r[c][e]));
      }
    }
    if constexpr (QUANT) {
      top = row_reduce<WAVES, true>(top, lds[1]);
      const bool fine = __builtin_isfinite(top) && __builtin_isfinite(sum);
      const float scale = top / 127.0f;
      if (lane == 0) p.scale[row] = fine ? scale : __builtin_nanf("");
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        // an exact quotient: a reciprocal of the smallest scales is not finite
        for (int e = 0; e < V; ++e) r[c][e] = fine && scale > 0.0f ? fminf(127.0f, fmaxf(-127.0f, rintf(r[c][e] / scale))) : 0.0f;
    }
    TY* y = (TY*)p.y + row * p.ldy;
#pragma unroll
    for (int c = 0; c < NC; ++c) store_chunk<TPR, VEC>(y, c, lane, p.width, r[c]);
    if constexpr (WAVES > 1) __syncthreads();   // lds is written again by the next row
  }
}

// Rows are dealt to the workgroups in turn; each adds up dweight of its rows in registers and leaves one partial row.
template <typename TX, typename TR, int WAVES, int NC, bool VEC>
__global__ __launch_bounds__(threads_of<WAVES>()) void norm_backward_kernel(NormBack p) {
  constexpr int TPR = WAVES * WAVE, ROWS = WAVES == 1 ? 4 : 1;
  constexpr bool AHEAD = WAVES < 16;
  __shared__ float lds[WAVES];
  __shared__ float waves_dw[WAVES == 1 ? 3 * NC * V * WAVE : 1];
  const int lane = threadIdx.x % TPR, sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);   // (uniform over a wave, and so are rows' addresses)
  float dw[NC][V];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[c][e] = 0.0f;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < p.rows; row += (int64_t)gridDim.x * ROWS) {
    float n[NC][V], g[NC][V];
    const float rstd = p.rstd[row];
    const TR* r = (const TR*)p.r + row * p.ldr;
    const TX* dy = (const TX*)p.dy + row * p.lddy;
    Raw<TR, VEC> rs[NC], os[NC];
    Raw<TX, VEC> gs[NC];
    Raw<float, VEC> ws[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(r, c, lane, p.width, rs[c]);
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(dy, c, lane, p.width, gs[c]);
    if (AHEAD && p.weight) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>(p.weight, c, lane, p.width, ws[c]);
    }
    if (AHEAD && p.dout) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<TPR, VEC>((const TR*)p.dout + row * p.lddo, c, lane, p.width, os[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      widen<TPR, VEC>(rs[c], c, lane, p.width, n[c]);
      widen<TPR, VEC>(gs[c], c, lane, p.width, g[c]);
    }
    float dot = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float w[V];
      if constexpr (!AHEAD) __builtin_amdgcn_sched_barrier(0);
      if (!AHEAD && p.weight) load_chunk<TPR, VEC>(p.weight, c, lane, p.width, ws[c]);
      if (p.weight) widen<TPR, VEC>(ws[c], c, lane, p.width, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        n[c][e] *= rstd;
        dw[c][e] += g[c][e] * n[c][e];
        if (p.weight) g[c][e] *= w[e];
        dot += g[c][e] * n[c][e];
      }
    }
    dot = row_reduce<WAVES, false>(dot, lds) / (float)p.width;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float d[V];
      if constexpr (!AHEAD) __builtin_amdgcn_sched_barrier(0);
      if (!AHEAD && p.dout) load_chunk<TPR, VEC>((const TR*)p.dout + row * p.lddo, c, lane, p.width, os[c]);
      if (p.dout) widen<TPR, VEC>(os[c], c, lane, p.width, d);
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = rstd * (g[c][e] - n[c][e] * dot) + (p.dout ? d[e] : 0.0f);
      if (p.dx) store_chunk<TPR, VEC>((TX*)p.dx + row * p.lddx, c, lane, p.width, d);
      if (p.dres) store_chunk<TPR, VEC>((TR*)p.dres + row * p.lddr, c, lane, p.width, d);
    }
    if constexpr (WAVES > 1) __syncthreads();
  }
  if (!p.parts) return;
  if constexpr (WAVES == 1) {   // the four waves' sums, in their order
    if (sub > 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) waves_dw[((sub - 1) * NC * V + c * V + e) * WAVE + lane] = dw[c][e];
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[c][e] += waves_dw[(w * NC * V + c * V + e) * WAVE + lane];
  }
  float* out = p.parts + (int64_t)blockIdx.x * p.width;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int k = column<TPR, VEC>(c, e, lane);
      if (k < p.width) out[k] = dw[c][e];
    }
}

// ---- launches ----------------------------------------------------------------------------------------

// A wave per row up to 2048 columns, 4 up to 8192, 16 beyond: at most 32 values of the row per thread, 16 in the largest workgroups,
// whose threads have 128 registers.
struct Shape { int waves, chunks; };
Shape shape_of(int width) {
  const int waves = width <= 2048 ? 1 : width <= 8192 ? 4 : 16;
  const int need = (int)ceil_div(width, waves * WAVE * V);
  return {waves, need <= 1 ? 1 : need <= 2 ? 2 : 4};
}

template <typename F>
int with_shape(Shape s, F&& f) {
  auto chunks = [&](auto w) {
    if (s.chunks == 1) return f(w, std::integral_constant<int, 1>{});
    if (s.chunks == 2) return f(w, std::integral_constant<int, 2>{});
    return f(w, std::integral_constant<int, 4>{});
  };
  if (s.waves == 1) return chunks(std::integral_constant<int, 1>{});
  if (s.waves == 4) return chunks(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
}

template <typename TX, typename TR, typename TY>
int forward(const Norm& p, bool vec, hipStream_t stream) {
  return with_shape(shape_of(p.width), [&](auto w, auto n) {
    constexpr int WAVES = decltype(w)::value, NC = decltype(n)::value;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.rows, WAVES == 1 ? 4 : 1), 1 << 20);
    if (vec) norm_forward_kernel<TX, TR, TY, WAVES, NC, true><<<grid, threads_of<WAVES>(), 0, stream>>>(p);
    else norm_forward_kernel<TX, TR, TY, WAVES, NC, false><<<grid, threads_of<WAVES>(), 0, stream>>>(p);
    return launched("mebptt_norm_forward");
  });
}

int64_t back_groups(const mebptt_norm_desc* d) {
  return std::min<int64_t>(ceil_div(d->rows, shape_of(d->width).waves == 1 ? 4 : 1), BACK_GROUPS);
}

template <typename TX, typename TR>
int backward(const NormBack& p, bool vec, int64_t groups, hipStream_t stream) {
  return with_shape(shape_of(p.width), [&](auto w, auto n) {
    constexpr int WAVES = decltype(w)::value, NC = decltype(n)::value;
    if (vec) norm_backward_kernel<TX, TR, WAVES, NC, true><<<(unsigned)groups, threads_of<WAVES>(), 0, stream>>>(p);
    else norm_backward_kernel<TX, TR, WAVES, NC, false><<<(unsigned)groups, threads_of<WAVES>(), 0, stream>>>(p);
    return launched("mebptt_norm_backward");
  });
}

int check(const mebptt_norm_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->rows < 0) return set_error(MEBPTT_EINVAL, "rows must not be negative");
  if (d->width < 1 || d->width > MAX_WIDTH) return set_error(MEBPTT_EINVAL, "width must be 1 .. %d", MAX_WIDTH);
  if (!float_dtype(d->x_dtype) || !float_dtype(d->residual_dtype) || (!float_dtype(d->y_dtype) && d->y_dtype != MEBPTT_INT8))
    return set_error(MEBPTT_EINVAL, "unknown dtype");
  if (!(d->eps >= 0.0f)) return set_error(MEBPTT_EINVAL, "eps must not be negative");
  return MEBPTT_OK;
}
int check_ld(const void* p, int64_t ld, int width, const char* what) {
  return p && ld < width ? set_error(MEBPTT_EINVAL, "row stride of %s is below the width", what) : MEBPTT_OK;
}

// [P][all] -> three outputs: 16 columns per workgroup, 64 threads per column, whose sums meet in LDS.
constexpr int SUM_COLS = 16, SUM_ROWS = 64;
struct Sum {
  const float* parts;
  int64_t P, all, end0, end1;
  float* outs[3];
};
__global__ __launch_bounds__(SUM_COLS* SUM_ROWS) void sum_parts_kernel(Sum p) {
  __shared__ float lds[SUM_ROWS][SUM_COLS];
  const int x = threadIdx.x % SUM_COLS, y = threadIdx.x / SUM_COLS;
  for (int64_t c0 = (int64_t)blockIdx.x * SUM_COLS; c0 < p.all; c0 += (int64_t)gridDim.x * SUM_COLS) {
    const int64_t c = c0 + x;
    float s = 0.0f;
    if (c < p.all) {
#pragma unroll 8
      for (int64_t i = y; i < p.P; i += SUM_ROWS) s += p.parts[i * p.all + c];
    }
    lds[y][x] = s;
    __syncthreads();
    if (y < 4) {
#pragma unroll
      for (int i = 4; i < SUM_ROWS; i += 4) s += lds[i + y][x];
      lds[y][x] = s;
    }
    __syncthreads();
    if (y == 0 && c < p.all) {
      s = lds[0][x] + lds[1][x] + lds[2][x] + lds[3][x];
      float* out = c < p.end0 ? p.outs[0] : c < p.end1 ? p.outs[1] : p.outs[2];
      if (out) out[c - (c < p.end0 ? 0 : c < p.end1 ? p.end0 : p.end1)] = s;
    }
    __syncthreads();
  }
}

}  // namespace

int mebptt::ops::sum_parts(const float* parts, int64_t P, int n, const int64_t* cols, float* const* outs, hipStream_t stream) {
  Sum p = {parts, P, cols[0], cols[0], cols[0], {outs[0], nullptr, nullptr}};
  if (n > 1) p.outs[1] = outs[1], p.all = p.end1 = cols[0] + cols[1];
  if (n > 2) p.outs[2] = outs[2], p.all += cols[2];
  if (p.all <= 0) return MEBPTT_OK;
  const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.all, SUM_COLS), 1 << 20);
  sum_parts_kernel<<<grid, SUM_COLS * SUM_ROWS, 0, stream>>>(p);
  return launched("sum of parts");
}

extern "C" {

int mebptt_norm_forward(const mebptt_norm_desc* d, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                        const float* weight, void* y, int64_t ldy, float* y_scale, void* residual_out, int64_t ldo, float* rstd,
                        void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->rows == 0) return MEBPTT_OK;
  if (!x || !y) return set_error(MEBPTT_EINVAL, "x and y are required");
  const bool quant = d->y_dtype == MEBPTT_INT8;
  if (quant && !y_scale) return set_error(MEBPTT_EINVAL, "an output in 8 bits needs y_scale");
  if ((rc = check_ld(x, ldx, d->width, "x")) || (rc = check_ld(residual, ldr, d->width, "residual")) ||
      (rc = check_ld(y, ldy, d->width, "y")) || (rc = check_ld(residual_out, ldo, d->width, "residual_out")))
    return rc;
  const Norm p = {x, residual, y, residual_out, weight, y_scale, rstd, d->rows, ldx, ldr, ldy, ldo, d->width, d->eps};
  const bool vec = d->width % V == 0 && rows_aligned(x, ldx, d->x_dtype, V) && rows_aligned(residual, ldr, d->residual_dtype, V) &&
                   rows_aligned(residual_out, ldo, d->residual_dtype, V) && rows_aligned(y, ldy, d->y_dtype, V) &&
                   rows_aligned(weight, 0, MEBPTT_FP32, V);
  hipStream_t s = (hipStream_t)stream;
  auto out = [&](auto tx, auto tr) {
    using TX = decltype(tx);
    using TR = decltype(tr);
    if (quant) return forward<TX, TR, int8_t>(p, vec, s);
    return d->y_dtype == MEBPTT_FP32 ? forward<TX, TR, float>(p, vec, s) : forward<TX, TR, __bf16>(p, vec, s);
  };
  if (d->x_dtype == MEBPTT_FP32) return d->residual_dtype == MEBPTT_FP32 ? out(float{}, float{}) : out(float{}, __bf16{});
  return d->residual_dtype == MEBPTT_FP32 ? out(__bf16{}, float{}) : out(__bf16{}, __bf16{});
}

size_t mebptt_norm_workspace_bytes(const mebptt_norm_desc* d) {
  if (check(d) != MEBPTT_OK) return 0;
  return align_up((size_t)back_groups(d) * d->width * sizeof(float));
}

int mebptt_norm_backward(const mebptt_norm_desc* d, const void* r, int64_t ldr, const float* weight, const float* rstd,
                         const void* dy, int64_t lddy, const void* dout, int64_t lddo, void* dx, int64_t lddx, void* dres,
                         int64_t lddr, float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->rows && (!r || !rstd || !dy)) return set_error(MEBPTT_EINVAL, "r, rstd and dy are required");
  if (d->rows && ((rc = check_ld(r, ldr, d->width, "r")) || (rc = check_ld(dy, lddy, d->width, "dy")) ||
                  (rc = check_ld(dout, lddo, d->width, "dresidual_out")) || (rc = check_ld(dx, lddx, d->width, "dx")) ||
                  (rc = check_ld(dres, lddr, d->width, "dresidual"))))
    return rc;
  if (dweight && (rc = check_workspace(workspace, workspace_bytes, mebptt_norm_workspace_bytes(d)))) return rc;
  const NormBack p = {r, dy, dout, dx, dres, weight, rstd, dweight ? (float*)workspace : nullptr,
                      d->rows, ldr, lddy, lddo, lddx, lddr, d->width};
  const bool vec = d->width % V == 0 && rows_aligned(r, ldr, d->residual_dtype, V) && rows_aligned(dy, lddy, d->x_dtype, V) &&
                   rows_aligned(dout, lddo, d->residual_dtype, V) && rows_aligned(dx, lddx, d->x_dtype, V) &&
                   rows_aligned(dres, lddr, d->residual_dtype, V) && rows_aligned(weight, 0, MEBPTT_FP32, V);
  const int64_t groups = back_groups(d);
  hipStream_t s = (hipStream_t)stream;
  if (groups) {
    if (d->x_dtype == MEBPTT_FP32)
      rc = d->residual_dtype == MEBPTT_FP32 ? backward<float, float>(p, vec, groups, s) : backward<float, __bf16>(p, vec, groups, s);
    else
      rc = d->residual_dtype == MEBPTT_FP32 ? backward<__bf16, float>(p, vec, groups, s) : backward<__bf16, __bf16>(p, vec, groups, s);
    if (rc) return rc;
  }
  if (!dweight) return MEBPTT_OK;
  const int64_t cols = d->width;
  return sum_parts((const float*)workspace, groups, 1, &cols, &dweight, s);
}

}  // extern "C"
