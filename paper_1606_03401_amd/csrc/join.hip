// What joins a block to the residual stream, forward and backward:
//     branch = n weight silu(z),  n = x rstd per group of columns;   r = scale residual + branch,   y = r rstd_next weight_next (without a residual: y = branch)
//     dr = rms_back(dy) + dresidual_out, from r as it was stored or (again) from the residual;  dresidual = scale dr;  dz = dr n weight silu'(z);  g = dr weight silu(z);  dx = rstd (g - n mean over the group(g n))
// A row stays in the registers of the threads that read it: one pass over memory each way.  Bound: HBM.
// Forward and backward at 32000 x 1024, bf16, groups of 128 and gate: 38 us (5.1 TB/s) and 57 (5.7); 64000 x 1024 with the residual in fp32: 146 and 236 (5.4, 5.0), 243 with the sum computed again;
// forward at 8192 x 4096, all parts: 65 (5.2).
// A row belongs to one wave up to 2048 columns, to 4 or 16 beyond.  L lanes (a power of two) share a group of columns, so that a group's sum takes
// shuffles among neighbours (and, where L is more than a wave, a few floats in LDS), and several groups of a row are summed at once.
// The kernels of 16 waves, for rows of over 8192 columns, have 128 registers to a thread and keep the rest in scratch memory: up to 23 values forward and 522 backward, of rows or groups that
// are no whole vectors 158 and 654.
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int MAX_WIDTH = 16384;
constexpr int V = 8;               // values of a thread's chunk
constexpr int BACK_GROUPS = 1024;  // workgroups of a backward launch, each with partial sums of dweight and dweight_next

struct Shape {
  int waves, chunks;   // per row, per thread
  int lanes, pieces;   // of a group: L lanes with `pieces` chunks each
};
struct Join {
  const void *x, *z, *residual;
  const float *weight, *weight_next;
  void *y, *residual_out;
  float *rstd, *rstd_next;
  int64_t rows, ldx, ldz, ldr, ldy, ldo;
  int width, group, lanes, pieces;
  float scale, eps;
};
struct JoinBack {
  const void *x, *z, *r, *dy, *dout;
  const float *weight, *weight_next, *rstd, *rstd_next;
  void *dx, *dz, *dres;
  float* parts;   // [workgroups][width, or 2 width], or NULL
  int64_t rows, ldx, ldz, ldr, lddy, lddo, lddx, lddz, lddr;
  int width, group, lanes, pieces;
  float scale;
  int again;   // r is the residual
};

template <int WAVES>
constexpr int threads_of() { return WAVES == 1 ? 4 * WAVE : WAVES * WAVE; }   // four rows of one wave each share a workgroup

// Where a thread's chunks are in a row.  VEC: V neighbouring columns at at[c]; else columns at[c] + L e.
template <int WAVES, int NC, bool VEC>
struct Place {
  int at[NC], count[NC];   // `count` of the V values exist (VEC: all or none)
  int slot[NC];            // the chunk's group
  __device__ inline Place(int width, int group, int lanes, int pieces) {
    const int t = threadIdx.x % (WAVES * WAVE), shift = __builtin_ctz(lanes), l = t & (lanes - 1), first = t >> shift, slots = WAVES * WAVE >> shift;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int it = pieces == 1 ? c : pieces == 2 ? c / 2 : c / 4, piece = pieces == 1 ? 0 : pieces == 2 ? c % 2 : c % 4;
      const int k = it * slots + first, in = VEC ? (piece * lanes + l) * V : piece * V * lanes + l;
      slot[c] = k;
      count[c] = k * group >= width || in >= group ? 0 : VEC ? V : min(V, (group - in + lanes - 1) >> shift);
      at[c] = count[c] ? k * group + in : 0;
    }
  }
  // Nothing that follows from the columns is kept from row to row: kept addresses of eight rows' chunks take more registers than there are.
  __device__ inline void fresh() {
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(at[c]));
  }
};
template <typename T, bool VEC>
struct Raw {
  typedef T Eight __attribute__((ext_vector_type(V), aligned(16)));
  std::conditional_t<VEC, Eight, T[V]> v;
};
// A chunk as it came (what does not exist reads the row's first values again, so that no branch stands between loads), then as floats.
template <bool VEC, typename T>
__device__ inline void load_chunk(const T* row, int at, int count, int lanes, Raw<T, VEC>& raw) {
  if constexpr (VEC) {
    raw.v = *reinterpret_cast<const typename Raw<T, VEC>::Eight*>(row + (unsigned)at);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) raw.v[e] = row[(unsigned)(e < count ? at + lanes * e : 0)];
  }
}
template <bool VEC, typename T>
__device__ inline void widen(const Raw<T, VEC>& raw, int count, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < count ? (float)raw.v[e] : 0.0f;
}
template <bool VEC, typename T>
__device__ inline void store_chunk(T* row, int at, int count, int lanes, const float (&v)[V]) {
  if constexpr (VEC) {
    if (count) store<V>(row + (unsigned)at, v);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < count) row[(unsigned)(at + lanes * e)] = (T)v[e];
  }
}

// A weight's values, or ones.
template <bool VEC>
__device__ inline void load_weight(const float* weight, int at, int count, int lanes, float (&w)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) w[e] = 1.0f;
  if (weight) {
    Raw<float, VEC> ws;
    load_chunk<VEC>(weight, at, count, lanes, ws);
    widen<VEC>(ws, count, w);
  }
}

// Sums of a row's groups, in every chunk of the group.  lds: [waves][NC].
template <int WAVES, int NC>
__device__ inline void group_sums(float (&s)[NC], int lanes, int pieces, float* lds) {
  for (int m = 1; m < min(lanes, WAVE); m <<= 1) {
#pragma unroll
    for (int c = 0; c < NC; ++c) s[c] += __shfl_xor(s[c], m);
  }
  if constexpr (WAVES > 1) {
    if (lanes > WAVE) {
      const int wave = threadIdx.x / WAVE, share = lanes / WAVE, w0 = wave / share * share;
      if (threadIdx.x % WAVE == 0) {
#pragma unroll
        for (int c = 0; c < NC; ++c) lds[wave * NC + c] = s[c];
      }
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float sum = 0.0f;
        for (int w = 0; w < share; ++w) sum += lds[(w0 + w) * NC + c];
        s[c] = sum;
      }
      __syncthreads();
    }
  }
  if constexpr (NC > 1) {
    if (pieces == 2) {
#pragma unroll
      for (int c = 0; c + 1 < NC; c += 2) s[c] = s[c + 1] = s[c] + s[c + 1];
    } else if (pieces == 4) {
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c) sum += s[c];
#pragma unroll
      for (int c = 0; c < NC; ++c) s[c] = sum;
    }
  }
}
template <int WAVES>
__device__ inline float row_sum(float v, float* lds) {
  v = wave_sum(v);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += lds[w];
    __syncthreads();
  }
  return v;
}

// NEXT: there is a residual and a second norm.
template <typename TX, typename TR, int WAVES, int NC, bool VEC, bool NEXT>
__global__ __launch_bounds__(threads_of<WAVES>()) void join_forward_kernel(Join p) {
  constexpr int ROWS = WAVES == 1 ? 4 : 1;
  __shared__ float lds[WAVES * NC];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);   // (uniform over a wave, and so are rows' addresses)
  Place<WAVES, NC, VEC> at(p.width, p.group, p.lanes, p.pieces);
  const int groups = p.width / p.group;
  const float per_group = 1.0f / (float)p.group;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < p.rows; row += (int64_t)gridDim.x * ROWS) {
    at.fresh();
    Raw<TX, VEC> xs[NC], zs[NC];
    Raw<TR, VEC> rs[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TX*)p.x + row * p.ldx, at.at[c], at.count[c], p.lanes, xs[c]);
    if (p.z) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TX*)p.z + row * p.ldz, at.at[c], at.count[c], p.lanes, zs[c]);
    }
    if constexpr (NEXT) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TR*)p.residual + row * p.ldr, at.at[c], at.count[c], p.lanes, rs[c]);
    }
    float a[NC][V], sums[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      widen<VEC>(xs[c], at.count[c], a[c]);
      sums[c] = 0.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) sums[c] += a[c][e] * a[c][e];
    }
    group_sums<WAVES, NC>(sums, p.lanes, p.pieces, lds);
    float total = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float rstd = rsqrtf(sums[c] * per_group + p.eps);
      if (p.rstd && at.count[c] && at.at[c] == at.slot[c] * p.group) p.rstd[row * groups + at.slot[c]] = rstd;
      float w[V];
      load_weight<VEC>(p.weight, at.at[c], at.count[c], p.lanes, w);
#pragma unroll
      for (int e = 0; e < V; ++e) a[c][e] *= rstd * w[e];
      if (p.z) {
        float z[V];
        widen<VEC>(zs[c], at.count[c], z);
#pragma unroll
        for (int e = 0; e < V; ++e) a[c][e] *= z[e] * sigmoid(z[e]);
      }
      if constexpr (NEXT) {
        float r[V];
        widen<VEC>(rs[c], at.count[c], r);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          a[c][e] = e < at.count[c] ? fmaf(p.scale, r[e], a[c][e]) : 0.0f;
          total += a[c][e] * a[c][e];
        }
      }
    }
    if constexpr (NEXT) {
      total = row_sum<WAVES>(total, lds);
      const float rstd = rsqrtf(total / (float)p.width + p.eps);
      if (p.rstd_next && threadIdx.x % (WAVES * WAVE) == 0) p.rstd_next[row] = rstd;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (p.residual_out) store_chunk<VEC>((TR*)p.residual_out + row * p.ldo, at.at[c], at.count[c], p.lanes, a[c]);
        float w[V];
        load_weight<VEC>(p.weight_next, at.at[c], at.count[c], p.lanes, w);
#pragma unroll
        for (int e = 0; e < V; ++e) a[c][e] *= rstd * w[e];
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) store_chunk<VEC>((TX*)p.y + row * p.ldy, at.at[c], at.count[c], p.lanes, a[c]);
  }
}

// Rows are dealt to the workgroups in turn; each adds up dweight and dweight_next of its rows in registers and leaves one partial row.
template <typename TX, typename TR, int WAVES, int NC, bool VEC, bool NEXT>
__global__ __launch_bounds__(threads_of<WAVES>()) void join_backward_kernel(JoinBack p) {
  constexpr int ROWS = WAVES == 1 ? 4 : 1;
  __shared__ float lds[WAVES * NC];
  __shared__ float waves_dw[WAVES == 1 ? 3 * NC * V * WAVE : 1];
  const int sub = ROWS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  Place<WAVES, NC, VEC> at(p.width, p.group, p.lanes, p.pieces);
  const int groups = p.width / p.group;
  const float per_group = 1.0f / (float)p.group;
  float dw[NC][V], dwn[NEXT ? NC : 1][V];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < V; ++e) dw[c][e] = dwn[NEXT ? c : 0][e] = 0.0f;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + sub; row < p.rows; row += (int64_t)gridDim.x * ROWS) {
    at.fresh();
    Raw<TX, VEC> xs[NC], zs[NC], ys[NC];
    Raw<TR, VEC> rs[NC], os[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TX*)p.dy + row * p.lddy, at.at[c], at.count[c], p.lanes, ys[c]);
    if constexpr (NEXT) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TR*)p.r + row * p.ldr, at.at[c], at.count[c], p.lanes, rs[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TX*)p.x + row * p.ldx, at.at[c], at.count[c], p.lanes, xs[c]);
    if (p.z) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TX*)p.z + row * p.ldz, at.at[c], at.count[c], p.lanes, zs[c]);
    }
    if (NEXT && p.dout) {
#pragma unroll
      for (int c = 0; c < NC; ++c) load_chunk<VEC>((const TR*)p.dout + row * p.lddo, at.at[c], at.count[c], p.lanes, os[c]);
    }
    float d[NC][V];   // gradient of the branch
#pragma unroll
    for (int c = 0; c < NC; ++c) widen<VEC>(ys[c], at.count[c], d[c]);
    if constexpr (NEXT) {
      const float rstd = p.rstd_next[row];
      float dot = 0.0f;
      float m[NC][V];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float w[V];
        load_weight<VEC>(p.weight_next, at.at[c], at.count[c], p.lanes, w);
        widen<VEC>(rs[c], at.count[c], m[c]);
        if (p.again) {   // the sum, operation by operation as the forward pass has it
          const float rstd_x = p.rstd[row * groups + (at.count[c] ? at.slot[c] : 0)];
          float a[V], wx[V];
          widen<VEC>(xs[c], at.count[c], a);
          load_weight<VEC>(p.weight, at.at[c], at.count[c], p.lanes, wx);
#pragma unroll
          for (int e = 0; e < V; ++e) a[e] *= rstd_x * wx[e];
          if (p.z) {
            float z[V];
            widen<VEC>(zs[c], at.count[c], z);
#pragma unroll
            for (int e = 0; e < V; ++e) a[e] *= z[e] * sigmoid(z[e]);
          }
#pragma unroll
          for (int e = 0; e < V; ++e) m[c][e] = e < at.count[c] ? fmaf(p.scale, m[c][e], a[e]) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          m[c][e] *= rstd;
          dwn[c][e] += d[c][e] * m[c][e];
          d[c][e] *= w[e];
          dot += d[c][e] * m[c][e];
        }
      }
      dot = row_sum<WAVES>(dot, lds) / (float)p.width;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float o[V], s[V];
        if (p.dout) widen<VEC>(os[c], at.count[c], o);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          d[c][e] = rstd * (d[c][e] - m[c][e] * dot) + (p.dout ? o[e] : 0.0f);
          s[e] = p.scale * d[c][e];
        }
        if (p.dres) store_chunk<VEC>((TR*)p.dres + row * p.lddr, at.at[c], at.count[c], p.lanes, s);
      }
    }
    float n[NC][V], rstd[NC], dots[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      // (0 for lanes that have no columns: another group's, were it not finite, would reach their own group's sum.  A select, since the load is there for all)
      const float own = p.rstd[row * groups + (at.count[c] ? at.slot[c] : 0)];
      rstd[c] = at.count[c] ? own : 0.0f;
      widen<VEC>(xs[c], at.count[c], n[c]);
      float w[V];
      load_weight<VEC>(p.weight, at.at[c], at.count[c], p.lanes, w);
      dots[c] = 0.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) n[c][e] *= rstd[c];
      if (p.z) {
        float z[V], dz[V];
        widen<VEC>(zs[c], at.count[c], z);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float s = sigmoid(z[e]), act = z[e] * s;
          dz[e] = d[c][e] * n[c][e] * w[e] * (s * (1.0f + z[e] * (1.0f - s)));
          d[c][e] *= act;
        }
        store_chunk<VEC>((TX*)p.dz + row * p.lddz, at.at[c], at.count[c], p.lanes, dz);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dw[c][e] += d[c][e] * n[c][e];
        d[c][e] *= w[e];
        dots[c] += d[c][e] * n[c][e];
      }
    }
    group_sums<WAVES, NC>(dots, p.lanes, p.pieces, lds);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int e = 0; e < V; ++e) d[c][e] = rstd[c] * (d[c][e] - n[c][e] * (dots[c] * per_group));
      store_chunk<VEC>((TX*)p.dx + row * p.lddx, at.at[c], at.count[c], p.lanes, d[c]);
    }
  }
  if (!p.parts) return;
  float* out = p.parts + (int64_t)blockIdx.x * p.width * (NEXT ? 2 : 1);
#pragma unroll
  for (int k = 0; k < (NEXT ? 2 : 1); ++k) {
    float t[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) t[c][e] = k ? dwn[NEXT ? c : 0][e] : dw[c][e];
    if constexpr (WAVES == 1) {   // the four waves' sums, in their order
      const int lane = threadIdx.x % WAVE;
      __syncthreads();
      if (sub > 0) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < V; ++e) waves_dw[((sub - 1) * NC * V + c * V + e) * WAVE + lane] = t[c][e];
      }
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) t[c][e] += waves_dw[(w * NC * V + c * V + e) * WAVE + lane];
      }
    }
    if (sub == 0) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e < at.count[c]) out[k * p.width + at.at[c] + (VEC ? e : p.lanes * e)] = t[c][e];
    }
  }
}

// ---- launches ----------------------------------------------------------------------------------------

int to_power(int64_t v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}
// The fewest waves whose threads hold the row in four chunks each, and then the fewest chunks.
bool shape_of(int width, int group, Shape* out) {
  for (int waves : {1, 4, 16}) {
    Shape best = {};
    for (int pieces : {1, 2, 4}) {
      const int lanes = to_power(ceil_div(ceil_div(group, V), pieces));
      if (lanes > waves * WAVE) continue;
      const int64_t chunks = ceil_div(width / group, waves * WAVE / lanes) * pieces;
      if (chunks <= 4 && (!best.waves || chunks < best.chunks)) best = {waves, (int)chunks, lanes, pieces};
    }
    if (best.waves) {
      best.chunks = best.chunks <= 1 ? 1 : best.chunks <= 2 ? 2 : 4;
      *out = best;
      return true;
    }
  }
  return false;
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
  return chunks(std::integral_constant<int, 16>{});
}
int64_t back_groups(const mebptt_join_desc* d, int waves) { return std::min<int64_t>(ceil_div(d->rows, waves == 1 ? 4 : 1), BACK_GROUPS); }

template <typename TX, typename TR, bool NEXT>
int forward(const Join& p, Shape s, bool vec, hipStream_t stream) {
  return with_shape(s, [&](auto w, auto n) {
    constexpr int WAVES = decltype(w)::value, NC = decltype(n)::value;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.rows, WAVES == 1 ? 4 : 1), 1 << 20);
    if (vec) join_forward_kernel<TX, TR, WAVES, NC, true, NEXT><<<grid, threads_of<WAVES>(), 0, stream>>>(p);
    else join_forward_kernel<TX, TR, WAVES, NC, false, NEXT><<<grid, threads_of<WAVES>(), 0, stream>>>(p);
    return launched("mebptt_join_forward");
  });
}
template <typename TX, typename TR, bool NEXT>
int backward(const JoinBack& p, Shape s, bool vec, int64_t groups, hipStream_t stream) {
  return with_shape(s, [&](auto w, auto n) {
    constexpr int WAVES = decltype(w)::value, NC = decltype(n)::value;
    if (vec) join_backward_kernel<TX, TR, WAVES, NC, true, NEXT><<<(unsigned)groups, threads_of<WAVES>(), 0, stream>>>(p);
    else join_backward_kernel<TX, TR, WAVES, NC, false, NEXT><<<(unsigned)groups, threads_of<WAVES>(), 0, stream>>>(p);
    return launched("mebptt_join_backward");
  });
}

int check(const mebptt_join_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->rows < 0) return set_error(MEBPTT_EINVAL, "rows must not be negative");
  if (d->width < 1 || d->width > MAX_WIDTH) return set_error(MEBPTT_EINVAL, "width must be 1 .. %d", MAX_WIDTH);
  if (d->group < 1 || d->width % d->group) return set_error(MEBPTT_EINVAL, "group must divide width");
  if (d->group < 8 && d->width > 4096 * d->group) return set_error(MEBPTT_EINVAL, "group must be at least 8 where width is over 4096 * group");
  if (!float_dtype(d->x_dtype) || !float_dtype(d->residual_dtype)) return set_error(MEBPTT_EINVAL, "unknown dtype");
  if (!(d->eps >= 0.0f)) return set_error(MEBPTT_EINVAL, "eps must not be negative");
  if ((d->again != 0 && d->again != 1) || d->reserved) return set_error(MEBPTT_EINVAL, "again must be 0 or 1, reserved 0");
  return MEBPTT_OK;
}
int check_ld(const void* p, int64_t ld, int width, const char* what) {
  return p && ld < width ? set_error(MEBPTT_EINVAL, "row stride of %s is below the width", what) : MEBPTT_OK;
}

}  // namespace

extern "C" {

int mebptt_join_forward(const mebptt_join_desc* d, const void* x, int64_t ldx, const void* z, int64_t ldz, const float* weight,
                        const void* residual, int64_t ldr, const float* weight_next, void* y, int64_t ldy, void* residual_out,
                        int64_t ldo, float* rstd, float* rstd_next, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (!residual && d->rows && (weight_next || residual_out || rstd_next))
    return set_error(MEBPTT_EINVAL, "weight_next, residual_out and rstd_next belong to a residual");
  if (d->rows == 0) return MEBPTT_OK;
  if (!x || !y) return set_error(MEBPTT_EINVAL, "x and y are required");
  if ((rc = check_ld(x, ldx, d->width, "x")) || (rc = check_ld(z, ldz, d->width, "z")) || (rc = check_ld(residual, ldr, d->width, "residual")) ||
      (rc = check_ld(y, ldy, d->width, "y")) || (rc = check_ld(residual_out, ldo, d->width, "residual_out")))
    return rc;
  const bool vec = d->group % V == 0 && rows_aligned(x, ldx, d->x_dtype, V) && rows_aligned(z, ldz, d->x_dtype, V) &&
                   rows_aligned(residual, ldr, d->residual_dtype, V) && rows_aligned(residual_out, ldo, d->residual_dtype, V) &&
                   rows_aligned(y, ldy, d->x_dtype, V) && rows_aligned(weight, 0, MEBPTT_FP32, V) && rows_aligned(weight_next, 0, MEBPTT_FP32, V);
  Shape s;
  if (!shape_of(d->width, d->group, &s)) return set_error(MEBPTT_EINVAL, "no shape for this width and group");
  const Join p = {x, z, residual, weight, weight_next, y, residual_out, rstd, rstd_next, d->rows, ldx, ldz, ldr, ldy, ldo,
                  d->width, d->group, s.lanes, s.pieces, d->scale, d->eps};
  hipStream_t st = (hipStream_t)stream;
  auto at = [&](auto tx) {
    using TX = decltype(tx);
    if (!residual) return forward<TX, float, false>(p, s, vec, st);
    return d->residual_dtype == MEBPTT_FP32 ? forward<TX, float, true>(p, s, vec, st) : forward<TX, __bf16, true>(p, s, vec, st);
  };
  return d->x_dtype == MEBPTT_FP32 ? at(float{}) : at(__bf16{});
}

size_t mebptt_join_workspace_bytes(const mebptt_join_desc* d) {
  if (check(d) != MEBPTT_OK) return 0;
  return align_up((size_t)std::min<int64_t>(d->rows, BACK_GROUPS) * 2 * d->width * sizeof(float));
}

int mebptt_join_backward(const mebptt_join_desc* d, const void* x, int64_t ldx, const void* z, int64_t ldz, const float* weight,
                         const void* r, int64_t ldr, const float* weight_next, const float* rstd, const float* rstd_next, const void* dy,
                         int64_t lddy, const void* dout, int64_t lddo, void* dx, int64_t lddx, void* dz, int64_t lddz, float* dweight,
                         void* dres, int64_t lddr, float* dweight_next, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  const int w = d->width;
  if (d->rows) {
    if (!x || !rstd || !dy || !dx) return set_error(MEBPTT_EINVAL, "x, rstd, dy and dx are required");
    if (!z != !dz) return set_error(MEBPTT_EINVAL, "z and dz belong together");
    if (!r && (weight_next || rstd_next || dout || dres || dweight_next))
      return set_error(MEBPTT_EINVAL, "weight_next, rstd_next, dresidual_out, dresidual and dweight_next belong to r");
    if (r && !rstd_next) return set_error(MEBPTT_EINVAL, "rstd_next is required");
    if ((rc = check_ld(x, ldx, w, "x")) || (rc = check_ld(z, ldz, w, "z")) || (rc = check_ld(r, ldr, w, "r")) || (rc = check_ld(dy, lddy, w, "dy")) ||
        (rc = check_ld(dout, lddo, w, "dresidual_out")) || (rc = check_ld(dx, lddx, w, "dx")) || (rc = check_ld(dz, lddz, w, "dz")) ||
        (rc = check_ld(dres, lddr, w, "dresidual")))
      return rc;
  }
  const bool sums = dweight || dweight_next;
  if (sums && (rc = check_workspace(workspace, workspace_bytes, mebptt_join_workspace_bytes(d)))) return rc;
  const bool vec = d->group % V == 0 && rows_aligned(x, ldx, d->x_dtype, V) && rows_aligned(z, ldz, d->x_dtype, V) &&
                   rows_aligned(r, ldr, d->residual_dtype, V) && rows_aligned(dy, lddy, d->x_dtype, V) && rows_aligned(dout, lddo, d->residual_dtype, V) &&
                   rows_aligned(dx, lddx, d->x_dtype, V) && rows_aligned(dz, lddz, d->x_dtype, V) && rows_aligned(dres, lddr, d->residual_dtype, V) &&
                   rows_aligned(weight, 0, MEBPTT_FP32, V) && rows_aligned(weight_next, 0, MEBPTT_FP32, V);
  Shape s;
  if (!shape_of(w, d->group, &s)) return set_error(MEBPTT_EINVAL, "no shape for this width and group");
  const int64_t groups = back_groups(d, s.waves);
  const JoinBack p = {x, z, r, dy, dout, weight, weight_next, rstd, rstd_next, dx, dz, dres, sums ? (float*)workspace : nullptr,
                      d->rows, ldx, ldz, ldr, lddy, lddo, lddx, lddz, lddr, w, d->group, s.lanes, s.pieces, d->scale, d->again};
  hipStream_t st = (hipStream_t)stream;
  if (groups) {
    auto at = [&](auto tx) {
      using TX = decltype(tx);
      if (!r) return backward<TX, float, false>(p, s, vec, groups, st);
      return d->residual_dtype == MEBPTT_FP32 ? backward<TX, float, true>(p, s, vec, groups, st) : backward<TX, __bf16, true>(p, s, vec, groups, st);
    };
    if ((rc = d->x_dtype == MEBPTT_FP32 ? at(float{}) : at(__bf16{}))) return rc;
  }
  if (!sums) return MEBPTT_OK;
  const int64_t cols[2] = {w, w};
  float* const outs[2] = {dweight, dweight_next};
  return sum_parts((const float*)workspace, groups, r || (!groups && dweight_next) ? 2 : 1, cols, outs, st);
}

}  // extern "C"
