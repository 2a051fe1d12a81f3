// Depthwise causal convolution of a few taps, forward, backward, and for single tokens:
//     y_s = act(bias + sum_j weight_j x_{s-W+1+j}),   act(v) = v sigmoid(v) or v
// A thread owns V neighbouring channels of one sequence and walks over a stretch of steps with the last W - 1 inputs in registers, so
// that x is read once (and W - 1 rows more per stretch).  Bound: HBM; where there is little to do, the rounds of rows that a thread waits for.
// 1000 x 64 x 2048, bf16, four taps: forward 115 us, 4.6 TB/s, backward 179, 4.4 TB/s; 256 tokens x 2048 6 us, most of it the launch and two
// dependent reads.
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int MAX_TAPS = 8;
constexpr int THREADS = 256;

struct Conv {
  const void *x, *state_in;
  void *y, *state_out;
  const float *weight, *bias;
  const int32_t* lengths;
  int64_t xt, xb, yt, yb;
  int t, B, C, silu;
  int stretch;         // steps per thread
  int groups;          // ceil(C / V)
  int stretches;       // ceil(t / stretch), at least 1
};
struct ConvBack {
  const void *x, *state_in, *dy, *dstate_out;
  void *dx, *dstate_in;
  const float *weight, *bias;
  const int32_t* lengths;
  float* parts;        // [workgroups along y][C][W + 1]
  int64_t xt, xb, gt, gb, dt, db;
  int t, B, C, silu, stretch, groups, stretches;
};
struct ConvStep {
  const void *x, *state_in;
  void *y, *state_out;
  const float *weight, *bias;
  const int32_t* index;
  int64_t ldx, ldy, slots;
  int B, C, silu, groups;
};

__device__ inline int length_of(const int32_t* lengths, int b, int t) { return lengths ? min(max(lengths[b], 0), t) : t; }

// (a group's V channels are all there)
template <int W, int V>
__device__ inline void load_weights(const float* weight, const float* bias, int c, float (&w)[W][V], float (&wb)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    wb[v] = bias ? bias[c + v] : 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][v] = weight[(int64_t)(c + v) * W + j];
  }
}

template <typename T, int V>
using Row = T __attribute__((ext_vector_type(V), aligned(std::min<size_t>(V * sizeof(T), 16))));
template <typename T, int V>
__device__ inline Row<T, V> row_at(const T* p) { return *reinterpret_cast<const Row<T, V>*>(p); }

// The input of step s (from -(W-1) on) of sequence b: x, the state's rows before step 0, zeros without a state and from `len` on.  As it came:
// what turns it into floats waits for it, and belongs behind the other rows' loads.
template <typename T, int W, int V>
__device__ inline Row<T, V> input(const T* x, int64_t xt, const T* state, int C, int s, int len) {
  Row<T, V> v = {};
  if (s < len && (s >= 0 || state)) v = row_at<T, V>(s >= 0 ? x + s * xt : state + (int64_t)(s + W - 1) * C);
  return v;
}
template <typename T, int V>
__device__ inline void widen(const Row<T, V>& r, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = (float)r[e];
}

constexpr int U = 4;   // rows on their way at once

template <typename T, int W, int V>
__global__ __launch_bounds__(THREADS) void conv_forward_kernel(Conv p) {
  const int64_t item = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (item >= (int64_t)p.groups * p.stretches) return;
  const int c = (int)(item % p.groups) * V, part = (int)(item / p.groups), b = blockIdx.y;
  const int len = length_of(p.lengths, b, p.t);
  const int s0 = part * p.stretch, s1 = min(p.t, s0 + p.stretch);
  const T* x = (const T*)p.x + b * p.xb + c;
  T* y = (T*)p.y + b * p.yb + c;
  const T* state = p.state_in ? (const T*)p.state_in + (int64_t)b * (W - 1) * p.C + c : nullptr;
  float w[W][V], wb[V], h[W][V];
  Row<T, V> before[W], last[W];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) before[j] = input<T, W, V>(x, p.xt, state, p.C, s0 - (W - 1) + j, len);
  const bool ends = part == 0 && p.state_out;   // the state may be written over the one read: this thread alone reads and writes these columns
  if (ends) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) last[j] = input<T, W, V>(x, p.xt, state, p.C, len - (W - 1) + j, len);
  }
  load_weights<W, V>(p.weight, p.bias, c, w, wb);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) widen<T, V>(before[j], h[j]);
  if (ends) {
    T* out = (T*)p.state_out + (int64_t)b * (W - 1) * p.C + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) *reinterpret_cast<Row<T, V>*>(out + (int64_t)j * p.C) = last[j];
  }
  const int live = min(s1, len);
  auto step = [&](int s, const Row<T, V>& row) {
    float v[V];
    widen<T, V>(row, h[W - 1]);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[e] = wb[e];
#pragma unroll
      for (int j = 0; j < W; ++j) v[e] += w[j][e] * h[j][e];
      if (p.silu) v[e] *= sigmoid(v[e]);
    }
    store<V>(y + s * p.yt, v);
#pragma unroll
    for (int j = 0; j < W - 1; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) h[j][e] = h[j + 1][e];
  };
  int s = s0;
  for (; s + U <= live; s += U) {
    Row<T, V> rows[U];
#pragma unroll
    for (int u = 0; u < U; ++u) rows[u] = row_at<T, V>(x + (s + u) * p.xt);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) step(s + u, rows[u]);
  }
  for (; s < live; ++s) step(s, row_at<T, V>(x + s * p.xt));
  const float none[V] = {};
  for (int s = max(s0, live); s < s1; ++s) store<V>(y + s * p.yt, none);
}

// dL/dx_p = sum_j w_j dpre_{p+W-1-j} (+ dstate_out where p is one of the last W - 1 inputs), dpre = dy act'(pre), for p from -(W-1), the
// state's rows, to the sequence's end.  A wave takes 64 groups of channels; its workgroup's four waves, and the workgroup's later turns, different
// stretches of steps and sequences, adding dweight and dbias up in registers.
template <typename T, int W, int V>
__global__ __launch_bounds__(THREADS, W <= 4 ? 3 : 2) void conv_backward_kernel(ConvBack p) {
  constexpr int WAVES = THREADS / WAVE;
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int group = blockIdx.x * WAVE + lane, c = group * V;
  const bool mine = group < p.groups;
  float dw[W][V] = {}, dbias[V] = {};
  if (mine) {
    float w[W][V], wb[V];
    load_weights<W, V>(p.weight, p.bias, c, w, wb);
    const int64_t items = (int64_t)p.B * p.stretches;
    for (int64_t item = (int64_t)blockIdx.y * WAVES + wave; item < items; item += (int64_t)gridDim.y * WAVES) {
      const int b = (int)(item / p.stretches), part = (int)(item % p.stretches);
      const int len = length_of(p.lengths, b, p.t);
      const int s0 = part * p.stretch, s1 = min(p.t, s0 + p.stretch), live = min(s1, len);
      const T* x = (const T*)p.x + b * p.xb + c;
      const T* dy = (const T*)p.dy + b * p.gb + c;
      T* dx = (T*)p.dx + b * p.db + c;
      const int64_t at = (int64_t)b * (W - 1) * p.C + c;
      const T* state = p.state_in ? (const T*)p.state_in + at : nullptr;
      const T* dlast = p.dstate_out ? (const T*)p.dstate_out + at : nullptr;
      T* dfirst = p.dstate_in ? (T*)p.dstate_in + at : nullptr;
      const int first = part == 0 ? -(W - 1) : s0;                 // the first position whose gradient is this item's
      float h[W][V], g[W][V];                                       // inputs s-W+1 .. s; dpre of the same steps
#pragma unroll
      for (int j = 0; j < W; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) g[j][e] = 0.0f;
      const int from = max(first, 0);
      Row<T, V> before[W];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) before[j] = input<T, W, V>(x, p.xt, state, p.C, from - (W - 1) + j, len);
#pragma unroll
      for (int j = 0; j < W - 1; ++j) widen<T, V>(before[j], h[j]);
      // dpre of a step, from its input (already the last of h) and d = dy; OWN: a step that dweight counts here.  (None past the sequence's end: its
      // zero times an infinite input would not be zero.)
      auto through = [&](float (&d)[V], bool own) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (p.silu) {
            float v = wb[e];
#pragma unroll
            for (int j = 0; j < W; ++j) v += w[j][e] * h[j][e];
            const float sg = sigmoid(v);
            d[e] *= sg * (1.0f + v * (1.0f - sg));
          }
          if (own) {
            dbias[e] += d[e];
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][e] += d[e] * h[j][e];
          }
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) h[j][e] = h[j + 1][e];
      };
      // what a step of dpre completes: the gradient of the position W - 1 before
      auto gather = [&](const float (&d)[V], float (&v)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          g[W - 1][e] = d[e];
#pragma unroll
          for (int j = 0; j < W; ++j) v[e] += w[W - 1 - j][e] * g[j][e];
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) g[j][e] = g[j + 1][e];
      };
      for (int s = first; s < live + W - 1; s += U) {               // U steps' rows at a time, all of them on their way
        Row<T, V> xs[U], ds[U];
        if (s >= from + W - 1 && s + U <= live) {
#pragma unroll
          for (int u = 0; u < U; ++u) xs[u] = row_at<T, V>(x + (s + u) * p.xt);
#pragma unroll
          for (int u = 0; u < U; ++u) ds[u] = row_at<T, V>(dy + (s + u) * p.gt);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float d[V], v[V] = {};
            widen<T, V>(xs[u], h[W - 1]);
            widen<T, V>(ds[u], d);
            through(d, true);
            gather(d, v);
            store<V>(dx + (s + u - (W - 1)) * p.dt, v);
          }
        } else {                                                    // steps before the first one, past the last, at a stretch's ends
          Row<T, V> ls[U];                                          // gradients of the state after the last step
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = s + u, q = k - (W - 1), r = k - len;      // the position that the step completes, and its row of that state
            xs[u] = ds[u] = ls[u] = Row<T, V>{};
            if (k >= 0 && k < len) {
              xs[u] = row_at<T, V>(x + k * p.xt);
              ds[u] = row_at<T, V>(dy + k * p.gt);
            }
            if (q >= first && r >= 0 && r < W - 1 && dlast) ls[u] = row_at<T, V>(dlast + (int64_t)r * p.C);
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = s + u, q = k - (W - 1);
            if (k < live + W - 1) {
              float d[V], v[V];
              widen<T, V>(ds[u], d);
              widen<T, V>(ls[u], v);
              if (k >= 0) {
                widen<T, V>(xs[u], h[W - 1]);
                through(d, k < live);
              }
              gather(d, v);
              if (q >= first) {
                if (q >= 0) store<V>(dx + q * p.dt, v);
                else if (dfirst) store<V>(dfirst + (int64_t)(q + W - 1) * p.C, v);
              }
            }
          }
        }
      }
      const float none[V] = {};
      for (int s = max(s0, live); s < s1; ++s) store<V>(dx + s * p.dt, none);
    }
  }
  // the four waves' sums, in their order
  __shared__ float lds[WAVES - 1][(W + 1) * V][WAVE];
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
      for (int j = 0; j < W; ++j) lds[wave - 1][j * V + e][lane] = dw[j][e];
      lds[wave - 1][W * V + e][lane] = dbias[e];
    }
  }
  __syncthreads();
  if (wave > 0 || !mine) return;
  float* out = p.parts + (int64_t)blockIdx.y * p.C * (W + 1);
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int k = 0; k < WAVES - 1; ++k) {
#pragma unroll
      for (int j = 0; j < W; ++j) dw[j][e] += lds[k][j * V + e][lane];
      dbias[e] += lds[k][W * V + e][lane];
    }
    if (c + e < p.C) {
#pragma unroll
      for (int j = 0; j < W; ++j) out[(int64_t)(c + e) * W + j] = dw[j][e];
      out[(int64_t)p.C * W + c + e] = dbias[e];
    }
  }
}

template <typename T, int W, int V>
__global__ __launch_bounds__(THREADS) void conv_step_kernel(ConvStep p) {
  const int64_t item = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (item >= (int64_t)p.groups * p.B) return;
  const int c = (int)(item % p.groups) * V, b = (int)(item / p.groups);
  const int64_t slot = p.index ? p.index[b] : b;
  T* y = (T*)p.y + b * p.ldy + c;
  if (slot < 0 || slot >= p.slots) {
    const float none[V] = {};
    store<V>(y, none);
    return;
  }
  const int64_t at = slot * (W - 1) * p.C + c;
  float w[W][V], wb[V], h[W][V], v[V];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) load<V>((const T*)p.state_in + at + (int64_t)j * p.C, h[j]);
  load<V>((const T*)p.x + b * p.ldx + c, h[W - 1]);
  load_weights<W, V>(p.weight, p.bias, c, w, wb);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    v[e] = wb[e];
#pragma unroll
    for (int j = 0; j < W; ++j) v[e] += w[j][e] * h[j][e];
    if (p.silu) v[e] *= sigmoid(v[e]);
  }
  store<V>(y, v);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) store<V>((T*)p.state_out + at + (int64_t)j * p.C, h[j + 1]);
}

// ---- launches ----------------------------------------------------------------------------------------

int check(const mebptt_conv_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->t < 0 || d->t > (1 << 30) || d->B < 0 || d->B > 65535 || d->C < 1 || d->C > (1 << 24))
    return set_error(MEBPTT_EINVAL, "0 <= t <= 2^30, 0 <= B <= 65535 and 1 <= C <= 2^24 are needed");
  if (d->taps < 1 || d->taps > MAX_TAPS) return set_error(MEBPTT_EINVAL, "taps must be 1 .. %d", MAX_TAPS);
  if (!float_dtype(d->dtype)) return set_error(MEBPTT_EINVAL, "dtype must be MEBPTT_FP32 or MEBPTT_BF16");
  return MEBPTT_OK;
}

// Steps per thread.  Long stretches read fewer rows twice (W - 1 of them each); short ones give more threads, and fewer rounds of U rows that a thread
// waits for: halved until two workgroups per compute unit have work (forward; 1536 waves backward), or no further.  Forward and backward, four
// taps, long stretches everywhere / these: 4000 x 1 x 2048 46 / 36 us, 512 x 8 x 1024 44 / 27, 1197 x 6 x 320 36 / 20, 100 x 2 x 128 36 / 16; with twice as
// much to fill 1000 x 64 x 512 84 instead of 77.
int stretch_for(int64_t t, int64_t B, int64_t per_stretch, int64_t enough, int longest, int shortest) {
  int s = longest;
  while (s > shortest && B * ceil_div(t, s) * per_stretch < enough) s /= 2;
  return s;
}
constexpr int STRETCH = 32, SHORT = 8;
constexpr int64_t FILLS = 512 * THREADS;   // threads
// The backward pass reads and computes W - 1 steps at both ends of a stretch twice; its workgroups, three on a compute unit at a time, take
// stretches in turn.  1000 x 64 x 2048, when it was chosen: 184 us; 212 with 1024 workgroups and stretches of 64, 193 with stretches of 32.
constexpr int BACK_STRETCH = 48, BACK_SHORT = 6, BACK_GROUPS = 768, BACK_FILLS = 1536;   // waves
constexpr int BACK_V = 4;

int64_t back_columns(const mebptt_conv_desc* d) { return ceil_div(ceil_div(d->C, d->C % BACK_V ? 1 : BACK_V), WAVE); }
int back_stretch(const mebptt_conv_desc* d) { return stretch_for(d->t, d->B, back_columns(d), BACK_FILLS, BACK_STRETCH, BACK_SHORT); }
int64_t back_parts(const mebptt_conv_desc* d) {
  const int64_t columns = back_columns(d);
  const int64_t items = d->B * std::max<int64_t>(1, ceil_div(d->t, back_stretch(d)));
  return std::max<int64_t>(1, std::min<int64_t>(ceil_div(items, THREADS / WAVE), ceil_div(BACK_GROUPS, columns)));
}

template <typename F>
int with_taps(int taps, F&& f) {
  switch (taps) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}

template <typename T, int V>
int forward(Conv p, int taps, hipStream_t stream) {
  p.groups = (int)ceil_div(p.C, V);
  p.stretch = stretch_for(p.t, p.B, p.groups, FILLS, STRETCH, SHORT);
  p.stretches = (int)std::max<int64_t>(1, ceil_div(p.t, p.stretch));
  const dim3 grid((unsigned)ceil_div((int64_t)p.groups * p.stretches, THREADS), p.B);
  return with_taps(taps, [&](auto w) {
    conv_forward_kernel<T, decltype(w)::value, V><<<grid, THREADS, 0, stream>>>(p);
    return launched("mebptt_conv_forward");
  });
}
template <typename T, int V>
int backward(ConvBack p, int taps, int64_t parts, hipStream_t stream) {
  p.groups = (int)ceil_div(p.C, V);
  p.stretches = (int)std::max<int64_t>(1, ceil_div(p.t, p.stretch));
  const dim3 grid((unsigned)ceil_div(p.groups, WAVE), (unsigned)parts);
  return with_taps(taps, [&](auto w) {
    conv_backward_kernel<T, decltype(w)::value, V><<<grid, THREADS, 0, stream>>>(p);
    return launched("mebptt_conv_backward");
  });
}
template <typename T, int V>
int step(ConvStep p, int taps, hipStream_t stream) {
  p.groups = (int)ceil_div(p.C, V);
  const unsigned grid = (unsigned)ceil_div((int64_t)p.groups * p.B, THREADS);
  return with_taps(taps, [&](auto w) {
    conv_step_kernel<T, decltype(w)::value, V><<<grid, THREADS, 0, stream>>>(p);
    return launched("mebptt_conv_step");
  });
}

int check_seq(const mebptt_seq& s, const mebptt_conv_desc* d, bool written, const char* what) {
  if (d->t && !s.data) return set_error(MEBPTT_EINVAL, "%s is NULL", what);
  if (written && !rows_apart(s, d->t, d->B, d->C)) return set_error(MEBPTT_EINVAL, "rows of %s overlap", what);
  return MEBPTT_OK;
}

}  // namespace

extern "C" {

int mebptt_conv_forward(const mebptt_conv_desc* d, mebptt_seq x, const float* weight, const float* bias, const int32_t* lengths,
                        const void* state_in, mebptt_seq y, void* state_out, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->B == 0 || (d->t == 0 && (!state_out || d->taps == 1))) return MEBPTT_OK;
  if (!weight) return set_error(MEBPTT_EINVAL, "weight is NULL");
  if ((rc = check_seq(x, d, false, "x")) || (rc = check_seq(y, d, true, "y"))) return rc;
  const Conv p = {x.data, state_in, y.data, state_out, weight, bias, lengths, x.stride_t, x.stride_b, y.stride_t, y.stride_b,
                  d->t, d->B, d->C, d->silu, 0, 0, 0};
  const bool vec = d->C % 8 == 0 && rows_aligned(x, d->dtype, 8) && rows_aligned(y, d->dtype, 8) &&
                   rows_aligned(state_in, d->C, d->dtype, 8) && rows_aligned(state_out, d->C, d->dtype, 8);
  hipStream_t s = (hipStream_t)stream;
  if (d->dtype == MEBPTT_FP32) return vec ? forward<float, 8>(p, d->taps, s) : forward<float, 1>(p, d->taps, s);
  return vec ? forward<__bf16, 8>(p, d->taps, s) : forward<__bf16, 1>(p, d->taps, s);
}

size_t mebptt_conv_workspace_bytes(const mebptt_conv_desc* d) {
  if (check(d) != MEBPTT_OK) return 0;
  return align_up((size_t)back_parts(d) * d->C * (d->taps + 1) * sizeof(float));
}

int mebptt_conv_backward(const mebptt_conv_desc* d, mebptt_seq x, const float* weight, const float* bias, const int32_t* lengths,
                         const void* state_in, mebptt_seq dy, const void* dstate_out, mebptt_seq dx, float* dweight, float* dbias,
                         void* dstate_in, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (!weight || !dweight) return set_error(MEBPTT_EINVAL, "weight and dweight are required");
  if (d->B && ((rc = check_seq(x, d, false, "x")) || (rc = check_seq(dy, d, false, "dy")) || (rc = check_seq(dx, d, true, "dx")))) return rc;
  if ((rc = check_workspace(workspace, workspace_bytes, mebptt_conv_workspace_bytes(d)))) return rc;
  const ConvBack p = {x.data, state_in, dy.data, dstate_out, dx.data, dstate_in, weight, bias, lengths, (float*)workspace,
                      x.stride_t, x.stride_b, dy.stride_t, dy.stride_b, dx.stride_t, dx.stride_b, d->t, d->B, d->C, d->silu, back_stretch(d), 0, 0};
  const bool vec = d->C % BACK_V == 0 && rows_aligned(x, d->dtype, BACK_V) && rows_aligned(dy, d->dtype, BACK_V) &&
                   rows_aligned(dx, d->dtype, BACK_V) && rows_aligned(state_in, d->C, d->dtype, BACK_V) &&
                   rows_aligned(dstate_out, d->C, d->dtype, BACK_V) && rows_aligned(dstate_in, d->C, d->dtype, BACK_V);
  const int64_t parts = back_parts(d);
  hipStream_t s = (hipStream_t)stream;
  if (d->dtype == MEBPTT_FP32)
    rc = vec ? backward<float, BACK_V>(p, d->taps, parts, s) : backward<float, 1>(p, d->taps, parts, s);
  else
    rc = vec ? backward<__bf16, BACK_V>(p, d->taps, parts, s) : backward<__bf16, 1>(p, d->taps, parts, s);
  if (rc) return rc;
  const int64_t cols[2] = {(int64_t)d->C * d->taps, d->C};
  float* const outs[2] = {dweight, dbias};
  return sum_parts((const float*)workspace, parts, 2, cols, outs, s);
}

int mebptt_conv_step(const mebptt_conv_desc* d, const void* x, int64_t ldx, const float* weight, const float* bias,
                     const void* state_in, int64_t slots, const int32_t* index, void* y, int64_t ldy, void* state_out,
                     void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->t != 1) return set_error(MEBPTT_EINVAL, "a single token's t is 1");
  if (d->B == 0) return MEBPTT_OK;
  if (!x || !weight || !y || (d->taps > 1 && (!state_in || !state_out))) return set_error(MEBPTT_EINVAL, "a required pointer is NULL");
  if (ldy < d->C && d->B > 1) return set_error(MEBPTT_EINVAL, "rows of y overlap");
  if (slots < 0 || (!index && slots < d->B)) return set_error(MEBPTT_EINVAL, "without an index every sequence needs its own slot");
  const ConvStep p = {x, state_in, y, state_out, weight, bias, index, ldx, ldy, slots, d->B, d->C, d->silu, 0};
  const bool vec = d->C % 8 == 0 && rows_aligned(x, ldx, d->dtype, 8) && rows_aligned(y, ldy, d->dtype, 8) &&
                   rows_aligned(state_in, d->C, d->dtype, 8) && rows_aligned(state_out, d->C, d->dtype, 8);
  hipStream_t s = (hipStream_t)stream;
  if (d->dtype == MEBPTT_FP32) return vec ? step<float, 8>(p, d->taps, s) : step<float, 1>(p, d->taps, s);
  return vec ? step<__bf16, 8>(p, d->taps, s) : step<__bf16, 1>(p, d->taps, s);
}

}  // extern "C"
