// Selective scan: D channels of N states each, a recurrence that is diagonal and depends on its input,
//     w = delta + delta_bias (through softplus);  h_s = exp(w_s A) h_{s-1} + w_s u_s B_s;  y_s = (C_s . h_s + skip u_s) silu(z_s)
// forward, backward, and for single tokens.
//
// A lane holds NB = 4 states of one or two channels in registers over all steps; NL lanes share a channel (4 NL >= N).  Steps come in blocks: a
// block's w, w u, B and C are put into LDS once, as floats, while the next block's inputs are already on their way, so that softplus and the
// gate are computed once per (step, channel) and not in each of the NL lanes.  Bound: the vector unit (per step, channel and
// state one exponential and four products or multiply-adds forward).
#include "dynamic_lds.h"
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int NB = 4;              // states per lane
constexpr int MAX_N = 64;
constexpr float LOG2E = 1.4426950408889634f;

struct Seq { const void* p; int64_t t, b; };
struct SeqOut { void* p; int64_t t, b; };
inline Seq in_seq(const mebptt_seq& s) { return {s.data, s.stride_t, s.stride_b}; }
inline SeqOut out_seq(const mebptt_seq& s) { return {s.data, s.stride_t, s.stride_b}; }

struct Scan {
  Seq u, delta, z, Bm, Cm;
  const float *A, *skip, *bias;
  const int32_t* lengths;
  int t, B, D, N, G, softplus;
  int tiles;                       // workgroups per group of channels
};
struct Forward {
  Scan in;
  SeqOut y;
  const float* h0;
  float *h_out, *states;
  int stretch;
};

template <typename T>
__device__ inline float at(const Seq& q, int64_t s, int64_t b, int64_t c) { return (float)((const T*)q.p)[s * q.t + b * q.b + c]; }
template <typename T>
__device__ inline void put(const SeqOut& q, int64_t s, int64_t b, int64_t c, float v) { ((T*)q.p)[s * q.t + b * q.b + c] = (T)v; }

__device__ inline int length_of(const int32_t* lengths, int b, int t) { return lengths ? min(max(lengths[b], 0), t) : t; }

// log(1 + e^x); small values keep their relative accuracy, steps of a thousandth being what such a model starts with.
__device__ inline float softplus_of(float x) { return fmaxf(x, 0.0f) + log1pf(__expf(-fabsf(x))); }

// Sum over the NL lanes that share a channel, in every one of them.
template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int NL>
__device__ inline float lanes_sum(float v) {
  if constexpr (NL >= 2) v = dpp_add<0xb1>(v);         // the other one of two
  if constexpr (NL >= 4) v = dpp_add<0x4e>(v);         // the other two of four
  if constexpr (NL >= 8) v = dpp_add<0x141>(v);        // mirrored within eight
  if constexpr (NL >= 16) v = dpp_add<0x128>(v);       // rotated by eight within sixteen
  return v;
}

// NB consecutive states of a channel's N.
__device__ inline void load_states(const float* p, int n0, int N, float (&v)[NB]) {
#pragma unroll
  for (int n = 0; n < NB; ++n) v[n] = n0 + n < N ? p[n0 + n] : 0.0f;
}
__device__ inline void store_states(float* p, int n0, int N, const float (&v)[NB]) {
#pragma unroll
  for (int n = 0; n < NB; ++n)
    if (n0 + n < N) p[n0 + n] = v[n];
}

// ---- forward ---------------------------------------------------------------------------------------

template <int NL>
struct ForwardShape {
  static constexpr int CPL = 2;                                       // channels per lane, which share what it reads of B and C
  static constexpr int CH = WAVE / NL * CPL;                          // channels per workgroup of one wave
  static constexpr int NP = NB * NL;                                  // N rounded up
  static constexpr int TS = NL == 1 || NL == 8 ? 8 : NL == 16 ? 4 : 16;   // steps per block
  static constexpr int ITEMS = (TS * CH + WAVE - 1) / WAVE;           // (step, channel) pairs per lane
  static constexpr int SHARED = (2 * TS * NP + WAVE - 1) / WAVE;      // values of B and C per lane
};

template <typename T, int NL>
__global__ __launch_bounds__(WAVE) void scan_forward_kernel(Forward p) {
  using S = ForwardShape<NL>;
  constexpr int CH = S::CH, TS = S::TS, NP = S::NP, CPL = S::CPL;
  __shared__ __align__(16) float wu[TS][CH][2];      // w and w u of a block; y takes w's place
  __shared__ __align__(16) float bc[TS][2][NP];
  const Scan& in = p.in;
  const int lane = threadIdx.x, b = blockIdx.y;
  const int group = blockIdx.x / in.tiles, per = in.D / in.G;
  const int c0 = group * per + (blockIdx.x % in.tiles) * CH;           // first channel
  const int nch = min(CH, group * per + per - c0);
  const int len = length_of(in.lengths, b, in.t);
  const int q = lane % NL, cl = lane / NL * CPL;                       // this lane's states NB q .. and channels cl, cl + 1

  float h[CPL][NB], A2[CPL][NB];
#pragma unroll
  for (int j = 0; j < CPL; ++j) {
    const int64_t d = min(c0 + cl + j, in.D - 1);
    load_states(in.A + d * in.N, q * NB, in.N, A2[j]);
    if (p.h0) load_states(p.h0 + ((int64_t)b * in.D + d) * in.N, q * NB, in.N, h[j]);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      A2[j][n] *= LOG2E;
      if (!p.h0) h[j][n] = 0.0f;
    }
  }

  float ru[S::ITEMS], rd[S::ITEMS], rz[S::ITEMS], rb[S::SHARED];
  const int64_t gn = (int64_t)group * in.N;
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      const int k = i * WAVE + lane, s = s0 + k / CH, c = k % CH;
      const bool live = k < TS * CH && s < len && c < nch;
      ru[i] = live ? at<T>(in.u, s, b, c0 + c) : 0.0f;
      rd[i] = live ? at<T>(in.delta, s, b, c0 + c) : 0.0f;
      rz[i] = live && in.z.p ? at<T>(in.z, s, b, c0 + c) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
      const int k = i * WAVE + lane, s = s0 + k / (2 * NP), n = k % NP;
      const bool live = k < 2 * TS * NP && s < len && n < in.N;
      rb[i] = !live ? 0.0f : k / NP % 2 ? at<T>(in.Cm, s, b, gn + n) : at<T>(in.Bm, s, b, gn + n);
    }
  };
  fetch(0);
  for (int s0 = 0; s0 < in.t; s0 += TS) {
    float cu[S::ITEMS], cz[S::ITEMS];
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      const int k = i * WAVE + lane, s = s0 + k / CH, c = k % CH;
      cu[i] = ru[i];
      cz[i] = rz[i];
      float w = rd[i] + (in.bias ? in.bias[min(c0 + c, in.D - 1)] : 0.0f);
      if (in.softplus) w = softplus_of(w);
      if (!(s < len && c < nch)) w = 0.0f;             // a step beyond the sequence: h stays as it is
      if (k < TS * CH) {
        wu[k / CH][c][0] = w;
        wu[k / CH][c][1] = w * ru[i];
      }
    }
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
      const int k = i * WAVE + lane;
      if (k < 2 * TS * NP) (&bc[0][0][0])[k] = rb[i];
    }
    __syncthreads();
    if (s0 + TS < in.t) fetch(s0 + TS);
#pragma unroll 4
    for (int s = 0; s < TS; ++s) {
      if (p.states && (s0 + s) % p.stretch == 0 && s0 + s < in.t) {
#pragma unroll
        for (int j = 0; j < CPL; ++j)
          if (cl + j < nch)
            store_states(p.states + (((int64_t)((s0 + s) / p.stretch) * in.B + b) * in.D + c0 + cl + j) * in.N, q * NB, in.N, h[j]);
      }
      const f32x4 w = *reinterpret_cast<const f32x4*>(&wu[s][cl][0]);
      const f32x4 vb = *reinterpret_cast<const f32x4*>(&bc[s][0][q * NB]), vc = *reinterpret_cast<const f32x4*>(&bc[s][1][q * NB]);
      float y[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        y[j] = 0.0f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const float a = __builtin_amdgcn_exp2f(w[2 * j] * A2[j][n]);
          h[j][n] = a * h[j][n] + w[2 * j + 1] * vb[n];
          y[j] += h[j][n] * vc[n];
        }
        y[j] = lanes_sum<NL>(y[j]);
      }
      if (q == 0) {
#pragma unroll
        for (int j = 0; j < CPL; ++j) wu[s][cl + j][0] = y[j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      const int k = i * WAVE + lane, s = s0 + k / CH, c = k % CH;
      if (k < TS * CH && s < in.t && c < nch) {
        float y = wu[k / CH][c][0];
        if (in.skip) y += in.skip[c0 + c] * cu[i];
        if (in.z.p) y *= cz[i] * sigmoid(cz[i]);
        put<T>(p.y, s, b, c0 + c, s < len ? y : 0.0f);
      }
    }
    __syncthreads();
  }
  if (p.h_out) {
#pragma unroll
    for (int j = 0; j < CPL; ++j)
      if (cl + j < nch) store_states(p.h_out + ((int64_t)b * in.D + c0 + cl + j) * in.N, q * NB, in.N, h[j]);
  }
}

// ---- backward --------------------------------------------------------------------------------------

struct Backward {
  Scan in;
  Seq dy;
  SeqOut du, ddelta, dz;
  const float *h0, *states, *dh_out;
  float* dh0;
  float *bc_parts;                 // [tiles][t][B][G][2][N]: sums of dB and dC over a workgroup's channels
  float *a_parts;                  // [B][D N | D | D]: dA, dskip, ddelta_bias of a sequence
  int stretch;
};

constexpr int BS = 16;             // steps per block: a lane's h and exp(w A) of a block stay in registers
constexpr int BACK_WAVES = 4;

template <int NL>
struct BackwardShape {
  static constexpr int CW = WAVE / NL;                                // channels per wave
  static constexpr int CH = CW * BACK_WAVES;                          // channels per workgroup
  static constexpr int NP = NB * NL;
  static constexpr int THREADS = BACK_WAVES * WAVE;
  static constexpr int ITEMS = (BS * CH + THREADS - 1) / THREADS;
  static constexpr int SHARED = (2 * BS * NP + THREADS - 1) / THREADS;
};

// Sums of a lane's eight values (four of dB, four of dC) over the channels of its wave, that is over the lanes with the same
// lane % NL, into red[2][NP].  Halves of the wave, then neighbouring rows of sixteen lanes, exchange one half of their values each, so that every addition
// adds two values that are wanted; what is left is rotated within the rows.
template <int NL>
__device__ inline void channels_sum(float (&v)[2 * NB], int lane, float* red) {
  constexpr int NP = NB * NL;
  const int q = lane % NL;
  float w[NB], x[2];
#pragma unroll
  for (int n = 0; n < NB; ++n) {       // lanes 0 .. 31: dB, 32 .. 63: dC
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[n]), __float_as_uint(v[NB + n]), false, false);
    w[n] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {        // even rows: states 0 and 2, odd rows: 1 and 3
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[2 * n]), __float_as_uint(w[2 * n + 1]), false, false);
    x[n] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    if constexpr (NL <= 8) x[n] = dpp_add<0x128>(x[n]);
    if constexpr (NL <= 4) x[n] = dpp_add<0x124>(x[n]);
    if constexpr (NL <= 2) x[n] = dpp_add<0x122>(x[n]);
    if constexpr (NL <= 1) x[n] = dpp_add<0x121>(x[n]);
  }
  if (lane % 16 < NL) {
    float* out = red + (lane / 32) * NP + q * NB + (lane / 16 % 2);
    out[0] = x[0];
    out[2] = x[1];
  }
}

template <typename T, int NL>
__global__ __launch_bounds__(BACK_WAVES* WAVE) void scan_backward_kernel(Backward p) {
  using S = BackwardShape<NL>;
  constexpr int CH = S::CH, NP = S::NP, THREADS = S::THREADS;
  extern __shared__ __align__(16) float lds[];
  float* wud = lds;                                   // [BS][CH][4]: w, w u, gated dy -> p, q, core
  float* bc = wud + BS * CH * 4;                      // [BS][2][NP]
  float* red = bc + BS * 2 * NP;                      // [BACK_WAVES][BS][2][NP]
  float* kept = red + BACK_WAVES * BS * 2 * NP;       // [stretch / BS][THREADS][NB]: states at the blocks' starts
  const Scan& in = p.in;
  const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, b = blockIdx.y;
  const int group = blockIdx.x / in.tiles, tile = blockIdx.x % in.tiles, per = in.D / in.G;
  const int c0 = group * per + tile * CH, nch = min(CH, group * per + per - c0);
  const int len = length_of(in.lengths, b, in.t);
  const int q = lane % NL, cl = wave * S::CW + lane / NL;
  const bool mine = cl < nch;
  const int64_t d = min(c0 + cl, in.D - 1);
  const int64_t gn = (int64_t)group * in.N;

  float A[NB], g[NB], dA[NB] = {};
  load_states(in.A + d * in.N, q * NB, in.N, A);
#pragma unroll
  for (int n = 0; n < NB; ++n) g[n] = 0.0f;
  if (p.dh_out) load_states(p.dh_out + ((int64_t)b * in.D + d) * in.N, q * NB, in.N, g);
  float dskip = 0.0f, dbias = 0.0f;
  const int ic = tid % CH;                            // this thread's channel in the (step, channel) pairs, THREADS being a multiple of CH
  const float bias = in.bias ? in.bias[min(c0 + ic, in.D - 1)] : 0.0f;
  const float skip = in.skip ? in.skip[min(c0 + ic, in.D - 1)] : 0.0f;

  // Puts a block's w, w u, gated dy and B, C into LDS; keeps u, w, dy and what softplus and the gate need.
  float iu[S::ITEMS], iw[S::ITEMS], idy[S::ITEMS], isig[S::ITEMS], idz[S::ITEMS];
  auto stage = [&](int s0, bool back) {
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      const int k = i * THREADS + tid, s = s0 + k / CH;
      const bool live = k < BS * CH && s < len && ic < nch;
      const float raw = (live ? at<T>(in.delta, s, b, c0 + ic) : 0.0f) + bias;
      iu[i] = live ? at<T>(in.u, s, b, c0 + ic) : 0.0f;
      iw[i] = !live ? 0.0f : in.softplus ? softplus_of(raw) : raw;
      isig[i] = in.softplus ? sigmoid(raw) : 1.0f;
      idy[i] = 0.0f;
      idz[i] = 0.0f;
      if (back) {
        idy[i] = live ? at<T>(p.dy, s, b, c0 + ic) : 0.0f;
        if (in.z.p) {
          const float z = live ? at<T>(in.z, s, b, c0 + ic) : 0.0f, sg = sigmoid(z);
          idz[i] = idy[i] * sg * (1.0f + z * (1.0f - sg));     // times what the gate multiplied
          idy[i] *= z * sg;
        }
      }
      if (k < BS * CH) *reinterpret_cast<f32x4*>(wud + 4 * k) = f32x4{iw[i], iw[i] * iu[i], idy[i], 0.0f};
    }
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
      const int k = i * THREADS + tid, s = s0 + k / (2 * NP), n = k % NP;
      if (k < 2 * BS * NP) bc[k] = !(s < len && n < in.N) ? 0.0f : k / NP % 2 ? at<T>(in.Cm, s, b, gn + n) : at<T>(in.Bm, s, b, gn + n);
    }
  };

  const int stretches = (in.t + p.stretch - 1) / p.stretch;
  for (int st = stretches - 1; st >= 0; --st) {
    const int first = st * p.stretch, blocks = (min(in.t, first + p.stretch) - first + BS - 1) / BS;
    float h[NB];
    load_states(p.states + (((int64_t)st * in.B + b) * in.D + d) * in.N, q * NB, in.N, h);
    // the states at the starts of the stretch's blocks
    for (int k = 0; k < blocks; ++k) {
      float* at_start = kept + (k * THREADS + tid) * NB;
#pragma unroll
      for (int n = 0; n < NB; ++n) at_start[n] = h[n];
      if (k + 1 == blocks) break;
      stage(first + k * BS, false);
      __syncthreads();
#pragma unroll 4
      for (int s = 0; s < BS; ++s) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(wud + 4 * (s * CH + cl));
        const f32x4 vb = *reinterpret_cast<const f32x4*>(bc + (2 * s) * NP + q * NB);
#pragma unroll
        for (int n = 0; n < NB; ++n) h[n] = __builtin_amdgcn_exp2f(w[0] * (A[n] * LOG2E)) * h[n] + w[1] * vb[n];
      }
      __syncthreads();
    }
    for (int k = blocks - 1; k >= 0; --k) {
      const int s0 = first + k * BS;
      stage(s0, true);
#pragma unroll
      for (int n = 0; n < NB; ++n) h[n] = kept[(k * THREADS + tid) * NB + n];
      __syncthreads();
      // forward through the block: exp(w A) and exp(w A) h_{s-1} of every step
      float a[BS][NB], ah[BS][NB];
#pragma unroll
      for (int s = 0; s < BS; ++s) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(wud + 4 * (s * CH + cl));
        const f32x4 vb = *reinterpret_cast<const f32x4*>(bc + (2 * s) * NP + q * NB);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          a[s][n] = __builtin_amdgcn_exp2f(w[0] * (A[n] * LOG2E));
          ah[s][n] = a[s][n] * h[n];
          h[n] = ah[s][n] + w[1] * vb[n];
        }
      }
      // and back
#pragma unroll
      for (int s = BS - 1; s >= 0; --s) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(wud + 4 * (s * CH + cl));
        const f32x4 vb = *reinterpret_cast<const f32x4*>(bc + (2 * s) * NP + q * NB);
        const f32x4 vc = *reinterpret_cast<const f32x4*>(bc + (2 * s + 1) * NP + q * NB);
        float v[2 * NB], through = 0.0f, dlog = 0.0f, core = 0.0f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const float hn = ah[s][n] + w[1] * vb[n];
          g[n] += w[2] * vc[n];
          v[n] = g[n] * w[1];                  // to dB
          v[NB + n] = w[2] * hn;               // to dC
          through += g[n] * vb[n];
          core += hn * vc[n];
          const float r = g[n] * ah[s][n];     // the exponent's gradient
          dlog += r * A[n];
          dA[n] += r * w[0];
          g[n] *= a[s][n];
        }
        if (!mine) {
#pragma unroll
          for (int n = 0; n < 2 * NB; ++n) v[n] = 0.0f;
        }
        channels_sum<NL>(v, lane, red + (wave * BS + s) * 2 * NP);
        through = lanes_sum<NL>(through);
        dlog = lanes_sum<NL>(dlog);
        if (in.z.p) core = lanes_sum<NL>(core);
        if (q == 0) *reinterpret_cast<f32x4*>(wud + 4 * (s * CH + cl)) = f32x4{through, dlog, core, 0.0f};
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        const int k2 = i * THREADS + tid, s = s0 + k2 / CH;
        if (k2 < BS * CH && s < in.t && ic < nch) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(wud + 4 * k2);
          const bool live = s < len;
          const float dw = live ? (iu[i] * v[0] + v[1]) * isig[i] : 0.0f;
          put<T>(p.du, s, b, c0 + ic, live ? iw[i] * v[0] + skip * idy[i] : 0.0f);
          put<T>(p.ddelta, s, b, c0 + ic, dw);
          if (in.z.p) put<T>(p.dz, s, b, c0 + ic, live ? idz[i] * (v[2] + skip * iu[i]) : 0.0f);
          dskip += idy[i] * iu[i];
          dbias += dw;
        }
      }
      for (int k2 = tid; k2 < BS * 2 * in.N; k2 += THREADS) {
        const int s = k2 / (2 * in.N), r = k2 % (2 * in.N), half = r / in.N, n = r % in.N;
        if (s0 + s < in.t) {
          float v = 0.0f;
#pragma unroll
          for (int w = 0; w < BACK_WAVES; ++w) v += red[(w * BS + s) * 2 * NP + half * NP + n];
          p.bc_parts[(((((int64_t)tile * in.t + s0 + s) * in.B + b) * in.G + group) * 2 + half) * in.N + n] = v;
        }
      }
      __syncthreads();
    }
  }
  if (mine && p.dh0) store_states(p.dh0 + ((int64_t)b * in.D + d) * in.N, q * NB, in.N, g);
  float* parts = p.a_parts + (int64_t)b * in.D * (in.N + 2);
  if (mine) store_states(parts + d * in.N, q * NB, in.N, dA);
  // dskip and ddelta_bias: the threads that share a channel, in their order
  red[tid] = dskip;
  red[THREADS + tid] = dbias;
  __syncthreads();
  if (tid < nch) {
    float s1 = 0.0f, s2 = 0.0f;
    for (int k = tid; k < THREADS; k += CH) {
      s1 += red[k];
      s2 += red[THREADS + k];
    }
    parts[(int64_t)in.D * in.N + c0 + tid] = s1;
    parts[(int64_t)in.D * (in.N + 1) + c0 + tid] = s2;
  }
}

// dB and dC from the workgroups' sums, in their order.
struct Shared {
  const float* parts;
  SeqOut dB, dC;
  int64_t t;
  int B, G, N, tiles;
};
template <typename T>
__global__ __launch_bounds__(256) void scan_shared_kernel(Shared p) {
  const int64_t row = (int64_t)p.G * 2 * p.N, all = p.t * p.B * row;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < all; k += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int i = 0; i < p.tiles; ++i) v += p.parts[i * all + k];
    const int r = (int)(k % row), group = r / (2 * p.N), half = r / p.N % 2, n = r % p.N;
    const int64_t sb = k / row;
    put<T>(half ? p.dC : p.dB, sb / p.B, sb % p.B, (int64_t)group * p.N + n, v);
  }
}

// [B][D N | D | D] -> dA, dskip, ddelta_bias
__global__ __launch_bounds__(256) void scan_params_kernel(const float* parts, int B, int64_t DN, int64_t D, float* dA, float* dskip, float* dbias) {
  const int64_t all = DN + 2 * D, k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= all) return;
  float v = 0.0f;
  for (int b = 0; b < B; ++b) v += parts[b * all + k];
  if (k < DN) dA[k] = v;
  else if (k < DN + D) { if (dskip) dskip[k - DN] = v; }
  else if (dbias) dbias[k - DN - D] = v;
}

// ---- single tokens -----------------------------------------------------------------------------------

struct Step {
  Scan in;
  SeqOut y;
  const float* state_in;
  float* state_out;
  const int32_t* index;
  int64_t slots;
};
// A lane per NB states: the pool's rows are read and written once.  Bound: HBM.
template <typename T, int NL>
__global__ __launch_bounds__(256) void scan_step_kernel(Step p) {
  const Scan& in = p.in;
  const int q = threadIdx.x % NL;
  for (int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / NL; item < (int64_t)in.B * in.D; item += (int64_t)gridDim.x * (256 / NL)) {
    const int b = (int)(item / in.D), d = (int)(item % in.D);
    const int64_t slot = p.index ? p.index[b] : b;
    if (slot < 0 || slot >= p.slots) {
      if (q == 0) put<T>(p.y, 0, b, d, 0.0f);
      continue;
    }
    const int64_t state = (slot * in.D + d) * in.N, gn = (int64_t)(d / (in.D / in.G)) * in.N;
    float h[NB], A[NB];
    load_states(p.state_in + state, q * NB, in.N, h);
    load_states(in.A + (int64_t)d * in.N, q * NB, in.N, A);
    const float u = at<T>(in.u, 0, b, d);
    float w = at<T>(in.delta, 0, b, d) + (in.bias ? in.bias[d] : 0.0f);
    if (in.softplus) w = softplus_of(w);
    float y = 0.0f;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const bool there = q * NB + n < in.N;
      const float vb = there ? at<T>(in.Bm, 0, b, gn + q * NB + n) : 0.0f, vc = there ? at<T>(in.Cm, 0, b, gn + q * NB + n) : 0.0f;
      h[n] = __builtin_amdgcn_exp2f(w * (A[n] * LOG2E)) * h[n] + w * u * vb;
      y += h[n] * vc;
    }
    y = lanes_sum<NL>(y);
    store_states(p.state_out + state, q * NB, in.N, h);
    if (q == 0) {
      if (in.skip) y += in.skip[d] * u;
      if (in.z.p) {
        const float z = at<T>(in.z, 0, b, d);
        y *= z * sigmoid(z);
      }
      put<T>(p.y, 0, b, d, y);
    }
  }
}

// ---- launches ----------------------------------------------------------------------------------------

template <typename F>
int with_lanes(int N, F&& f) {
  if (N <= 4) return f(std::integral_constant<int, 1>{});
  if (N <= 8) return f(std::integral_constant<int, 2>{});
  if (N <= 16) return f(std::integral_constant<int, 4>{});
  if (N <= 32) return f(std::integral_constant<int, 8>{});
  return f(std::integral_constant<int, 16>{});
}

int check(const mebptt_scan_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->t < 0 || d->B < 0 || d->B > 65535 || d->D < 1 || d->D > (1 << 22))
    return set_error(MEBPTT_EINVAL, "t >= 0, 0 <= B <= 65535 and 1 <= D <= 2^22 are needed");
  if (d->N < 1 || d->N > MAX_N) return set_error(MEBPTT_EINVAL, "N must be 1 .. %d", MAX_N);
  if (d->G < 1 || d->D % d->G) return set_error(MEBPTT_EINVAL, "G must divide D");
  if (!float_dtype(d->dtype)) return set_error(MEBPTT_EINVAL, "dtype must be MEBPTT_FP32 or MEBPTT_BF16");
  return MEBPTT_OK;
}
int check_stretch(const mebptt_scan_desc* d) {
  const int s = d->stretch;
  return s == 16 || s == 32 || s == 64 || s == 128 || s == 256 ? MEBPTT_OK : set_error(MEBPTT_EINVAL, "stretch must be 16, 32, 64, 128 or 256");
}
int check_inputs(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  if (!in) return set_error(MEBPTT_EINVAL, "inputs are NULL");
  if (!in->A) return set_error(MEBPTT_EINVAL, "A is NULL");
  if (d->t && d->B && (!in->u.data || !in->delta.data || !in->Bm.data || !in->Cm.data))
    return set_error(MEBPTT_EINVAL, "u, delta, B and C are required");
  return MEBPTT_OK;
}
int check_out(const mebptt_scan_desc* d, const mebptt_seq& s, int64_t channels, const char* what) {
  if (d->t && d->B && !s.data) return set_error(MEBPTT_EINVAL, "%s is NULL", what);
  if (!rows_apart(s, d->t, d->B, channels)) return set_error(MEBPTT_EINVAL, "rows of %s overlap", what);
  return MEBPTT_OK;
}
Scan scan_of(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  return {in_seq(in->u), in_seq(in->delta), in_seq(in->z), in_seq(in->Bm), in_seq(in->Cm), in->A, in->skip, in->delta_bias, in->lengths,
          d->t, d->B, d->D, d->N, d->G, d->softplus, 0};
}

int64_t back_tiles(const mebptt_scan_desc* d) {
  int64_t tiles = 0;
  with_lanes(d->N, [&](auto l) {
    tiles = ceil_div(d->D / d->G, BackwardShape<decltype(l)::value>::CH);
    return 0;
  });
  return tiles;
}
size_t bc_bytes(const mebptt_scan_desc* d) {
  return align_up((size_t)back_tiles(d) * d->t * d->B * d->G * 2 * d->N * sizeof(float));
}
size_t a_bytes(const mebptt_scan_desc* d) { return align_up((size_t)d->B * d->D * (d->N + 2) * sizeof(float)); }

template <typename T, int NL>
size_t back_lds(int stretch) {
  using S = BackwardShape<NL>;
  // (the last part also holds two floats per thread at the end)
  return ((size_t)BS * S::CH * 4 + BS * 2 * S::NP + std::max(BACK_WAVES * BS * 2 * S::NP, 2 * S::THREADS) +
          (size_t)stretch / BS * S::THREADS * NB) * sizeof(float);
}

}  // namespace

extern "C" {

size_t mebptt_scan_state_bytes(const mebptt_scan_desc* d) {
  if (check(d) != MEBPTT_OK || check_stretch(d) != MEBPTT_OK) return 0;
  return (size_t)ceil_div(d->t, d->stretch) * d->B * d->D * d->N * sizeof(float);
}

size_t mebptt_scan_workspace_bytes(const mebptt_scan_desc* d, int32_t backward) {
  if (check(d) != MEBPTT_OK) return 0;
  return backward ? bc_bytes(d) + a_bytes(d) : 0;
}

int mebptt_scan_forward(const mebptt_scan_desc* d, const mebptt_scan_inputs* in, mebptt_seq y, float* h_out, void* states,
                        size_t states_bytes, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d);
  if (rc || (rc = check_inputs(d, in)) || (rc = check_out(d, y, d->D, "y"))) return rc;
  if (states) {
    if ((rc = check_stretch(d))) return rc;
    if (states_bytes < mebptt_scan_state_bytes(d))
      return set_error(MEBPTT_EWORKSPACE, "states have %zu bytes, %zu needed", states_bytes, mebptt_scan_state_bytes(d));
    if (!aligned(states, ALIGN)) return set_error(MEBPTT_EWORKSPACE, "states must be 256-byte aligned");
  }
  if ((rc = check_workspace(workspace, workspace_bytes, mebptt_scan_workspace_bytes(d, 0)))) return rc;
  if (d->B == 0) return MEBPTT_OK;
  Forward p = {scan_of(d, in), out_seq(y), in->h0, h_out, (float*)states, d->stretch};
  return with_lanes(d->N, [&](auto l) {
    constexpr int NL = decltype(l)::value;
    p.in.tiles = (int)ceil_div(d->D / d->G, ForwardShape<NL>::CH);
    const dim3 grid((unsigned)(p.in.tiles * d->G), d->B);
    if (d->dtype == MEBPTT_FP32) scan_forward_kernel<float, NL><<<grid, WAVE, 0, (hipStream_t)stream>>>(p);
    else scan_forward_kernel<__bf16, NL><<<grid, WAVE, 0, (hipStream_t)stream>>>(p);
    return launched("mebptt_scan_forward");
  });
}

int mebptt_scan_backward(const mebptt_scan_desc* d, const mebptt_scan_inputs* in, mebptt_seq dy, const float* dh_out, const void* states,
                         size_t states_bytes, const mebptt_scan_grads* grads, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d);
  if (rc || (rc = check_stretch(d)) || (rc = check_inputs(d, in))) return rc;
  if (!grads || !grads->dA) return set_error(MEBPTT_EINVAL, "grads and dA are required");
  if (d->t && d->B && (!dy.data || !states)) return set_error(MEBPTT_EINVAL, "dy and states are required");
  if ((rc = check_out(d, grads->du, d->D, "du")) || (rc = check_out(d, grads->ddelta, d->D, "ddelta")) ||
      (rc = check_out(d, grads->dBm, (int64_t)d->G * d->N, "dB")) || (rc = check_out(d, grads->dCm, (int64_t)d->G * d->N, "dC")) ||
      (in->z.data && (rc = check_out(d, grads->dz, d->D, "dz"))))
    return rc;
  if (states_bytes < mebptt_scan_state_bytes(d))
    return set_error(MEBPTT_EWORKSPACE, "states have %zu bytes, %zu needed", states_bytes, mebptt_scan_state_bytes(d));
  if ((rc = check_workspace(workspace, workspace_bytes, mebptt_scan_workspace_bytes(d, 1)))) return rc;
  hipStream_t s = (hipStream_t)stream;
  float *bc = (float*)workspace, *ap = (float*)((char*)workspace + bc_bytes(d));
  if (d->B) {
    Backward p = {scan_of(d, in), in_seq(dy), out_seq(grads->du), out_seq(grads->ddelta), out_seq(grads->dz), in->h0,
                  (const float*)states, dh_out, grads->dh0, bc, ap, d->stretch};
    rc = with_lanes(d->N, [&](auto l) {
      constexpr int NL = decltype(l)::value;
      p.in.tiles = (int)back_tiles(d);
      const dim3 grid((unsigned)(p.in.tiles * d->G), d->B);
      auto go = [&](auto elem) {
        using T = decltype(elem);
        const size_t lds = back_lds<T, NL>(d->stretch);
        const hipError_t e = allow_dynamic_lds<scan_backward_kernel<T, NL>>(back_lds<T, NL>(256));
        if (e != hipSuccess) return set_error(MEBPTT_EHIP, "mebptt_scan_backward: %s", hipGetErrorString(e));
        scan_backward_kernel<T, NL><<<grid, BACK_WAVES * WAVE, lds, s>>>(p);
        return launched("mebptt_scan_backward");
      };
      return d->dtype == MEBPTT_FP32 ? go(float{}) : go(__bf16{});
    });
    if (rc) return rc;
    if (d->t) {
      const Shared q = {bc, out_seq(grads->dBm), out_seq(grads->dCm), d->t, d->B, d->G, d->N, p.in.tiles};
      const unsigned grid = (unsigned)std::min<int64_t>(ceil_div((int64_t)d->t * d->B * d->G * 2 * d->N, 256), 4096);
      if (d->dtype == MEBPTT_FP32) scan_shared_kernel<float><<<grid, 256, 0, s>>>(q);
      else scan_shared_kernel<__bf16><<<grid, 256, 0, s>>>(q);
      if ((rc = launched("mebptt_scan_backward"))) return rc;
    }
  }
  const int64_t DN = (int64_t)d->D * d->N;
  scan_params_kernel<<<(unsigned)ceil_div(DN + 2 * (int64_t)d->D, 256), 256, 0, s>>>(ap, d->B, DN, d->D, grads->dA, grads->dskip, grads->ddelta_bias);
  return launched("mebptt_scan_backward");
}

int mebptt_scan_step(const mebptt_scan_desc* d, const mebptt_scan_inputs* in, const float* state_in, int64_t slots, const int32_t* index,
                     mebptt_seq y, float* state_out, void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->t != 1) return set_error(MEBPTT_EINVAL, "a single token's t is 1");
  if ((rc = check_inputs(d, in)) || (rc = check_out(d, y, d->D, "y"))) return rc;
  if (d->B == 0) return MEBPTT_OK;
  if (!state_in || !state_out) return set_error(MEBPTT_EINVAL, "state_in and state_out are required");
  if (slots < 0 || (!index && slots < d->B)) return set_error(MEBPTT_EINVAL, "without an index every sequence needs its own slot");
  const Step p = {scan_of(d, in), out_seq(y), state_in, state_out, index, slots};
  return with_lanes(d->N, [&](auto l) {
    constexpr int NL = decltype(l)::value;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div((int64_t)d->B * d->D * NL, 256), 1 << 22);
    if (d->dtype == MEBPTT_FP32) scan_step_kernel<float, NL><<<grid, 256, 0, (hipStream_t)stream>>>(p);
    else scan_step_kernel<__bf16, NL><<<grid, 256, 0, (hipStream_t)stream>>>(p);
    return launched("mebptt_scan_step");
  });
}

}  // extern "C"
