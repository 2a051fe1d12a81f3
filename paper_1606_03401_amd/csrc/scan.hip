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
  int chunk, chunks;               // steps per chunk, a multiple of a block's
  float *starts, *sums;            // [chunks][B][D][N], the first left out; [chunks][B][D]
};

template <typename T>
__device__ inline float at(const Seq& q, int64_t s, int64_t b, int64_t c) { return (float)((const T*)q.p)[s * q.t + b * q.b + c]; }
template <typename T>
__device__ inline void put(const SeqOut& q, int64_t s, int64_t b, int64_t c, float v) { ((T*)q.p)[s * q.t + b * q.b + c] = (T)v; }

// The same with an address in two parts: uniform over the wave, and a lane's own, at most seven rows in bytes.
template <typename T>
__device__ inline unsigned lane_bytes(int64_t stride, int row, int c) { return (unsigned)((row * stride + c) * (int64_t)sizeof(T)); }
__device__ inline unsigned opaque(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}
template <typename T>
__device__ inline float elem(const T* base, unsigned bytes) { return (float)*reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes); }
template <typename T>
__device__ inline void set_elem(T* base, unsigned bytes, float v) { *reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes) = (T)v; }

__device__ inline int length_of(const int32_t* lengths, int b, int t) { return lengths ? min(max(lengths[b], 0), t) : t; }

// log(1 + e^x).  Small values keep their relative accuracy, steps of a thousandth being what such a model starts with: what 1 + e lost of e is
// added to the logarithm of the sum.
__device__ inline float softplus_of(float x) {
  const float e = __expf(-fabsf(x)), w = 1.0f + e;
  return fmaxf(x, 0.0f) + (__builtin_amdgcn_logf(w) * 0.6931471805599453f + (e - (w - 1.0f)));
}

// Sum over the NL lanes that share a channel, in every one of them.
template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
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
  static constexpr int SHARED = (TS * NP + WAVE - 1) / WAVE;          // values of B, and of C, per lane
};

// One wave's channels over a chunk of steps.  ENDS: only the state at the chunk's end (from a start of zeros, the first chunk's
// apart) and the sum of w, for the chunks after it.
//
// Addresses are a uniform part, advanced per block and per pair, and a lane's own 32 bits.
template <typename T, int NL, bool ENDS>
__global__ __launch_bounds__(WAVE) void scan_forward_kernel(Forward p) {
  using S = ForwardShape<NL>;
  constexpr int CH = S::CH, TS = S::TS, NP = S::NP, CPL = S::CPL;
  constexpr int WIDE = CH > WAVE ? CH / WAVE : 1;                      // pairs of one step per lane
  __shared__ __align__(16) float wu[TS][CH][2];                        // w and w u of a block
  __shared__ __align__(16) float sb[TS][NP], sc[TS][NP];
  __shared__ __align__(16) float sy[TS][CH];
  const Scan& in = p.in;
  const int lane = threadIdx.x, b = blockIdx.y, chunk = blockIdx.z;
  const int group = blockIdx.x / in.tiles, per = in.D / in.G;
  const int c0 = group * per + (blockIdx.x % in.tiles) * CH;           // first channel
  const int nch = min(CH, group * per + per - c0);
  const int len = length_of(in.lengths, b, in.t);
  const int begin = chunk * p.chunk, end = min(in.t, begin + p.chunk);
  const int q = lane % NL, cl = lane / NL * CPL;                       // this lane's states NB q .. and channels cl, cl + 1

  float h[CPL][NB], A2[CPL][NB], sum_w[CPL] = {};
  const float* start = chunk == 0 ? p.h0 : ENDS ? nullptr : p.starts + (int64_t)chunk * in.B * in.D * in.N;
#pragma unroll
  for (int j = 0; j < CPL; ++j) {
    const int64_t d = min(c0 + cl + j, in.D - 1);
    load_states(in.A + d * in.N, q * NB, in.N, A2[j]);
    if (start) load_states(start + ((int64_t)b * in.D + d) * in.N, q * NB, in.N, h[j]);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      A2[j][n] *= LOG2E;
      if (!start) h[j][n] = 0.0f;
    }
  }

  // the pairs of a lane: step i * ROWS + row (WIDE: i / WIDE), channel ch (+ 64 for every second one)
  constexpr int ROWS = CH < WAVE ? WAVE / CH : 1;
  const int row = CH < WAVE ? lane / CH : 0, ch = lane % CH;
  const bool pair = TS * CH >= WAVE || lane < TS * CH;
  auto step_of = [&](int i) { return i / WIDE * ROWS; };              // uniform part
  auto channel_of = [&](int i) { return i % WIDE * WAVE; };
  float bias[WIDE], skip[WIDE];
#pragma unroll
  for (int i = 0; i < WIDE; ++i) {
    const int d = min(c0 + ch + i * WAVE, in.D - 1);
    bias[i] = in.bias ? in.bias[d] : 0.0f;
    skip[i] = in.skip ? in.skip[d] : 0.0f;
  }
  const unsigned ou_ = lane_bytes<T>(in.u.t, row, ch), od_ = lane_bytes<T>(in.delta.t, row, ch), oz_ = lane_bytes<T>(in.z.t, row, ch),
                 oy_ = lane_bytes<T>(p.y.t, row, ch);
  const int srow = lane / NP, sn = lane % NP;
  const bool shared = TS * NP >= WAVE || lane < TS * NP;
  const int sk = min(sn, in.N - 1);
  const unsigned ob_ = lane_bytes<T>(in.Bm.t, srow, sk), oc_ = lane_bytes<T>(in.Cm.t, srow, sk);
  const int64_t gn = (int64_t)group * in.N;
  const T* const pu = (const T*)in.u.p + b * in.u.b + c0;
  const T* const pd = (const T*)in.delta.p + b * in.delta.b + c0;
  const T* const pz = (const T*)in.z.p + b * in.z.b + c0;
  const T* const pb = (const T*)in.Bm.p + b * in.Bm.b + gn;
  const T* const pc = (const T*)in.Cm.p + b * in.Cm.b + gn;
  T* const py = (T*)p.y.p + b * p.y.b + c0;

  // The next block's inputs, fetched while a block is worked on.  A whole block (all its steps within the sequence, all its channels
  // there) needs no masks; which it is, is the same for the whole wave.
  float ru[S::ITEMS], rd[S::ITEMS], rz[S::ITEMS], rb[S::SHARED], rc[S::SHARED];
  auto whole = [&](int s0) { return TS * CH >= WAVE && TS * NP >= WAVE && s0 + TS <= min(len, end) && nch == CH; };
  auto fetch = [&](int s0) {
    // (opaque, or the sums of the parts are formed ahead in registers)
    const unsigned ou = opaque(ou_), od = opaque(od_), oz = opaque(oz_), ob = opaque(ob_), oc = opaque(oc_);
    const T *au = pu + s0 * in.u.t, *ad = pd + s0 * in.delta.t, *az = pz + s0 * in.z.t, *ab = pb + s0 * in.Bm.t, *ac = pc + s0 * in.Cm.t;
    const int64_t iu = ROWS * in.u.t, id = ROWS * in.delta.t, iz = ROWS * in.z.t, ib = WAVE / NP * in.Bm.t, ic = WAVE / NP * in.Cm.t;
    if (whole(s0)) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        ru[i] = elem(au + channel_of(i), ou);
        rd[i] = elem(ad + channel_of(i), od);
        if (i % WIDE == WIDE - 1) au += iu, ad += id;
      }
      if (!ENDS && in.z.p) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          rz[i] = elem(az + channel_of(i), oz);
          if (i % WIDE == WIDE - 1) az += iz;
        }
      }
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        rb[i] = elem(ab, ob);
        ab += ib;
        if (!ENDS) rc[i] = elem(ac, oc);
        ac += ic;
      }
    } else {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        const int c = channel_of(i);
        ru[i] = rd[i] = rz[i] = 0.0f;
        if (pair && s0 + step_of(i) + row < len && ch + c < nch) {
          ru[i] = elem(au + c, ou);
          rd[i] = elem(ad + c, od);
          if (!ENDS && in.z.p) rz[i] = elem(az + c, oz);
        }
        if (i % WIDE == WIDE - 1) au += iu, ad += id, az += iz;
      }
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        rb[i] = rc[i] = 0.0f;
        if (shared && s0 + i * (WAVE / NP) + srow < len) {
          rb[i] = elem(ab, ob);
          if (!ENDS) rc[i] = elem(ac, oc);
        }
        ab += ib;
        ac += ic;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < S::ITEMS; ++i) rz[i] = 0.0f;
  const int stop = ENDS ? min(end, len) : end;                         // (beyond its length a sequence's state stays as it is)
  if (begin < stop) fetch(begin);
  for (int s0 = begin; s0 < stop; s0 += TS) {
    const bool all = whole(s0);
    float cu[S::ITEMS], cz[S::ITEMS];
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      cu[i] = ru[i];
      cz[i] = rz[i];
      rd[i] += bias[i % WIDE];
    }
    if (in.softplus) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) rd[i] = softplus_of(rd[i]);
    }
    if (!all) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i)      // a step beyond the sequence
        if (!(s0 + step_of(i) + row < len && ch + channel_of(i) < nch)) rd[i] = 0.0f;
    }
    if (pair) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) *reinterpret_cast<float2*>(&wu[step_of(i) + row][ch + channel_of(i)][0]) = float2{rd[i], rd[i] * cu[i]};
    }
    if (shared) {
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        sb[i * (WAVE / NP) + srow][sn] = sn < in.N ? rb[i] : 0.0f;
        if (!ENDS) sc[i * (WAVE / NP) + srow][sn] = sn < in.N ? rc[i] : 0.0f;
      }
    }
    __syncthreads();
    if (s0 + TS < stop) fetch(s0 + TS);
    if (!ENDS && p.states && s0 % p.stretch == 0) {
#pragma unroll
      for (int j = 0; j < CPL; ++j)
        if (cl + j < nch)
          store_states(p.states + (((int64_t)(s0 / p.stretch) * in.B + b) * in.D + c0 + cl + j) * in.N, q * NB, in.N, h[j]);
    }
#pragma unroll
    for (int s = 0; s < TS; ++s) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(&wu[s][cl][0]);
      const f32x4 vb = *reinterpret_cast<const f32x4*>(&sb[s][q * NB]);
      f32x4 vc = {};
      if constexpr (!ENDS) vc = *reinterpret_cast<const f32x4*>(&sc[s][q * NB]);
      float y[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const float a = __builtin_amdgcn_exp2f(w[2 * j] * A2[j][n]);
          h[j][n] = a * h[j][n] + w[2 * j + 1] * vb[n];
          if constexpr (!ENDS) y[j] = n ? y[j] + h[j][n] * vc[n] : h[j][n] * vc[n];
        }
        if constexpr (ENDS) sum_w[j] += w[2 * j];
        else y[j] = lanes_sum<NL>(y[j]);
      }
      // every lane of a channel writes the same value to the same place
      if constexpr (!ENDS) *reinterpret_cast<float2*>(&sy[s][cl]) = float2{y[0], y[1]};
    }
    __syncthreads();
    if constexpr (!ENDS) {
      float y[S::ITEMS];
      if (pair) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) y[i] = sy[step_of(i) + row][ch + channel_of(i)] + skip[i % WIDE] * cu[i];
      }
      if (in.z.p) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) y[i] *= cz[i] * sigmoid(cz[i]);
      }
      T* ay = py + s0 * p.y.t;
      const unsigned oy = opaque(oy_);
      const int64_t iy = ROWS * p.y.t;
      if (all) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          set_elem(ay + channel_of(i), oy, y[i]);
          if (i % WIDE == WIDE - 1) ay += iy;
        }
      } else {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          const int s = s0 + step_of(i) + row;
          if (pair && s < end && ch + channel_of(i) < nch) set_elem(ay + channel_of(i), oy, s < len ? y[i] : 0.0f);
          if (i % WIDE == WIDE - 1) ay += iy;
        }
      }
    }
  }
  float* last = ENDS ? p.starts + (int64_t)(chunk + 1) * in.B * in.D * in.N : chunk + 1 == p.chunks ? p.h_out : nullptr;
#pragma unroll
  for (int j = 0; j < CPL; ++j) {
    if (cl + j >= nch) continue;
    const int64_t d = (int64_t)b * in.D + c0 + cl + j;
    if (last) store_states(last + d * in.N, q * NB, in.N, h[j]);
    if (ENDS && q == 0) p.sums[(int64_t)chunk * in.B * in.D + d] = sum_w[j];
  }
}

// starts[c] holds the state that chunk c - 1 reached from zeros; adds what it started from, decayed by exp(A sum w).
__global__ __launch_bounds__(256) void scan_join_kernel(float* starts, const float* sums, const float* A, int64_t BD, int D, int N, int chunks) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= BD * N) return;
  const int64_t bd = k / N;
  const float a2 = A[(bd % D) * N + k % N] * LOG2E;
  float h = starts[BD * N + k];
#pragma unroll 8
  for (int c = 2; c < chunks; ++c) {
    h = starts[c * BD * N + k] + __builtin_amdgcn_exp2f(a2 * sums[(c - 1) * BD + bd]) * h;
    starts[c * BD * N + k] = h;
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
// A lane's part of an address is 32 bits, of up to seven rows of four bytes.
bool stride_fits(const mebptt_seq& s) { return s.stride_t >= 0 && s.stride_t <= (1 << 26); }
int check_inputs(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  if (!in) return set_error(MEBPTT_EINVAL, "inputs are NULL");
  if (!in->A) return set_error(MEBPTT_EINVAL, "A is NULL");
  if (d->t && d->B && (!in->u.data || !in->delta.data || !in->Bm.data || !in->Cm.data))
    return set_error(MEBPTT_EINVAL, "u, delta, B and C are required");
  if (d->t > 1)
    for (const mebptt_seq* q : {&in->u, &in->delta, &in->z, &in->Bm, &in->Cm})
      if (q->data && !stride_fits(*q)) return set_error(MEBPTT_EINVAL, "stride_t must be 0 .. 2^26");
  return MEBPTT_OK;
}
int check_out(const mebptt_scan_desc* d, const mebptt_seq& s, int64_t channels, const char* what) {
  if (d->t && d->B && !s.data) return set_error(MEBPTT_EINVAL, "%s is NULL", what);
  if (d->t > 1 && !stride_fits(s)) return set_error(MEBPTT_EINVAL, "stride_t must be 0 .. 2^26");
  if (!rows_apart(s, d->t, d->B, channels)) return set_error(MEBPTT_EINVAL, "rows of %s overlap", what);
  return MEBPTT_OK;
}
Scan scan_of(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  return {in_seq(in->u), in_seq(in->delta), in_seq(in->z), in_seq(in->Bm), in_seq(in->Cm), in->A, in->skip, in->delta_bias, in->lengths,
          d->t, d->B, d->D, d->N, d->G, d->softplus, 0};
}

// How many chunks the time axis is cut into: enough workgroups for two waves on each of the 1024 SIMDs, in chunks of at least MIN_CHUNK steps.  The
// chunks' ends are computed first, which is most of the work once more, so nothing is cut that fills the chip by itself.
constexpr int MIN_CHUNK = 64;
int64_t forward_tiles(const mebptt_scan_desc* d) {
  int64_t tiles = 0;
  with_lanes(d->N, [&](auto l) {
    tiles = ceil_div(d->D / d->G, ForwardShape<decltype(l)::value>::CH);
    return 0;
  });
  return tiles;
}
struct Cut { int chunk, chunks; };
Cut cut_of(const mebptt_scan_desc* d, int64_t workgroups, int unit) {
  const int64_t t = std::max(d->t, 1), want = ceil_div(2048, std::max<int64_t>(1, workgroups));
  int64_t chunk = std::max<int64_t>(MIN_CHUNK, ceil_div(t, want));
  chunk = ceil_div(chunk, unit) * unit;
  const int64_t chunks = ceil_div(t, chunk);
  return workgroups >= 1024 || chunks < 2 ? Cut{(int)(ceil_div(t, unit) * unit), 1} : Cut{(int)chunk, (int)chunks};
}
Cut forward_cut(const mebptt_scan_desc* d) { return cut_of(d, forward_tiles(d) * d->G * d->B, 16); }
size_t starts_bytes(const mebptt_scan_desc* d, int chunks) { return chunks < 2 ? 0 : align_up((size_t)chunks * d->B * d->D * d->N * sizeof(float)); }
size_t sums_bytes(const mebptt_scan_desc* d, int chunks) { return chunks < 2 ? 0 : align_up((size_t)chunks * d->B * d->D * sizeof(float)); }

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
  if (backward) return bc_bytes(d) + a_bytes(d);
  const int chunks = forward_cut(d).chunks;
  return starts_bytes(d, chunks) + sums_bytes(d, chunks);
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
  const Cut cut = forward_cut(d);
  Forward p = {scan_of(d, in), out_seq(y), in->h0, h_out, (float*)states, d->stretch, cut.chunk, cut.chunks,
               (float*)workspace, (float*)((char*)workspace + starts_bytes(d, cut.chunks))};
  hipStream_t s = (hipStream_t)stream;
  return with_lanes(d->N, [&](auto l) {
    constexpr int NL = decltype(l)::value;
    p.in.tiles = (int)ceil_div(d->D / d->G, ForwardShape<NL>::CH);
    const unsigned wide = (unsigned)(p.in.tiles * d->G);
    auto go = [&](auto elem) {
      using T = decltype(elem);
      if (cut.chunks > 1) {
        scan_forward_kernel<T, NL, true><<<dim3(wide, d->B, cut.chunks - 1), WAVE, 0, s>>>(p);
        const int64_t BD = (int64_t)d->B * d->D;
        if (cut.chunks > 2)
          scan_join_kernel<<<(unsigned)ceil_div(BD * d->N, 256), 256, 0, s>>>(p.starts, p.sums, in->A, BD, d->D, d->N, cut.chunks);
      }
      scan_forward_kernel<T, NL, false><<<dim3(wide, d->B, cut.chunks), WAVE, 0, s>>>(p);
      return launched("mebptt_scan_forward");
    };
    return d->dtype == MEBPTT_FP32 ? go(float{}) : go(__bf16{});
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
