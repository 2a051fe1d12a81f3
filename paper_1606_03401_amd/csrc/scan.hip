// Selective scan: D channels of N states each, a recurrence that is diagonal and depends on its input,
//     w = delta + delta_bias (through softplus);  h_s = exp(w_s A) h_{s-1} + w_s u_s B_s;  y_s = (C_s . h_s + skip u_s) silu(z_s)
// forward, backward, and for single tokens.
//
// A channel's states are spread over NL neighbouring lanes, four of them in each lane's registers over all steps (eight forward beyond
// N = 32).  Steps come in blocks: a block's w, w u, B and C are put into LDS once, as floats, while the next block's inputs are already on their
// way, so that softplus and the gate are computed once per (step, channel) and not in each of the NL lanes.
//
// Bound: the vector unit.  Per step, channel and state the forward pass needs an exponential and four products or multiply-adds, 24 cycles
// of a SIMD for 64 of them, the backward pass 60; what staging, sums over lanes and addresses add to that makes 36 and 133.  Measured, bf16 with
// a gate, N = 16: 1000 x 32 x 1024, forward 175 us and backward 640 (the operations above alone 80 and 200, the bytes 35 and 73), two
// thirds of the cycles with a vector instruction; 10000 x 1 x 2048, forward, 150 us in three launches (50; 33).
#include "dynamic_lds.h"
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int NB = 4;              // states per lane, single tokens
constexpr int MAX_N = 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

constexpr int64_t MAX_STRIDE = 1 << 25;   // over steps, in elements: 15 rows of 4 bytes are below 2^32
struct Seq { const void* p; int64_t b; int t; };
struct SeqOut { void* p; int64_t b; int t; };
// (a stride that is never used, of a sequence of one step, may be anything)
inline Seq in_seq(const mebptt_seq& s) { return {s.data, s.stride_b, (int)std::min(std::max<int64_t>(s.stride_t, 0), MAX_STRIDE)}; }
inline SeqOut out_seq(const mebptt_seq& s) { return {s.data, s.stride_b, (int)std::min(std::max<int64_t>(s.stride_t, 0), MAX_STRIDE)}; }

struct Scan {
  Seq u, delta, z, Bm, Cm;
  const float *A, *skip, *bias;
  const int32_t* lengths;
  int t, B, D, N, G, softplus;
  int tiles;                       // workgroups per group of channels
};
template <typename T>
__device__ inline void put(const SeqOut& q, int64_t s, int64_t b, int64_t c, float v) { ((T*)q.p)[s * q.t + b * q.b + c] = (T)v; }

// The same with an address in two parts: uniform over the wave, and a lane's own, of at most 15 rows, in bytes.
template <typename T>
__device__ inline unsigned lane_bytes(int stride, int row, int c) { return (unsigned)(row * stride + c) * (unsigned)sizeof(T); }
template <typename T>
__device__ inline const T* row_of(const Seq& q, int s, int b, int64_t c) { return (const T*)q.p + (int64_t)s * q.t + b * q.b + c; }
template <typename T>
__device__ inline T* row_of(const SeqOut& q, int s, int b, int64_t c) { return (T*)q.p + (int64_t)s * q.t + b * q.b + c; }
__device__ inline unsigned opaque(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}
template <typename T>
__device__ inline T raw(const T* base, unsigned bytes) { return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes); }
template <typename T>
__device__ inline void set_elem(T* base, unsigned bytes, float v) { *reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes) = (T)v; }

__device__ inline int length_of(const int32_t* lengths, int b, int t) { return lengths ? min(max(lengths[b], 0), t) : t; }

// A log2 e, finite: where nothing happens (w = 0: beyond a sequence's end, in lanes without a channel) exp(w A) is 1 for an infinite A as well.
__device__ inline float log2_decay(float A) {
  constexpr float MOST = 3.402823466e38f;
  const float v = A * LOG2E;
  return v < -MOST ? -MOST : v > MOST ? MOST : v;      // (a NaN stays one)
}

// log(1 + e^x).  Small values are as accurate as e^x is, (4 + 1.5 |x|) 2^-24 of themselves, steps of a thousandth being what such a model starts with:
// what 1 + e lost of e is added to the logarithm of the sum.
__device__ inline float softplus_of(float x) {
  const float e = __expf(-fabsf(x)), w = 1.0f + e;
  return fmaxf(x, 0.0f) + (__builtin_amdgcn_logf(w) * LN2 + (e - (w - 1.0f)));
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

// K consecutive states of a channel's N.
template <int K>
__device__ inline void load_states(const float* p, int n0, int N, float (&v)[K]) {
#pragma unroll
  for (int n = 0; n < K; ++n) v[n] = n0 + n < N ? p[n0 + n] : 0.0f;
}
template <int K>
__device__ inline void store_states(float* p, int n0, int N, const float (&v)[K]) {
#pragma unroll
  for (int n = 0; n < K; ++n)
    if (n0 + n < N) p[n0 + n] = v[n];
}

// ---- forward ---------------------------------------------------------------------------------------

struct Forward {
  Scan in;
  SeqOut y;
  const float* h0;
  float *h_out, *states;
  int stretch;
  int chunk, chunks;               // steps per chunk, a multiple of a block's
  float *starts, *sums;            // [chunks][B][D][N]: what the chunk before reached (ENDS: by itself), the first one's h0; [chunks][B][D]: sum of w
};

constexpr int FORWARD_WAVES = 4;   // waves of neighbouring channels per workgroup: they share cache lines, and nothing else

template <int NL_, int NB_>
struct ForwardShape {
  static constexpr int NL = NL_, NB = NB_;                            // lanes per channel, states per lane
  static constexpr int CH = WAVE / NL;                                // channels per wave
  static constexpr int NP = NB * NL;                                  // N rounded up
  static constexpr int TS = NL <= 8 ? 16 : 8;                         // steps per block
  static constexpr int ITEMS = (TS * CH + WAVE - 1) / WAVE;           // (step, channel) pairs per lane
  static constexpr int SHARED = (TS * NP + WAVE - 1) / WAVE;          // values of B, and of C, per lane
};

// What the lanes of one wave hand each other through LDS is in order by itself; the compiler has to keep it so.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wave's channels over a chunk of steps.  ENDS: only the state at the chunk's end (from zeros, the first chunk's from h0) and the
// sum of w, for the chunks after it.  Addresses are a uniform part, advanced per block and per pair, and a lane's own 32 bits.
template <typename T, typename S, bool ENDS>
__global__ __launch_bounds__(FORWARD_WAVES* WAVE) void scan_forward_kernel(Forward p) {
  constexpr int CH = S::CH, TS = S::TS, NP = S::NP, NL = S::NL, NB = S::NB;
  struct Lds { float wu[TS][CH][2], sb[TS][NP], sc[ENDS ? 1 : TS][NP], sy[ENDS ? 1 : TS][CH]; };   // w and w u of a block, B, C, y
  __shared__ __align__(16) Lds lds[FORWARD_WAVES];
  const Scan& in = p.in;
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), b = blockIdx.y, chunk = blockIdx.z;
  auto& [wu, sb, sc, sy] = lds[wave];
  const int group = blockIdx.x / in.tiles, per = in.D / in.G;
  const int c0 = group * per + (blockIdx.x % in.tiles * FORWARD_WAVES + wave) * CH;   // first channel
  const int nch = min(CH, group * per + per - c0);
  if (nch <= 0) return;                                                // (waves of a workgroup never wait for each other)
  const int len = length_of(in.lengths, b, in.t);
  const int begin = chunk * p.chunk, end = min(in.t, begin + p.chunk);
  const int q = lane % NL, cl = lane / NL;                             // this lane's states NB q .. and channel
  const int64_t d = min(c0 + cl, in.D - 1), bd = (int64_t)b * in.D + d, all_states = (int64_t)in.B * in.D * in.N;

  float h[NB], A2[NB], sum_w = 0.0f;
  load_states(in.A + d * in.N, q * NB, in.N, A2);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    A2[n] = log2_decay(A2[n]);
    h[n] = 0.0f;
  }
  // h0 of launches in chunks: from its copy, as another workgroup may be writing h_out over it
  const float* start = chunk == 0 ? (ENDS || p.chunks == 1 || !p.h0 ? p.h0 : p.starts) : ENDS ? nullptr : p.starts + chunk * all_states;
  if (start) load_states(start + bd * in.N, q * NB, in.N, h);
  if (ENDS && chunk == 0 && p.h0 && cl < nch) store_states(p.starts + bd * in.N, q * NB, in.N, h);

  // the pairs of a lane: step i * ROWS + row, channel ch; its values of B and C: step i * SROWS + srow, state sn
  constexpr int ROWS = WAVE / CH, SROWS = WAVE / NP;
  const int row = lane / CH, ch = lane % CH, srow = lane / NP, sn = lane % NP;
  const bool pair = TS * CH >= WAVE || lane < TS * CH, shared = TS * NP >= WAVE || lane < TS * NP;
  const float bias = in.bias ? in.bias[min(c0 + ch, in.D - 1)] : 0.0f, skip = in.skip ? in.skip[min(c0 + ch, in.D - 1)] : 0.0f;
  const int64_t gn = (int64_t)group * in.N;

  // The next block's inputs, fetched while a block is worked on, and kept as they came: what turns them into floats would wait for them.  A whole block (all its steps within the sequence, all its channels
  // there) needs no masks; which it is, is the same for the whole wave.
  T ru[S::ITEMS], rd[S::ITEMS], rz[S::ITEMS], rb[S::SHARED], rc[S::SHARED];
  auto whole = [&](int s0) { return TS * CH >= WAVE && TS * NP >= WAVE && s0 + TS <= min(len, end) && nch == CH; };
  auto fetch = [&](int s0) {
    // (opaque: the sums of an address's parts are not to be formed ahead, in registers)
    const int sk = min(sn, in.N - 1);
    const unsigned ou = opaque(lane_bytes<T>(in.u.t, row, ch)), od = opaque(lane_bytes<T>(in.delta.t, row, ch)),
                   oz = opaque(lane_bytes<T>(in.z.t, row, ch)), ob = opaque(lane_bytes<T>(in.Bm.t, srow, sk)),
                   oc = opaque(lane_bytes<T>(in.Cm.t, srow, sk));
    const T *au = row_of<T>(in.u, s0, b, c0), *ad = row_of<T>(in.delta, s0, b, c0), *az = row_of<T>(in.z, s0, b, c0),
            *ab = row_of<T>(in.Bm, s0, b, gn), *ac = row_of<T>(in.Cm, s0, b, gn);
    const int iu = ROWS * in.u.t, id = ROWS * in.delta.t, iz = ROWS * in.z.t, ib = SROWS * in.Bm.t, ic = SROWS * in.Cm.t;
    if (whole(s0)) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        ru[i] = raw(au, ou);
        rd[i] = raw(ad, od);
        au += iu;
        ad += id;
      }
      if (!ENDS && in.z.p) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          rz[i] = raw(az, oz);
          az += iz;
        }
      }
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        rb[i] = raw(ab, ob);
        ab += ib;
        if (!ENDS) rc[i] = raw(ac, oc);
        ac += ic;
      }
    } else {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        ru[i] = rd[i] = rz[i] = (T)0.0f;
        if (pair && s0 + i * ROWS + row < len && ch < nch) {
          ru[i] = raw(au, ou);
          rd[i] = raw(ad, od);
          if (!ENDS && in.z.p) rz[i] = raw(az, oz);
        }
        au += iu;
        ad += id;
        az += iz;
      }
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        rb[i] = rc[i] = (T)0.0f;
        if (shared && s0 + i * SROWS + srow < len) {
          rb[i] = raw(ab, ob);
          if (!ENDS) rc[i] = raw(ac, oc);
        }
        ab += ib;
        ac += ic;
      }
    }
  };
#pragma unroll
  for (int i = 0; i < S::ITEMS; ++i) rz[i] = (T)0.0f;
  const int stop = min(end, len);                                      // beyond its length a sequence's state stays as it is
  if (begin < stop) fetch(begin);
  int s0 = begin;
  for (; s0 < stop; s0 += TS) {
    const bool all = whole(s0);
    float cu[S::ITEMS], cz[S::ITEMS], cw[S::ITEMS];
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      cu[i] = (float)ru[i];
      cz[i] = (float)rz[i];
      cw[i] = (float)rd[i] + bias;
    }
    if (in.softplus) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) cw[i] = softplus_of(cw[i]);
    }
    if (!all) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i)      // a step beyond the sequence
        if (!(s0 + i * ROWS + row < len && ch < nch)) cw[i] = 0.0f;
    }
    if (pair) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) *reinterpret_cast<f32x2*>(&wu[i * ROWS + row][ch][0]) = f32x2{cw[i], cw[i] * cu[i]};
    }
    if (shared) {
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) {
        sb[i * SROWS + srow][sn] = sn < in.N ? (float)rb[i] : 0.0f;
        if (!ENDS) sc[i * SROWS + srow][sn] = sn < in.N ? (float)rc[i] : 0.0f;
      }
    }
    wave_sync();
    if (s0 + TS < stop) fetch(s0 + TS);
    if (!ENDS && p.states && s0 % p.stretch == 0) {
      if (cl < nch) store_states(p.states + (int64_t)(s0 / p.stretch) * all_states + bd * in.N, q * NB, in.N, h);
    }
    // a step's operands are read from LDS while the one before is worked on
    f32x2 next_w = *reinterpret_cast<const f32x2*>(&wu[0][cl][0]);
    float next_b[NB], next_c[NB];
    load<NB>(&sb[0][q * NB], next_b);
    if constexpr (!ENDS) load<NB>(&sc[0][q * NB], next_c);
#pragma unroll
    for (int s = 0; s < TS; ++s) {
      const f32x2 w = next_w;
      float vb[NB], vc[NB], y = 0.0f;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        vb[n] = next_b[n];
        if constexpr (!ENDS) vc[n] = next_c[n];
      }
      if (s + 1 < TS) {
        next_w = *reinterpret_cast<const f32x2*>(&wu[s + 1][cl][0]);
        load<NB>(&sb[s + 1][q * NB], next_b);
        if constexpr (!ENDS) load<NB>(&sc[s + 1][q * NB], next_c);
      }
      __builtin_amdgcn_sched_barrier(0);   // (they would be read where they are used)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float a = __builtin_amdgcn_exp2f(w[0] * A2[n]);
        h[n] = a * h[n] + w[1] * vb[n];
        if constexpr (!ENDS) y = n ? y + h[n] * vc[n] : h[n] * vc[n];
      }
      // (every lane of a channel writes the same value to the same place)
      if constexpr (ENDS) sum_w += w[0];
      else sy[s][cl] = lanes_sum<NL>(y);
    }
    wave_sync();
    if constexpr (!ENDS) {
      float y[S::ITEMS];
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) y[i] = pair ? sy[i * ROWS + row][ch] + skip * cu[i] : 0.0f;
      if (in.z.p) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) y[i] *= cz[i] * sigmoid(cz[i]);
      }
      T* ay = row_of<T>(p.y, s0, b, c0);
      const unsigned oy = opaque(lane_bytes<T>(p.y.t, row, ch));
      const int iy = ROWS * p.y.t;
      if (all) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          set_elem(ay, oy, y[i]);
          ay += iy;
        }
      } else {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          const int s = s0 + i * ROWS + row;
          if (pair && s < end && ch < nch) set_elem(ay, oy, s < len ? y[i] : 0.0f);
          ay += iy;
        }
      }
      wave_sync();
    }
  }
  if constexpr (!ENDS) {
    for (; s0 < end; s0 += TS) {
      if (p.states && s0 % p.stretch == 0 && cl < nch) store_states(p.states + (int64_t)(s0 / p.stretch) * all_states + bd * in.N, q * NB, in.N, h);
      T* ay = row_of<T>(p.y, s0, b, c0);
      const unsigned oy = opaque(lane_bytes<T>(p.y.t, row, ch));
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        if (pair && s0 + i * ROWS + row < end && ch < nch) set_elem(ay, oy, 0.0f);
        ay += ROWS * p.y.t;
      }
    }
  }
  if (cl >= nch) return;
  float* last = ENDS ? p.starts + (chunk + 1) * all_states : chunk + 1 == p.chunks ? p.h_out : nullptr;
  if (last) store_states(last + bd * in.N, q * NB, in.N, h);
  if (ENDS && q == 0) p.sums[(int64_t)chunk * in.B * in.D + bd] = sum_w;
}

// What the chunks reached by themselves, one after the other: slot k of `starts`, k = first, first + step, .., `count` of them, adds the slot
// before it (`before` for the first one, NULL: nothing) times exp(A sum w) of the chunk in between, which is k + shift.
struct Join {
  float* starts;
  const float *sums, *A, *before;
  int64_t BD;
  int D, N, first, step, count, shift;
};
__global__ __launch_bounds__(256) void scan_join_kernel(Join p) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = p.BD * p.N;
  if (i >= all) return;
  const int64_t bd = i / p.N;
  const float a2 = log2_decay(p.A[(bd % p.D) * p.N + i % p.N]);
  float h = p.before ? p.before[i] : 0.0f;
  constexpr int U = 16;                                // slots read at once
  for (int c = 0; c < p.count; c += U) {
    float e[U], w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = p.first + min(c + u, p.count - 1) * p.step;
      e[u] = p.starts[k * all + i];
      w[u] = p.sums[(k + p.shift) * p.BD + bd];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c + u < p.count) {
        h = e[u] + __builtin_amdgcn_exp2f(a2 * w[u]) * h;
        p.starts[(p.first + (c + u) * p.step) * all + i] = h;
      }
  }
}

// ---- backward --------------------------------------------------------------------------------------

struct Backward {
  Scan in;
  Seq dy;
  SeqOut du, ddelta, dz;
  const float *states, *dh_out;
  float* dh0;
  float *bc_parts;                 // [tiles][B][G][t][2][N]: sums of dB and dC over a workgroup's channels
  float *a_parts;                  // [chunks][B][D N | D | D]: dA, dskip, ddelta_bias of a chunk of a sequence
  int stretch;
  int chunk, chunks;               // steps per chunk, a multiple of the stretch
  float *starts, *sums;            // [chunks][B][D][N]: dL/dh at a chunk's start from its own steps; [chunks][B][D]: sum of w
};

// Steps per block: exp(w A) and exp(w A) h of a block stay in a lane's registers.  With 8, and so three waves per SIMD instead of two,
// 1353 instead of 1279 us at 1000 x 64 x 1024: what a block costs apart from its steps comes up twice as often.
constexpr int BS = 16;

template <int NL_, int NB_>
struct BackwardShape {
  static constexpr int NL = NL_, NB = NB_;
  static constexpr int BACK_WAVES = 4;                                // (what fits into LDS with stretches of 256)
  static constexpr int CW = WAVE / NL;                                // channels per wave
  static constexpr int CH = CW * BACK_WAVES;                          // channels per workgroup
  static constexpr int NP = NB * NL;
  static constexpr int THREADS = BACK_WAVES * WAVE;
  static constexpr int ITEMS = BS * CH / THREADS;                     // (step, channel) pairs per thread
  static constexpr int SHARED = (BS * NP + THREADS - 1) / THREADS;    // values of B, and of C, per thread
  static constexpr int WAVES_PER_SIMD = 2;
};

// Sums of a lane's 2 NB values (of dB, then of dC) over the channels of its wave, that is over the lanes with the same lane % NL, into
// red[2][NP].  Halves of the wave, then neighbouring rows of sixteen lanes, exchange one half of their values each, so that every addition
// adds two values that are wanted; what is left is rotated within the rows.
template <typename S>
__device__ inline void channels_sum(const float (&v)[2 * S::NB], int lane, float* red) {
  constexpr int NL = S::NL, NB = S::NB;
  float w[NB], x[NB / 2];
#pragma unroll
  for (int n = 0; n < NB; ++n) {         // lanes 0 .. 31: dB, 32 .. 63: dC
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[n]), __float_as_uint(v[NB + n]), false, false);
    w[n] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int n = 0; n < NB / 2; ++n) {     // even rows: even states, odd rows: odd ones
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[2 * n]), __float_as_uint(w[2 * n + 1]), false, false);
    x[n] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    if constexpr (NL <= 8) x[n] = dpp_add<0x128>(x[n]);
    if constexpr (NL <= 4) x[n] = dpp_add<0x124>(x[n]);
    if constexpr (NL <= 2) x[n] = dpp_add<0x122>(x[n]);
  }
  // (every lane that has a sum writes it)
#pragma unroll
  for (int n = 0; n < NB / 2; ++n) red[(lane / 32) * S::NP + lane % NL * NB + 2 * n + lane / 16 % 2] = x[n];
}

// A workgroup's channels over a chunk of steps, from its end to its start, stretch by stretch: the states at the starts of the stretch's blocks
// are recomputed from the one kept at its start and put into LDS; then block by block, the last one first, the block's steps
// are run forward into registers and back.
template <typename T, typename S, bool GATE>
__global__ __launch_bounds__(S::THREADS, S::WAVES_PER_SIMD) void scan_backward_kernel(Backward p) {
  constexpr int CH = S::CH, NP = S::NP, THREADS = S::THREADS, NL = S::NL, NB = S::NB, BACK_WAVES = S::BACK_WAVES;
  extern __shared__ __align__(16) float lds[];
  const int tid = threadIdx.x;
  // what a block stages, twice: the next one's is written while slower waves still read
  constexpr int STAGED = BS * (CH * 4 + 2 * NP);
  float* red = lds + 2 * STAGED;                      // [BACK_WAVES][BS][2][NP]
  // [stretch / BS - 2][THREADS][NB]: states at the starts of a stretch's blocks from its second one to its last but one
  float* const kept = red + BACK_WAVES * BS * 2 * NP + tid * NB;
  const Scan& in = p.in;
  const int lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), b = blockIdx.y, chunk = blockIdx.z;
  const int group = blockIdx.x / in.tiles, tile = blockIdx.x % in.tiles, per = in.D / in.G;
  const int c0 = group * per + tile * CH, nch = min(CH, group * per + per - c0);
  const int len = length_of(in.lengths, b, in.t);
  const int q = lane % NL, cl = wave * S::CW + lane / NL;
  const bool mine = cl < nch;
  const int64_t d = min(c0 + cl, in.D - 1), bd = (int64_t)b * in.D + d, all_states = (int64_t)in.B * in.D * in.N;
  const int64_t gn = (int64_t)group * in.N;

  float A2[NB], g[NB], dA[NB], h[NB];
  load_states(in.A + d * in.N, q * NB, in.N, A2);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    A2[n] = log2_decay(A2[n]);
    dA[n] = g[n] = h[n] = 0.0f;
  }
  // (channels beyond the workgroup's keep zeros in h and g: their w, w u and dy are zeros, and so is what they add to dB and dC)
  const float* into = chunk + 1 == p.chunks ? p.dh_out : p.starts + (chunk + 1) * all_states;
  if (into && mine) load_states(into + bd * in.N, q * NB, in.N, g);

  // a thread's (step, channel) pairs: step i * ROWS + wrow + lrow, channel ic; a wave shares wrow
  constexpr int ROWS = THREADS / CH;
  const int ic = tid % CH, wrow = wave * WAVE / CH, lrow = CH < WAVE ? lane / CH : 0, row = wrow + lrow;
  const int lane_c = CH < WAVE ? ic : lane, wave_c = CH < WAVE ? 0 : wave * WAVE % CH;   // ic = wave_c + lane_c
  const float bias = in.bias ? in.bias[min(c0 + ic, in.D - 1)] : 0.0f, skip = in.skip ? in.skip[min(c0 + ic, in.D - 1)] : 0.0f;
  float dskip = 0.0f, dbias = 0.0f;
  // and its values of B and C: step i * SROWS + srow, state sn
  constexpr int SROWS = THREADS / NP;
  const int srow = tid / NP, sn = tid % NP;
  const bool shared = BS * NP >= THREADS || tid < BS * NP;

  // (s, b and the wave's part of an address are uniform)
  const T *const pu = row_of<T>(in.u, wrow, b, c0 + wave_c), *const pd = row_of<T>(in.delta, wrow, b, c0 + wave_c),
          *const pg = row_of<T>(p.dy, wrow, b, c0 + wave_c), *const pz = row_of<T>(in.z, wrow, b, c0 + wave_c),
          *const pb = row_of<T>(in.Bm, 0, b, gn), *const pc = row_of<T>(in.Cm, 0, b, gn);
  T *const qu = row_of<T>(p.du, wrow, b, c0 + wave_c), *const qd = row_of<T>(p.ddelta, wrow, b, c0 + wave_c),
    *const qz = row_of<T>(p.dz, wrow, b, c0 + wave_c);
  float* const bc = p.bc_parts + (((int64_t)tile * in.B + b) * in.G + group) * in.t * 2 * in.N;

  T ru[S::ITEMS], rd[S::ITEMS], rg[S::ITEMS], rz[S::ITEMS], rb[S::SHARED], rc[S::SHARED];
  float rh[NB];
  auto fetch = [&](int st, int k, bool back) {
    const int s0 = st * p.stretch + k * BS;
    if (mine && k == 0) load_states(p.states + st * all_states + bd * in.N, q * NB, in.N, rh);   // (its first block comes up twice)
    const unsigned ou = opaque(lane_bytes<T>(in.u.t, lrow, lane_c)), od = opaque(lane_bytes<T>(in.delta.t, lrow, lane_c)),
                   og = opaque(lane_bytes<T>(p.dy.t, lrow, lane_c)), oz = opaque(lane_bytes<T>(in.z.t, lrow, lane_c));
    const T *au = pu + (int64_t)s0 * in.u.t, *ad = pd + (int64_t)s0 * in.delta.t, *ag = pg + (int64_t)s0 * p.dy.t, *az = pz + (int64_t)s0 * in.z.t;
    if (s0 + BS <= len && nch == CH) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        ru[i] = raw(au, ou);
        rd[i] = raw(ad, od);
        au += ROWS * in.u.t;
        ad += ROWS * in.delta.t;
      }
      if (back) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          rg[i] = raw(ag, og);
          if (GATE) rz[i] = raw(az, oz);
          ag += ROWS * p.dy.t;
          az += ROWS * in.z.t;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        ru[i] = rd[i] = rg[i] = rz[i] = (T)0.0f;
        if (s0 + i * ROWS + row < len && ic < nch) {
          ru[i] = raw(au, ou);
          rd[i] = raw(ad, od);
          if (back) {
            rg[i] = raw(ag, og);
            if (GATE) rz[i] = raw(az, oz);
          }
        }
        au += ROWS * in.u.t;
        ad += ROWS * in.delta.t;
        ag += ROWS * p.dy.t;
        az += ROWS * in.z.t;
      }
    }
    const T *ab = pb + (int64_t)s0 * in.Bm.t, *ac = pc + (int64_t)s0 * in.Cm.t;
    const unsigned ob = opaque(lane_bytes<T>(in.Bm.t, srow, sn)), oc = opaque(lane_bytes<T>(in.Cm.t, srow, sn));
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
      rb[i] = rc[i] = (T)0.0f;
      if (shared && s0 + i * SROWS + srow < len && sn < in.N) {
        rb[i] = raw(ab, ob);
        if (back) rc[i] = raw(ac, oc);
      }
      ab += SROWS * in.Bm.t;
      ac += SROWS * in.Cm.t;
    }
  };
#pragma unroll
  for (int i = 0; i < S::ITEMS; ++i) rg[i] = rz[i] = (T)0.0f;
#pragma unroll
  for (int n = 0; n < NB; ++n) rh[n] = 0.0f;

  const int from = chunk * p.chunk / p.stretch, last_step = min(in.t, (chunk + 1) * p.chunk);
  auto blocks_of = [&](int st) { return (min(last_step, (st + 1) * p.stretch) - st * p.stretch + BS - 1) / BS; };
  int st = (last_step - 1) / p.stretch, k = 0;        // stretch; block in it
  bool back = blocks_of(st) == 1;
  if (in.t) fetch(st, 0, back);
  int turn = 0;
  while (in.t && st >= from) {
    float* const wud = lds + turn * STAGED;           // [BS][CH][4]: w, w u, gated dy -> through, dlog, core; softplus' slope
    float* const sb = wud + BS * CH * 4;              // [BS][NP]
    float* const sc = sb + BS * NP;                   // [BS][NP]
    const int s0 = st * p.stretch + k * BS, blocks = blocks_of(st);
    const bool beyond = s0 >= len;                      // no step of the sequence in it: gradients of zero, h and g stay as they are
    // stage the block: w, w u, gated dy; what softplus' and the gate's gradients need stays in registers
    float iu[S::ITEMS], iw[S::ITEMS], idy[S::ITEMS], idz[S::ITEMS];
    const bool whole = s0 + BS <= len && nch == CH;
    if (!beyond) {
      float slope[S::ITEMS];                            // softplus'
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        iu[i] = (float)ru[i];
        iw[i] = (float)rd[i] + bias;
        idy[i] = (float)rg[i];
        slope[i] = 1.0f;
        if (GATE) {
          const float z = (float)rz[i], sg = sigmoid(z);
          idz[i] = idy[i] * sg * (1.0f + z * (1.0f - sg));    // times what the gate multiplied
          idy[i] *= z * sg;
        }
      }
      if (in.softplus) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          slope[i] = sigmoid(iw[i]);
          iw[i] = softplus_of(iw[i]);
        }
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i)
          if (!(s0 + i * ROWS + row < len && ic < nch)) iw[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i)
        *reinterpret_cast<f32x4*>(wud + 4 * ((i * ROWS + row) * CH + ic)) = f32x4{iw[i], iw[i] * iu[i], idy[i], slope[i]};
      if (shared) {
#pragma unroll
        for (int i = 0; i < S::SHARED; ++i) {
          sb[(i * SROWS + srow) * NP + sn] = (float)rb[i];
          sc[(i * SROWS + srow) * NP + sn] = (float)rc[i];
        }
      }
    }
    if (k == 0) {       // (twice, and the same)
#pragma unroll
      for (int n = 0; n < NB; ++n) h[n] = rh[n];
    }
    if (!beyond) __syncthreads();
    // the block after this one
    int next_st = st, next_k = k;
    bool next_back = true;
    if (!back) {
      next_back = k + 1 == blocks - 1;
      next_k = k + 1;
    } else if (k > 0) {
      next_k = k - 1;
    } else {
      next_st = st - 1;
      next_back = p.stretch == BS;
    }
    if (next_st >= from) fetch(next_st, next_k, next_back);

    if (!back) {
      if (k > 0) store<NB>(kept + (k - 1) * THREADS * NB, h);
      if (!beyond) {
#pragma unroll
        for (int s = 0; s < BS; ++s) {
          const f32x2 w = *reinterpret_cast<const f32x2*>(wud + 4 * (s * CH + cl));
          float vb[NB];
          load<NB>(sb + s * NP + q * NB, vb);
#pragma unroll
          for (int n = 0; n < NB; ++n) h[n] = __builtin_amdgcn_exp2f(w[0] * A2[n]) * h[n] + w[1] * vb[n];
        }
      }
    } else if (beyond) {
      T *bu = qu + (int64_t)s0 * p.du.t, *bd2 = qd + (int64_t)s0 * p.ddelta.t, *bz = qz + (int64_t)s0 * p.dz.t;
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        if (s0 + i * ROWS + row < last_step && ic < nch) {
          set_elem(bu, lane_bytes<T>(p.du.t, lrow, lane_c), 0.0f);
          set_elem(bd2, lane_bytes<T>(p.ddelta.t, lrow, lane_c), 0.0f);
          if (GATE) set_elem(bz, lane_bytes<T>(p.dz.t, lrow, lane_c), 0.0f);
        }
        bu += ROWS * p.du.t;
        bd2 += ROWS * p.ddelta.t;
        bz += ROWS * p.dz.t;
      }
      for (int m = tid; m < BS * 2 * NP; m += THREADS) {
        if (s0 + m / (2 * NP) < last_step && m % NP < in.N) bc[(int64_t)s0 * 2 * in.N + m / NP * in.N + m % NP] = 0.0f;
      }
    } else {
      if (k > 0 && k + 1 < blocks) load<NB>(kept + (k - 1) * THREADS * NB, h);   // (the last block goes on from the one before)
      // forward through the block: exp(w A) and exp(w A) h_{s-1} of every step
      float a[BS][NB], ah[BS][NB];
#pragma unroll
      for (int s = 0; s < BS; ++s) {
        const f32x2 w = *reinterpret_cast<const f32x2*>(wud + 4 * (s * CH + cl));
        float vb[NB];
        load<NB>(sb + s * NP + q * NB, vb);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          a[s][n] = __builtin_amdgcn_exp2f(w[0] * A2[n]);
          ah[s][n] = a[s][n] * h[n];
          h[n] = ah[s][n] + w[1] * vb[n];
        }
      }
      // Steps that only fill up the block keep no state: with their w of zero an infinite one would make NaN of dA.  In a branch of its own here, or, with
      // two lanes per channel, step by step below: 1000 x 32 x 1024, N = 16 634 / 660 us, N = 32 1180 / 1217, N = 8 480 / 458.
      constexpr bool APART = NL > 2;
      if (APART && s0 + BS > len) {
#pragma unroll
        for (int s = 1; s < BS; ++s)
#pragma unroll
          for (int n = 0; n < NB; ++n) ah[s][n] = s0 + s < len ? ah[s][n] : 0.0f;
      }
      // and back; a step's operands are read while the one before is worked on, whose results go over its own
      f32x3 next_w = *reinterpret_cast<const f32x3*>(wud + 4 * ((BS - 1) * CH + cl));
      float next_b[NB], next_c[NB];
      load<NB>(sb + (BS - 1) * NP + q * NB, next_b);
      load<NB>(sc + (BS - 1) * NP + q * NB, next_c);
#pragma unroll
      for (int s = BS - 1; s >= 0; --s) {
        const f32x3 w = next_w;
        float vb[NB], vc[NB], v[2 * NB], through = 0.0f, dlog = 0.0f, core = 0.0f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          vb[n] = next_b[n];
          vc[n] = next_c[n];
        }
        if (s > 0) {
          next_w = *reinterpret_cast<const f32x3*>(wud + 4 * ((s - 1) * CH + cl));
          load<NB>(sb + (s - 1) * NP + q * NB, next_b);
          load<NB>(sc + (s - 1) * NP + q * NB, next_c);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if (!APART && s > 0 && s0 + s >= len) ah[s][n] = 0.0f;
          const float hn = ah[s][n] + w[1] * vb[n];
          g[n] += w[2] * vc[n];
          v[n] = g[n] * w[1];                  // to dB
          v[NB + n] = w[2] * hn;               // to dC
          through = n ? through + g[n] * vb[n] : g[n] * vb[n];
          if (GATE) core = n ? core + hn * vc[n] : hn * vc[n];
          const float r = g[n] * ah[s][n];     // the exponent's gradient
          dlog = n ? dlog + r * A2[n] : r * A2[n];   // times log2 e
          dA[n] += r * w[0];
          g[n] *= a[s][n];
        }
        channels_sum<S>(v, lane, red + (wave * BS + s) * 2 * NP);
        through = lanes_sum<NL>(through);
        dlog = lanes_sum<NL>(dlog);
        if (GATE) core = lanes_sum<NL>(core);
        *reinterpret_cast<f32x3*>(wud + 4 * (s * CH + cl)) = f32x3{through, dlog, core};   // (all lanes of a channel the same)
      }
      __syncthreads();
      T *bu = qu + (int64_t)s0 * p.du.t, *bd2 = qd + (int64_t)s0 * p.ddelta.t, *bz = qz + (int64_t)s0 * p.dz.t;
      const unsigned ou = opaque(lane_bytes<T>(p.du.t, lrow, lane_c)), od = opaque(lane_bytes<T>(p.ddelta.t, lrow, lane_c)),
                     oz = opaque(lane_bytes<T>(p.dz.t, lrow, lane_c));
      if (whole && s0 + BS <= last_step) {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(wud + 4 * ((i * ROWS + row) * CH + ic));
          const float dw = (iu[i] * v[0] + LN2 * v[1]) * v[3];
          set_elem(bu, ou, iw[i] * v[0] + skip * idy[i]);
          set_elem(bd2, od, dw);
          if (GATE) set_elem(bz, oz, idz[i] * (v[2] + skip * iu[i]));
          dskip += idy[i] * iu[i];
          dbias += dw;
          bu += ROWS * p.du.t;
          bd2 += ROWS * p.ddelta.t;
          bz += ROWS * p.dz.t;
        }
      } else {
#pragma unroll
        for (int i = 0; i < S::ITEMS; ++i) {
          const int s = s0 + i * ROWS + row;
          const f32x4 v = *reinterpret_cast<const f32x4*>(wud + 4 * ((i * ROWS + row) * CH + ic));
          const bool live = s < len;
          const float dw = live ? (iu[i] * v[0] + LN2 * v[1]) * v[3] : 0.0f;
          if (s < last_step && ic < nch) {
            set_elem(bu, ou, live ? iw[i] * v[0] + skip * idy[i] : 0.0f);
            set_elem(bd2, od, dw);
            if (GATE) set_elem(bz, oz, live ? idz[i] * (v[2] + skip * iu[i]) : 0.0f);
            dskip += idy[i] * iu[i];
            dbias += dw;
          }
          bu += ROWS * p.du.t;
          bd2 += ROWS * p.ddelta.t;
          bz += ROWS * p.dz.t;
        }
      }
      float* const to = bc + (int64_t)s0 * 2 * in.N;
#pragma unroll
      for (int i = 0; i < (BS * 2 * NP + THREADS - 1) / THREADS; ++i) {
        const int m = i * THREADS + tid;
        if (BS * 2 * NP % THREADS && m >= BS * 2 * NP) break;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < BACK_WAVES; ++w) v += red[w * BS * 2 * NP + m];
        const int s = s0 + m / (2 * NP);
        if (s < last_step && m % NP < in.N) to[m / NP * in.N + m % NP] = s < len ? v : 0.0f;   // (zero times what may be infinite)
      }
    }
    if (!beyond) turn ^= 1;
    st = next_st;
    k = next_k;
    back = next_back;
    if (st < from) break;
  }
  if (mine && p.dh0 && chunk == 0) store_states(p.dh0 + bd * in.N, q * NB, in.N, g);
  float* parts = p.a_parts + ((int64_t)chunk * in.B + b) * in.D * (in.N + 2);
  if (mine) store_states(parts + d * in.N, q * NB, in.N, dA);
  // dskip and ddelta_bias: the threads that share a channel, in their order
  __syncthreads();
  red[tid] = dskip;
  red[THREADS + tid] = dbias;
  __syncthreads();
  if (tid < nch) {
    float s1 = 0.0f, s2 = 0.0f;
    for (int i = tid; i < THREADS; i += CH) {
      s1 += red[i];
      s2 += red[THREADS + i];
    }
    parts[(int64_t)in.D * in.N + c0 + tid] = s1;
    parts[(int64_t)in.D * (in.N + 1) + c0 + tid] = s2;
  }
}

// dL/dh just before a chunk, from the chunk's own steps: g_{s-1} = exp(w_s A) (g_s + C_s dy_s) from its end to its start; and the sum of w.
// One wave's channels, as in the forward launches.
template <typename T, typename S, bool GATE>
__global__ __launch_bounds__(FORWARD_WAVES* WAVE) void scan_back_ends_kernel(Backward p) {
  constexpr int CH = S::CH, TS = S::TS, NP = S::NP, NL = S::NL, NB = S::NB, ROWS = WAVE / CH, SROWS = WAVE / NP;
  struct Lds { float wg[TS][CH][2], sc[TS][NP]; };
  __shared__ __align__(16) Lds lds[FORWARD_WAVES];
  const Scan& in = p.in;
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), b = blockIdx.y, chunk = blockIdx.z + 1;
  auto& [wg, sc] = lds[wave];
  const int group = blockIdx.x / in.tiles, per = in.D / in.G;
  const int c0 = group * per + (blockIdx.x % in.tiles * FORWARD_WAVES + wave) * CH;
  const int nch = min(CH, group * per + per - c0);
  if (nch <= 0) return;
  const int len = length_of(in.lengths, b, in.t);
  const int begin = chunk * p.chunk, stop = min(len, min(in.t, begin + p.chunk));
  const int q = lane % NL, cl = lane / NL;
  const int64_t d = min(c0 + cl, in.D - 1), bd = (int64_t)b * in.D + d, gn = (int64_t)group * in.N;
  float g[NB], A2[NB], sum_w = 0.0f;
  load_states(in.A + d * in.N, q * NB, in.N, A2);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    A2[n] = log2_decay(A2[n]);
    g[n] = 0.0f;
  }
  const int row = lane / CH, ch = lane % CH, srow = lane / NP, sn = lane % NP;
  const bool pair = TS * CH >= WAVE || lane < TS * CH, shared = TS * NP >= WAVE || lane < TS * NP;
  const float bias = in.bias ? in.bias[min(c0 + ch, in.D - 1)] : 0.0f;
  T rd[S::ITEMS], rg[S::ITEMS], rz[S::ITEMS], rc[S::SHARED];
  auto fetch = [&](int s0) {
    const bool all = s0 + TS <= stop && nch == CH;
    const unsigned od = opaque(lane_bytes<T>(in.delta.t, row, ch)), og = opaque(lane_bytes<T>(p.dy.t, row, ch)),
                   oz = opaque(lane_bytes<T>(in.z.t, row, ch)), oc = opaque(lane_bytes<T>(in.Cm.t, srow, min(sn, in.N - 1)));
    const T *ad = row_of<T>(in.delta, s0, b, c0), *ag = row_of<T>(p.dy, s0, b, c0), *az = row_of<T>(in.z, s0, b, c0),
            *ac = row_of<T>(in.Cm, s0, b, gn);
#pragma unroll
    for (int i = 0; i < S::ITEMS; ++i) {
      rd[i] = rg[i] = rz[i] = (T)0.0f;
      if (pair && (all || (s0 + i * ROWS + row < stop && ch < nch))) {
        rd[i] = raw(ad, od);
        rg[i] = raw(ag, og);
        if (GATE) rz[i] = raw(az, oz);
      }
      ad += ROWS * in.delta.t;
      ag += ROWS * p.dy.t;
      az += ROWS * in.z.t;
    }
#pragma unroll
    for (int i = 0; i < S::SHARED; ++i) {
      rc[i] = (T)0.0f;
      if (shared && s0 + i * SROWS + srow < stop) rc[i] = raw(ac, oc);
      ac += SROWS * in.Cm.t;
    }
  };
  int s0 = begin + (stop - 1 - begin) / TS * TS;
  if (begin < stop) fetch(s0);
  for (; begin < stop && s0 >= begin; s0 -= TS) {
    if (pair) {
#pragma unroll
      for (int i = 0; i < S::ITEMS; ++i) {
        const bool live = s0 + i * ROWS + row < stop && ch < nch;
        const float v = (float)rd[i] + bias, w = !live ? 0.0f : in.softplus ? softplus_of(v) : v, dy = (float)rg[i], z = (float)rz[i];
        *reinterpret_cast<f32x2*>(&wg[i * ROWS + row][ch][0]) = f32x2{w, GATE ? dy * z * sigmoid(z) : dy};
      }
    }
    if (shared) {
#pragma unroll
      for (int i = 0; i < S::SHARED; ++i) sc[i * SROWS + srow][sn] = sn < in.N ? (float)rc[i] : 0.0f;
    }
    wave_sync();
    if (s0 - TS >= begin) fetch(s0 - TS);
#pragma unroll
    for (int s = TS - 1; s >= 0; --s) {
      const f32x2 w = *reinterpret_cast<const f32x2*>(&wg[s][cl][0]);
      float vc[NB];
      load<NB>(&sc[s][q * NB], vc);
#pragma unroll
      for (int n = 0; n < NB; ++n) g[n] = __builtin_amdgcn_exp2f(w[0] * A2[n]) * (g[n] + w[1] * vc[n]);
      sum_w += w[0];
    }
    wave_sync();
  }
  if (cl >= nch) return;
  store_states(p.starts + chunk * ((int64_t)in.B * in.D * in.N) + bd * in.N, q * NB, in.N, g);
  if (q == 0) p.sums[(int64_t)chunk * in.B * in.D + bd] = sum_w;
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
  constexpr int U = 8;                                 // parts on their way at once
  const int64_t row = p.t * 2 * p.N, all = (int64_t)p.B * p.G * row;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < all; k += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    int i = 0;
    for (; i + U <= p.tiles; i += U) {
      float part[U];
#pragma unroll
      for (int u = 0; u < U; ++u) part[u] = p.parts[(i + u) * all + k];
#pragma unroll
      for (int u = 0; u < U; ++u) v += part[u];
    }
    for (; i < p.tiles; ++i) v += p.parts[i * all + k];
    const int64_t bg = k / row, r = k % row;
    const unsigned step = (unsigned)(r / (2 * p.N)), rest = (unsigned)(r % (2 * p.N)), half = rest / p.N, n = rest % p.N;
    put<T>(half ? p.dC : p.dB, step, bg / p.G, bg % p.G * p.N + n, v);
  }
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
// A lane per NB states: the pool's rows are read and written once.  VEC: a channel's states, and its group's B and C, in whole vectors of NB.
// Bound: HBM.  256 x 2048 x 16: 16 us, 4.4 TB/s (a value at a time 41 us).
template <typename T, int NL, bool VEC>
__global__ __launch_bounds__(256) void scan_step_kernel(Step p) {
  const Scan& in = p.in;
  const int q = threadIdx.x % NL, b = blockIdx.y;
  const unsigned d = blockIdx.x * (256 / NL) + threadIdx.x / NL;
  if (d >= (unsigned)in.D) return;                       // (all lanes of a channel)
  const int64_t slot = p.index ? p.index[b] : b;
  T* const y_at = (T*)p.y.p + b * p.y.b + d;
  if (slot < 0 || slot >= p.slots) {
    if (q == 0) *y_at = (T)0.0f;
    return;
  }
  const unsigned group = in.G == 1 ? 0u : d / (unsigned)(in.D / in.G);
  const int64_t state = (slot * in.D + d) * in.N;
  const T* const pb = (const T*)in.Bm.p + b * in.Bm.b + (int64_t)group * in.N;
  const T* const pc = (const T*)in.Cm.p + b * in.Cm.b + (int64_t)group * in.N;
  float h[NB], A[NB], vb[NB], vc[NB];
  if constexpr (VEC) {
    if (q * NB >= in.N) {
#pragma unroll
      for (int n = 0; n < NB; ++n) h[n] = A[n] = vb[n] = vc[n] = 0.0f;
    } else {
      load<NB>(p.state_in + state + q * NB, h);
      load<NB>(in.A + (int64_t)d * in.N + q * NB, A);
      load<NB>(pb + q * NB, vb);
      load<NB>(pc + q * NB, vc);
    }
  } else {
    load_states(p.state_in + state, q * NB, in.N, h);
    load_states(in.A + (int64_t)d * in.N, q * NB, in.N, A);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const bool there = q * NB + n < in.N;
      vb[n] = there ? (float)pb[q * NB + n] : 0.0f;
      vc[n] = there ? (float)pc[q * NB + n] : 0.0f;
    }
  }
  const float u = (float)*((const T*)in.u.p + b * in.u.b + d), z = in.z.p ? (float)*((const T*)in.z.p + b * in.z.b + d) : 0.0f;
  float w = (float)*((const T*)in.delta.p + b * in.delta.b + d) + (in.bias ? in.bias[d] : 0.0f);
  const float skip = in.skip ? in.skip[d] : 0.0f;
  if (in.softplus) w = softplus_of(w);
  float y = 0.0f;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    h[n] = __builtin_amdgcn_exp2f(w * log2_decay(A[n])) * h[n] + w * u * vb[n];
    y += h[n] * vc[n];
  }
  y = lanes_sum<NL>(y);
  if constexpr (VEC) {
    if (q * NB < in.N) store<NB>(p.state_out + state + q * NB, h);
  } else {
    store_states(p.state_out + state, q * NB, in.N, h);
  }
  if (q == 0) {
    y += skip * u;
    if (in.z.p) y *= z * sigmoid(z);
    *y_at = (T)y;
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
  if (d->t < 0 || d->t > (1 << 30) || d->B < 0 || d->B > 65535 || d->D < 1 || d->D > (1 << 22))
    return set_error(MEBPTT_EINVAL, "0 <= t <= 2^30, 0 <= B <= 65535 and 1 <= D <= 2^22 are needed");
  if (d->N < 1 || d->N > MAX_N) return set_error(MEBPTT_EINVAL, "N must be 1 .. %d", MAX_N);
  if (d->G < 1 || d->D % d->G) return set_error(MEBPTT_EINVAL, "G must divide D");
  if (!float_dtype(d->dtype)) return set_error(MEBPTT_EINVAL, "dtype must be MEBPTT_FP32 or MEBPTT_BF16");
  return MEBPTT_OK;
}
int check_stretch(const mebptt_scan_desc* d) {
  const int s = d->stretch;
  return s == 16 || s == 32 || s == 64 || s == 128 || s == 256 ? MEBPTT_OK : set_error(MEBPTT_EINVAL, "stretch must be 16, 32, 64, 128 or 256");
}
bool stride_fits(const mebptt_seq& s) { return s.stride_t >= 0 && s.stride_t <= MAX_STRIDE; }
int check_inputs(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  if (!in) return set_error(MEBPTT_EINVAL, "inputs are NULL");
  if (!in->A) return set_error(MEBPTT_EINVAL, "A is NULL");
  if (d->t && d->B && (!in->u.data || !in->delta.data || !in->Bm.data || !in->Cm.data))
    return set_error(MEBPTT_EINVAL, "u, delta, B and C are required");
  if (d->t > 1)
    for (const mebptt_seq* q : {&in->u, &in->delta, &in->z, &in->Bm, &in->Cm})
      if (q->data && !stride_fits(*q)) return set_error(MEBPTT_EINVAL, "stride_t must be 0 .. 2^25");
  return MEBPTT_OK;
}
int check_out(const mebptt_scan_desc* d, const mebptt_seq& s, int64_t channels, const char* what) {
  if (d->t && d->B && !s.data) return set_error(MEBPTT_EINVAL, "%s is NULL", what);
  if (d->t > 1 && !stride_fits(s)) return set_error(MEBPTT_EINVAL, "stride_t must be 0 .. 2^25");
  if (!rows_apart(s, d->t, d->B, channels)) return set_error(MEBPTT_EINVAL, "rows of %s overlap", what);
  return MEBPTT_OK;
}
Scan scan_of(const mebptt_scan_desc* d, const mebptt_scan_inputs* in) {
  return {in_seq(in->u), in_seq(in->delta), in_seq(in->z), in_seq(in->Bm), in_seq(in->Cm), in->A, in->skip, in->delta_bias, in->lengths,
          d->t, d->B, d->D, d->N, d->G, d->softplus, 0};
}

void join(const Join& j, hipStream_t s) { scan_join_kernel<<<(unsigned)ceil_div(j.BD * j.N, 256), 256, 0, s>>>(j); }

// Forward launches.  A SIMD issues a vector instruction of one wave only every other turn, and more waves hide what the recurrence waits
// for, so what counts is waves.  Where the channels give fewer than 2048, two per SIMD, the time axis is cut into chunks, up to eight
// waves per SIMD, whose ends are computed first (70 % of the work once more).  Measured, 10000 x 1 x 2048: 4096 / 6144 / 8192 waves wanted
// 174 / 173 / 172 us, uncut 1173; 4000 x 8 x 512 122 / 122 / 119, uncut 476; 1000 x 32 x 1024, which gives 2048: uncut 193, in four chunks 245.
constexpr int ENOUGH_WAVES = 2048, WANT_WAVES = 8192, MIN_CHUNK = 32, MAX_CHUNKS = 64;
struct Cut {
  int tiles;           // workgroups per group of channels
  int chunk, chunks;   // steps per chunk, a multiple of a block's
};
// Lanes per channel and states per lane.  1000 x 32 x 1024, N = 16: 4 lanes of 4 states 188 us, 8 of 2 213, 2 of 8 257 (at four times as many
// sequences 593, 857, 556).
template <typename F>
int with_shape(int N, F&& f) {
  if (N <= 4) return f(ForwardShape<1, 4>{});
  if (N <= 8) return f(ForwardShape<2, 4>{});
  if (N <= 16) return f(ForwardShape<4, 4>{});
  if (N <= 32) return f(ForwardShape<8, 4>{});
  return f(ForwardShape<8, 8>{});   // (16 lanes of 4 have four channels per wave to stage B and C for: 631 instead of 475 us at 1000 x 32 x 1024)
}
Cut forward_cut(const mebptt_scan_desc* d) {
  Cut c = {};
  int64_t waves = 0;
  with_shape(d->N, [&](auto shape) {
    using S = decltype(shape);
    c.tiles = (int)ceil_div(d->D / d->G, S::CH * FORWARD_WAVES);
    waves = ceil_div(d->D / d->G, S::CH) * d->G * std::max(d->B, 1);
    return 0;
  });
  const int64_t t = std::max(d->t, 1);
  const int64_t want = waves >= ENOUGH_WAVES ? 1 : std::min<int64_t>(MAX_CHUNKS, ceil_div(WANT_WAVES, waves));
  c.chunk = (int)(ceil_div(std::max<int64_t>(want > 1 ? MIN_CHUNK : t, ceil_div(t, want)), 16) * 16);
  c.chunks = (int)ceil_div(t, c.chunk);
  return c;
}
size_t starts_bytes(const mebptt_scan_desc* d, int chunks) { return chunks < 2 ? 0 : align_up((size_t)chunks * d->B * d->D * d->N * sizeof(float)); }
size_t sums_bytes(const mebptt_scan_desc* d, int chunks) { return chunks < 2 ? 0 : align_up((size_t)chunks * d->B * d->D * sizeof(float)); }

// Backward launches: 4 states per lane, two waves per SIMD, where what a block keeps (exp(w A) and exp(w A) h of 16 steps) takes half the
// registers.  (With stretches of 256, and of 128 up to N = 8, the states at the starts of their blocks take so much LDS that a compute unit holds one
// workgroup, one wave per SIMD: below.)  With 2 states per lane and twice the waves, when that was chosen: 1000 x 32 x 1024, N = 8 473 us instead of 465, N = 16 883 instead of 711, N = 32
// 1619 instead of 1240.  The time axis is cut as the forward pass's is, in whole stretches: 1000 x 32 x 1024, which gives 2048 waves, 711 us
// uncut, 778 in two; 10000 x 1 x 2048, both passes, 660 us, 1827 uncut.
constexpr int BACK_ENOUGH = 2048, BACK_WANT = 4096;   // waves
struct BackCut {
  int tiles, ends_tiles, chunk, chunks;
};
template <typename F>
int with_back_shape(int N, F&& f) {
  if (N <= 8) return f(BackwardShape<2, 4>{});
  if (N <= 16) return f(BackwardShape<4, 4>{});
  if (N <= 32) return f(BackwardShape<8, 4>{});
  return f(BackwardShape<16, 4>{});
}
BackCut back_cut(const mebptt_scan_desc* d) {
  BackCut c = {};
  int64_t waves = 0;
  with_back_shape(d->N, [&](auto shape) {
    using S = decltype(shape);
    c.tiles = (int)ceil_div(d->D / d->G, S::CH);
    waves = ceil_div(d->D / d->G, S::CW) * d->G * std::max(d->B, 1);
    return 0;
  });
  with_shape(d->N, [&](auto shape) {
    c.ends_tiles = (int)ceil_div(d->D / d->G, decltype(shape)::CH * FORWARD_WAVES);
    return 0;
  });
  const int64_t t = std::max(d->t, 1);
  const int64_t want = waves >= BACK_ENOUGH ? 1 : std::min<int64_t>(MAX_CHUNKS, ceil_div(BACK_WANT, waves));
  c.chunk = (int)(ceil_div(ceil_div(t, want), d->stretch) * d->stretch);
  c.chunks = (int)ceil_div(t, c.chunk);
  return c;
}
size_t bc_bytes(const mebptt_scan_desc* d, const BackCut& c) {
  return align_up((size_t)c.tiles * d->t * d->B * d->G * 2 * d->N * sizeof(float));
}
size_t a_bytes(const mebptt_scan_desc* d, const BackCut& c) { return align_up((size_t)c.chunks * d->B * d->D * (d->N + 2) * sizeof(float)); }

// Per workgroup at stretches of 64 / 128 / 256: N = 8 80 / 96 / 129 thousand bytes, N = 16 53 / 70 / 102, N = 32 49 / 66 / 98, of a compute unit's 164.  Time by stretch,
// 16 / 32 / 64 / 128 / 256: 1000 x 32 x 1024, N = 8 390 / 436 / 464 / 711 / 724 us, N = 16 524 / 603 / 635 / 651 / 1003 (the forward pass, which writes the
// states, 207 / 177 / 170 / 168 / 165).
template <typename S>
size_t back_lds(int stretch) {
  return (2 * ((size_t)BS * S::CH * 4 + 2 * BS * S::NP) + S::BACK_WAVES * BS * 2 * S::NP + std::max(stretch / BS - 2, 0) * S::THREADS * S::NB) * sizeof(float);
}

}  // namespace

extern "C" {

size_t mebptt_scan_state_bytes(const mebptt_scan_desc* d) {
  if (check(d) != MEBPTT_OK || check_stretch(d) != MEBPTT_OK) return 0;
  return (size_t)ceil_div(d->t, d->stretch) * d->B * d->D * d->N * sizeof(float);
}

size_t mebptt_scan_workspace_bytes(const mebptt_scan_desc* d, int32_t backward) {
  if (check(d) != MEBPTT_OK) return 0;
  if (backward) {
    if (check_stretch(d) != MEBPTT_OK) return 0;
    const BackCut c = back_cut(d);
    return std::max(bc_bytes(d, c) + a_bytes(d, c) + starts_bytes(d, c.chunks) + sums_bytes(d, c.chunks), mebptt_scan_workspace_bytes(d, 0));
  }
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
  p.in.tiles = cut.tiles;
  const unsigned wide = (unsigned)(cut.tiles * d->G);
  hipStream_t s = (hipStream_t)stream;
  return with_shape(d->N, [&](auto shape) {
    using S = decltype(shape);
    auto go = [&](auto elem) {
      using T = decltype(elem);
      if (cut.chunks > 1) scan_forward_kernel<T, S, true><<<dim3(wide, d->B, cut.chunks - 1), FORWARD_WAVES * WAVE, 0, s>>>(p);
      if (cut.chunks > 2) join({p.starts, p.sums, in->A, p.starts + (int64_t)d->B * d->D * d->N, (int64_t)d->B * d->D, d->D, d->N, 2, 1, cut.chunks - 2, -1}, s);
      scan_forward_kernel<T, S, false><<<dim3(wide, d->B, cut.chunks), FORWARD_WAVES * WAVE, 0, s>>>(p);
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
  const BackCut cut = back_cut(d);
  hipStream_t s = (hipStream_t)stream;
  float *bc = (float*)workspace, *ap = (float*)((char*)bc + bc_bytes(d, cut)), *starts = (float*)((char*)ap + a_bytes(d, cut));
  if (d->B) {
    Backward p = {scan_of(d, in), in_seq(dy), out_seq(grads->du), out_seq(grads->ddelta), out_seq(grads->dz), (const float*)states, dh_out,
                  grads->dh0, bc, ap, d->stretch, cut.chunk, cut.chunks, starts, (float*)((char*)starts + starts_bytes(d, cut.chunks))};
    auto go = [&](auto elem, auto gate) {
      using T = decltype(elem);
      constexpr bool GATE = decltype(gate)::value;
      if (cut.chunks > 1)
        with_shape(d->N, [&](auto shape) {
          p.in.tiles = cut.ends_tiles;
          scan_back_ends_kernel<T, decltype(shape), GATE>
              <<<dim3((unsigned)(cut.ends_tiles * d->G), d->B, cut.chunks - 1), FORWARD_WAVES * WAVE, 0, s>>>(p);
          join({p.starts, p.sums, in->A, dh_out, (int64_t)d->B * d->D, d->D, d->N, cut.chunks - 1, -1, cut.chunks - 1, 0}, s);
          return 0;
        });
      return with_back_shape(d->N, [&](auto shape) {
        using S = decltype(shape);
        const hipError_t e = allow_dynamic_lds<scan_backward_kernel<T, S, GATE>>(back_lds<S>(256));
        if (e != hipSuccess) {
          (void)hipGetLastError();   // reported here, and not by the next call as well
          return set_error(MEBPTT_EHIP, "mebptt_scan_backward: %s", hipGetErrorString(e));
        }
        p.in.tiles = cut.tiles;
        scan_backward_kernel<T, S, GATE>
            <<<dim3((unsigned)(cut.tiles * d->G), d->B, cut.chunks), S::THREADS, back_lds<S>(d->stretch), s>>>(p);
        return launched("mebptt_scan_backward");
      });
    };
    const std::true_type gate{};
    const std::false_type none{};
    if (d->dtype == MEBPTT_FP32) rc = in->z.data ? go(float{}, gate) : go(float{}, none);
    else rc = in->z.data ? go(__bf16{}, gate) : go(__bf16{}, none);
    if (rc) return rc;
    if (d->t) {
      const Shared q = {bc, out_seq(grads->dBm), out_seq(grads->dCm), d->t, d->B, d->G, d->N, cut.tiles};
      const unsigned grid = (unsigned)std::min<int64_t>(ceil_div((int64_t)d->t * d->B * d->G * 2 * d->N, 256), 4096);
      if (d->dtype == MEBPTT_FP32) scan_shared_kernel<float><<<grid, 256, 0, s>>>(q);
      else scan_shared_kernel<__bf16><<<grid, 256, 0, s>>>(q);
      if ((rc = launched("mebptt_scan_backward"))) return rc;
    }
  }
  const int64_t DN = (int64_t)d->D * d->N;
  float* const outs[3] = {grads->dA, grads->dskip, grads->ddelta_bias};
  const int64_t cols[3] = {DN, d->D, d->D};
  return sum_parts(ap, d->B ? (int64_t)cut.chunks * d->B : 0, 3, cols, outs, s);
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
  const bool vec = d->N % NB == 0 && aligned(state_in, 16) && aligned(state_out, 16) && aligned(in->A, 16) &&
                   rows_aligned(in->Bm.data, in->Bm.stride_b, d->dtype, NB) && rows_aligned(in->Cm.data, in->Cm.stride_b, d->dtype, NB);
  hipStream_t s = (hipStream_t)stream;
  return with_lanes(d->N, [&](auto l) {
    constexpr int NL = decltype(l)::value;
    const dim3 grid((unsigned)ceil_div(d->D, 256 / NL), d->B);
    auto go = [&](auto elem) {
      using T = decltype(elem);
      if (vec) scan_step_kernel<T, NL, true><<<grid, 256, 0, s>>>(p);
      else scan_step_kernel<T, NL, false><<<grid, 256, 0, s>>>(p);
      return launched("mebptt_scan_step");
    };
    return d->dtype == MEBPTT_FP32 ? go(float{}) : go(__bf16{});
  });
}

}  // extern "C"
