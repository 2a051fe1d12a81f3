// What the kernels of the gated delta rule share: the recurrence cut into chunks, matrix products out of registers and LDS, what a chunk's
// preparation leaves for the kernels that walk over chunks.  Not part of the ABI.
//
// Per sequence and head, with a state S [dk, dv], k^ = k / |k| and q~ = scale q / |q| (or k and scale q as they are), alpha = exp(g):
//     r_s = v_s - alpha_s S_{s-1}^T k^_s,   S_s = alpha_s S_{s-1} + beta_s k^_s r_s^T,   y_s = S_s^T q~_s.
// Over a chunk of 64 steps, with G the running sum of g, gamma = exp(G), D_ij = exp(G_i - G_j) (j <= i), M = K^ K^^T o D below the diagonal,
// P = Q~ K^^T o D up to it:
//     R = T (V - gamma K^ S),  T = (I + M beta)^-1,   Y = gamma Q~ S + P beta R,   S' = gamma_C S + (gamma_C / gamma K^)^T beta R.
// T and P do not depend on the state: one launch prepares them for all chunks at once, another walks over the chunks with the state in
// registers.  Backward, with dS' the gradient of the state behind the chunk:
//     dU = P^T dY + (gamma_C / gamma K^) dS',   Z = T^T beta dU = dV,   dS = gamma_C dS' + (gamma Q~)^T dY - (gamma K^)^T Z,
// and the other gradients from q, k, dY, R, Z, S and dS' of the chunk alone.
#pragma once

#include <type_traits>

#include "ops.h"

namespace mebptt {
namespace delta {

using namespace mebptt::ops;

constexpr int C = 64;            // steps of a chunk
constexpr int MAX_DK = 128, MAX_DV = 256, MAX_HEADS = 1024;

// ---- products ----------------------------------------------------------------------------------------
//
// An operand of one instruction's worth: 16 rows (or columns) by 32 of what is summed over.  Lane l holds row l % 16 and, with g = l / 16, the eight
// values 4 g .. 4 g + 3 and 16 + 4 g .. of the 32.  A result tile has column l % 16 and rows 4 g .. 4 g + 3 in lane l, so two tiles above each
// other are an operand of the next product as they stand: what a wave computes in a column never leaves its registers.
//
// bf16 inputs go to the bf16 matrix instruction as they are; what has 32 bits is cut into N parts of 8 significant bits each, h = bf16(x), m =
// bf16(x - h), l = bf16(x - h - m): with three of them 24 bits arrive, with two 16 (errors of about 2^-18).  fp32 inputs go to the fp32 instruction.
template <typename T, int N>
struct Op;
template <int N>
struct Op<__bf16, N> {
  bf16x8 p[N];
};
template <int N>
struct Op<float, N> {
  f32x4 v[2];
};

template <typename T, int N>
__device__ inline Op<T, N> cut(f32x4 a, f32x4 b) {
  Op<T, N> o;
  if constexpr (std::is_same<T, float>::value) {
    o.v[0] = a;
    o.v[1] = b;
  } else {
    // in pairs: one instruction rounds two values, and a pair is a register of the operand
    float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      u32x4 pairs;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x2 two = {x[2 * e], x[2 * e + 1]};
        const unsigned pair = __builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2));
        pairs[e] = pair;
        if (n + 1 < N) {
          x[2 * e] -= __uint_as_float(pair << 16);
          x[2 * e + 1] -= __uint_as_float(pair & 0xFFFF0000u);
        }
      }
      o.p[n] = __builtin_bit_cast(bf16x8, pairs);
    }
  }
  return o;
}

// The operand whose row `row` (of this lane) stands at p, 32 values from p on.
__device__ inline Op<__bf16, 1> from_row(const __bf16* p, int g) {
  const bf16x4 a = *reinterpret_cast<const bf16x4*>(p + 4 * g), b = *reinterpret_cast<const bf16x4*>(p + 16 + 4 * g);
  Op<__bf16, 1> o;
  o.p[0] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return o;
}
__device__ inline Op<float, 1> from_row(const float* p, int g) {
  Op<float, 1> o;
  o.v[0] = *reinterpret_cast<const f32x4*>(p + 4 * g);
  o.v[1] = *reinterpret_cast<const f32x4*>(p + 16 + 4 * g);
  return o;
}

// c[r] += a[r] b for R tiles; of the products of parts those that matter.  Tiles innermost: an instruction's result can be added to four or more
// instructions later without a pause.
template <int R, int M, int NA, int NB>
__device__ inline void mma(f32x4 (&c)[M], const Op<__bf16, NA> (&a)[R], const Op<__bf16, NB>& b, int first = 0) {
  constexpr int MOST = NA > NB ? NA : NB;
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j < MOST) {
#pragma unroll
        for (int r = 0; r < R; ++r) c[first + r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r].p[i], b.p[j], c[first + r], 0, 0, 0);
      }
}
template <int R, int M, int NA, int NB>
__device__ inline void mma(f32x4 (&c)[M], const Op<float, NA> (&a)[R], const Op<float, NB>& b, int first = 0) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int r = 0; r < R; ++r) c[first + r] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r].v[h][e], b.v[h][e], c[first + r], 0, 0, 0);
}
// The same with another operand's cutting between: left to itself the compiler puts matrix instructions in a row and the cutting behind them, and a wave
// that is alone on its SIMD uses one unit at a time.  `next` is what the cutting of (x, y) gives.
template <int R, int M, int NA, int NB, int N>
__device__ inline void mma_and_cut(f32x4 (&c)[M], const Op<__bf16, NA> (&a)[R], const Op<__bf16, NB>& b, int first, float (&x)[8], Op<__bf16, N>& next, int step0, int every) {
  constexpr int MOST = NA > NB ? NA : NB;
  int count = 0;
#pragma unroll
  for (int i = NA - 1; i >= 0; --i)
#pragma unroll
    for (int j = NB - 1; j >= 0; --j)
      if (i + j < MOST) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          c[first + r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r].p[i], b.p[j], c[first + r], 0, 0, 0);
          const int step = step0 + count / every;
          if (count % every == every - 1 && step < 4 * N) {
            const int n = step / 4, e = step % 4;
            const f32x2 two = {x[2 * e], x[2 * e + 1]};
            const unsigned pair = __builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2));
            u32x4 pairs = __builtin_bit_cast(u32x4, next.p[n]);
            pairs[e] = pair;
            next.p[n] = __builtin_bit_cast(bf16x8, pairs);
            if (n + 1 < N) {
              x[2 * e] -= __uint_as_float(pair << 16);
              x[2 * e + 1] -= __uint_as_float(pair & 0xFFFF0000u);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          ++count;
        }
      }
}
template <typename T, int NA, int NB>
__device__ inline void mma(f32x4& c, const Op<T, NA>& a, const Op<T, NB>& b) {
  const Op<T, NA> row[1] = {a};
  mma(*reinterpret_cast<f32x4(*)[1]>(&c), row, b);
}

// ---- a chunk's rows in LDS -----------------------------------------------------------------------------

// [C][KD] values of T as rows, padded so that 16 of them begin in different banks.
template <typename T>
struct Lds {
  static constexpr int PAD = 16 / sizeof(T);
  static constexpr int ld(int KD) { return KD + PAD; }
  static constexpr int row_bytes(int KD) { return C * ld(KD) * (int)sizeof(T); }
};
// The operand with column c0 + l % 16 and steps s0 .. s0 + 31.  bf16: LDS turns 4 steps x 16 columns round on the way (lane i of 16 gives the address of 4
// columns of step i / 4 and receives column i of the four steps); fp32: single values.
template <int LD>
__device__ inline Op<__bf16, 1> from_columns(const __bf16* rows, int c0, int s0, int lane) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* At;
  const int i = lane % 16;
  const __bf16* p = rows + (s0 + lane / 16 * 4 + i / 4) * LD + c0 + i % 4 * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p + 16 * LD));
  Op<__bf16, 1> o;
  o.p[0] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  return o;
}
template <int LD>
__device__ inline Op<float, 1> from_columns(const float* rows, int c0, int s0, int lane) {
  Op<float, 1> o;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) o.v[h][e] = rows[(s0 + 16 * h + lane / 16 * 4 + e) * LD + c0 + lane % 16];
  return o;
}

// What a chunk's loads go by.  Loads are never conditional, since each would be waited for in its branch: steps that do not exist read the last one that
// does, columns that do not exist the last ones, and both become zeros afterwards.  A lane's address is a uniform base and 32 bits.
constexpr int64_t NEAR = 1 << 23;   // elements between steps, at most, for that
struct Window {
  int stride, live;   // live: at least one (a chunk of none is read all the same, and not used)
  __device__ inline Window(int64_t stride, int live) : stride((int)stride), live(min(max(live, 1), C)) {}
  // Offset of a step, `first` being its offset were they all there.
  __device__ inline unsigned row(unsigned first) const { return min(first, (unsigned)((live - 1) * stride)); }
};
template <typename T>
__device__ inline T* near(T* base, unsigned bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<std::conditional_t<std::is_const<T>::value, const char, char>*>(base) + bytes);
}

// Numbers that the compiler knows nothing of: what is computed from them stays where it is used.  Taken out of the loop over chunks, the addresses of
// rows would fill the registers.
__device__ inline int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ inline int here_uniform(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

// Rows of an input that are whole 16-byte vectors at 16-byte boundaries: head h of step s of sequence b is at data + s stride_t + b stride_b + h head, `width`
// values, zeros behind those that the input has.
struct Rows {
  const void* data;
  int64_t stride_t, stride_b;
  int head, width;
};
// [C][COLS] of such rows from column c0 on, on their way from memory to LDS by THREADS threads; 16 or more neighbours have a row.
template <typename T, int COLS, int THREADS>
struct Fetch {
  static constexpr int E = 16 / sizeof(T), PER_ROW = COLS / E, VECS = C * PER_ROW, N = (VECS + THREADS - 1) / THREADS;
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(16)));
  Vec v[N];
  // (where there are more threads than vectors the last ones do the same as others)
  static __device__ inline int number(int i) { return (VECS % THREADS ? min(i * THREADS + (int)threadIdx.x, VECS - 1) : i * THREADS + (int)threadIdx.x); }
  __device__ inline void load(const Rows& r, int64_t s0, int b, int h, int c0, int live) {
    const Window w(r.stride_t, live);
    const T* p = (const T*)r.data + s0 * r.stride_t + b * r.stride_b + (int64_t)h * r.head;
    const unsigned at = (unsigned)min(c0 + number(0) % PER_ROW * E, r.width - E);
    static_assert(THREADS % PER_ROW == 0, "all of a thread's vectors are in the same columns");
#pragma unroll
    for (int i = 0; i < N; ++i)
      v[i] = *reinterpret_cast<const Vec*>(near(p, (w.row((unsigned)(number(i) / PER_ROW * w.stride)) + at) * (unsigned)sizeof(T)));
  }
  // What does not exist becomes zero.
  __device__ inline void put(T* rows, const Rows& r, int c0, int live) {
    if (r.width < c0 + COLS && c0 + number(0) % PER_ROW * E >= r.width) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = Vec{};
    }
    if (live < C) {
      const int first = here(number(0) / PER_ROW);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (first + i * (THREADS / PER_ROW) >= live) v[i] = Vec{};
    }
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<Vec*>(rows + number(i) / PER_ROW * Lds<T>::ld(COLS) + number(i) % PER_ROW * E) = v[i];
  }
};

// ---- what a chunk's preparation leaves ---------------------------------------------------------------

// Per step, in rows of C floats; the walks need the first five.  GA: gamma, BE: beta, LA: gamma_C / gamma, SK: 1 / |k|, SQ: scale / |q|, RQ: 1 / |q|.
enum { GA_SK = 0, GA_SQ = 1, BE = 2, LA_SK = 3, GA = 4, LA = 5, SK = 6, SQ = 7, RQ = 8, GATES = 9, WALK_GATES = 5 };

// Matrices [C][C] as operands in the order in which lanes read them.  A lower triangle has six pieces of 16 rows by 32 columns: (0,0) (1,0)
// (2,0) (2,1) (3,0) (3,1); its transpose (0,0) (0,1) (1,0) (1,1) (2,1) (3,1).
constexpr int FRAGS = 6;
__device__ inline constexpr int lower(int rt, int pb) { return rt < 2 ? rt : 2 + (rt - 2) * 2 + pb; }
__device__ inline constexpr int upper(int rt, int pb) { return rt < 2 ? rt * 2 + pb : 4 + rt - 2; }
// KiB per piece: parts of bf16, or two halves of fp32.
template <typename T>
constexpr int units(int parts) { return sizeof(T) == 2 ? parts : 2; }
template <typename T>
constexpr int frag_bytes(int parts) { return FRAGS * units<T>(parts) * 1024; }
template <typename T, int N>
__device__ inline Op<T, N> from_frag(const char* at, int f, int lane) {
  Op<T, N> o;
  const char* p = at + f * units<T>(N) * 1024 + lane * 16;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int n = 0; n < N; ++n) o.p[n] = *reinterpret_cast<const bf16x8*>(p + n * 1024);
  } else {
    o.v[0] = *reinterpret_cast<const f32x4*>(p);
    o.v[1] = *reinterpret_cast<const f32x4*>(p + 1024);
  }
  return o;
}

// Also of P, which reaches y only: with two its terms would have 16 bits, which a y shows that is little of what they are (10000 x 1 x 16 heads: 257 us, 247 with two).
constexpr int PARTS = 3;
// A chunk's record: forward [T | P | gates | G], backward [T | T^T | P^T | gates | G], G in 64 bits.
template <typename T, bool BACK>
struct Record {
  static constexpr int T_ = 0;
  static constexpr int TT = frag_bytes<T>(PARTS);
  static constexpr int P = BACK ? TT + frag_bytes<T>(PARTS) : TT;     // P, or its transpose
  static constexpr int GATE = P + frag_bytes<T>(PARTS);
  static constexpr int SUMS = GATE + GATES * C * 4;
  static constexpr int BYTES = SUMS + C * 8;
};
inline size_t record_bytes(int dtype, bool back) {
  if (dtype == MEBPTT_FP32) return back ? Record<float, true>::BYTES : Record<float, false>::BYTES;
  return back ? Record<__bf16, true>::BYTES : Record<__bf16, false>::BYTES;
}

// ---- arguments -----------------------------------------------------------------------------------------

struct Args {
  Rows q, k, v, dy;
  mebptt_seq a, b, y;
  const float *A, *bias;
  const int32_t* lengths;
  int t, B, Hk, H, dk, dv, dvp;         // dvp: dv rounded up to 32
  int activate, normalise;
  float scale, eps;
  int c0, c1;                           // chunks of this launch
  char* records;                        // [c1 - c0][B H]
  int seg;                              // chunks of a segment: a launch walks over its segments side by side
  const float* from;                    // states [B][H][dk][dv] before the first chunk, or NULL
  float* starts;                        // [segments][B][H][start_rows][start_width] before every segment; NULL: one segment, that starts with `from`
  int start_rows, start_width;
  float* to;                            // after the last one, or NULL
  float *moves, *ends;                  // of a survey: [segments][B][H][KD][KD] and [KD][dvp], see there
  float* states;                        // kept states, or NULL
  int keep;                             // every keep-th chunk's
  float *S, *R, *Z, *dS;                // of every chunk of the launch: [KD][dvp] and [C][dvp]
  mebptt_seq dq, dkey, dval, da, db;
  int vec_out;                          // rows of y, or of dval, are whole vectors of four
  float* parts;                         // [c1 - c0][B][2 H]: sums of dg softplus and da
};

__device__ inline int ends_at(const Args& p, int b) { return p.lengths ? min(max(p.lengths[b], 0), p.t) : p.t; }

// Steps of a launch.
inline int launch_steps(const Args& p) { return std::min((p.c1 - p.c0) * C, p.t - p.c0 * C); }

// Rows that are no whole vectors, copied to ones that are, in one launch: the launch's steps, [B][..][heads][width].
struct Padded {
  struct One {
    mebptt_seq from;
    void* to;
    int heads, d, width;
  } one[4];
  int n;
};
int pad_rows(const Padded& all, const Args& p, int dtype, hipStream_t stream);
int prepare(const Args& p, int dtype, bool back, hipStream_t stream);
enum { WALK = 0, AGAIN = 1, SURVEY = 2 };   // y; S and R of every chunk; what segments do to the state
int walk(const Args& p, int dtype, int mode, hipStream_t stream);
int join_segments(const Args& p, int dtype, hipStream_t stream);
int walk_back(const Args& p, int dtype, hipStream_t stream);
int gradients(const Args& p, int dtype, hipStream_t stream);

inline int padded(int dk) { return dk <= 32 ? 32 : dk <= 64 ? 64 : 128; }
template <typename F>
int with_size(int dtype, int dk, F&& f) {
  auto at = [&](auto t) {
    if (dk <= 32) return f(t, std::integral_constant<int, 32>{});
    if (dk <= 64) return f(t, std::integral_constant<int, 64>{});
    return f(t, std::integral_constant<int, 128>{});
  };
  return dtype == MEBPTT_FP32 ? at(float{}) : at(__bf16{});
}

}  // namespace delta
}  // namespace mebptt
