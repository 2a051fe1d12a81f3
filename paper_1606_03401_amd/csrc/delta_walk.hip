// Gated delta rule: the walks over a launch's chunks, forward and back.  A workgroup of W waves owns 16 W of the state's columns for one sequence and
// head, a wave 16 of them: all rows of the state in its registers, and with them everything that is computed in these columns.  Waves share a
// chunk's keys, queries and matrices in LDS, nothing else.
// Bound: the chain of products over a sequence's chunks, one workgroup to a compute unit; there the matrix instructions of three bf16 parts (of an fp32
// state, to the state's full width) and the cutting take turns.  128 x 128, bf16: 1000 x 32 x 8 heads 151 us forward (the matrix unit busy 40 % of the time, the
// vector unit as long), 4 x 39 to run it again with S and R written, 4 x 53 back; 10000 x 1 x 16 heads in eight segments 100 for the survey and 116.
#include "delta.h"
#include "dynamic_lds.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

// A record's [bytes] from one place to LDS, by way of registers.  (The last threads' share may be another's: the same bytes twice.)
template <int BYTES, int THREADS>
struct Copy {
  static constexpr int N = (BYTES / 16 + THREADS - 1) / THREADS;
  u32x4 v[N];
  static __device__ inline unsigned at(int i) { return (unsigned)min((i * THREADS + (int)threadIdx.x) * 16, BYTES - 16); }
  __device__ inline void load(const char* from) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const u32x4*>(near(from, at(i)));
  }
  __device__ inline void put(char* to) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(to + at(i)) = v[i];
  }
};

// Nothing is moved across: operands are fetched a product ahead, where that is written, and not all at once, for which there are no registers.
__device__ inline void next_product() { __builtin_amdgcn_sched_barrier(0); }

__device__ inline f32x4 steps_of(const float* gate, int row, int rt, int g) { return *reinterpret_cast<const f32x4*>(gate + row * C + 16 * rt + 4 * g); }

// Columns c0 + l % 16 of rows in LDS, as result tiles.
template <int LD>
__device__ inline void load_tiles(f32x4 (&x)[4], const __bf16* rows, int c0, int lane) {
#pragma unroll
  for (int pb = 0; pb < 2; ++pb) {
    const Op<__bf16, 1> o = from_columns<LD>(rows, c0, 32 * pb, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[2 * pb + e / 4][e % 4] = (float)o.p[0][e];
  }
}
template <int LD>
__device__ inline void load_tiles(f32x4 (&x)[4], const float* rows, int c0, int lane) {
#pragma unroll
  for (int pb = 0; pb < 2; ++pb) {
    const Op<float, 1> o = from_columns<LD>(rows, c0, 32 * pb, lane);
    x[2 * pb] = o.v[0], x[2 * pb + 1] = o.v[1];
  }
}
// Result tiles to `steps` rows of an output, column c0 + l % 16 of `width`, zeros from `live` on.  bf16 rows that are whole vectors of four go there by way of the wave's
// own 16 columns of LDS, which turns them round, so that a lane has four neighbouring columns.
constexpr int TURN_LD = C + 8, TURN = 16 * TURN_LD;   // values of LDS for it
template <typename T>
__device__ inline void store_tiles(T* p, int step, const f32x4 (&x)[4], int steps, int live, int c0, int width, bool vec, T* turn, int lane) {
  const int g = lane / 16, i = lane % 16;
  const int64_t stride = here_uniform(step);
  if constexpr (sizeof(T) == 2) {
    if (vec) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* At;
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
        *reinterpret_cast<bf16x4*>(turn + i * TURN_LD + 16 * rt + 4 * g) = bf16x4{(__bf16)x[rt][0], (__bf16)x[rt][1], (__bf16)x[rt][2], (__bf16)x[rt][3]};
      __builtin_amdgcn_wave_barrier();
      const unsigned off = (unsigned)(i * (int)stride + c0 + 4 * g) * 2u;
      s16x4 y[4];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) y[rt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(turn + (4 * g + i / 4) * TURN_LD + 16 * rt + i % 4 * 4));
      if (c0 + 4 * g < width) {
        if (live >= C) {
#pragma unroll
          for (int rt = 0; rt < 4; ++rt) *reinterpret_cast<s16x4*>(near(p + 16 * rt * stride, off)) = y[rt];
        } else {
          const int first = here(i);
#pragma unroll
          for (int rt = 0; rt < 4; ++rt)
            if (16 * rt + first < steps) *reinterpret_cast<s16x4*>(near(p + 16 * rt * stride, off)) = 16 * rt + first < live ? y[rt] : s16x4{};
        }
      }
      return;
    }
  }
  if (c0 + i >= width) return;
  const unsigned off = (unsigned)(4 * g * (int)stride + c0 + i) * (unsigned)sizeof(T);
  const int first = here(4 * g);
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int s = 16 * rt + first + e;
      if (s < steps) *near(p + (16 * rt + e) * stride, off) = (T)(s < live ? x[rt][e] : 0.0f);
    }
}
// Zeros where a whole chunk is behind the sequence's end.
template <typename T>
__device__ inline void store_zeros(T* p, int64_t stride, int steps, int col, int width, int g) {
  if (col < width)
    for (int s = g; s < steps; s += 4) p[s * stride + col] = (T)0.0f;
}

// Waves of a SIMD: the registers of one of four waves that hold 128 rows and fetch the next chunk's are more than half.
template <int KD, int W, int MODE>
constexpr int per_simd() { return W == 4 && KD == 128 && MODE != SURVEY ? 1 : 2; }

// The state's tiles: rows 16 n + 4 g + e of column `col`, of `rows` rows with `width` columns.
template <int NT>
__device__ inline void load_state(f32x4 (&S)[NT], const float* from, int rows, int width, int col, int g) {
  const int left = rows - 4 * g;
  const unsigned off = (unsigned)(4 * g * width + col) * 4u;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) S[n][e] = from && col < width && 16 * n + e < left ? *near(from + (16 * n + e) * width, off) : 0.0f;
}
template <int NT>
__device__ inline void store_state(const f32x4 (&S)[NT], float* to, int rows, int width, int col, int g) {
  g = here(g);
  width = here_uniform(width);
  const unsigned off = (unsigned)(4 * g * width + col) * 4u;
  if (rows == 16 * NT) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) *near(to + (16 * n + e) * width, off) = S[n][e];
  } else {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * n + e < rows - 4 * g) *near(to + (16 * n + e) * width, off) = S[n][e];
  }
}

// ---- forward -------------------------------------------------------------------------------------------

template <typename T, int KD, int W, int MODE>
struct Layout {   // of LDS
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), T_ = MODE ? Q : Q + Lds<T>::row_bytes(KD), P = T_ + frag_bytes<T>(PARTS),
                       GATE = MODE ? P : P + frag_bytes<T>(PARTS), V = GATE + WALK_GATES * C * 4, Y = V + Lds<T>::row_bytes(16 * W),
                       BYTES = MODE || sizeof(T) == 4 ? Y : Y + W * TURN * 2;
};

// WALK: y.  AGAIN: the backward pass's recomputation, from its records, of S and R of every chunk.
// SURVEY: S behind a segment is linear in S before it, A S + B.  Workgroups of the first columns walk from S = 0 (the first segment: from what it
// is) and leave B in `ends`, the others from the columns of I without a v and leave A in `moves`.  For few sequences: with A and B of every segment joined
// one after another the segments can be walked side by side.
template <typename T, int KD, int W, int MODE>
__global__ __launch_bounds__(W* WAVE, (per_simd<KD, W, MODE>())) void delta_walk_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD, W, MODE>;
  using R = Record<T, MODE == AGAIN>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  constexpr bool DEEP = per_simd<KD, W, MODE>() == 1;
  T *K = reinterpret_cast<T*>(lds + L::K), *Q = reinterpret_cast<T*>(lds + L::Q), *VL = reinterpret_cast<T*>(lds + L::V);
  const float* gate = reinterpret_cast<const float*>(lds + L::GATE);
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE, g = lane / 16;
  const int blocks = (p.dv + 16 * W - 1) / (16 * W);
  const bool unit = MODE == SURVEY && blockIdx.y >= blocks;   // columns of I
  const int c0 = (blockIdx.y - (unit ? blocks : 0)) * W * 16, col = c0 + 16 * wave + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b), segment = blockIdx.z, first = p.c0 + segment * p.seg, behind = min(first + p.seg, p.c1);
  if (unit && segment == 0) return;   // (its start is known)

  f32x4 S[NT];
  if (unit) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[n][e] = 16 * n + 4 * g + e == col ? 1.0f : 0.0f;
  } else if (MODE == SURVEY ? segment == 0 : !p.starts) {
    load_state(S, p.from ? p.from + (int64_t)bh * p.dk * p.dv : nullptr, p.dk, p.dv, col, g);
    // (a copy for the walk, whose last segment may end where the first one started)
    if (MODE == SURVEY && col < p.dvp) store_state(S, p.starts + (int64_t)bh * KD * p.dvp, KD, p.dvp, col, g);
  } else {
    load_state(S, MODE == SURVEY ? nullptr : p.starts + ((int64_t)segment * BH + bh) * p.start_rows * p.start_width, p.start_rows, p.start_width, col, g);
  }

  Fetch<T, KD, W * WAVE> ck, cq;
  Fetch<T, 16 * W, W * WAVE> cv;
  // of the record: T, P and the gates as one, or T and the gates
  Copy<MODE == WALK ? L::V - L::T_ : frag_bytes<T>(PARTS), W * WAVE> ct;
  Copy<WALK_GATES * C * 4, W * WAVE> cg;
  auto fetch = [&](int chunk) {
    const int live = end - chunk * C;
    ck.load(p.k, (int64_t)chunk * C, b, hk, 0, live);
    if (MODE == WALK) cq.load(p.q, (int64_t)chunk * C, b, hk, 0, live);
    if (!unit) cv.load(p.v, (int64_t)chunk * C, b, h, c0, live);
    const char* rec = p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES;
    ct.load(rec + R::T_);
    if (MODE != WALK) cg.load(rec + R::GATE);
  };
  auto keep = [&](int chunk) {
    if (MODE == WALK && p.states && chunk % p.keep == 0 && there)
      store_state(S, p.states + ((int64_t)(chunk / p.keep) * BH + bh) * p.dk * p.dv, p.dk, p.dv, col, g);
  };
  auto y_of = [&](int chunk) { return (T*)p.y.data + (int64_t)(chunk * C) * p.y.stride_t + b * p.y.stride_b + h * p.dv; };
  const int dead = max(first, min(behind, (end + C - 1) / C));   // the first chunk behind the sequence's end
  if (first < dead) fetch(first);
  for (int chunk = first; chunk < dead; ++chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    keep(chunk);
    if (MODE == AGAIN && col < p.dvp) store_state(S, p.S + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp, KD, p.dvp, col, g);
    __syncthreads();   // the chunk before has been read
    ck.put(K, p.k, 0, live);
    ct.put(lds + L::T_);
    if (MODE == WALK) cq.put(Q, p.q, 0, live);
    else cg.put(lds + L::GATE);
    if (!unit) cv.put(VL, p.v, c0, live);
    __syncthreads();
    fetch(min(chunk + 1, dead - 1));   // (not under a condition, see there)
    next_product();

    // K S and Q S: tiles 0 .. 3 and 4 .. 7
    constexpr int ROWS = MODE ? 4 : 8;
    f32x4 KQ[ROWS] = {};
    auto rows = [&](Op<T, 1>(&o)[4], int rt0, int n) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) o[rt] = from_row((rt0 ? Q : K) + (16 * rt + lane % 16) * LD + 32 * n, g);
    };
    if constexpr (DEEP) {   // operands a product ahead, and cut while it runs
      Op<T, 1> a[2][ROWS / 4][4];
      Op<T, 3> s[2];
#pragma unroll
      for (int r = 0; r < ROWS; r += 4) rows(a[0][r / 4], r, 0);
      s[0] = cut<T, 3>(S[0], S[1]);
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) {
        if (n + 1 < NT / 2) {
#pragma unroll
          for (int r = 0; r < ROWS; r += 4) rows(a[(n + 1) % 2][r / 4], r, n + 1);
        }
        next_product();
        if constexpr (sizeof(T) == 2) {
          if (n + 1 < NT / 2) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = S[2 * n + 2][e], x[4 + e] = S[2 * n + 3][e];
#pragma unroll
            for (int r = 0; r < ROWS; r += 4) mma_and_cut(KQ, a[n % 2][r / 4], s[n % 2], r, x, s[(n + 1) % 2], ROWS == 8 ? r / 4 * 6 : 0, ROWS == 8 ? 2 : 1);
            next_product();
            continue;
          }
        }
#pragma unroll
        for (int r = 0; r < ROWS; r += 4) mma(KQ, a[n % 2][r / 4], s[n % 2], r);
        if (n + 1 < NT / 2) s[(n + 1) % 2] = cut<T, 3>(S[2 * n + 2], S[2 * n + 3]);
        next_product();
      }
    } else {
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) {
        Op<T, 1> a[4];
        rows(a, 0, n);
        const Op<T, 3> s = cut<T, 3>(S[2 * n], S[2 * n + 1]);
        mma(KQ, a, s);
        if constexpr (MODE == WALK) {
          rows(a, 4, n);
          mma(KQ, a, s, 4);
        }
        next_product();
      }
    }
    f32x4 X[4] = {};
    if (!unit) load_tiles<Lds<T>::ld(16 * W)>(X, VL, 16 * wave, lane);
    f32x4 U[4] = {};
    {
      Op<T, PARTS> t0[4], t1[2];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) t0[rt] = from_frag<T, PARTS>(lds + L::T_, lower(rt, 0), lane);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) X[rt] -= steps_of(gate, GA_SK, rt, g) * KQ[rt];
      next_product();
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) t1[rt] = from_frag<T, PARTS>(lds + L::T_, lower(2 + rt, 1), lane);
      mma(U, t0, cut<T, 3>(X[0], X[1]));
      next_product();
      mma(U, t1, cut<T, 3>(X[2], X[3]), 2);
    }
    Op<T, 1> columns[DEEP ? 2 : 1][NT];
    auto fetch_columns = [&](int pb) {
#pragma unroll
      for (int n = 0; n < NT; ++n) columns[DEEP ? pb : 0][n] = from_columns<LD>(K, 16 * n, 32 * pb, lane);
    };
    if (MODE == AGAIN && col < p.dvp) store_state(U, p.R + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp, C, p.dvp, col, g);
    if constexpr (MODE == WALK) {
      f32x4 Y[4];
      Op<T, PARTS> p0[4], p1[2];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) p0[rt] = from_frag<T, PARTS>(lds + L::P, lower(rt, 0), lane);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        Y[rt] = steps_of(gate, GA_SQ, rt, g) * KQ[4 + rt];
        U[rt] *= steps_of(gate, BE, rt, g);
      }
      if (DEEP) next_product();
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) p1[rt] = from_frag<T, PARTS>(lds + L::P, lower(2 + rt, 1), lane);
      mma(Y, p0, cut<T, PARTS>(U[0], U[1]));
      next_product();
      if (DEEP) fetch_columns(0);
      mma(Y, p1, cut<T, PARTS>(U[2], U[3]), 2);
      store_tiles(y_of(chunk), (int)p.y.stride_t, Y, steps, live, c0 + 16 * wave, p.dv, p.vec_out, reinterpret_cast<T*>(lds + L::Y) + wave * TURN, lane);
      next_product();
    } else {
      if (DEEP) fetch_columns(0);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, BE, rt, g);
    }
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, LA_SK, rt, g);
#pragma unroll
    for (int n = 0; n < NT; ++n) S[n] *= last;
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      if (!DEEP || pb == 0) fetch_columns(DEEP ? 1 : pb);
      mma(S, columns[DEEP ? pb : 0], cut<T, 3>(U[2 * pb], U[2 * pb + 1]));
      next_product();
    }
  }
  if constexpr (MODE == WALK) {   // zeros, the state stays
    for (int chunk = dead; chunk < behind; ++chunk) {
      keep(chunk);
      store_zeros(y_of(chunk), p.y.stride_t, min(p.t - chunk * C, C), col, p.dv, g);
    }
  }
  if constexpr (MODE == SURVEY) {
    const int64_t at = (int64_t)segment * BH + bh;
    if (unit && col < KD) store_state(S, p.moves + at * KD * KD, KD, KD, col, g);
    if (!unit && col < p.dvp) store_state(S, p.ends + at * KD * p.dvp, KD, p.dvp, col, g);
  } else if (p.to && there && behind == p.c1) {
    store_state(S, p.to + (int64_t)bh * p.dk * p.dv, p.dk, p.dv, col, g);
  }
}

// ---- back ----------------------------------------------------------------------------------------------

template <typename T, int KD, int W>
struct BackLayout {   // of LDS: the record's part from T^T on as it is
  using R = Record<T, true>;
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), REC = Q + Lds<T>::row_bytes(KD), RBYTES = R::GATE + WALK_GATES * C * 4 - R::TT,
                       T_ = REC, P = REC + R::P - R::TT, GATE = REC + R::GATE - R::TT, N = REC + RBYTES, Y = N + Lds<T>::row_bytes(16 * W),
                       BYTES = sizeof(T) == 4 ? Y : Y + W * TURN * 2;
};

template <typename T, int KD, int W>
__global__ __launch_bounds__(W* WAVE, (per_simd<KD, W, WALK>())) void delta_walk_back_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = BackLayout<T, KD, W>;
  using R = Record<T, true>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  constexpr bool DEEP = per_simd<KD, W, WALK>() == 1;
  T *K = reinterpret_cast<T*>(lds + L::K), *Q = reinterpret_cast<T*>(lds + L::Q), *NL = reinterpret_cast<T*>(lds + L::N);
  const float* gate = reinterpret_cast<const float*>(lds + L::GATE);
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE, g = lane / 16;
  const int c0 = blockIdx.y * W * 16, col = c0 + 16 * wave + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b);

  f32x4 S[NT];   // gradient of the state behind the chunk
  load_state(S, p.from ? p.from + (int64_t)bh * p.dk * p.dv : nullptr, p.dk, p.dv, col, g);

  Fetch<T, KD, W * WAVE> ck, cq;
  Fetch<T, 16 * W, W * WAVE> cn;
  Copy<L::RBYTES, W * WAVE> cr;
  auto fetch = [&](int chunk) {
    const int live = end - chunk * C;
    ck.load(p.k, (int64_t)chunk * C, b, hk, 0, live);
    cq.load(p.q, (int64_t)chunk * C, b, hk, 0, live);
    cn.load(p.dy, (int64_t)chunk * C, b, h, c0, live);
    cr.load(p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES + R::TT);
  };
  if (p.c0 < p.c1) fetch(p.c1 - 1);
  for (int chunk = p.c1 - 1; chunk >= p.c0; --chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    T* dv = (T*)p.dval.data + (int64_t)s0 * p.dval.stride_t + b * p.dval.stride_b + h * p.dv;
    if (live <= 0) {
      store_zeros(dv, p.dval.stride_t, steps, col, p.dv, g);
      fetch(max(chunk - 1, p.c0));
      continue;
    }
    if (col < p.dvp) store_state(S, p.dS + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp, KD, p.dvp, col, g);
    __syncthreads();   // the chunk before has been read
    ck.put(K, p.k, 0, live);
    cq.put(Q, p.q, 0, live);
    cr.put(lds + L::REC);
    cn.put(NL, p.dy, c0, live);
    __syncthreads();
    fetch(max(chunk - 1, p.c0));   // (not under a condition, see there)
    next_product();

    f32x4 U[4] = {};
    {
      Op<T, 1> a[2][4];
      Op<T, 3> x[2];
      auto rows = [&](Op<T, 1>(&o)[4], int n) {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) o[rt] = from_row(K + (16 * rt + lane % 16) * LD + 32 * n, g);
      };
      rows(a[0], 0);
      x[0] = cut<T, 3>(S[0], S[1]);
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) {
        if (n + 1 < NT / 2) rows(a[(n + 1) % 2], n + 1);
        next_product();
        mma(U, a[n % 2], x[n % 2]);
        if (n + 1 < NT / 2) x[(n + 1) % 2] = cut<T, 3>(S[2 * n + 2], S[2 * n + 3]);
        next_product();
      }
    }
    f32x4 dY[4];
    load_tiles<Lds<T>::ld(16 * W)>(dY, NL, 16 * wave, lane);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, LA_SK, rt, g);
    {
      Op<T, PARTS> p0[2], p1[4];
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) p0[rt] = from_frag<T, PARTS>(lds + L::P, upper(rt, 0), lane);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) p1[rt] = from_frag<T, PARTS>(lds + L::P, upper(rt, 1), lane);
      mma(U, p0, cut<T, 1>(dY[0], dY[1]));   // (exact: dY has T's bits)
      mma(U, p1, cut<T, 1>(dY[2], dY[3]));
      next_product();
    }
    f32x4 Z[4] = {};
    {
      Op<T, PARTS> t0[2], t1[4];
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) t0[rt] = from_frag<T, PARTS>(lds + L::T_, upper(rt, 0), lane);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) t1[rt] = from_frag<T, PARTS>(lds + L::T_, upper(rt, 1), lane);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, BE, rt, g);
      mma(Z, t0, cut<T, 3>(U[0], U[1]));
      mma(Z, t1, cut<T, 3>(U[2], U[3]));
      next_product();
    }
    if (col < p.dvp) store_state(Z, p.Z + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp, C, p.dvp, col, g);
    store_tiles(dv, (int)p.dval.stride_t, Z, steps, live, c0 + 16 * wave, p.dv, p.vec_out, reinterpret_cast<T*>(lds + L::Y) + wave * TURN, lane);
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) S[n] *= last;
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
      dY[rt] *= steps_of(gate, GA_SQ, rt, g);
      Z[rt] *= -steps_of(gate, GA_SK, rt, g);
    }
    {
      Op<T, 1> a[DEEP ? 2 : 1][NT];   // columns of q, of k, the first 32 steps, then the others
      auto columns = [&](int i) {
#pragma unroll
        for (int n = 0; n < NT; ++n) a[DEEP ? i % 2 : 0][n] = from_columns<LD>(i % 2 ? K : Q, 16 * n, 32 * (i / 2), lane);
      };
      if (DEEP) columns(0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!DEEP) columns(i);
        else if (i < 3) columns(i + 1);
        if (DEEP) next_product();
        mma(S, a[DEEP ? i % 2 : 0], i % 2 ? cut<T, 3>(Z[i - 1], Z[i]) : cut<T, 3>(dY[i], dY[i + 1]));
        next_product();
      }
    }
  }
  if (p.to && there) store_state(S, p.to + (int64_t)bh * p.dk * p.dv, p.dk, p.dv, col, g);
}

// ---- segments ------------------------------------------------------------------------------------------

// States before all segments but the first, one after another: S <- A S + B.  A wave has 16 rows of 16 columns, waves give each other theirs in LDS.
template <int KD>
__global__ __launch_bounds__(KD * 4) void delta_join_segments_kernel(Args p, int segments) {
  constexpr int NT = KD / 16, LD = 20;
  __shared__ __align__(16) float S[2][KD][LD];
  const int bh = blockIdx.x, BH = p.B * p.H, wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16, c16 = lane % 16;
  const int c0 = blockIdx.y * 16;
  const unsigned off = (unsigned)((16 * wave + 4 * g) * p.dvp + c0 + c16), row = (unsigned)((16 * wave + c16) * KD + 4 * g);
  f32x4 x, A[NT] = {};
  auto of = [&](const float* m, int s) { return m + ((int64_t)s * BH + bh) * KD * p.dvp; };
  auto rows = [&](int s) {
#pragma unroll
    for (int n = 0; n < NT; ++n) A[n] = *reinterpret_cast<const f32x4*>(p.moves + ((int64_t)s * BH + bh) * KD * KD + row + 16 * n);
  };
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = of(p.ends, 0)[off + e * p.dvp];
  if (segments > 2) rows(1);
  for (int s = 0; s + 1 < segments; ++s) {
    if (s) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = of(p.ends, s)[off + e * p.dvp];
      f32x4 sum[2] = {};
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[n % 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[n][e], S[s % 2][16 * n + 4 * g + e][c16], sum[n % 2], 0, 0, 0);
      x = y + (sum[0] + sum[1]);
      rows(min(s + 1, segments - 2));
    }
    float* to = p.starts + ((int64_t)(s + 1) * BH + bh) * KD * p.dvp;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      to[off + e * p.dvp] = x[e];
      S[(s + 1) % 2][16 * wave + 4 * g + e][c16] = x[e];
    }
    __syncthreads();
  }
}

// ---- launches ------------------------------------------------------------------------------------------

template <auto Kernel>
int launch(const Args& p, int W, int bytes, const char* what, hipStream_t stream, int columns, int segments = 1) {
  const hipError_t e = allow_dynamic_lds<Kernel>(bytes);
  if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
  const dim3 grid((unsigned)(p.B * p.H), (unsigned)columns, (unsigned)segments);
  Kernel<<<grid, W * WAVE, bytes, stream>>>(p);
  return launched(what);
}

// 128 columns in one workgroup, which reads a chunk once and whose waves hide each other's latencies; in two, whose waves fetch operands ahead, where there
// are compute units for both (10000 x 1 x 16 heads of 128 x 128 in eight segments: 165 us with eight waves, 102 with four).
bool eight_waves(const Args& p, int segments) { return p.dv > 64 && (int64_t)p.B * p.H * segments > 128; }

template <typename T, int KD, int W>
int forward(const Args& p, int mode, int segments, hipStream_t stream) {
  const int columns = (int)ceil_div(p.dv, 16 * W);
  if (mode == WALK) return launch<delta_walk_kernel<T, KD, W, WALK>>(p, W, Layout<T, KD, W, WALK>::BYTES, "delta rule, forward", stream, columns, segments);
  return launch<delta_walk_kernel<T, KD, W, AGAIN>>(p, W, Layout<T, KD, W, AGAIN>::BYTES, "delta rule, recomputation", stream, columns, segments);
}

}  // namespace

int mebptt::delta::walk(const Args& p, int dtype, int mode, hipStream_t stream) {
  const int segments = (int)std::max<int64_t>(1, ceil_div(p.c1 - p.c0, p.seg));
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    if (mode == SURVEY) {   // (of the last segment nothing has to be known)
      const int columns = (int)ceil_div(p.dv, 64) + (int)ceil_div(KD, 64);
      return launch<delta_walk_kernel<T, KD, 4, SURVEY>>(p, 4, Layout<T, KD, 4, SURVEY>::BYTES, "delta rule, survey", stream, columns, segments - 1);
    }
    return eight_waves(p, segments) ? forward<T, KD, 8>(p, mode, segments, stream) : forward<T, KD, 4>(p, mode, segments, stream);
  });
}

int mebptt::delta::join_segments(const Args& p, int dtype, hipStream_t stream) {
  const int segments = (int)ceil_div(p.c1 - p.c0, p.seg);
  return with_size(dtype, p.dk, [&](auto, auto n) {
    constexpr int KD = decltype(n)::value;
    delta_join_segments_kernel<KD><<<dim3((unsigned)(p.B * p.H), (unsigned)(p.dvp / 16)), KD * 4, 0, stream>>>(p, segments);
    return launched("delta rule, segments");
  });
}

int mebptt::delta::walk_back(const Args& p, int dtype, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    if (eight_waves(p, 1)) return launch<delta_walk_back_kernel<T, KD, 8>>(p, 8, BackLayout<T, KD, 8>::BYTES, "delta rule, back", stream, (int)ceil_div(p.dv, 128));
    return launch<delta_walk_back_kernel<T, KD, 4>>(p, 4, BackLayout<T, KD, 4>::BYTES, "delta rule, back", stream, (int)ceil_div(p.dv, 64));
  });
}
