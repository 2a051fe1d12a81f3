// Gated delta rule: the walks over a launch's chunks, forward and back.  A workgroup of W waves owns 16 W of the state's columns for one sequence and
// head, a wave 16 of them: all rows of the state in its registers, and with them everything that is computed in these columns.  Waves share a
// chunk's keys, queries and matrices in LDS, nothing else.
#include "delta.h"
#include "dynamic_lds.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

// A record's [bytes] from one place to LDS, by way of registers.
template <int BYTES, int THREADS>
struct Copy {
  static constexpr int N = (BYTES / 16 + THREADS - 1) / THREADS;
  u32x4 v[N];
  __device__ inline void load(const char* from) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * THREADS + (int)threadIdx.x;
      if (N * THREADS * 16 == BYTES || u * 16 < BYTES) v[i] = *reinterpret_cast<const u32x4*>(from + u * 16);
    }
  }
  __device__ inline void put(char* to) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * THREADS + (int)threadIdx.x;
      if (N * THREADS * 16 == BYTES || u * 16 < BYTES) *reinterpret_cast<u32x4*>(to + u * 16) = v[i];
    }
  }
};

template <typename T, int KD, int W>
struct Chunk {   // [C][KD] of one of the inputs
  static constexpr int N = (pieces<T>(KD) + W * WAVE - 1) / (W * WAVE);
  static constexpr bool ALL = N * W * WAVE == pieces<T>(KD);
  Piece<T> x[N];
  __device__ inline void load(const T* p, const Window& w, int width) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * W * WAVE + (int)threadIdx.x;
      if (ALL || u < pieces<T>(KD)) load_piece<T, KD>(x[i], p, w, width, u);
    }
  }
  __device__ inline void put(T* rows, const Window& w, int width) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * W * WAVE + (int)threadIdx.x;
      if (ALL || u < pieces<T>(KD)) {
        clear_piece<T, KD>(x[i], w, width, u);
        put_rows<T, KD>(x[i], rows, u);
      }
    }
  }
};

// Between a chunk's products: operands of the next one are not to be fetched early, which would take more registers than there are.
__device__ inline void next_product() { __builtin_amdgcn_sched_barrier(0); }

__device__ inline f32x4 steps_of(const float* gate, int row, int rt, int g) { return *reinterpret_cast<const f32x4*>(gate + row * C + 16 * rt + 4 * g); }

// A column of a chunk's rows: [rt][e] is step 16 rt + 4 g + e of column `col`.
template <typename T>
struct Column {
  unsigned v[4][4];   // (a register each: two in one would have to be waited for)
  static __device__ inline unsigned raw(const T* p) {
    if constexpr (sizeof(T) == 2) return *reinterpret_cast<const unsigned short*>(p);
    else return *reinterpret_cast<const unsigned*>(p);
  }
  __device__ inline void load(const T* p, const Window& w, int col, int g) {
    if (w.live >= C) {
      const unsigned off = (unsigned)(4 * g * w.stride + col) * (unsigned)sizeof(T);
      const int64_t stride = here_uniform(w.stride);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[rt][e] = raw(near(p + (16 * rt + e) * stride, off));
    } else {
      const int first = here(4 * g);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[rt][e] = raw(near(p, (unsigned)(min(16 * rt + first + e, w.live - 1) * w.stride + col) * (unsigned)sizeof(T)));
    }
  }
  __device__ inline void get(f32x4 (&x)[4], const Window& w, bool there, int g) const {
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[rt][e] = __uint_as_float(sizeof(T) == 2 ? v[rt][e] << 16 : v[rt][e]);
    if (w.live < C) {
      const int first = here(4 * g);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[rt][e] = 16 * rt + first + e < w.live ? x[rt][e] : 0.0f;
    }
    if (!there) x[0] = x[1] = x[2] = x[3] = f32x4{};
  }
};
// The first `steps` of a column, zeros from `live` on.
template <typename T>
__device__ inline void store_column(T* p, int step, const f32x4 (&x)[4], int steps, int live, int col, int g) {
  const int64_t stride = here_uniform(step);
  const unsigned off = (unsigned)(4 * g * (int)stride + col) * (unsigned)sizeof(T);
  if (live >= C) {
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
      for (int e = 0; e < 4; ++e) *near(p + (16 * rt + e) * stride, off) = (T)x[rt][e];
  } else {
    const int first = here(4 * g);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int s = 16 * rt + first + e;
        if (s < steps) *near(p + (16 * rt + e) * stride, off) = (T)(s < live ? x[rt][e] : 0.0f);
      }
  }
}

// Waves of a SIMD: the registers of one of four waves that hold 128 rows and fetch the next chunk's are more than half.
template <int KD, int W>
constexpr int per_simd() { return W == 4 && KD == 128 ? 1 : 2; }

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

template <typename T, int KD, bool AGAIN>
struct Layout {   // of LDS
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), T_ = AGAIN ? Q : Q + Lds<T>::row_bytes(KD), P = T_ + frag_bytes<T>(T_PARTS),
                       GATE = AGAIN ? P : P + frag_bytes<T>(P_PARTS), BYTES = GATE + WALK_GATES * C * 4;
};

// AGAIN: the backward pass's recomputation, from its records, of S and R of every chunk.
template <typename T, int KD, int W, bool AGAIN>
__global__ __launch_bounds__(W* WAVE, (per_simd<KD, W>())) void delta_walk_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD, AGAIN>;
  using R = Record<T, AGAIN>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  T *K = reinterpret_cast<T*>(lds + L::K), *Q = reinterpret_cast<T*>(lds + L::Q);
  const float* gate = reinterpret_cast<const float*>(lds + L::GATE);
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16;
  const int col = (blockIdx.y * W + wave) * 16 + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b), near_col = min(col, p.dv - 1);

  f32x4 S[NT];
  load_state(S, p.from ? p.from + (int64_t)bh * p.dk * p.dv : nullptr, p.dk, p.dv, col, g);

  Chunk<T, KD, W> ck, cq;
  Copy<frag_bytes<T>(T_PARTS), W * WAVE> ct;
  Copy<frag_bytes<T>(P_PARTS), W * WAVE> cp;
  Copy<WALK_GATES * C * 4, W * WAVE> cg;
  Column<T> V;
  auto fetch = [&](int chunk) {
    const int64_t s0 = (int64_t)chunk * C;
    const int live = min(end - chunk * C, C);
    if (live <= 0) return;
    ck.load((const T*)p.k.data + s0 * p.k.stride_t + b * p.k.stride_b + hk * p.head, Window(p.k.stride_t, live), p.width);
    if (!AGAIN) cq.load((const T*)p.q.data + s0 * p.q.stride_t + b * p.q.stride_b + hk * p.head, Window(p.q.stride_t, live), p.width);
    const char* rec = p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES;
    ct.load(rec + R::T_);
    if (!AGAIN) cp.load(rec + R::P);
    cg.load(rec + R::GATE);
    V.load((const T*)p.v.data + s0 * p.v.stride_t + b * p.v.stride_b + h * p.dv, Window(p.v.stride_t, live), near_col, g);
  };
  if (p.c0 < p.c1) fetch(p.c0);
  for (int chunk = p.c0; chunk < p.c1; ++chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    if (p.states && chunk % p.keep == 0 && there)
      store_state(S, p.states + ((int64_t)(chunk / p.keep) * BH + bh) * p.dk * p.dv, p.dk, p.dv, col, g);
    T* y = AGAIN ? nullptr : (T*)p.y.data + (int64_t)s0 * p.y.stride_t + b * p.y.stride_b + h * p.dv;
    if (live <= 0) {   // behind the sequence's end: zeros, the state stays
      if (!AGAIN && there)
        for (int s = g; s < steps; s += 4) y[(int64_t)s * p.y.stride_t + col] = (T)0.0f;
      continue;
    }
    if (AGAIN && col < p.dvp) store_state(S, p.S + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp, KD, p.dvp, col, g);
    __syncthreads();   // the chunk before has been read
    ck.put(K, Window(p.k.stride_t, live), p.width);
    ct.put(lds + L::T_);
    if (!AGAIN) cq.put(Q, Window(p.q.stride_t, live), p.width), cp.put(lds + L::P);
    cg.put(lds + L::GATE);
    f32x4 X[4];
    V.get(X, Window(p.v.stride_t, live), there, g);
    __syncthreads();
    if (chunk + 1 < p.c1) fetch(chunk + 1);
    next_product();

    f32x4 KS[4] = {}, Y[4] = {};
#pragma unroll
    for (int n = 0; n < NT / 2; ++n) {
      const Op<T, 3> s = cut<T, 3>(S[2 * n], S[2 * n + 1]);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        mma(KS[rt], from_row(K + (16 * rt + lane % 16) * LD + 32 * n, g), s);
        if (!AGAIN) mma(Y[rt], from_row(Q + (16 * rt + lane % 16) * LD + 32 * n, g), s);
      }
      next_product();
    }
    f32x4 U[4] = {};
    {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) X[rt] -= steps_of(gate, GA_SK, rt, g) * KS[rt];
      const Op<T, 3> Xp[2] = {cut<T, 3>(X[0], X[1]), cut<T, 3>(X[2], X[3])};
#pragma unroll
      for (int pb = 0; pb < 2; ++pb)
#pragma unroll
        for (int rt = 2 * pb; rt < 4; ++rt) mma(U[rt], from_frag<T, T_PARTS>(lds + L::T_, lower(rt, pb), lane), Xp[pb]);
    }
    next_product();
    if (AGAIN && col < p.dvp) store_state(U, p.R + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp, C, p.dvp, col, g);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, BE, rt, g);
    if constexpr (!AGAIN) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) Y[rt] *= steps_of(gate, GA_SQ, rt, g);
#pragma unroll
      for (int pb = 0; pb < 2; ++pb) {
        const Op<T, 2> u = cut<T, 2>(U[2 * pb], U[2 * pb + 1]);
#pragma unroll
        for (int rt = 2 * pb; rt < 4; ++rt) mma(Y[rt], from_frag<T, P_PARTS>(lds + L::P, lower(rt, pb), lane), u);
        next_product();
      }
      if (there) store_column(y, (int)p.y.stride_t, Y, steps, live, col, g);
    }
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) S[n] *= last;
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      U[2 * pb] *= steps_of(gate, LA_SK, 2 * pb, g);
      U[2 * pb + 1] *= steps_of(gate, LA_SK, 2 * pb + 1, g);
      const Op<T, 3> u = cut<T, 3>(U[2 * pb], U[2 * pb + 1]);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma(S[n], from_columns<LD>(K, 16 * n, 32 * pb, lane), u);
      next_product();
    }
  }
  if (p.to && there) store_state(S, p.to + (int64_t)bh * p.dk * p.dv, p.dk, p.dv, col, g);
}

// ---- back ----------------------------------------------------------------------------------------------

template <typename T, int KD>
struct BackLayout {   // of LDS: the record's part from T^T on as it is
  using R = Record<T, true>;
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), REC = Q + Lds<T>::row_bytes(KD), RBYTES = R::GATE + WALK_GATES * C * 4 - R::TT,
                       T_ = REC, P = REC + R::P - R::TT, GATE = REC + R::GATE - R::TT, BYTES = REC + RBYTES;
};

template <typename T, int KD, int W>
__global__ __launch_bounds__(W* WAVE, (per_simd<KD, W>())) void delta_walk_back_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = BackLayout<T, KD>;
  using R = Record<T, true>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  T *K = reinterpret_cast<T*>(lds + L::K), *Q = reinterpret_cast<T*>(lds + L::Q);
  const float* gate = reinterpret_cast<const float*>(lds + L::GATE);
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16;
  const int col = (blockIdx.y * W + wave) * 16 + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b), near_col = min(col, p.dv - 1);

  f32x4 S[NT];   // gradient of the state behind the chunk
  load_state(S, p.from ? p.from + (int64_t)bh * p.dk * p.dv : nullptr, p.dk, p.dv, col, g);

  Chunk<T, KD, W> ck, cq;
  Copy<L::RBYTES, W * WAVE> cr;
  Column<T> N;
  auto fetch = [&](int chunk) {
    const int64_t s0 = (int64_t)chunk * C;
    const int live = min(end - chunk * C, C);
    if (live <= 0) return;
    ck.load((const T*)p.k.data + s0 * p.k.stride_t + b * p.k.stride_b + hk * p.head, Window(p.k.stride_t, live), p.width);
    cq.load((const T*)p.q.data + s0 * p.q.stride_t + b * p.q.stride_b + hk * p.head, Window(p.q.stride_t, live), p.width);
    cr.load(p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES + R::TT);
    N.load((const T*)p.dy.data + s0 * p.dy.stride_t + b * p.dy.stride_b + h * p.dv, Window(p.dy.stride_t, live), near_col, g);
  };
  if (p.c0 < p.c1) fetch(p.c1 - 1);
  for (int chunk = p.c1 - 1; chunk >= p.c0; --chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    T* dv = (T*)p.dval.data + (int64_t)s0 * p.dval.stride_t + b * p.dval.stride_b + h * p.dv;
    if (live <= 0) {
      if (there)
        for (int s = g; s < steps; s += 4) dv[(int64_t)s * p.dval.stride_t + col] = (T)0.0f;
      if (chunk > p.c0) fetch(chunk - 1);
      continue;
    }
    if (col < p.dvp) store_state(S, p.dS + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp, KD, p.dvp, col, g);
    __syncthreads();   // the chunk before has been read
    ck.put(K, Window(p.k.stride_t, live), p.width);
    cq.put(Q, Window(p.q.stride_t, live), p.width);
    cr.put(lds + L::REC);
    f32x4 dY[4];
    N.get(dY, Window(p.dy.stride_t, live), there, g);
    __syncthreads();
    if (chunk > p.c0) fetch(chunk - 1);
    next_product();

    f32x4 U[4] = {};
#pragma unroll
    for (int n = 0; n < NT / 2; ++n) {
      const Op<T, 3> s = cut<T, 3>(S[2 * n], S[2 * n + 1]);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) mma(U[rt], from_row(K + (16 * rt + lane % 16) * LD + 32 * n, g), s);
      next_product();
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) U[rt] *= steps_of(gate, LA_SK, rt, g);
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      const Op<T, 1> y = cut<T, 1>(dY[2 * pb], dY[2 * pb + 1]);   // (exact: dY has T's bits)
#pragma unroll
      for (int rt = 0; rt < 2 * pb + 2; ++rt) mma(U[rt], from_frag<T, PT_PARTS>(lds + L::P, upper(rt, pb), lane), y);
      next_product();
    }
    f32x4 Z[4] = {};
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      const Op<T, 3> u = cut<T, 3>(U[2 * pb] * steps_of(gate, BE, 2 * pb, g), U[2 * pb + 1] * steps_of(gate, BE, 2 * pb + 1, g));
#pragma unroll
      for (int rt = 0; rt < 2 * pb + 2; ++rt) mma(Z[rt], from_frag<T, T_PARTS>(lds + L::T_, upper(rt, pb), lane), u);
      next_product();
    }
    if (col < p.dvp) store_state(Z, p.Z + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp, C, p.dvp, col, g);
    if (there) store_column(dv, (int)p.dval.stride_t, Z, steps, live, col, g);
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) S[n] *= last;
#pragma unroll
    for (int pb = 0; pb < 2; ++pb) {
      const Op<T, 3> y = cut<T, 3>(dY[2 * pb] * steps_of(gate, GA_SQ, 2 * pb, g), dY[2 * pb + 1] * steps_of(gate, GA_SQ, 2 * pb + 1, g));
      const Op<T, 3> z = cut<T, 3>(-Z[2 * pb] * steps_of(gate, GA_SK, 2 * pb, g), -Z[2 * pb + 1] * steps_of(gate, GA_SK, 2 * pb + 1, g));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma(S[n], from_columns<LD>(Q, 16 * n, 32 * pb, lane), y);
        mma(S[n], from_columns<LD>(K, 16 * n, 32 * pb, lane), z);
      }
      next_product();
    }
  }
  if (p.to && there) store_state(S, p.to + (int64_t)bh * p.dk * p.dv, p.dk, p.dv, col, g);
}

template <auto Kernel>
int launch(const Args& p, int W, int bytes, const char* what, hipStream_t stream) {
  const hipError_t e = allow_dynamic_lds<Kernel>(bytes);
  if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
  const dim3 grid((unsigned)(p.B * p.H), (unsigned)ceil_div(p.dv, 16 * W));
  Kernel<<<grid, W * WAVE, bytes, stream>>>(p);
  return launched(what);
}

// 128 columns in one workgroup, which reads a chunk once; in two where there are compute units to spare.
bool eight_waves(const Args& p) { return p.dv > 64 && p.B * p.H >= 128; }

template <typename T, int KD, int W>
int forward(const Args& p, bool again, hipStream_t stream) {
  if (!again) return launch<delta_walk_kernel<T, KD, W, false>>(p, W, Layout<T, KD, false>::BYTES, "delta rule, forward", stream);
  return launch<delta_walk_kernel<T, KD, W, true>>(p, W, Layout<T, KD, true>::BYTES, "delta rule, recomputation", stream);
}

}  // namespace

int mebptt::delta::walk(const Args& p, int dtype, bool again, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    return eight_waves(p) ? forward<T, KD, 8>(p, again, stream) : forward<T, KD, 4>(p, again, stream);
  });
}

int mebptt::delta::walk_back(const Args& p, int dtype, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    if (eight_waves(p)) return launch<delta_walk_back_kernel<T, KD, 8>>(p, 8, BackLayout<T, KD>::BYTES, "delta rule, back", stream);
    return launch<delta_walk_back_kernel<T, KD, 4>>(p, 4, BackLayout<T, KD>::BYTES, "delta rule, back", stream);
  });
}
