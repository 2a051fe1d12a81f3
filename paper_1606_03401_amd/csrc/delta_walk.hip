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

template <typename T, int KD, int W, bool ROWS, bool COLUMNS>
struct Chunk {   // pieces of [C][KD] of one of the inputs
  static constexpr int N = (pieces<T>(KD) + W * WAVE - 1) / (W * WAVE);
  Piece<T> x[N];
  __device__ inline void load(const T* p, int64_t stride, int width, int live, bool vec) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * W * WAVE + (int)threadIdx.x;
      if (u < pieces<T>(KD)) load_piece<T, KD>(x[i], p, stride, width, live, vec, u);
    }
  }
  __device__ inline void put(T* rows, T* columns) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * W * WAVE + (int)threadIdx.x;
      if (u < pieces<T>(KD)) {
        if constexpr (ROWS || sizeof(T) == 4) put_rows<T, KD>(x[i], rows, u);
        if constexpr (COLUMNS) put_columns<T, KD>(x[i], columns, u);
      }
    }
  }
};

template <typename T, int KD, bool BACK>
struct Layout {   // of LDS
  static constexpr int K = 0;
  static constexpr int KT = K + Lds<T>::row_bytes(KD);
  static constexpr int Q = KT + Lds<T>::column_bytes(KD);    // forward (and fp32): rows; backward: columns
  static constexpr int REC = Q + (BACK && sizeof(T) == 2 ? Lds<T>::column_bytes(KD) : Lds<T>::row_bytes(KD));
  using R = Record<T, BACK>;
  static constexpr int FROM = BACK ? R::TT : R::T_;          // of the record
  static constexpr int TO = R::SUMS;
  static constexpr int BYTES = REC + TO - FROM;
};

// [rt][e] is step 16 rt + 4 g + e of a column, zero where `inside` is not set.
template <typename T>
__device__ inline void load_column(f32x4 (&v)[4], const T* p, int64_t stride, int live, bool inside, int g) {
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int s = 16 * rt + 4 * g + e;
      v[rt][e] = inside && s < live ? (float)p[(int64_t)s * stride] : 0.0f;
    }
}

// ---- forward -------------------------------------------------------------------------------------------

template <typename T, int KD, int W, bool AGAIN>
__global__ __launch_bounds__(W* WAVE) void delta_walk_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD, AGAIN>;
  // (a second walk has the backward pass's records: T and the gates, without the matrices between them)
  using R = Record<T, AGAIN>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  constexpr int TBYTES = frag_bytes<T>(T_PARTS), PBYTES = AGAIN ? 0 : frag_bytes<T>(P_PARTS), GBYTES = GATES * C * 4;
  T* K = reinterpret_cast<T*>(lds);
  T* KT = reinterpret_cast<T*>(lds + L::KT);
  T* Q = reinterpret_cast<T*>(lds + L::Q);
  char* Tm = lds + (AGAIN ? L::Q : L::REC);
  char* Pm = Tm + TBYTES;
  const float* gate = reinterpret_cast<const float*>(Pm + PBYTES);
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16;
  const int col = (blockIdx.y * W + wave) * 16 + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b);

  f32x4 S[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 16 * n + 4 * g + e;
      S[n][e] = p.from && there && d < p.dk ? p.from[((int64_t)bh * p.dk + d) * p.dv + col] : 0.0f;
    }

  Chunk<T, KD, W, true, true> ck;
  Chunk<T, KD, W, true, false> cq;
  Copy<TBYTES, W * WAVE> ct;
  Copy<AGAIN ? 16 : PBYTES, W * WAVE> cp;
  Copy<GBYTES, W * WAVE> cg;
  f32x4 V[4];
  auto fetch = [&](int chunk) {
    const int64_t s0 = (int64_t)chunk * C;
    const int live = min(end - chunk * C, C);
    if (live <= 0) return;
    ck.load((const T*)p.k.data + s0 * p.k.stride_t + b * p.k.stride_b + hk * p.dk, p.k.stride_t, p.dk, live, p.vec);
    if (!AGAIN) cq.load((const T*)p.q.data + s0 * p.q.stride_t + b * p.q.stride_b + hk * p.dk, p.q.stride_t, p.dk, live, p.vec);
    const char* rec = p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES;
    ct.load(rec + R::T_);
    if (!AGAIN) cp.load(rec + R::P);
    cg.load(rec + R::GATE);
    load_column(V, (const T*)p.v.data + s0 * p.v.stride_t + b * p.v.stride_b + h * p.dv + col, p.v.stride_t, live, there, g);
  };
  if (p.c0 < p.c1) fetch(p.c0);
  for (int chunk = p.c0; chunk < p.c1; ++chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    if (p.states && chunk % p.keep == 0 && there) {
      float* to = p.states + ((int64_t)(chunk / p.keep) * BH + bh) * p.dk * p.dv + col;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 16 * n + 4 * g + e;
          if (d < p.dk) to[(int64_t)d * p.dv] = S[n][e];
        }
    }
    T* y = AGAIN ? nullptr : (T*)p.y.data + (int64_t)s0 * p.y.stride_t + b * p.y.stride_b + h * p.dv + col;
    if (live <= 0) {   // behind the sequence's end: zeros, the state stays
      if (!AGAIN && there)
        for (int s = g; s < steps; s += 4) y[(int64_t)s * p.y.stride_t] = (T)0.0f;
      continue;
    }
    if (AGAIN && col < p.dvp) {
      float* to = p.S + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp + col;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(16 * n + 4 * g + e) * p.dvp] = S[n][e];
    }
    __syncthreads();   // the chunk before has been read
    ck.put(K, KT);
    ct.put(Tm);
    if (!AGAIN) cq.put(Q, nullptr), cp.put(Pm);
    cg.put(const_cast<char*>(reinterpret_cast<const char*>(gate)));
    f32x4 X[4];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) X[rt] = V[rt];
    __syncthreads();
    if (chunk + 1 < p.c1) fetch(chunk + 1);

    Op<T, 3> Sp[NT / 2];
#pragma unroll
    for (int n = 0; n < NT / 2; ++n) Sp[n] = cut<T, 3>(S[2 * n], S[2 * n + 1]);
    f32x4 Y[4];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
      f32x4 x = {}, z = {};
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) mma(x, from_row(K + (16 * rt + lane % 16) * LD + 32 * n, g), Sp[n]);
      const f32x4 ga = *reinterpret_cast<const f32x4*>(gate + GA * C + 16 * rt + 4 * g);
      const f32x4 sk = *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
      X[rt] -= ga * sk * x;
      if constexpr (!AGAIN) {
#pragma unroll
        for (int n = 0; n < NT / 2; ++n) mma(z, from_row(Q + (16 * rt + lane % 16) * LD + 32 * n, g), Sp[n]);
        const f32x4 sq = *reinterpret_cast<const f32x4*>(gate + SQ * C + 16 * rt + 4 * g);
        Y[rt] = ga * sq * z;
      }
    }
    f32x4 U[4];
    {
      const Op<T, 3> Xp[2] = {cut<T, 3>(X[0], X[1]), cut<T, 3>(X[2], X[3])};
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4 r = {};
#pragma unroll
        for (int pb = 0; pb <= rt / 2; ++pb) mma(r, from_frag<T, T_PARTS>(Tm, lower(rt, pb), lane), Xp[pb]);
        U[rt] = r;
      }
    }
    if (AGAIN && col < p.dvp) {
      float* to = p.R + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp + col;
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(16 * rt + 4 * g + e) * p.dvp] = U[rt][e];
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) U[rt] *= *reinterpret_cast<const f32x4*>(gate + BE * C + 16 * rt + 4 * g);
    if constexpr (!AGAIN) {
      const Op<T, 2> Up[2] = {cut<T, 2>(U[0], U[1]), cut<T, 2>(U[2], U[3])};
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
#pragma unroll
        for (int pb = 0; pb <= rt / 2; ++pb) mma(Y[rt], from_frag<T, P_PARTS>(Pm, lower(rt, pb), lane), Up[pb]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int s = 16 * rt + 4 * g + e;
          if (there && s < steps) y[(int64_t)s * p.y.stride_t] = (T)(s < live ? Y[rt][e] : 0.0f);
        }
      }
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
      U[rt] *= *reinterpret_cast<const f32x4*>(gate + LA * C + 16 * rt + 4 * g) * *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
    const Op<T, 3> Up[2] = {cut<T, 3>(U[0], U[1]), cut<T, 3>(U[2], U[3])};
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      S[n] *= last;
#pragma unroll
      for (int pb = 0; pb < 2; ++pb) mma(S[n], from_column<KD>(K, KT, 16 * n + lane % 16, 32 * pb, g), Up[pb]);
    }
  }
  if (p.to && there) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = 16 * n + 4 * g + e;
        if (d < p.dk) p.to[((int64_t)bh * p.dk + d) * p.dv + col] = S[n][e];
      }
  }
}

// ---- back ----------------------------------------------------------------------------------------------

template <typename T, int KD, int W>
__global__ __launch_bounds__(W* WAVE) void delta_walk_back_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD, true>;
  using R = Record<T, true>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16;
  T* K = reinterpret_cast<T*>(lds);
  T* KT = reinterpret_cast<T*>(lds + L::KT);
  T* Q = reinterpret_cast<T*>(lds + L::Q);
  char* Tm = lds + L::REC;
  char* Pm = Tm + (R::P - L::FROM);
  const float* gate = reinterpret_cast<const float*>(Tm + (R::GATE - L::FROM));
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk), BH = p.B * p.H;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16;
  const int col = (blockIdx.y * W + wave) * 16 + lane % 16;
  const bool there = col < p.dv;
  const int end = ends_at(p, b);

  f32x4 S[NT];   // gradient of the state behind the chunk
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 16 * n + 4 * g + e;
      S[n][e] = p.from && there && d < p.dk ? p.from[((int64_t)bh * p.dk + d) * p.dv + col] : 0.0f;
    }

  Chunk<T, KD, W, true, true> ck;
  Chunk<T, KD, W, false, true> cq;
  Copy<L::TO - L::FROM, W * WAVE> cr;
  f32x4 N[4];
  auto fetch = [&](int chunk) {
    const int64_t s0 = (int64_t)chunk * C;
    const int live = min(end - chunk * C, C);
    if (live <= 0) return;
    ck.load((const T*)p.k.data + s0 * p.k.stride_t + b * p.k.stride_b + hk * p.dk, p.k.stride_t, p.dk, live, p.vec);
    cq.load((const T*)p.q.data + s0 * p.q.stride_t + b * p.q.stride_b + hk * p.dk, p.q.stride_t, p.dk, live, p.vec);
    cr.load(p.records + ((int64_t)(chunk - p.c0) * BH + bh) * R::BYTES + L::FROM);
    load_column(N, (const T*)p.dy.data + s0 * p.dy.stride_t + b * p.dy.stride_b + h * p.dv + col, p.dy.stride_t, live, there, g);
  };
  if (p.c0 < p.c1) fetch(p.c1 - 1);
  for (int chunk = p.c1 - 1; chunk >= p.c0; --chunk) {
    const int s0 = chunk * C, live = min(end - s0, C), steps = min(p.t - s0, C);
    T* dv = (T*)p.dval.data + (int64_t)s0 * p.dval.stride_t + b * p.dval.stride_b + h * p.dv + col;
    if (live <= 0) {
      if (there)
        for (int s = g; s < steps; s += 4) dv[(int64_t)s * p.dval.stride_t] = (T)0.0f;
      if (chunk > p.c0) fetch(chunk - 1);
      continue;
    }
    if (col < p.dvp) {
      float* to = p.dS + ((int64_t)(chunk - p.c0) * BH + bh) * KD * p.dvp + col;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(16 * n + 4 * g + e) * p.dvp] = S[n][e];
    }
    __syncthreads();
    ck.put(K, KT);
    cq.put(Q, Q);
    cr.put(Tm);
    f32x4 dY[4];
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) dY[rt] = N[rt];
    __syncthreads();
    if (chunk > p.c0) fetch(chunk - 1);

    f32x4 Z[4];
    {
      Op<T, 3> Sp[NT / 2];
#pragma unroll
      for (int n = 0; n < NT / 2; ++n) Sp[n] = cut<T, 3>(S[2 * n], S[2 * n + 1]);
      const Op<T, 1> Yp[2] = {cut<T, 1>(dY[0], dY[1]), cut<T, 1>(dY[2], dY[3])};   // (exact: dY has T's bits)
      f32x4 U[4];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4 u = {};
#pragma unroll
        for (int n = 0; n < NT / 2; ++n) mma(u, from_row(K + (16 * rt + lane % 16) * LD + 32 * n, g), Sp[n]);
        u *= *reinterpret_cast<const f32x4*>(gate + LA * C + 16 * rt + 4 * g) * *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
#pragma unroll
        for (int pb = rt / 2; pb < 2; ++pb) mma(u, from_frag<T, PT_PARTS>(Pm, upper(rt, pb), lane), Yp[pb]);
        U[rt] = u * *reinterpret_cast<const f32x4*>(gate + BE * C + 16 * rt + 4 * g);
      }
      const Op<T, 3> Up[2] = {cut<T, 3>(U[0], U[1]), cut<T, 3>(U[2], U[3])};
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4 z = {};
#pragma unroll
        for (int pb = rt / 2; pb < 2; ++pb) mma(z, from_frag<T, T_PARTS>(Tm, upper(rt, pb), lane), Up[pb]);
        Z[rt] = z;
      }
    }
    if (col < p.dvp) {
      float* to = p.Z + ((int64_t)(chunk - p.c0) * BH + bh) * C * p.dvp + col;
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int s = 16 * rt + 4 * g + e;
          to[s * p.dvp] = Z[rt][e];
          if (there && s < steps) dv[(int64_t)s * p.dval.stride_t] = (T)(s < live ? Z[rt][e] : 0.0f);
        }
    }
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) {
      const f32x4 ga = *reinterpret_cast<const f32x4*>(gate + GA * C + 16 * rt + 4 * g);
      dY[rt] *= ga * *reinterpret_cast<const f32x4*>(gate + SQ * C + 16 * rt + 4 * g);
      Z[rt] *= -ga * *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
    }
    const Op<T, 3> Yp[2] = {cut<T, 3>(dY[0], dY[1]), cut<T, 3>(dY[2], dY[3])};
    const Op<T, 3> Zp[2] = {cut<T, 3>(Z[0], Z[1]), cut<T, 3>(Z[2], Z[3])};
    const float last = gate[GA * C + C - 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      S[n] *= last;
#pragma unroll
      for (int pb = 0; pb < 2; ++pb) {
        mma(S[n], from_column<KD>(Q, Q, 16 * n + lane % 16, 32 * pb, g), Yp[pb]);
        mma(S[n], from_column<KD>(K, KT, 16 * n + lane % 16, 32 * pb, g), Zp[pb]);
      }
    }
  }
  if (p.to && there) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = 16 * n + 4 * g + e;
        if (d < p.dk) p.to[((int64_t)bh * p.dk + d) * p.dv + col] = S[n][e];
      }
  }
}

template <auto Kernel>
int launch(const Args& p, int W, int bytes, const char* what, hipStream_t stream) {
  const hipError_t e = allow_dynamic_lds<Kernel>(bytes);
  if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
  const dim3 grid((unsigned)(p.B * p.H), (unsigned)ceil_div(p.dv, 16 * W));
  Kernel<<<grid, W * WAVE, bytes, stream>>>(p);
  return launched(what);
}

template <typename T, int KD, int W>
int forward(const Args& p, bool again, hipStream_t stream) {
  if (!again) return launch<delta_walk_kernel<T, KD, W, false>>(p, W, Layout<T, KD, false>::BYTES, "delta rule, forward", stream);
  constexpr int BYTES = Layout<T, KD, true>::Q + frag_bytes<T>(T_PARTS) + GATES * C * 4;
  return launch<delta_walk_kernel<T, KD, W, true>>(p, W, BYTES, "delta rule, recomputation", stream);
}

}  // namespace

int mebptt::delta::walk(const Args& p, int dtype, bool again, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) { return forward<decltype(t), decltype(n)::value, 4>(p, again, stream); });
}

int mebptt::delta::walk_back(const Args& p, int dtype, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    return launch<delta_walk_back_kernel<T, KD, 4>>(p, 4, Layout<T, KD, true>::BYTES, "delta rule, back", stream);
  });
}
