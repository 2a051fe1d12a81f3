// Gated delta rule: the gradients of a chunk's q, k, a and b, all chunks of a launch at once, from what the two walks left: R, Z and the states
// before and behind the chunk (S, and its gradient dS').  With E = Z R^T below the diagonal,
//     dP = (dY R^T) beta,   dM = -E beta,   W1 = dP o D,   W3 = dM o D,
//     dq~ = W1 K^ + gamma dY S^T,   dk^ = W1^T Q~ + (W3 + W3^T) K^ + beta gamma_C / gamma R dS'^T - gamma Z S^T,
//     dbeta_j = sum_i (P o dY R^T)_ij - sum_i (M o E)_ij + (gamma_C / gamma k^)_j . (R dS'^T)_j,
//     dG_i = sum_j F_ij - sum_j F_ji + q~_i . (gamma dY S^T)_i - k^_i . (gamma Z S^T)_i - e_i,   F = dP o P + dM o M,
//     e_j = beta_j (gamma_C / gamma k^)_j . (R dS'^T)_j,   the last step's dG also sum e + gamma_C <dS', S>,   dg_s = sum_{i >= s} dG_i.
// A workgroup of eight waves has a chunk of a sequence and one key head, and goes through the value heads that share it.  Wave w computes
// 16 columns of dq and dk; in what is 64 x 64, waves 0 .. 3 have column tiles of dY R^T and P, 4 .. 7 those of E and M.
#include "delta.h"
#include "dynamic_lds.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

constexpr int WAVES = 8, THREADS = WAVES * WAVE;
// Parts of R, Z, S and dS' in the products, and of W1 .. W3, which reach dq and dk only.
constexpr int N32 = 3, NW = 2;

template <typename T, int KD>
struct Layout {
  static constexpr int VB = sizeof(T) == 2 ? 64 : 32;     // columns of a block of dY, Z and R
  static constexpr int VLD = VB + Lds<T>::PAD, VSIZE = C * VLD * (int)sizeof(T);
  static constexpr int NV = sizeof(T) == 2 ? N32 : 1;
  static constexpr int WLD = C + Lds<T>::PAD, WSIZE = C * WLD * (int)sizeof(T);
  static constexpr int NM = sizeof(T) == 2 ? NW : 1;
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), BLOCK = Q + Lds<T>::row_bytes(KD);
  static constexpr int DY = BLOCK, Z = DY + VSIZE, R = Z + NV * VSIZE;
  static constexpr int W1 = BLOCK, W2 = W1 + NM * WSIZE, W3 = W2 + NM * WSIZE;      // over the blocks, when they have been read
  static constexpr int SUMS = BLOCK + ((1 + 2 * NV) * VSIZE > 3 * NM * WSIZE ? (1 + 2 * NV) * VSIZE : 3 * NM * WSIZE);
  static constexpr int GATE = SUMS + C * 8, ROWF = GATE + GATES * C * 4, COLS = ROWF + WAVES * C * 4, DOTS = COLS + 4 * C * 4,
                       MORE = DOTS + 2 * WAVES * C * 4, BYTES = MORE + WAVES * 4;
};

// An operand with N parts whose row stands at p; parts `apart` values from each other.
template <int N>
__device__ inline Op<__bf16, N> from_parts(const __bf16* p, int apart, int g) {
  Op<__bf16, N> o;
#pragma unroll
  for (int n = 0; n < N; ++n) o.p[n] = from_row(p + n * apart, g).p[0];
  return o;
}
template <int N>
__device__ inline Op<float, N> from_parts(const float* p, int, int g) {
  const Op<float, 1> x = from_row(p, g);
  Op<float, N> o;
  o.v[0] = x.v[0];
  o.v[1] = x.v[1];
  return o;
}
// A value as its parts.
template <int N>
__device__ inline void put_parts(__bf16* p, int apart, float x) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const __bf16 part = (__bf16)x;
    p[n * apart] = part;
    x -= (float)part;
  }
}
template <int N>
__device__ inline void put_parts(float* p, int, float x) { *p = x; }
template <int N>
__device__ inline void put_parts(__bf16* p, int apart, f32x4 x) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    bf16x4 part;
#pragma unroll
    for (int e = 0; e < 4; ++e) part[e] = (__bf16)x[e], x[e] -= (float)part[e];
    *reinterpret_cast<bf16x4*>(p + n * apart) = part;
  }
}
template <int N>
__device__ inline void put_parts(float* p, int, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }

__device__ inline float over_columns(float v) {   // sum over a tile's 16 columns
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

template <typename T, int KD>
__global__ __launch_bounds__(THREADS) void delta_gradients_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD>;
  using Rec = Record<T, true>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16, VB = L::VB, VLD = L::VLD, WLD = L::WLD;
  T *K = (T*)(lds + L::K), *Q = (T*)(lds + L::Q);
  T *DY = (T*)(lds + L::DY), *ZL = (T*)(lds + L::Z), *RL = (T*)(lds + L::R), *W1 = (T*)(lds + L::W1), *W2 = (T*)(lds + L::W2), *W3 = (T*)(lds + L::W3);
  double* G = (double*)(lds + L::SUMS);
  float *gate = (float*)(lds + L::GATE), *rowF = (float*)(lds + L::ROWF), *cols = (float*)(lds + L::COLS), *dots = (float*)(lds + L::DOTS),
        *more = (float*)(lds + L::MORE);
  const int per = p.B * p.Hk, chunk = p.c0 + blockIdx.x / per, b = blockIdx.x % per / p.Hk, hk = blockIdx.x % p.Hk, group = p.H / p.Hk;
  const int s0 = chunk * C, steps = min(p.t - s0, C), live = min(ends_at(p, b) - s0, C), BH = p.B * p.H;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE, g = lane / 16, c16 = lane % 16;
  const bool mine = wave < NT;               // waves with columns of dq and dk
  const int jt = wave % 4, col = 16 * wave + c16;
  float* parts = p.parts + ((int64_t)(chunk - p.c0) * p.B + b) * 2 * p.H;
  T* dq = (T*)p.dq.data + (int64_t)s0 * p.dq.stride_t + b * p.dq.stride_b + hk * p.dk + col;
  T* dk = (T*)p.dkey.data + (int64_t)s0 * p.dkey.stride_t + b * p.dkey.stride_b + hk * p.dk + col;
  if (live <= 0) {   // behind the sequence's end
    if (mine && col < p.dk)
      for (int s = g; s < steps; s += 4) dq[(int64_t)s * p.dq.stride_t] = dk[(int64_t)s * p.dkey.stride_t] = (T)0.0f;
    for (int i = threadIdx.x; i < steps * group; i += THREADS) {
      const int s = s0 + i / group, h = hk * group + i % group;
      ((T*)p.db.data)[s * p.db.stride_t + b * p.db.stride_b + h] = (T)0.0f;
      if (p.a.data) ((T*)p.da.data)[s * p.da.stride_t + b * p.da.stride_b + h] = (T)0.0f;
    }
    for (int i = threadIdx.x; i < group; i += THREADS) parts[hk * group + i] = parts[p.H + hk * group + i] = 0.0f;
    return;
  }
  for (int u = threadIdx.x; u < pieces<T>(KD); u += THREADS) {
    Piece<T> x, y;
    const Window wk(p.k.stride_t, live), wq(p.q.stride_t, live);
    load_piece<T, KD>(x, (const T*)p.k.data + (int64_t)s0 * p.k.stride_t + b * p.k.stride_b + hk * p.head, wk, p.width, u);
    load_piece<T, KD>(y, (const T*)p.q.data + (int64_t)s0 * p.q.stride_t + b * p.q.stride_b + hk * p.head, wq, p.width, u);
    clear_piece<T, KD>(x, wk, p.width, u);
    clear_piece<T, KD>(y, wq, p.width, u);
    put_rows<T, KD>(x, K, u);
    put_rows<T, KD>(y, Q, u);
  }
  f32x4 dQ[4] = {}, dK[4] = {};
  for (int h = hk * group; h < (hk + 1) * group; ++h) {
    const int64_t at = (int64_t)(chunk - p.c0) * BH + b * p.H + h;
    const char* rec = p.records + at * Rec::BYTES;
    const float *Sg = p.S + at * KD * p.dvp, *dSg = p.dS + at * KD * p.dvp, *Rg = p.R + at * C * p.dvp, *Zg = p.Z + at * C * p.dvp;
    const T* dyg = (const T*)p.dy.data + (int64_t)s0 * p.dy.stride_t + b * p.dy.stride_b + h * p.dv;
    __syncthreads();   // the head before has been read
    for (int i = threadIdx.x; i < GATES * C; i += THREADS) gate[i] = reinterpret_cast<const float*>(rec + Rec::GATE)[i];
    if (threadIdx.x < C) G[threadIdx.x] = reinterpret_cast<const double*>(rec + Rec::SUMS)[threadIdx.x];
    f32x4 YS[4] = {}, ZS[4] = {}, RS[4] = {}, AA[4] = {};
    float inner = 0.0f;
    for (int v0 = 0; v0 < p.dvp; v0 += VB) {
      if (v0) __syncthreads();
      for (int u = threadIdx.x; u < C * VB / 4; u += THREADS) {   // four values of a step
        const int s = u / (VB / 4), v = u % (VB / 4) * 4;
        f32x4 z = {}, r = {}, y = {};
        if (v0 + v < p.dvp) {
          z = *reinterpret_cast<const f32x4*>(Zg + s * p.dvp + v0 + v);
          r = *reinterpret_cast<const f32x4*>(Rg + s * p.dvp + v0 + v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (s < live && v0 + v + e < p.dv) y[e] = (float)dyg[(int64_t)s * p.dy.stride_t + v0 + v + e];
        put_parts<1>(DY + s * VLD + v, 0, y);
        put_parts<L::NV>(ZL + s * VLD + v, L::VSIZE / (int)sizeof(T), z);
        put_parts<L::NV>(RL + s * VLD + v, L::VSIZE / (int)sizeof(T), r);
      }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < VB; v += 32) {
        if (v0 + v >= p.dvp) break;
        // R's (waves 0 .. 3) or Z's pairs with column tile jt of R
        const auto rj = from_parts<N32>(RL + (16 * jt + c16) * VLD + v, L::VSIZE / (int)sizeof(T), g);
        Op<T, N32> s, ds;
        if (mine) {
          f32x4 x[2], y[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int c = v0 + v + 16 * i + 4 * g;
            x[i] = y[i] = f32x4{};
            if (c < p.dvp) {
              x[i] = *reinterpret_cast<const f32x4*>(Sg + col * p.dvp + c);
              y[i] = *reinterpret_cast<const f32x4*>(dSg + col * p.dvp + c);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) inner += x[i][e] * y[i][e];
          }
          s = cut<T, N32>(x[0], x[1]);
          ds = cut<T, N32>(y[0], y[1]);
        }
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
          const auto y = from_row(DY + (16 * rt + c16) * VLD + v, g);
          const auto z = from_parts<N32>(ZL + (16 * rt + c16) * VLD + v, L::VSIZE / (int)sizeof(T), g);
          if (rt >= jt) {
            if (wave < 4) mma(AA[rt], y, rj);
            else mma(AA[rt], z, rj);
          }
          if (mine) {
            mma(YS[rt], y, s);
            mma(ZS[rt], z, s);
            mma(RS[rt], from_parts<N32>(RL + (16 * rt + c16) * VLD + v, L::VSIZE / (int)sizeof(T), g), ds);
          }
        }
      }
    }
    __syncthreads();   // the blocks have been read: W1 .. W3 go there
    {
      const int j = 16 * jt + c16;
      const float skj = gate[SK * C + j], bej = gate[BE * C + j];
      float down = 0.0f, colF = 0.0f;
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        f32x4 x = {};
        if (rt >= jt) {
#pragma unroll
          for (int c = 0; c < KD; c += 32)
            mma(x, from_row((wave < 4 ? Q : K) + (16 * rt + c16) * LD + c, g), from_row(K + j * LD + c, g));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * rt + 4 * g + e;
          float f = 0.0f;
          if (wave < 4) {
            float w1 = 0.0f, w2 = 0.0f;
            if (j <= i) {
              const float d = expf((float)(G[i] - G[j])), m = x[e] * gate[SQ * C + i] * skj * d;
              const float dp = AA[rt][e] * bej;
              down += m * AA[rt][e];
              f = dp * m;
              w1 = dp * d * skj;
              w2 = dp * d * gate[SQ * C + i];
            }
            put_parts<L::NM>(W1 + i * WLD + j, L::WSIZE / (int)sizeof(T), w1);
            put_parts<L::NM>(W2 + j * WLD + i, L::WSIZE / (int)sizeof(T), w2);
          } else {
            if (j < i) {
              const float d = expf((float)(G[i] - G[j])), m = x[e] * gate[SK * C + i] * skj * d;
              const float dm = -AA[rt][e] * bej;
              down -= m * AA[rt][e];
              f = dm * m;
              put_parts<L::NM>(W3 + i * WLD + j, L::WSIZE / (int)sizeof(T), dm * d * skj);
              put_parts<L::NM>(W3 + j * WLD + i, L::WSIZE / (int)sizeof(T), dm * d * gate[SK * C + i]);
            } else if (j == i) {
              put_parts<L::NM>(W3 + i * WLD + i, L::WSIZE / (int)sizeof(T), 0.0f);
            }
          }
          colF += f;
          f = over_columns(f);
          if (c16 == 0) rowF[wave * C + i] = f;
        }
      }
      down += __shfl_xor(down, 16);
      colF += __shfl_xor(colF, 16);
      down += __shfl_xor(down, 32);
      colF += __shfl_xor(colF, 32);
      if (g == 0) {
        cols[(wave / 4) * C + j] = down;
        cols[(2 + wave / 4) * C + j] = colF;
      }
    }
    inner = wave_sum(inner);
    if (lane == 0) more[wave] = mine ? inner : 0.0f;
    __syncthreads();
    if (mine) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const f32x4 ga = *reinterpret_cast<const f32x4*>(gate + GA * C + 16 * rt + 4 * g);
        const f32x4 be = *reinterpret_cast<const f32x4*>(gate + BE * C + 16 * rt + 4 * g);
        const f32x4 la = *reinterpret_cast<const f32x4*>(gate + LA * C + 16 * rt + 4 * g);
        const f32x4 sk = *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
        const f32x4 sq = *reinterpret_cast<const f32x4*>(gate + SQ * C + 16 * rt + 4 * g);
        const f32x4 y = ga * YS[rt], z = ga * ZS[rt], r = la * RS[rt];
        f32x4 x = {}, w = {};
#pragma unroll
        for (int pb = 0; pb < 2; ++pb) {
          const auto kc = from_columns<LD>(K, 16 * wave, 32 * pb, lane), qc = from_columns<LD>(Q, 16 * wave, 32 * pb, lane);
          mma(x, from_parts<NW>(W1 + (16 * rt + c16) * WLD + 32 * pb, L::WSIZE / (int)sizeof(T), g), kc);
          mma(w, from_parts<NW>(W2 + (16 * rt + c16) * WLD + 32 * pb, L::WSIZE / (int)sizeof(T), g), qc);
          mma(w, from_parts<NW>(W3 + (16 * rt + c16) * WLD + 32 * pb, L::WSIZE / (int)sizeof(T), g), kc);
        }
        dQ[rt] += x + y;
        dK[rt] += w + be * r - z;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * rt + 4 * g + e;
          const float k = (float)K[i * LD + col] * sk[e], q = (float)Q[i * LD + col] * sq[e];
          const float first = over_columns(q * y[e] - k * z[e]), second = over_columns(k * r[e]);
          if (c16 == 0) {
            dots[wave * C + i] = first;
            dots[(WAVES + wave) * C + i] = second;
          }
        }
      }
    }
    __syncthreads();
    if (wave == 0) {
      const int i = lane;
      float rows = 0.0f, first = 0.0f, second = 0.0f, all = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) rows += rowF[w * C + i];
#pragma unroll
      for (int w = 0; w < NT; ++w) {
        first += dots[w * C + i];
        second += dots[(WAVES + w) * C + i];
        all += more[w];
      }
      const float beta = gate[BE * C + i], e = beta * second;
      float dG = rows - (cols[2 * C + i] + cols[3 * C + i]) + first - e;
      const float ends = wave_sum(e);
      if (i == C - 1) dG += ends + gate[GA * C + C - 1] * all;
      // sum from this step to the last one
#pragma unroll
      for (int m = 1; m < WAVE; m <<= 1) {
        const float behind = __shfl_down(dG, m);
        if (lane + m < WAVE) dG += behind;
      }
      const float dbeta = cols[i] + cols[C + i] + second;
      float dlog = 0.0f, da = 0.0f;
      const int64_t s = s0 + i;
      if (i < steps) {
        const bool in = i < live;
        if (p.a.data && in) {
          const float raw = (float)((const T*)p.a.data)[s * p.a.stride_t + b * p.a.stride_b + h] + (p.activate && p.bias ? p.bias[h] : 0.0f);
          if (p.activate) {
            dlog = dG * (fmaxf(raw, 0.0f) + log1pf(expf(-fabsf(raw))));
            da = dG * p.A[h] / (1.0f + expf(-raw));
          } else {
            da = dG;
          }
        }
        if (p.a.data) ((T*)p.da.data)[s * p.da.stride_t + b * p.da.stride_b + h] = (T)da;
        ((T*)p.db.data)[s * p.db.stride_t + b * p.db.stride_b + h] = (T)(!in ? 0.0f : p.activate ? dbeta * beta * (1.0f - beta) : dbeta);
      }
      dlog = wave_sum(dlog);
      da = wave_sum(da);
      if (lane == 0) {
        parts[h] = dlog;
        parts[p.H + h] = da;
      }
    }
  }
  // through the norms of q and k
  if (p.normalise) {
    __syncthreads();
    if (mine) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * rt + 4 * g + e;
          const float first = over_columns(dQ[rt][e] * (float)Q[i * LD + col]), second = over_columns(dK[rt][e] * (float)K[i * LD + col]);
          if (c16 == 0) {
            dots[wave * C + i] = first;
            dots[(WAVES + wave) * C + i] = second;
          }
        }
    }
    __syncthreads();
  }
  if (!mine || col >= p.dk) return;
#pragma unroll
  for (int rt = 0; rt < 4; ++rt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 16 * rt + 4 * g + e;
      float x = p.scale * dQ[rt][e], y = dK[rt][e];
      if (p.normalise) {
        float first = 0.0f, second = 0.0f;
#pragma unroll
        for (int w = 0; w < NT; ++w) {
          first += dots[w * C + i];
          second += dots[(WAVES + w) * C + i];
        }
        const float rq = gate[RQ * C + i], rk = gate[SK * C + i];
        x = rq * (x - (float)Q[i * LD + col] * rq * rq * p.scale * first);
        y = rk * (y - (float)K[i * LD + col] * rk * rk * second);
      }
      if (i < steps) {
        dq[(int64_t)i * p.dq.stride_t] = (T)(i < live ? x : 0.0f);
        dk[(int64_t)i * p.dkey.stride_t] = (T)(i < live ? y : 0.0f);
      }
    }
}

}  // namespace

int mebptt::delta::gradients(const Args& p, int dtype, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value, BYTES = Layout<T, KD>::BYTES;
    static_assert(BYTES <= 160 * 1024, "LDS of a compute unit");
    const hipError_t e = allow_dynamic_lds<delta_gradients_kernel<T, KD>>(BYTES);
    if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
    delta_gradients_kernel<T, KD><<<(unsigned)((p.c1 - p.c0) * p.B * p.Hk), THREADS, BYTES, stream>>>(p);
    return launched("delta rule, gradients");
  });
}
