// Gated delta rule: what a chunk's steps need of each other, T = (I + M beta)^-1 and P, for all chunks of a launch at once, and the
// factors of its steps.  One workgroup of four waves per chunk, sequence and head.
// Bound: short dependent steps (products, a substitution over 16 rows, two levels of joined blocks) with a barrier between any two; half of the
// waves' time is waiting, which four or five workgroups on a compute unit fill.  1000 steps x 32 sequences x 8 heads of 128, bf16: 74 us (for the
// backward pass, which needs T^T as well, 4 x 26), of which 227 MB take 44 at a copy's rate; 132 while k and q kept LDS of their own.
#include "delta.h"
#include "dynamic_lds.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

constexpr int LM = C + 4;        // floats between rows of the 64 x 64 matrices
constexpr float LEAST = -1e4f;   // exp of it is zero; sums of it stay far from infinity

// M and P take the place of the rows of k and q that they come from: four workgroups to a compute unit in place of two, which is what hides the
// waits between the short steps here.
template <typename T, int KD>
constexpr int matrix_bytes() { return 2 * (Lds<T>::row_bytes(KD) > C * LM * 4 ? Lds<T>::row_bytes(KD) : C * LM * 4); }
template <typename T, int KD>
constexpr int lds_bytes() { return matrix_bytes<T, KD>() + GATES * C * 4 + C * 8; }

// c += a b of one 16 x 16 x 16 in fp32: a as rows in LDS, b as a result tile.
__device__ inline void mma16(f32x4& c, const float* a, f32x4 b, int lane) {
  const f32x4 x = *reinterpret_cast<const f32x4*>(a + (lane % 16) * LM + lane / 16 * 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], b[e], c, 0, 0, 0);
}
__device__ inline f32x4 tile(const float* a, int lane) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = a[(lane / 16 * 4 + e) * LM + lane % 16];
  return v;
}
__device__ inline void put_tile(float* a, f32x4 v, int lane) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a[(lane / 16 * 4 + e) * LM + lane % 16] = v[e];
}

// The pieces of a triangle, or of its transpose, in the order of the operands.
template <typename T, bool TRANSPOSED>
__device__ inline void put_frags(char* out, const float* m) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = here(threadIdx.x % WAVE), g = lane / 16;
  for (int f = wave; f < FRAGS; f += 4) {
    const int rt = TRANSPOSED ? (f < 4 ? f / 2 : f - 2) : (f < 2 ? f : f / 2 + 1);
    const int pb = TRANSPOSED ? (f < 4 ? f % 2 : 1) : (f < 2 ? 0 : f % 2);
    const int row = 16 * rt + lane % 16, col = 32 * pb + 4 * g;
    f32x4 x, y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = TRANSPOSED ? m[(col + e) * LM + row] : m[row * LM + col + e];
      y[e] = TRANSPOSED ? m[(col + 16 + e) * LM + row] : m[row * LM + col + 16 + e];
    }
    const Op<T, PARTS> o = cut<T, PARTS>(x, y);
    char* p = out + f * units<T>(PARTS) * 1024 + lane * 16;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int n = 0; n < PARTS; ++n) *reinterpret_cast<bf16x8*>(p + n * 1024) = o.p[n];
    } else {
      *reinterpret_cast<f32x4*>(p) = o.v[0];
      *reinterpret_cast<f32x4*>(p + 1024) = o.v[1];
    }
  }
}

template <typename T, int KD, bool BACK>
__global__ __launch_bounds__(256, 4) void delta_prepare_kernel(Args p) {
  extern __shared__ __align__(16) char lds[];
  T* K = reinterpret_cast<T*>(lds);
  T* Q = reinterpret_cast<T*>(lds + Lds<T>::row_bytes(KD));
  float* M = reinterpret_cast<float*>(lds);
  float* P = M + C * LM;
  double* G = reinterpret_cast<double*>(lds + matrix_bytes<T, KD>());
  float* gate = reinterpret_cast<float*>(G + C);
  constexpr int LD = Lds<T>::ld(KD);
  const int BH = p.B * p.H, chunk = p.c0 + blockIdx.x / BH, bh = blockIdx.x % BH, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk);
  const int s0 = chunk * C, live = min(ends_at(p, b) - s0, C);
  if (live <= 0) return;   // (nobody reads the record)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE, g = lane / 16;
  using R = Record<T, BACK>;
  char* out = p.records + (int64_t)blockIdx.x * R::BYTES;

  Fetch<T, KD, 256> fk, fq;
  fk.load(p.k, s0, b, hk, 0, live);
  fq.load(p.q, s0, b, hk, 0, live);
  const int64_t step = s0 + min(lane, live - 1);   // (a and b are read before k and q are waited for)
  const T raw_b = ((const T*)p.b.data)[step * p.b.stride_t + b * p.b.stride_b + h];
  const T raw_a = p.a.data ? ((const T*)p.a.data)[step * p.a.stride_t + b * p.a.stride_b + h] : (T)0.0f;
  fk.put(K, p.k, 0, live);
  fq.put(Q, p.q, 0, live);
  if (wave == 0) {   // decays and betas of the steps
    float lg = 0.0f, beta = 0.0f;
    if (lane < live) {
      const float bv = (float)raw_b;
      beta = p.activate ? 1.0f / (1.0f + expf(-bv)) : bv;
      if (p.a.data) {
        lg = (float)raw_a;
        if (p.activate) {
          lg += p.bias ? p.bias[h] : 0.0f;
          lg = p.A[h] * (fmaxf(lg, 0.0f) + log1pf(expf(-fabsf(lg))));
        }
        // (a NaN stays one)
        if (lg < LEAST) lg = LEAST;
      }
    }
    // in 64 bits: after one step that forgets all, differences of the sums behind it would have few bits left in 32
    double sum = lg;
#pragma unroll
    for (int m = 1; m < WAVE; m <<= 1) {
      const double before = __shfl_up(sum, m);
      if (lane >= m) sum += before;
    }
    G[lane] = sum;
    gate[GA * C + lane] = expf((float)sum);
    gate[BE * C + lane] = beta;
    gate[LA * C + lane] = expf((float)(__shfl(sum, C - 1) - sum));
  }
  __syncthreads();
  // row tile `wave` of M beta and P; what stands above the diagonal is zero
  f32x4 kk[4] = {}, qk[4] = {}, qq = {};
  {
    Op<T, 1> ki[KD / 32], qi[KD / 32];
#pragma unroll
    for (int c = 0; c < KD / 32; ++c) {
      ki[c] = from_row(K + (16 * wave + lane % 16) * LD + 32 * c, g);
      qi[c] = from_row(Q + (16 * wave + lane % 16) * LD + 32 * c, g);
      mma(qq, qi[c], qi[c]);
    }
#pragma unroll
    for (int jt = 0; jt < 4; ++jt)
      if (jt <= wave) {
#pragma unroll
        for (int c = 0; c < KD / 32; ++c) {
          const auto kj = from_row(K + (16 * jt + lane % 16) * LD + 32 * c, g);
          mma(kk[jt], ki[c], kj);
          mma(qk[jt], qi[c], kj);
        }
      }
  }
  {   // squared lengths of k and q are the diagonals of their products with themselves
    f32x4 k2 = kk[0];
#pragma unroll
    for (int jt = 1; jt < 4; ++jt) k2 = jt == wave ? kk[jt] : k2;
    const int e = lane % 4;
    if (lane % 16 / 4 == g) {
      const float k = e == 0 ? k2[0] : e == 1 ? k2[1] : e == 2 ? k2[2] : k2[3], q = e == 0 ? qq[0] : e == 1 ? qq[1] : e == 2 ? qq[2] : qq[3];
      const int row = 16 * wave + lane % 16;
      // (nothing of a step that does not exist: without an eps its length of zero would make infinities, and those NaNs of the chunk's other steps)
      const float rq = row >= live ? 0.0f : p.normalise ? 1.0f / sqrtf(q + p.eps) : 1.0f;
      gate[SK * C + row] = row >= live ? 0.0f : p.normalise ? 1.0f / sqrtf(k + p.eps) : 1.0f;
      gate[SQ * C + row] = p.scale * rq;
      gate[RQ * C + row] = rq;
    }
  }
  __syncthreads();   // k and q have been read
  {
    const int i0 = 16 * wave + 4 * g;
    const f32x4 sk = *reinterpret_cast<const f32x4*>(gate + SK * C + i0), sq = *reinterpret_cast<const f32x4*>(gate + SQ * C + i0);
    double Gi[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) Gi[e] = G[i0 + e];
#pragma unroll
    for (int jt = 0; jt < 4; ++jt) {
      const int j = 16 * jt + lane % 16;
      const float skj = gate[SK * C + j], bej = gate[BE * C + j];
      const double Gj = G[j];
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // (what is above the diagonal may be infinite before it is dropped)
        const float d = __expf((float)(Gi[e] - Gj)) * skj, m = kk[jt][e] * d * sk[e] * bej, q = qk[jt][e] * d * sq[e];
        kk[jt][e] = j < i0 + e ? m : 0.0f;
        qk[jt][e] = j <= i0 + e ? q : 0.0f;
      }
      put_tile(M + 16 * wave * LM + 16 * jt, kk[jt], lane);
      put_tile(P + 16 * wave * LM + 16 * jt, qk[jt], lane);
    }
  }
  __syncthreads();
  // T over M.  Diagonal tiles by substitution, a column per lane; then from two diagonal blocks' inverses the block below: -T22 M21 T11.
  const int lane_ = lane;
  {
    float* m = M + 16 * wave * (LM + 1);
    const int c = lane % 16;
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s = r == c ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < r; j += 4) {
        const f32x4 row = *reinterpret_cast<const f32x4*>(m + r * LM + j);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < r) s -= row[e] * x[j + e];
      }
      x[r] = s;
      if (r % 4 == 3) asm volatile("" : "+v"(x[r]) : : "memory");   // (all rows at once would not fit the registers)
    }
    __builtin_amdgcn_wave_barrier();
    if (lane < 16) {
#pragma unroll
      for (int r = 0; r < 16; ++r) m[r * LM + c] = x[r];
    }
  }
  __syncthreads();
  if (wave < 2) {
    const int lane = here(lane_);
    float* m = M + 32 * wave * (LM + 1);
    f32x4 w = {}, x = {};
    mma16(w, m + 16 * LM, tile(m, lane), lane);
    mma16(x, m + 16 * (LM + 1), w, lane);
    __builtin_amdgcn_wave_barrier();
    put_tile(m + 16 * LM, -x, lane);
  }
  __syncthreads();
  f32x4 low[2] = {};
  if (wave < 2) {   // column tile `wave` of the lower left 32 x 32
    const int lane = here(lane_);
    f32x4 w[2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) mma16(w[i], M + (32 + 16 * i) * LM + 16 * k, tile(M + 16 * k * LM + 16 * wave, lane), lane);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k <= i; ++k) mma16(low[i], M + (32 + 16 * i) * LM + 32 + 16 * k, w[k], lane);
  }
  __syncthreads();
  if (wave < 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) put_tile(M + (32 + 16 * i) * LM + 16 * wave, -low[i], lane);
  }
  __syncthreads();
  put_frags<T, false>(out + R::T_, M);
  if constexpr (BACK) {
    put_frags<T, true>(out + R::TT, M);
    put_frags<T, true>(out + R::P, P);
  } else {
    put_frags<T, false>(out + R::P, P);
  }
  if (threadIdx.x < C) {
    const int i = threadIdx.x;
    gate[GA_SK * C + i] = gate[GA * C + i] * gate[SK * C + i];
    gate[GA_SQ * C + i] = gate[GA * C + i] * gate[SQ * C + i];
    gate[LA_SK * C + i] = gate[LA * C + i] * gate[SK * C + i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < GATES * C; i += 256) reinterpret_cast<float*>(out + R::GATE)[i] = gate[i];
  if (threadIdx.x < C) reinterpret_cast<double*>(out + R::SUMS)[threadIdx.x] = G[threadIdx.x];
}

// PAD_ROWS neighbouring rows a workgroup, four columns of one a thread at a time: 333 x 20 rows of 50 and 75 floats in 10 us, 15 with a wave a row.
constexpr int PAD_ROWS = 64;
template <typename T>
__global__ __launch_bounds__(256) void delta_pad_kernel(Padded all, int B, int s0, int steps) {
  typedef T Quad __attribute__((ext_vector_type(4), aligned(sizeof(T) * 4)));
  const Padded::One& p = all.one[blockIdx.y];
  const int64_t rows = (int64_t)steps * B * p.heads;
  const int quads = p.width / 4;
  for (int64_t row0 = (int64_t)blockIdx.x * PAD_ROWS; row0 < rows; row0 += (int64_t)gridDim.x * PAD_ROWS) {
    const unsigned r0 = (unsigned)(row0 / p.heads), h0 = (unsigned)(row0 - (int64_t)r0 * p.heads);
    const int n = (int)min((int64_t)PAD_ROWS, rows - row0) * quads;
    for (int i = threadIdx.x; i < n; i += 256) {
      const unsigned row = (unsigned)i / (unsigned)quads, c = ((unsigned)i - row * quads) * 4;
      const unsigned h1 = h0 + row, more = h1 / (unsigned)p.heads, h = h1 - more * p.heads, r = r0 + more, b = r / (unsigned)steps, s = r - b * (unsigned)steps;
      const T* from = (const T*)p.from.data + (int64_t)(s0 + (int)s) * p.from.stride_t + (int64_t)b * p.from.stride_b + (int64_t)h * p.d;
      Quad v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = from[min(c + e, (unsigned)p.d - 1)];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = c + e < (unsigned)p.d ? v[e] : (T)0.0f;
      *reinterpret_cast<Quad*>((T*)p.to + (row0 + row) * p.width + c) = v;
    }
  }
}

template <typename T, int KD, bool BACK>
int launch(const Args& p, hipStream_t stream) {
  constexpr int BYTES = lds_bytes<T, KD>();
  const hipError_t e = allow_dynamic_lds<delta_prepare_kernel<T, KD, BACK>>(BYTES);
  if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
  delta_prepare_kernel<T, KD, BACK><<<(unsigned)((p.c1 - p.c0) * p.B * p.H), 256, BYTES, stream>>>(p);
  return launched("delta rule, preparation");
}

}  // namespace

int mebptt::delta::pad_rows(const Padded& all, const Args& p, int dtype, hipStream_t stream) {
  if (!all.n) return MEBPTT_OK;
  const int steps = launch_steps(p);
  int64_t most = 1;
  for (int i = 0; i < all.n; ++i) most = std::max(most, (int64_t)steps * p.B * all.one[i].heads);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(most, PAD_ROWS), 1 << 14), (unsigned)all.n);
  if (dtype == MEBPTT_FP32) delta_pad_kernel<float><<<grid, 256, 0, stream>>>(all, p.B, p.c0 * C, steps);
  else delta_pad_kernel<__bf16><<<grid, 256, 0, stream>>>(all, p.B, p.c0 * C, steps);
  return launched("delta rule, rows");
}

int mebptt::delta::prepare(const Args& p, int dtype, bool back, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value;
    return back ? launch<T, KD, true>(p, stream) : launch<T, KD, false>(p, stream);
  });
}
