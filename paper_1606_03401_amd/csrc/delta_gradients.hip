// Gated delta rule: the gradients of a chunk's q, k, a and b, all chunks of a launch at once, from what the two walks left: R, Z and the states
// before and behind the chunk (S, and its gradient dS').  With E = Z R^T below the diagonal,
//     dP = (dY R^T) beta,   dM = -E beta,   W1 = dP o D,   W3 = dM o D,
//     dq~ = W1 K^ + gamma dY S^T,   dk^ = W1^T Q~ + (W3 + W3^T) K^ + beta gamma_C / gamma R dS'^T - gamma Z S^T,
//     dbeta_j = sum_i (P o dY R^T)_ij - sum_i (M o E)_ij + (gamma_C / gamma k^)_j . (R dS'^T)_j,
//     dG_i = sum_j F_ij - sum_j F_ji + q~_i . (gamma dY S^T)_i - k^_i . (gamma Z S^T)_i - e_i,   F = dP o P + dM o M,
//     e_j = beta_j (gamma_C / gamma k^)_j . (R dS'^T)_j,   the last step's dG also sum e + gamma_C <dS', S>,   dg_s = sum_{i >= s} dG_i.
// A workgroup of eight waves, one to a compute unit, goes through chunks of sequences with one head each; or, where value heads share a key head, has one
// chunk and key head and goes through its value heads.  Wave w computes 16 columns of dq and dk; in what is 64 x 64, waves 0 .. 3 have column tiles of
// dY R^T and P, 4 .. 7 those of E and M.
// Bound: what a chunk reads (R, Z, S and dS' in fp32: 243 KB a chunk of 128 x 128, 2 TB/s over all), in bursts between which the products stand; eight waves
// of 240 registers and 157 KB of LDS leave no room for a second workgroup to fill the gaps.  1000 x 32 x 8 heads of 128 x 128, bf16, in four launches: 497 us,
// of a chunk's 62 thousand cycles 25 in the loop over columns of v (13 of them products), 12 for the 64 x 64 products, 8 for sums, the rest writing and waiting.
// Tried: two bf16 parts for R, Z, S and dS', 3 % faster and dA off by 10^-6; loads spread over the products, workgroups started apart, blocks in another order in
// each workgroup: none faster.
#include "delta.h"
#include "dynamic_lds.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

constexpr int WAVES = 8, THREADS = WAVES * WAVE;
// Parts of R, Z, S, dS' and W1 .. W3 in the products.  (With two for W1 .. W3, which reach dq and dk only, a launch takes 120 us in place of 124, and a dq that is little of
// its terms shows their 16 bits.)
constexpr int N32 = PARTS;
constexpr int COMPUTE_UNITS = 256;
constexpr int VB = 32;      // columns of a block of dY, Z and R

template <typename T, int KD>
struct Layout {
  static constexpr int VLD = VB + Lds<T>::PAD, VSIZE = C * VLD * (int)sizeof(T), NV = sizeof(T) == 2 ? N32 : 1, BLOCK_BYTES = (1 + 2 * NV) * VSIZE;
  static constexpr int WLD = C + Lds<T>::PAD, WSIZE = C * WLD * (int)sizeof(T);
  static constexpr int K = 0, Q = K + Lds<T>::row_bytes(KD), BLOCK = Q + Lds<T>::row_bytes(KD);    // two blocks, one being filled
  static constexpr int W = BLOCK;                                                                    // four matrices, over them
  static constexpr int SUMS = BLOCK + (2 * BLOCK_BYTES > 4 * NV * WSIZE ? 2 * BLOCK_BYTES : 4 * NV * WSIZE);
  static constexpr int GATE = SUMS + C * 8, ROWF = GATE + GATES * C * 4, COLF = ROWF + WAVES * C * 8, COLS = COLF + 2 * C * 8, DOTS = COLS + 2 * C * 4,
                       NORMS = DOTS + 3 * WAVES * C * 4, MORE = NORMS + 2 * C * 4, BYTES = MORE + WAVES * 4;
};

// An operand in the order in which it stands in a block: places 8 g .. 8 g + 7 hold columns 4 g .. and 16 + 4 g .., so that a load of S for one lane group
// takes 64 neighbouring bytes of a row.
template <int N>
__device__ inline Op<__bf16, N> as_it_stands(const __bf16* p, int apart, int g) {
  Op<__bf16, N> o;
#pragma unroll
  for (int n = 0; n < N; ++n) o.p[n] = *reinterpret_cast<const bf16x8*>(p + n * apart + 8 * g);
  return o;
}
template <int N>
__device__ inline Op<float, N> as_it_stands(const float* p, int, int g) {
  Op<float, N> o;
  o.v[0] = *reinterpret_cast<const f32x4*>(p + 8 * g);
  o.v[1] = *reinterpret_cast<const f32x4*>(p + 8 * g + 4);
  return o;
}
// An operand with N parts whose row stands at p, or (columns) whose rows c0 .. stand as columns; parts `apart` values from each other.
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
template <int N, int LD>
__device__ inline Op<__bf16, N> from_part_columns(const __bf16* p, int apart, int c0, int s0, int lane) {
  Op<__bf16, N> o;
#pragma unroll
  for (int n = 0; n < N; ++n) o.p[n] = from_columns<LD>(p + n * apart, c0, s0, lane).p[0];
  return o;
}
template <int N, int LD>
__device__ inline Op<float, N> from_part_columns(const float* p, int, int c0, int s0, int lane) {
  const Op<float, 1> x = from_columns<LD>(p, c0, s0, lane);
  Op<float, N> o;
  o.v[0] = x.v[0];
  o.v[1] = x.v[1];
  return o;
}
// Four values as their parts.
template <int N>
__device__ inline void put_parts(__bf16* p, int apart, f32x4 x) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x2 pairs;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const f32x2 two = {x[2 * e], x[2 * e + 1]};
      pairs[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2));
      x[2 * e] -= __uint_as_float(pairs[e] << 16);
      x[2 * e + 1] -= __uint_as_float(pairs[e] & 0xFFFF0000u);
    }
    *reinterpret_cast<u32x2*>(p + n * apart) = pairs;
  }
}
template <int N>
__device__ inline void put_parts(float* p, int, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }

// Sum over 16 neighbouring lanes, a tile's columns, in each of them.
__device__ inline float over_columns(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));   // from 8 lanes on, round the row of 16
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, false));
  return v;
}

// Sums of 16 values over 16 neighbouring lanes; lane c's is that of value c.  In each step a lane hands the half that it does not keep to its mirror
// image: 45 operations where 16 sums of their own take 64.
__device__ inline float over_columns(float (&v)[16], int c16) {
  auto half = [&](auto n, auto mirror) {
    constexpr int N = decltype(n)::value;
    const bool upper = c16 & N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float keep = upper ? v[i + N] : v[i], give = upper ? v[i] : v[i + N];
      v[i] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(give), decltype(mirror)::value, 0xf, 0xf, false));
    }
  };
  half(std::integral_constant<int, 8>{}, std::integral_constant<int, 0x140>{});   // 15 - c
  half(std::integral_constant<int, 4>{}, std::integral_constant<int, 0x141>{});   // 7 - c of 8
  half(std::integral_constant<int, 2>{}, std::integral_constant<int, 0x1B>{});    // 3 - c of 4
  half(std::integral_constant<int, 1>{}, std::integral_constant<int, 0xB1>{});    // 1 - c of 2
  return v[0];
}

// Sum over a wave in each lane: rows of 16 lanes, then the four rows.
__device__ inline float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ inline float over_wave(float v) {
  v = over_columns(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// The same in 64 bits.
template <int CONTROL>
__device__ inline double moved(double v) {
  const u32x2 x = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{(unsigned)__builtin_amdgcn_update_dpp(0, (int)x[0], CONTROL, 0xf, 0xf, true), (unsigned)__builtin_amdgcn_update_dpp(0, (int)x[1], CONTROL, 0xf, 0xf, true)});
}
__device__ inline double over_columns(double v) {
  v += moved<0x128>(v);
  v += moved<0x124>(v);
  v += moved<0x122>(v);
  v += moved<0x121>(v);
  return v;
}
__device__ inline double lane_of(double v, int lane) {
  const u32x2 x = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{(unsigned)__builtin_amdgcn_readlane((int)x[0], lane), (unsigned)__builtin_amdgcn_readlane((int)x[1], lane)});
}
__device__ inline double over_wave(double v) {
  v = over_columns(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// Sum of the values of this lane and those behind it.
__device__ inline double from_lane_on(double v, int lane) {
  v += moved<0x101>(v);   // (lanes behind the row's end count as zero)
  v += moved<0x102>(v);
  v += moved<0x104>(v);
  v += moved<0x108>(v);
  const double last = lane_of(v, 48), two = lane_of(v, 32) + last, three = lane_of(v, 16) + two;
  return v + (lane < 16 ? three : lane < 32 ? two : lane < 48 ? last : 0.0);
}

// The kernel's first argument where the launch put it.
__device__ inline const Args* fresh_arguments() {
  auto* at = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return (const Args*)at;
}

// SHARED: more than one value head to a key head.  (Without the loop over them the compiler keeps what belongs to it out of registers.  With it 24 values of a thread are in
// scratch memory at 128 rows in bf16, 125 in fp32, 3 at 64.)
template <typename T, int KD, bool SHARED>
__global__ __launch_bounds__(THREADS) void delta_gradients_kernel(Args arguments) {
  (void)arguments;
  const Args* now = fresh_arguments();   // (read again for each head: kept over the loop, they would fill the scalar registers)
  extern __shared__ __align__(16) char lds[];
  using L = Layout<T, KD>;
  using Rec = Record<T, true>;
  constexpr int LD = Lds<T>::ld(KD), NT = KD / 16, VLD = L::VLD, WLD = L::WLD, VA = L::VSIZE / (int)sizeof(T), WA = L::WSIZE / (int)sizeof(T);
  T *K = (T*)(lds + L::K), *Q = (T*)(lds + L::Q);
  // [j][i], i >= j: W1 and W3 with the factor of column j's key, and with that of row i's query or key
  T *W1 = (T*)(lds + L::W), *W1q = W1 + L::NV * WA, *W3 = W1q + L::NV * WA, *W3k = W3 + L::NV * WA;
  double *G = (double*)(lds + L::SUMS), *rowF = (double*)(lds + L::ROWF), *colF_ = (double*)(lds + L::COLF);
  float *gate = (float*)(lds + L::GATE), *cols = (float*)(lds + L::COLS), *dots = (float*)(lds + L::DOTS),
        *norms = (float*)(lds + L::NORMS), *more = (float*)(lds + L::MORE);
  const int per = now->B * now->Hk, items = (now->c1 - now->c0) * per, group = SHARED ? now->H / now->Hk : 1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane_ = threadIdx.x % WAVE;
  const bool mine = wave < NT;               // waves with columns of dq and dk
  // column tiles with many rows and with few are paired: waves w and w + 4 share a SIMD
  const int jt = wave < 4 ? wave : 7 - wave;
  struct Item {
    int chunk, b, hk, s0, live;   // chunk: from the launch's first one on
  };
  auto item_at = [&](int item) {
    const Args& p = *now;
    Item w;
    w.chunk = item / per;
    w.b = (item - w.chunk * per) / p.Hk;
    w.hk = item - w.chunk * per - w.b * p.Hk;
    w.s0 = (p.c0 + w.chunk) * C;
    w.live = min(ends_at(p, w.b) - w.s0, C);
    return w;
  };
  auto parts_of = [&](const Item& w) { return now->parts + ((int64_t)w.chunk * now->B + w.b) * 2 * now->H; };
  auto out_of = [&](const mebptt_seq& s, const Item& w) {
    const Args& p = *now;
    return (T*)s.data + (int64_t)w.s0 * s.stride_t + w.b * s.stride_b + w.hk * p.dk + 16 * wave + here(lane_) % 16;
  };
  // The first item from `item` on, of those that this workgroup takes, that has steps in it; gradients behind a sequence's end are zero.
  auto next_live = [&](int item) {
    const Args& p = *now;
    for (; item < items; item += gridDim.x) {
      const Item w = item_at(item);
      if (w.live > 0) break;
      const int steps = min(p.t - w.s0, C), lane = here(lane_);
      if (mine && 16 * wave + lane % 16 < p.dk) {
        T *dq = out_of(p.dq, w), *dk = out_of(p.dkey, w);
        for (int s = lane / 16; s < steps; s += 4) dq[(int64_t)s * p.dq.stride_t] = dk[(int64_t)s * p.dkey.stride_t] = (T)0.0f;
      }
      for (int i = threadIdx.x; i < steps * group; i += THREADS) {
        const int s = w.s0 + i / group, h = w.hk * group + i % group;
        ((T*)p.db.data)[s * p.db.stride_t + w.b * p.db.stride_b + h] = (T)0.0f;
        if (p.a.data) ((T*)p.da.data)[s * p.da.stride_t + w.b * p.da.stride_b + h] = (T)0.0f;
      }
      float* parts = parts_of(w);
      for (int i = threadIdx.x; i < group; i += THREADS) parts[w.hk * group + i] = parts[p.H + w.hk * group + i] = 0.0f;
    }
    return item;
  };
  static_assert(C * VB / 4 == THREADS, "a block is four values a thread");
  constexpr int FACTORS = (GATES * C * 4 + C * 8) / 16;   // the gates and behind them G: whole vectors of a record
  static_assert(FACTORS <= THREADS && L::GATE == L::SUMS + C * 8 && Rec::SUMS == Rec::GATE + GATES * C * 4, "a vector a thread");
  // What an item needs first is read while the item before it is being finished.  (Where heads are shared no registers are left for that: dq and dk are kept
  // from head to head.)
  typedef T Quad __attribute__((ext_vector_type(4), aligned(sizeof(T) * 4)));
  Fetch<T, KD, THREADS> fk, fq;
  f32x4 z, r, x[2], y[2], factors;
  Quad q4;
  T raw_a;
  // WHAT: 0 rows of dY, Z and R, 1 of S, 2 of dS'
  auto fetch = [&](const Item& w, int h, int v0, auto what) {
    constexpr int WHAT = decltype(what)::value;
    const Args& p = *now;
    const int lane = here(lane_), vs = (64 * wave + lane) / (VB / 4), vc = lane % (VB / 4) * 4;   // a thread's step and four columns of a block
    const int64_t at = (int64_t)w.chunk * (p.B * p.H) + w.b * p.H + h;
    if constexpr (WHAT == 0) {
      const unsigned off_v = (unsigned)(vs * p.dvp + vc) * 4u, off_y = (unsigned)(min(vs, w.live - 1) * (int)p.dy.stride_t);
      const T* dyg = (const T*)p.dy.data + (int64_t)w.s0 * p.dy.stride_t + w.b * p.dy.stride_b + (int64_t)h * p.dy.head;
      z = *reinterpret_cast<const f32x4*>(near(p.Z + at * C * p.dvp + v0, off_v));
      r = *reinterpret_cast<const f32x4*>(near(p.R + at * C * p.dvp + v0, off_v));
      q4 = *reinterpret_cast<const Quad*>(near(dyg, (off_y + (unsigned)min(v0 + vc, p.dy.width - 4)) * (unsigned)sizeof(T)));
    } else {
      const unsigned off_s = (unsigned)((16 * (mine ? wave : 0) + lane % 16) * p.dvp + lane / 16 * 4) * 4u;
      const float* from = (WHAT == 1 ? p.S : p.dS) + at * KD * p.dvp + v0;
#pragma unroll
      for (int i = 0; i < 2; ++i) (WHAT == 1 ? x : y)[i] = *reinterpret_cast<const f32x4*>(near(from + 16 * i, off_s));
    }
  };
  constexpr std::integral_constant<int, 0> ROWS{};
  constexpr std::integral_constant<int, 1> STATE{};
  constexpr std::integral_constant<int, 2> STATE_GRAD{};
  auto fetch_first = [&](const Item& w, int n) {
    const Args& p = *now;
    const int h = w.hk * group + n, lane = here(lane_);
    if (n == 0) {
      fk.load(p.k, w.s0, w.b, w.hk, 0, w.live);
      fq.load(p.q, w.s0, w.b, w.hk, 0, w.live);
    }
    factors = *reinterpret_cast<const f32x4*>(p.records + ((int64_t)w.chunk * (p.B * p.H) + w.b * p.H + h) * Rec::BYTES + Rec::GATE +
                                              min((int)threadIdx.x, FACTORS - 1) * 16);
    fetch(w, h, 0, ROWS);
    fetch(w, h, 0, STATE);
    fetch(w, h, 0, STATE_GRAD);
    raw_a = p.a.data ? ((const T*)p.a.data)[(w.s0 + min(lane, w.live - 1)) * p.a.stride_t + w.b * p.a.stride_b + h] : (T)0.0f;
  };
  int item = next_live(blockIdx.x), n = 0;
  if (item >= items) return;
  Item at = item_at(item);
  if constexpr (!SHARED) fetch_first(at, 0);
  f32x4 dQ[4], dK[4];
  while (true) {
    now = fresh_arguments();
    const Args& p = *now;
    if (!SHARED || n == 0) {
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) dQ[rt] = dK[rt] = f32x4{};
    }
    const int lane = here(lane_), g = lane / 16, c16 = lane % 16, col = 16 * wave + c16, h = at.hk * group + n;
    const int b = at.b, s0 = at.s0, live = at.live, steps = min(p.t - s0, C);
    const int vs = (64 * wave + lane) / (VB / 4), vc = lane % (VB / 4) * 4;
    if constexpr (SHARED) fetch_first(at, n);
    const T this_a = raw_a;
    auto put = [&](int v0, int buffer) {
      T* dy = (T*)(lds + L::BLOCK + buffer * L::BLOCK_BYTES);
      if (vs >= live || v0 + vc >= p.dy.width) q4 = Quad{};
      T* place = dy + vs * VLD + vc % 16 * 2 + vc / 16 * 4;
      *reinterpret_cast<Quad*>(place) = q4;
      put_parts<L::NV>(place + VA, VA, z);
      put_parts<L::NV>(place + (1 + L::NV) * VA, VA, r);
    };
    if (n == 0) {
      fk.put(K, p.k, 0, live);
      fq.put(Q, p.q, 0, live);
    }
    const int fi = min((int)threadIdx.x, FACTORS - 1);
    *reinterpret_cast<f32x4*>(fi < GATES * C / 4 ? reinterpret_cast<char*>(gate) + fi * 16 : reinterpret_cast<char*>(G) + (fi * 16 - GATES * C * 4)) = factors;
    f32x4 YS[4] = {}, ZS[4] = {}, RS[4] = {}, AA[4] = {};
    float inner = 0.0f;
    for (int v0 = 0, buffer = 0; v0 < p.dvp; v0 += VB, buffer ^= 1) {
      put(v0, buffer);
      const Op<T, N32> s = cut<T, N32>(x[0], x[1]), ds = cut<T, N32>(y[0], y[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) inner += x[i][e] * y[i][e];
      __syncthreads();   // (and the block before the last one has been read)
      // The next block, or the last one again: under a condition it would be waited for there.  (Shared heads leave fewer registers: a few loads at a time there.
      // Where there are enough, that was no faster.)
      const int ahead = min(v0 + VB, p.dvp - VB);
      if constexpr (!SHARED) {
        fetch(at, h, ahead, ROWS);
        fetch(at, h, ahead, STATE);
        fetch(at, h, ahead, STATE_GRAD);
      }
      const T *DY = (const T*)(lds + L::BLOCK + buffer * L::BLOCK_BYTES), *ZL = DY + VA, *RL = ZL + L::NV * VA;
      const auto rj = as_it_stands<N32>(RL + (16 * jt + c16) * VLD, VA, g);
      Op<T, 1> dy[4];
      Op<T, N32> zr[4];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        dy[rt] = as_it_stands<1>(DY + (16 * rt + c16) * VLD, VA, g);
        zr[rt] = as_it_stands<N32>(ZL + (16 * rt + c16) * VLD, VA, g);
      }
      if constexpr (SHARED) fetch(at, h, ahead, ROWS);
      // (all four tiles: the ones above the diagonal cost less than branches)
      if (wave < 4) mma(AA, dy, rj);
      else mma(AA, zr, rj);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (SHARED) {
        fetch(at, h, ahead, STATE);
        if (mine) mma(YS, dy, s);
        __builtin_amdgcn_sched_barrier(0);
        fetch(at, h, ahead, STATE_GRAD);
      }
      if (mine) {
        if constexpr (!SHARED) mma(YS, dy, s);
        mma(ZS, zr, s);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) zr[rt] = as_it_stands<N32>(RL + (16 * rt + c16) * VLD, VA, g);
        mma(RS, zr, ds);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();   // the blocks have been read: W1 .. W3 go there
    {
      const int j = 16 * jt + c16;
      const float skj = gate[SK * C + j], bej = gate[BE * C + j];
      const double Gj = G[j];
      float down = 0.0f;
      double colF = 0.0;
      T *first = wave < 4 ? W1 : W3, *second = wave < 4 ? W1q : W3k;
      const T* rows = wave < 4 ? Q : K;
      const float* factor = gate + (wave < 4 ? SQ : SK) * C;
      Op<T, 1> kj[KD / 32];
#pragma unroll
      for (int c = 0; c < KD / 32; ++c) kj[c] = from_row(K + j * LD + 32 * c, g);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const int i0 = 16 * rt + 4 * g;
        f32x4 w1 = {}, w2 = {};   // (above the diagonal too, as far as the products read)
        double row[4] = {};
        if (rt >= jt) {
          f32x4 m = {};
#pragma unroll
          for (int c = 0; c < KD / 32; ++c) mma(m, from_row(rows + (16 * rt + c16) * LD + 32 * c, g), kj[c]);
          const f32x4 fi = *reinterpret_cast<const f32x4*>(factor + i0);
          double Gi[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) Gi[e] = G[i0 + e];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool in = wave < 4 ? j <= i0 + e : j < i0 + e;
            const float far = __expf((float)(Gi[e] - Gj)), d = in ? far : 0.0f, a = wave < 4 ? AA[rt][e] : -AA[rt][e], u = a * bej;
            m[e] *= fi[e] * skj * d;
            down += m[e] * a;
            const float f = u * m[e];
            w1[e] = u * d * skj;
            w2[e] = u * d * fi[e];
            colF += f;
            row[e] = over_columns((double)f);
          }
        }
        put_parts<L::NV>(first + j * WLD + i0, WA, w1);
        put_parts<L::NV>(second + j * WLD + i0, WA, w2);
        if (c16 == 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) rowF[wave * C + i0 + e] = row[e];
        }
      }
      down += __shfl_xor(down, 16);
      colF += __shfl_xor(colF, 16);
      down += __shfl_xor(down, 32);
      colF += __shfl_xor(colF, 32);
      if (g == 0) {
        cols[(wave / 4) * C + j] = down;
        colF_[(wave / 4) * C + j] = colF;
      }
    }
    inner = over_wave(inner);
    if (lane == 0) more[wave] = inner;
    __syncthreads();
    f32x4 wx[4] = {}, w[4] = {};
    if (mine) {
      // lower triangles have tiles 0 .. 3 of the first 32 columns and 2, 3 of the others, their transposes 0, 1 of the first and all of the others
#pragma unroll
      for (int pb = 0; pb < 2; ++pb) {
        const auto kc = from_columns<LD>(K, 16 * wave, 32 * pb, lane), qc = from_columns<LD>(Q, 16 * wave, 32 * pb, lane);
        constexpr int LOW = 4;
        Op<T, N32> a[LOW];
        auto products = [&](const T* m, bool transposed, f32x4(&to)[4], const Op<T, 1>& x) {
          // (what a triangle leaves empty is zero in LDS as far as it is read)
#pragma unroll
          for (int rt = 0; rt < 4; ++rt)
            a[rt] = transposed ? from_parts<N32>(m + (16 * rt + c16) * WLD + 32 * pb, WA, g) : from_part_columns<N32, WLD>(m, WA, 16 * rt, 32 * pb, lane);
          if (transposed ? pb == 1 : pb == 0) {
            mma(to, a, x);
          } else {
            const Op<T, N32> part[2] = {a[transposed ? 0 : 2], a[transposed ? 1 : 3]};
            mma(to, part, x, transposed ? 0 : 2);
          }
          __builtin_amdgcn_sched_barrier(0);
        };
        products(W1, false, wx, kc);
        products(W1q, true, w, qc);
        products(W3, false, w, kc);
        products(W3k, true, w, kc);
      }
    }
    now = fresh_arguments();
    const bool last_head = !SHARED || n == group - 1;
    const int item_then = SHARED ? items : next_live(item + gridDim.x);
    const bool more_items = item_then < items;
    const Item then = more_items ? item_at(item_then) : at;
    if constexpr (!SHARED) fetch_first(then, 0);   // (not under a condition: it would be waited for there)
    if (mine) {
      // q~ . (gamma dY S^T), k^ . (gamma Z S^T), k^ . (gamma_C / gamma R dS'^T) of each step, over this wave's columns
      float v[16];
      float* dot = dots + wave * C + 16 * (c16 / 4) + 4 * g + c16 % 4;
      auto factors_of = [&](int which, int rt) { return *reinterpret_cast<const f32x4*>(gate + which * C + 16 * rt + 4 * g); };
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const f32x4 ys = factors_of(GA, rt) * YS[rt], sq = factors_of(SQ, rt);
        dQ[rt] += wx[rt] + ys;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * rt + e] = (float)Q[(16 * rt + 4 * g + e) * LD + col] * sq[e] * ys[e];
      }
      dot[0] = over_columns(v, c16);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 k[4];
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const f32x4 zs = factors_of(GA, rt) * ZS[rt], sk = factors_of(SK, rt);
        dK[rt] += w[rt] - zs;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k[rt][e] = (float)K[(16 * rt + 4 * g + e) * LD + col] * sk[e];
          v[4 * rt + e] = k[rt][e] * zs[e];
        }
      }
      dot[WAVES * C] = over_columns(v, c16);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        const f32x4 rs = factors_of(LA, rt) * RS[rt];
        dK[rt] += factors_of(BE, rt) * rs;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * rt + e] = k[rt][e] * rs[e];
      }
      dot[2 * WAVES * C] = over_columns(v, c16);
    }
    __syncthreads();
    if (p.normalise && wave >= 6) {
      // q . dq and k . dk with the factors of both norms; the terms of dq and dk make sums that are there already, of rows and columns of F and those above
      const int i = lane;
      float sum = 0.0f;
      if (wave == 6) {
#pragma unroll
        for (int w = 0; w < 4; ++w) sum += (float)rowF[w * C + i];
#pragma unroll
        for (int w = 0; w < NT; ++w) sum += dots[w * C + i];
        sum *= gate[RQ * C + i];
      } else {
        float e = 0.0f, zs = 0.0f;
#pragma unroll
        for (int w = 4; w < 8; ++w) sum += (float)rowF[w * C + i];
#pragma unroll
        for (int w = 0; w < NT; ++w) zs += dots[(WAVES + w) * C + i], e += dots[(2 * WAVES + w) * C + i];
        sum = (sum + (float)colF_[i] + (float)colF_[C + i] + gate[BE * C + i] * e - zs) * gate[SK * C + i];
      }
      float* norm = norms + (wave - 6) * C + i;
      *norm = SHARED && n ? *norm + sum : sum;
    }
    if (wave == 0) {
      const int i = lane;
      // In 64 bits: of a sum from one step to the last what belongs to pairs of steps both behind it cancels, and each product's own rounding with it.
      double dG = 0.0;
      float second = 0.0f, all = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) dG += rowF[w * C + i];
      dG -= colF_[i] + colF_[C + i];
#pragma unroll
      for (int w = 0; w < NT; ++w) {
        dG += (double)dots[w * C + i] - dots[(WAVES + w) * C + i];
        second += dots[(2 * WAVES + w) * C + i];
        all += more[w];
      }
      const float beta = gate[BE * C + i], e = beta * second;
      const double ends = over_wave((double)e);
      dG -= e;
      if (i == C - 1) dG += ends + gate[GA * C + C - 1] * all;
      const float dlast = (float)from_lane_on(dG, i);   // sum from this step to the last one
      const float dbeta = cols[i] + cols[C + i] + second;
      float dlog = 0.0f, da = 0.0f;
      const int64_t s = s0 + i;
      const float bias_h = p.a.data && p.activate && p.bias ? p.bias[h] : 0.0f, A_h = p.a.data && p.activate ? p.A[h] : 0.0f;
      if (i < steps) {
        const bool in = i < live;
        if (p.a.data && in) {
          const float raw = (float)this_a + bias_h;
          if (p.activate) {
            dlog = dlast * (fmaxf(raw, 0.0f) + log1pf(expf(-fabsf(raw))));
            da = dlast * A_h / (1.0f + expf(-raw));
          } else {
            da = dlast;
          }
        }
        if (p.a.data) ((T*)p.da.data)[s * p.da.stride_t + b * p.da.stride_b + h] = (T)da;
        ((T*)p.db.data)[s * p.db.stride_t + b * p.db.stride_b + h] = (T)(!in ? 0.0f : p.activate ? dbeta * beta * (1.0f - beta) : dbeta);
      }
      dlog = over_wave(dlog);
      da = over_wave(p.activate ? da : 0.0f);
      if (lane == 0) {
        float* parts = parts_of(at);
        parts[h] = dlog;
        parts[p.H + h] = da;
      }
    }
    __syncthreads();   // `norms`; and this head has been read
    if (last_head) {
      if (mine && col < p.dk) {
        T *dq = out_of(p.dq, at), *dk = out_of(p.dkey, at);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
          f32x4 dqt = p.scale * dQ[rt], dkt = dK[rt];
          if (p.normalise) {
            const f32x4 rq = *reinterpret_cast<const f32x4*>(gate + RQ * C + 16 * rt + 4 * g), rk = *reinterpret_cast<const f32x4*>(gate + SK * C + 16 * rt + 4 * g);
            const f32x4 a = *reinterpret_cast<const f32x4*>(norms + 16 * rt + 4 * g), c = *reinterpret_cast<const f32x4*>(norms + C + 16 * rt + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = 16 * rt + 4 * g + e;
              dqt[e] = rq[e] * (dqt[e] - (float)Q[i * LD + col] * a[e]);
              dkt[e] = rk[e] * (dkt[e] - (float)K[i * LD + col] * c[e]);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 16 * rt + 4 * g + e;
            if (i < steps) {
              dq[(int64_t)i * p.dq.stride_t] = (T)(i < live ? dqt[e] : 0.0f);
              dk[(int64_t)i * p.dkey.stride_t] = (T)(i < live ? dkt[e] : 0.0f);
            }
          }
        }
      }
      if (!more_items) return;
      __syncthreads();   // k, q, gates and `norms` have been read
    }
    if constexpr (SHARED) {
      ++n;
    } else {
      item = item_then;
      at = then;
    }
  }
}

}  // namespace

int mebptt::delta::gradients(const Args& p, int dtype, hipStream_t stream) {
  return with_size(dtype, p.dk, [&](auto t, auto n) {
    using T = decltype(t);
    constexpr int KD = decltype(n)::value, BYTES = Layout<T, KD>::BYTES;
    static_assert(BYTES <= 160 * 1024, "LDS of a compute unit");
    auto go = [&](auto shared) {
      constexpr bool SHARED = decltype(shared)::value;
      const hipError_t e = allow_dynamic_lds<delta_gradients_kernel<T, KD, SHARED>>(BYTES);
      if (e != hipSuccess) return set_error(MEBPTT_EHIP, "LDS of the delta rule: %s", hipGetErrorString(e));
      const int64_t items = (int64_t)(p.c1 - p.c0) * p.B * p.Hk;
      const unsigned groups = (unsigned)(SHARED ? items : std::min<int64_t>(items, COMPUTE_UNITS));
      delta_gradients_kernel<T, KD, SHARED><<<groups, THREADS, BYTES, stream>>>(p);
      return launched("delta rule, gradients");
    };
    return p.H > p.Hk ? go(std::true_type{}) : go(std::false_type{});
  });
}
