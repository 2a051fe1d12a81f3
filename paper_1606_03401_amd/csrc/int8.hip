// Product of 8-bit integers with a scale per token and per channel:
//     out[m][n] = a_scale[m] * b_scale[n] * sum_k a[m][k] b[n][k] + bias[n]
// on the 8-bit matrix instructions: exact 32-bit sums, scaled in fp32 at the end.  b's rows are the instruction's rows, a's its columns, so a
// lane's four results are neighbours along n and are stored at once.  Three kernels: many rows by large tiles, few rows with b read once, and
// one for a K so short that neither's loads fit.
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int MAX_K = 131071;   // 2^14 * MAX_K < 2^31
constexpr int KB = 64;          // bytes of K per step: one instruction

struct Product {
  const int8_t *a, *b;
  const float *a_scale, *b_scale, *bias;
  void* out;
  int64_t M, lda, ldb, ldo;
  int N, K;
  bool wide_store, whole_store;   // four neighbours of a row of out, or 16 bytes, lie on a boundary of their size
};

typedef unsigned u32x4u __attribute__((ext_vector_type(4), aligned(1)));

// 16 bytes of a row from k on, zeros from K on.
__device__ inline u32x4 fetch(const int8_t* row, int k, int K) {
  if (k + 16 <= K) return *reinterpret_cast<const u32x4u*>(row + k);
  union { uint8_t b[16]; u32x4 v; } r;
  r.v = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (k + e < K) r.b[e] = (uint8_t)row[k + e];
  return r.v;
}

__device__ inline void pack4(float* to, const float (&v)[4]) { *reinterpret_cast<f32x4*>(to) = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ inline void pack4(__bf16* to, const float (&v)[4]) {
  union { __bf16 b[4]; u32x2 u; } r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.b[i] = (__bf16)v[i];
  *reinterpret_cast<u32x2*>(to) = r.u;
}

// sum * sa * sb + bias for any scales.  Their product alone may leave fp32's range where the result does not (2^-75 each and a sum of 2^26; a
// sum of zero and two large ones), so the sum is multiplied by one after the other.  Nothing is lost below the normal numbers on the way, as sums are
// whole numbers; a row's scale of 2^96 or more is taken 2^64 times smaller until the end, so that only a result that is too large overflows.
// One product more per value, which costs at most 1 % at 8192 x 4096 x 4096.
struct RowScale {
  float scale, rest;
  __device__ RowScale() = default;
  __device__ explicit RowScale(float sa) {
    const bool large = fabsf(sa) >= 0x1p96f;
    scale = large ? sa * 0x1p-64f : sa;
    rest = large ? 0x1p64f : 1.0f;
  }
  __device__ float operator()(int sum, float sb, float bias) const { return (float)sum * scale * sb * rest + bias; }
};

// Four neighbours along n of row m.
template <typename T>
__device__ inline void store4(const Product& p, int64_t m, int n, i32x4 acc) {
  if (m >= p.M || n >= p.N) return;
  const RowScale sa(p.a_scale[m]);
  T* out = (T*)p.out + m * p.ldo + n;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = min(n + i, p.N - 1);
    v[i] = sa(acc[i], p.b_scale[c], p.bias ? p.bias[c] : 0.0f);
  }
  if (p.wide_store && n + 4 <= p.N) {
    pack4(out, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.N) out[i] = (T)v[i];
  }
}

// LDS rows of KB bytes; the four 16-byte parts of a row change places with the row, so that eight neighbouring rows' same part
// (what eight lanes read at a time) lie in eight different places of 128 bytes.  (The counters have eight cycles to a read of 1 KB, 128 bytes a cycle,
// and count half of them as conflicts.)
__device__ inline int place(int row, int part) { return row * KB + ((part ^ ((row >> 1) & 3)) * 16); }

// 64 x 64 outputs per workgroup, 32 x 32 per wave, operands through LDS one step ahead in registers.  Any size, stride and alignment; in use
// where K is below 16, less than a lane's load of the others.
template <typename T>
__global__ __launch_bounds__(256) void int8_product_kernel(Product p) {
  __shared__ __align__(16) int8_t la[64 * KB], lb[64 * KB];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE;
  const int64_t m0 = (int64_t)blockIdx.x * 64;
  const int n0 = blockIdx.y * 64;
  const int row = tid / 4, part = tid % 4;
  const int8_t* arow = p.a + min(m0 + row, p.M - 1) * p.lda;
  const int8_t* brow = p.b + (int64_t)min(n0 + row, p.N - 1) * p.ldb;
  i32x4 acc[2][2] = {};
  u32x4 ra = fetch(arow, part * 16, p.K), rb = fetch(brow, part * 16, p.K);
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32, r = lane & 15, g = lane >> 4;
  for (int k = 0; k < p.K; k += KB) {
    *reinterpret_cast<u32x4*>(la + place(row, part)) = ra;
    *reinterpret_cast<u32x4*>(lb + place(row, part)) = rb;
    __syncthreads();
    if (k + KB < p.K) {
      ra = fetch(arow, k + KB + part * 16, p.K);
      rb = fetch(brow, k + KB + part * 16, p.K);
    }
    i32x4 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *reinterpret_cast<const i32x4*>(la + place(wm + 16 * i + r, g));
      fb[i] = *reinterpret_cast<const i32x4*>(lb + place(wn + 16 * i + r, g));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) store4<T>(p, m0 + wm + 16 * i + r, n0 + wn + 16 * j + 4 * g, acc[i][j]);
}

// ---- large tiles -------------------------------------------------------------------------------------
//
// BM x BN outputs per workgroup of four waves, (BM / 2) x (BN / 2) each.  Both operands come into LDS by the loads that write
// it directly, 64 bytes of K per stage, four stages: while a stage is multiplied, the next one's fragments are read into a second set of
// registers and three more are on their way.  Rows begin at 16-byte boundaries; only the last stage may be short, and goes through registers.
//
// Bound: the card's power, the matrix instructions, and what a tile does before and after them, with no other workgroup on its compute unit.  A stage of
// 256 x 256 is 1024 cycles of matrix instructions on every SIMD, 0.43 us at 2.4 GHz; its 32 KB written to LDS and 64 KB read take 768 at 128 bytes a
// cycle.  Measured with the chip full, K from 4096 to 16384: 0.54 us a stage on zeros, 0.85 on random operands, at 1.9 GHz, and 14 to 16 us a tile
// besides.  8192 x 4096 x 4096, two tiles per compute unit, 137 - 141 us, 2.0 POP/s, on zeros 100, the matrix unit 51 % busy; 8192^3 480 us, 2.3 POP/s, on
// zeros 366 (the library's 8-bit product 2.0 POP/s).  The order of K and the places in LDS make no difference to that.

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;
constexpr int vmcnt(int n) { return (n & 15) | 0x0f70 | (n >> 4) << 14; }

// Nothing moves across: the compiler would have every fragment read just before its product, and waited for.
__device__ inline void in_order() { __builtin_amdgcn_sched_barrier(0); }

template <typename T, int BM, int BN>
__global__ __launch_bounds__(256) void int8_tile_kernel(Product p, int tiles_m, int tiles_n) {
  constexpr int STAGE = (BM + BN) * KB, PIECES = (BM + BN) / 16 / 4;   // 1 KB pieces of 16 rows, per wave
  constexpr int TM = BM / 64, TN = BN / 64, KK = 2;                     // 32 x 32 tiles per wave; instructions per stage
  __shared__ __align__(16) int8_t s0[STAGE], s1[STAGE], s2[STAGE], s3[STAGE];   // apart, so that waits are told apart
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  // workgroups go to the eight XCDs in turn: each gets a run of tiles, which share rows of a or of b in its L2
  const int all = tiles_m * tiles_n, each = (all + 7) / 8;
  const int id = blockIdx.x % 8 * each + blockIdx.x / 8;
  if (id >= all) return;
  constexpr int BAND = 4;                                               // tiles along n before the next row of tiles
  const int band = id / (BAND * tiles_m), in_band = id % (BAND * tiles_m), width = min(BAND, tiles_n - band * BAND);
  const int tm = in_band / width, tn = band * BAND + in_band % width;
  const int64_t m0 = (int64_t)tm * BM;
  const int n0 = tn * BN;

  const int8_t* src[PIECES];        // this lane's 16 bytes of its pieces, stage 0
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int piece = wave * PIECES + i, r = lane >> 2, part = (lane & 3) ^ ((r >> 1) & 3);
    src[i] = (piece < BM / 16 ? p.a + min(m0 + piece * 16 + r, p.M - 1) * p.lda
                              : p.b + (int64_t)min(n0 + (piece - BM / 16) * 16 + r, p.N - 1) * p.ldb) + part * 16;
  }
  const int full = p.K / KB;
  auto fill_piece = [&](int8_t* buf, int64_t k, int i) {
    __builtin_amdgcn_global_load_lds((global_void*)(src[i] + k), (lds_void*)(buf + (wave * PIECES + i) * 1024), 16, 0, 0);
  };
  auto fill = [&](int8_t* buf, int s) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) fill_piece(buf, (int64_t)s * KB, i);
  };
  const int r = lane & 31, g = lane >> 5, wm = (wave & 1) * (BM / 2), wn = BM + (wave >> 1) * (BN / 2);
  i32x16 acc[TM][TN] = {};
  i32x4 f[2][TM + TN][KK];            // fragments of a, then of b, of this stage and of the next
  constexpr int READS = (TM + TN) * KK, PRODUCTS = TM * TN * KK, HALF = PRODUCTS / 2;
  auto read = [&](const int8_t* buf, i32x4 (&to)[TM + TN][KK], int n) {
    const int i = n / KK, k = n % KK;
    to[i][k] = *reinterpret_cast<const i32x4*>(buf + place((i < TM ? wm + 32 * i : wn + 32 * (i - TM)) + r, 2 * k + g));
  };
  auto multiply = [&](i32x4 (&from)[TM + TN][KK], int n) {
    const int i = n / KK / TN, j = n / KK % TN, k = n % KK;
    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(from[TM + j][k], from[i][k], acc[i][j], 0, 0, 0);
  };
  // Waits until a stage is in LDS for every wave; behind it are the loads of exactly two more.
  auto arrive = [&]() {
    __builtin_amdgcn_s_waitcnt(vmcnt(2 * PIECES));
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): what this wave read of the stage before
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Stage s, whose fragments are in `now`.  Half of its products, while the next stage arrives; once the barrier is passed the stage's own buffer
  // has been read by all and is filled with the stage four later, and the next stage is read, an instruction or two after every one of the
  // other products, which take long enough to hide them.  Past the last stage the fills repeat it and what is read is not used, so that every
  // step is the same.
  const int fours = full & ~3;
  auto step = [&](int s, int8_t* own, const int8_t* following, i32x4 (&now)[TM + TN][KK], i32x4 (&next)[TM + TN][KK]) {
#pragma unroll
    for (int n = 0; n < HALF; ++n) multiply(now, n);
    in_order();
    arrive();
    in_order();
    const int64_t later = (int64_t)min(s + 4, fours - 1) * KB;
#pragma unroll
    for (int n = 0; n < HALF; ++n) {
      multiply(now, HALF + n);
      in_order();
#pragma unroll
      for (int m = n * READS / HALF; m < (n + 1) * READS / HALF; ++m) read(following, next, m);
#pragma unroll
      for (int m = n * PIECES / HALF; m < (n + 1) * PIECES / HALF; ++m) fill_piece(own, later, m);
      in_order();
    }
  };
  if (fours > 0) {
    fill(s0, 0);
    fill(s1, 1);
    fill(s2, 2);
    arrive();
    fill(s3, 3);
#pragma unroll
    for (int n = 0; n < READS; ++n) read(s0, f[0], n);
    for (int s = 0; s < fours; s += 4) {
      step(s, s0, s1, f[0], f[1]);
      step(s + 1, s1, s2, f[1], f[0]);
      step(s + 2, s2, s3, f[0], f[1]);
      step(s + 3, s3, s0, f[1], f[0]);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt(0));   // nothing may still be written into LDS when it is used otherwise, or given back
  }
  if (fours * KB < p.K) {   // up to three stages and a short one, all at once
    __syncthreads();
    if (full > fours) fill(s0, fours);
    if (full > fours + 1) fill(s1, fours + 1);
    if (full > fours + 2) fill(s2, fours + 2);
    if (p.K % KB) {
      const int k = full * KB, part = (lane & 3) ^ ((lane >> 3) & 3);
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        *reinterpret_cast<u32x4*>(s3 + (wave * PIECES + i) * 1024 + lane * 16) = fetch(src[i] + k, 0, p.K - k - part * 16);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt(0));
    __syncthreads();
    for (int s = fours; s * KB < p.K; ++s) {
      const int8_t* buf = s == full ? s3 : s == fours ? s0 : s == fours + 1 ? s1 : s2;
#pragma unroll
      for (int n = 0; n < READS; ++n) read(buf, f[0], n);
#pragma unroll
      for (int n = 0; n < PRODUCTS; ++n) multiply(f[0], n);
    }
  }

  // Out by way of LDS, whole rows of the wave's part at a time: a lane has 4 neighbours along n of one row, 16 bytes of which meet with
  // another lane's.  A row's 16-byte parts change places with the row, so that 16 rows written at once lie in different banks.
  constexpr int ROWS = BM / 2, PASS = std::min(BN / 2, 256 / (int)sizeof(T)), ROW = PASS * (int)sizeof(T), PARTS = ROW / 16;
  static_assert(ROWS * ROW <= STAGE, "");
  __syncthreads();
  int8_t* mine = wave == 0 ? s0 : wave == 1 ? s1 : wave == 2 ? s2 : s3;
  RowScale sa[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) sa[i] = RowScale(p.a_scale[min(m0 + wm + 32 * i + r, p.M - 1)]);
  const int first_n = n0 + wn - BM;
#pragma unroll
  for (int pass = 0; pass < BN / 2 / PASS; ++pass) {
#pragma unroll
    for (int j = pass * PASS / 32; j < (pass + 1) * PASS / 32; ++j) {
      float sb[16], bias[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int n = min(first_n + 32 * j + 8 * (e / 4) + 4 * g + e % 4, p.N - 1);
        sb[e] = p.b_scale[n];
        bias[e] = p.bias ? p.bias[n] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = sa[i](acc[i][j][4 * e + c], sb[4 * e + c], bias[4 * e + c]);
          const int at = (32 * j + 8 * e + 4 * g - pass * PASS) * (int)sizeof(T), row = 32 * i + r;
          pack4(reinterpret_cast<T*>(mine + row * ROW + ((at / 16) ^ (row & (PARTS - 1))) * 16 + at % 16), v);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (a wave's own part)
    __builtin_amdgcn_wave_barrier();
#pragma unroll 4
    for (int t = 0; t < ROWS * PARTS / WAVE; ++t) {
      const int row = (t * WAVE + lane) / PARTS, part = lane % PARTS;
      const u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * ROW + (part ^ (row & (PARTS - 1))) * 16);
      const int64_t m = m0 + wm + row;
      const int n = first_n + pass * PASS + part * (16 / (int)sizeof(T));
      if (m < p.M && n < p.N) {
        T* out = (T*)p.out + m * p.ldo + n;
        if (p.whole_store && n + 16 / (int)sizeof(T) <= p.N) {
          *reinterpret_cast<u32x4*>(out) = v;
        } else {
          union { u32x4 u; T e[16 / sizeof(T)]; } x;
          x.u = v;
#pragma unroll
          for (int e = 0; e < 16 / (int)sizeof(T); ++e)
            if (n + e < p.N) out[e] = x.e[e];
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- few rows ----------------------------------------------------------------------------------------
//
// Single tokens of some sequences: every weight is read once, and its bytes are the bound (32 x 16384 x 4096: 18.8 us, 3.6 TB/s, of which launch and first
// bytes take 4).  A workgroup takes 16 MT rows of a and, in turn, tiles
// of 16 rows of b; its eight waves share K.  A wave reads its part of b's tile straight into the instruction's registers, all of it at
// once and a tile ahead, and the waves' sums meet in LDS.  HELD: a wave's part of a (at most STEPS steps of K) stays in registers for
// all tiles; otherwise it is read again, STEPS steps at a time.
//
// K is at least 16.  A lane whose 16 bytes would pass K's end reads the last 16 of both rows, those of a that it should not have as zeros.
template <typename T, int MT, int STEPS, bool HELD>
__global__ __launch_bounds__(512) void int8_rows_kernel(Product p, int tiles, int gx) {
  constexpr int WAVES = 8;
  __shared__ i32x4 red[2][WAVES][MT][WAVE];
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), r = lane & 15, g = lane >> 4;
  const int bx = blockIdx.x % gx;
  const int64_t m0 = (int64_t)(blockIdx.x / gx) * 16 * MT;
  const int8_t* arow[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) arow[i] = p.a + min(m0 + 16 * i + r, p.M - 1) * p.lda;
  const int steps = (p.K + KB - 1) / KB, each = (steps + WAVES - 1) / WAVES;
  const int first = wave * each, last = min(steps, first + each);       // (last < first: a wave without work)
  auto offset = [&](int s) { return min(s * KB + 16 * g, p.K - 16); };
  auto read_b = [&](int tile, int s0, u32x4 (&b)[STEPS]) {
    const int8_t* row = p.b + (int64_t)min(tile * 16 + r, p.N - 1) * p.ldb;
#pragma unroll
    for (int u = 0; u < STEPS; ++u) b[u] = *reinterpret_cast<const u32x4u*>(row + offset(s0 + u));
  };
  auto read_a = [&](int s0, u32x4 (&a)[STEPS][MT]) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i) a[u][i] = *reinterpret_cast<const u32x4u*>(arow[i] + offset(s0 + u));
    if (s0 + STEPS <= last && (s0 + STEPS) * KB <= p.K) return;
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int skip = s0 + u < last ? (s0 + u) * KB + 16 * g - offset(s0 + u) : 16;   // bytes that another lane has, or that are not this wave's
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int drop = min(max(skip - 4 * e, 0), 4);
          a[u][i][e] = drop >= 4 ? 0u : a[u][i][e] >> (8 * drop) << (8 * drop);
        }
    }
  };
  auto mma = [&](const u32x4 (&b)[STEPS], const u32x4 (&a)[STEPS][MT], i32x4 (&acc)[MT]) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
        acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, b[u]), __builtin_bit_cast(i32x4, a[u][i]), acc[i], 0, 0, 0);
  };
  u32x4 a[STEPS][MT], b[STEPS], ahead[STEPS];
  read_b(bx, first, b);
  if (HELD) read_a(first, a);
  int turn = 0;
  for (int tile = bx; tile < tiles; tile += gx, turn ^= 1) {
    i32x4 acc[MT] = {};
    if constexpr (HELD) {
      if (tile + gx < tiles) read_b(tile + gx, first, ahead);
      __builtin_amdgcn_sched_barrier(0);   // the loads first, all of them
      mma(b, a, acc);
    } else {
      for (int s = first; s < last; s += STEPS) {
        read_a(s, a);
        if (s + STEPS < last) read_b(tile, s + STEPS, ahead);
        else if (tile + gx < tiles) read_b(tile + gx, first, ahead);
        __builtin_amdgcn_sched_barrier(0);
        mma(b, a, acc);
#pragma unroll
        for (int u = 0; u < STEPS; ++u) b[u] = ahead[u];
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) red[turn][wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < MT) {
      i32x4 sum = red[turn][0][wave][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum += red[turn][w][wave][lane];
      store4<T>(p, m0 + 16 * wave + r, tile * 16 + 4 * g, sum);
    }
    if constexpr (HELD) {
#pragma unroll
      for (int u = 0; u < STEPS; ++u) b[u] = ahead[u];
    }
  }
}

int check(const mebptt_int8_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->M < 0 || d->M > (1 << 28)) return set_error(MEBPTT_EINVAL, "M must be 0 .. 2^28");
  if (d->N < 1 || d->N > (1 << 21)) return set_error(MEBPTT_EINVAL, "N must be 1 .. 2^21");
  if (d->M * d->N > (int64_t)1 << 38) return set_error(MEBPTT_EINVAL, "M * N must not exceed 2^38");
  if (d->K < 0 || d->K > MAX_K) return set_error(MEBPTT_EINVAL, "K must be 0 .. %d: the sums are 32 bits wide", MAX_K);
  if (!float_dtype(d->out_dtype)) return set_error(MEBPTT_EINVAL, "out_dtype must be MEBPTT_FP32 or MEBPTT_BF16");
  return MEBPTT_OK;
}

// ---- operands whose rows begin anywhere -----------------------------------------------------------------

// Copies of rows that do not begin at 16-byte boundaries, with zeros up to the next one: 16 bytes per thread.
struct Copy {
  const int8_t* from;
  int8_t* to;
  int64_t rows, ld, to_ld;
  int K;
};
__global__ __launch_bounds__(256) void int8_copy_kernel(Copy a, Copy b) {
  const int64_t parts = a.to_ld / 16;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < (a.rows + b.rows) * parts; k += (int64_t)gridDim.x * 256) {
    const int64_t row = k / parts, part = k % parts;
    const bool second = row >= a.rows;
    const Copy& c = second ? b : a;
    const int64_t r = second ? row - a.rows : row;
    *reinterpret_cast<u32x4*>(c.to + r * c.to_ld + part * 16) = fetch(c.from + r * c.ld, (int)part * 16, c.K);
  }
}

// The three kernels by what a launch is estimated to take, in us, fitted to 15 shapes timed on all of them (M 1 .. 8192, N 512 .. 16384,
// K 512 .. 8192; within a quarter of the times measured).  A tile's stages take longer the fuller the
// chip is.  Measured, rows / 128 / 256: 32 x 16384 x 4096 20 / 30 / 66, 512 x 512 x 4096 11.5 / 18.8 / 45, 1024 x 4096 x 4096 48 / 25 / 49,
// 8192 x 4096 x 4096 310 / 221 / 169.
struct Estimate {
  double rows, t128, t256;
  double tiles() const { return std::min(t128, t256); }
};
constexpr int ROWS_GROUPS = 256;   // a workgroup per compute unit; two read a twice as often: 26 instead of 20 us at 32 x 16384 x 4096
Estimate estimate(int64_t M, int N, int K) {
  const double stages = (double)ceil_div(K, KB);
  const int64_t m_tiles = ceil_div(M, M <= 16 ? 16 : M <= 32 ? 32 : 64);
  const int64_t t128 = ceil_div(M, 128) * ceil_div(N, 128), t256 = ceil_div(M, 256) * ceil_div(N, 256);
  Estimate e;
  e.rows = 3 + K / 600.0 + (double)ceil_div(ceil_div(N, 16) * m_tiles, ROWS_GROUPS) * (1.1 + K / 2700.0);
  e.t128 = 4 + stages * (t128 <= 256 ? 0.3 : 0.86 * (double)ceil_div(t128, 512));
  e.t256 = (double)ceil_div(t256, 256) * (13 + stages * (0.52 + 0.58 * (double)std::min<int64_t>(t256, 256) / 256));
  return e;
}

// Where K is no multiple of 16, rows that follow each other begin anywhere, and reading them so by rows takes up to three times as long, copies and
// their launch at least 10 us.  Measured, by rows / from copies: 777 x 1301 x 650 16 / 20, 1000 x 1000 x 1001 12 / 20, 512 x 4096 x 1022
// 28 / 21, 4000 x 4096 x 510 110 / 41, 8192 x 4096 x 4095 980 / 198.  Whether copies of both operands and tiles are faster:
bool copies_pay(int64_t M, int N, int K) {
  if (K % 16 == 0 || K < 16 || M <= 64) return false;
  const Estimate e = estimate(M, N, K);
  return e.tiles() + 10 + (double)(M + N) * K / 3.0e6 < 1.6 * e.rows;
}
int64_t copied_ld(int K) { return ceil_div(K, 16) * 16; }
size_t copy_bytes(int64_t rows, int K) { return align_up((size_t)rows * copied_ld(K)); }

template <typename T>
int launch(const Product& p, hipStream_t stream) {
  using std::integral_constant;
  auto tiles = [&](auto size) {
    constexpr int SIZE = decltype(size)::value;
    const int64_t tm = ceil_div(p.M, SIZE), tn = ceil_div(p.N, SIZE);
    int8_tile_kernel<T, SIZE, SIZE><<<(unsigned)(ceil_div(tm * tn, 8) * 8), 256, 0, stream>>>(p, (int)tm, (int)tn);
  };
  // fewer steps of K per wave than 8 where K is short
  auto rows = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    const int n = (int)ceil_div(p.N, 16);
    const int64_t my = ceil_div(p.M, 16 * MT), each = ceil_div(ceil_div(p.K, KB), 8);
    const int64_t gx = std::min<int64_t>(n, std::max<int64_t>(1, ROWS_GROUPS / my));
    const unsigned grid = (unsigned)(gx * my);
    if (each <= 1) int8_rows_kernel<T, MT, 1, true><<<grid, 512, 0, stream>>>(p, n, (int)gx);
    else if (each <= 2) int8_rows_kernel<T, MT, 2, true><<<grid, 512, 0, stream>>>(p, n, (int)gx);
    else if (each <= 4) int8_rows_kernel<T, MT, 4, true><<<grid, 512, 0, stream>>>(p, n, (int)gx);
    else if (each <= 8) int8_rows_kernel<T, MT, 8, true><<<grid, 512, 0, stream>>>(p, n, (int)gx);
    else int8_rows_kernel<T, MT, 4, false><<<grid, 512, 0, stream>>>(p, n, (int)gx);
  };
  const Estimate e = estimate(p.M, p.N, p.K);
  const bool rows16 = aligned(p.a, 16) && aligned(p.b, 16) && p.lda % 16 == 0 && p.ldb % 16 == 0;   // what the tiles' loads need
  if (p.K < 16) {
    const dim3 grid((unsigned)ceil_div(p.M, 64), (unsigned)ceil_div(p.N, 64));
    int8_product_kernel<T><<<grid, 256, 0, stream>>>(p);
  } else if (!rows16 || (e.rows <= e.t128 && e.rows <= e.t256)) {
    if (p.M <= 16) rows(integral_constant<int, 1>{});
    else if (p.M <= 32) rows(integral_constant<int, 2>{});
    else rows(integral_constant<int, 4>{});
  } else if (e.t128 <= e.t256) {
    tiles(integral_constant<int, 128>{});
  } else {
    tiles(integral_constant<int, 256>{});
  }
  return launched("mebptt_int8_product");
}

}  // namespace

extern "C" {

size_t mebptt_int8_workspace_bytes(const mebptt_int8_desc* d) {
  if (check(d) != MEBPTT_OK || !copies_pay(d->M, d->N, d->K)) return 0;
  return copy_bytes(d->M, d->K) + copy_bytes(d->N, d->K);
}

int mebptt_int8_product(const mebptt_int8_desc* d, const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb,
                        const float* b_scale, const float* bias, void* out, int64_t ldo, void* workspace, size_t workspace_bytes,
                        void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->M == 0) return MEBPTT_OK;
  if (!a_scale || !b_scale || !out || (d->K && (!a || !b))) return set_error(MEBPTT_EINVAL, "a required pointer is NULL");
  if ((d->K && (lda < d->K || ldb < d->K)) || ldo < d->N) return set_error(MEBPTT_EINVAL, "a row stride is below the row's length");
  Product p = {a, b, a_scale, b_scale, bias, out, d->M, lda, ldb, ldo, d->N, d->K, rows_aligned(out, ldo, d->out_dtype, 4),
               rows_aligned(out, ldo, d->out_dtype, 8)};
  const hipStream_t st = (hipStream_t)stream;
  if (copies_pay(d->M, d->N, d->K)) {
    const int64_t ld = copied_ld(d->K);
    auto ready = [](const int8_t* x, int64_t ldx) { return aligned(x, 16) && ldx % 16 == 0; };
    Copy ca = {a, nullptr, ready(a, lda) ? 0 : d->M, lda, ld, d->K}, cb = {b, nullptr, ready(b, ldb) ? 0 : d->N, ldb, ld, d->K};
    // (rows that are ready need no room)
    if ((rc = check_workspace(workspace, workspace_bytes, copy_bytes(ca.rows, d->K) + copy_bytes(cb.rows, d->K)))) return rc;
    ca.to = (int8_t*)workspace;
    cb.to = ca.to + copy_bytes(ca.rows, d->K);
    if (ca.rows) p.a = ca.to, p.lda = ld;
    if (cb.rows) p.b = cb.to, p.ldb = ld;
    if (ca.rows + cb.rows) {
      int8_copy_kernel<<<(unsigned)std::min<int64_t>(ceil_div((ca.rows + cb.rows) * (ld / 16), 256), 1 << 16), 256, 0, st>>>(ca, cb);
      if ((rc = launched("mebptt_int8_product"))) return rc;
    }
  }
  return d->out_dtype == MEBPTT_FP32 ? launch<float>(p, st) : launch<__bf16>(p, st);
}

}  // extern "C"
