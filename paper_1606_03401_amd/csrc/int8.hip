// Product of 8-bit integers with a scale per token and per channel:
//     out[m][n] = a_scale[m] * b_scale[n] * sum_k a[m][k] b[n][k] + bias[n]
// on v_mfma_i32_16x16x64_i8: exact 32-bit sums, one rounding at the end.  b's rows are the instruction's rows, a's its columns, so a
// lane's four results are neighbours along n and are stored at once.
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
  bool wide_store;   // four neighbours of a row of out lie on a boundary of their size
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

// Four neighbours along n of row m.
template <typename T>
__device__ inline void store4(const Product& p, int64_t m, int n, i32x4 acc) {
  if (m >= p.M || n >= p.N) return;
  const float sa = p.a_scale[m];
  T* out = (T*)p.out + m * p.ldo + n;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = min(n + i, p.N - 1);
    v[i] = (float)acc[i] * (sa * p.b_scale[c]) + (p.bias ? p.bias[c] : 0.0f);
  }
  if (p.wide_store && n + 4 <= p.N) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(out) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      union { __bf16 b[4]; u32x2 u; } r;
#pragma unroll
      for (int i = 0; i < 4; ++i) r.b[i] = (__bf16)v[i];
      *reinterpret_cast<u32x2*>(out) = r.u;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.N) out[i] = (T)v[i];
  }
}

// LDS rows of KB bytes; the four 16-byte parts of a row change places with the row, so that eight neighbouring rows' same part
// (what eight lanes read at a time) lie in eight different places of 128 bytes.
__device__ inline int place(int row, int part) { return row * KB + ((part ^ ((row >> 1) & 3)) * 16); }

// 64 x 64 outputs per workgroup, 32 x 32 per wave, operands through LDS one step ahead in registers.  Any size, stride and alignment.
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

int check(const mebptt_int8_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->M < 0 || d->M > (1 << 29)) return set_error(MEBPTT_EINVAL, "M must be 0 .. 2^29");
  if (d->N < 1 || d->N > (1 << 21)) return set_error(MEBPTT_EINVAL, "N must be 1 .. 2^21");
  if (d->K < 0 || d->K > MAX_K) return set_error(MEBPTT_EINVAL, "K must be 0 .. %d: the sums are 32 bits wide", MAX_K);
  if (!float_dtype(d->out_dtype)) return set_error(MEBPTT_EINVAL, "out_dtype must be MEBPTT_FP32 or MEBPTT_BF16");
  return MEBPTT_OK;
}

}  // namespace

extern "C" {

size_t mebptt_int8_workspace_bytes(const mebptt_int8_desc* d) {
  (void)d;
  return 0;
}

int mebptt_int8_product(const mebptt_int8_desc* d, const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb,
                        const float* b_scale, const float* bias, void* out, int64_t ldo, void* workspace, size_t workspace_bytes,
                        void* stream) {
  int rc = check(d);
  if (rc) return rc;
  if (d->M == 0) return MEBPTT_OK;
  if (!a_scale || !b_scale || !out || (d->K && (!a || !b))) return set_error(MEBPTT_EINVAL, "a required pointer is NULL");
  if ((d->K && (lda < d->K || ldb < d->K)) || ldo < d->N) return set_error(MEBPTT_EINVAL, "a row stride is below the row's length");
  if ((rc = check_workspace(workspace, workspace_bytes, mebptt_int8_workspace_bytes(d)))) return rc;
  Product p = {a, b, a_scale, b_scale, bias, out, d->M, lda, ldb, ldo, d->N, d->K, rows_aligned(out, ldo, d->out_dtype, 4)};
  const dim3 grid((unsigned)ceil_div(d->M, 64), (unsigned)ceil_div(d->N, 64));
  if (d->out_dtype == MEBPTT_FP32) int8_product_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(p);
  else int8_product_kernel<__bf16><<<grid, 256, 0, (hipStream_t)stream>>>(p);
  return launched("mebptt_int8_product");
}

}  // extern "C"
