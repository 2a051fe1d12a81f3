// AdamW over many tensors at once, states in 32 or 8 bits:
//     g = factor grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - rate decay) - rate (m / c1) / (sqrt(v / c2) + eps).
// Tensors are cut into pieces of at most PIECE values, a workgroup each; a table in device memory, written once, names every piece's tensor, so that
// any number of tensors takes one launch.  Bound: HBM.  40 tensors, 80 million values in all: 430 us with states in 32 bits and bf16 copies (30 bytes a value, 5.6
// TB/s), 264 with states in 8 bits, gradients in bf16 and copies (16 bytes, 4.8 TB/s; the vector unit's square root and division a value come close), the norm's
// pass over fp32 gradients 94 (3.4 TB/s, where a library's sum of as much takes 87).
#include "ops.h"

using namespace mebptt;
using namespace mebptt::ops;

namespace {

constexpr int BLOCK = 256;            // values that share a scale
constexpr int PIECE = 4096;           // whole blocks
constexpr int THREADS = 256, V = 8;   // neighbouring values of a thread
constexpr int SHARE = BLOCK / V;      // threads of a block: half a wave
constexpr int64_t MAX_TENSORS = 65536;
constexpr int NORM_GROUPS = 2048;

struct Entry {
  float* param;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  __bf16* copy;
  int64_t n, first;        // first: number of its first piece
  int64_t block;           // number of its first block over all tensors
  int grad_bf16, state8, no_decay, vec;
};
// An entry as a kernel reads it: through scalar loads, once, in place of loads after each store that might have changed it, and with pointers of which
// the compiler knows that they are to global memory.
template <typename T>
__device__ inline T* global(uint64_t address) { return (T*)(__attribute__((address_space(1))) T*)address; }
template <typename T>
__device__ inline T scalar(const void* p, int64_t at) { return ((const __attribute__((address_space(4))) T*)(uint64_t)p)[at]; }
__device__ inline Entry entry_of(const Entry* entries, int32_t tensor) {
  static_assert(sizeof(Entry) == 96 && offsetof(Entry, n) == 56 && offsetof(Entry, grad_bf16) == 80, "");
  uint64_t w[12];
#pragma unroll
  for (int i = 0; i < 12; ++i) w[i] = scalar<uint64_t>(entries + tensor, i);
  return {global<float>(w[0]), global<const void>(w[1]), global<void>(w[2]), global<void>(w[3]), global<float>(w[4]), global<float>(w[5]), global<__bf16>(w[6]),
          (int64_t)w[7], (int64_t)w[8], (int64_t)w[9], (int)w[10], (int)(w[10] >> 32), (int)w[11], (int)(w[11] >> 32)};
}
// [entries][a piece's tensor]
size_t map_at(int count) { return align_up((size_t)count * sizeof(Entry)); }

// ---- the table -----------------------------------------------------------------------------------------

constexpr int BATCH = 24;             // entries that one launch's arguments hold
struct Batch {
  Entry e[BATCH];
  int first, count;
};
__global__ void adamw_table_kernel(Batch b, Entry* entries, int32_t* map) {
  for (int i = blockIdx.x; i < b.count; i += gridDim.x) {
    if (threadIdx.x == 0 && blockIdx.y == 0) entries[b.first + i] = b.e[i];
    const int64_t pieces = (b.e[i].n + PIECE - 1) / PIECE;
    for (int64_t k = (int64_t)blockIdx.y * blockDim.x + threadIdx.x; k < pieces; k += (int64_t)gridDim.y * blockDim.x) map[b.e[i].first + k] = b.first + i;
  }
}

// ---- codes of 8 bits -----------------------------------------------------------------------------------

// 32 bits out of 32, each of which depends on all.
__device__ inline uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 17)) * 0x2C9277B5u;
  x = (x ^ (x >> 14)) * 0x5851F42Du;
  return x ^ (x >> 16);
}
// With bits of an fp32 below 2: exponent and three bits of the fraction, the exponent counted from 2^-15 or 2^-31.
template <bool SIGNED>
__device__ inline float value_of(uint32_t code, float scale) {
  const uint32_t low = SIGNED ? code & 127u : code;
  const float size = low ? __uint_as_float((low + ((SIGNED ? 112u : 96u) << 3)) << 20) * scale : 0.0f;
  return SIGNED && (code & 128u) ? -size : size;
}
// x / scale, correctly rounded, for x and scale of at least zero, by Markstein's correction: of a quotient that is off by one unit at most, the remainder
// is exact in a fused multiply-add, and its product with the nearest number to 1 / scale settles the rounding.  The first step of the two makes it so.
// (Where a remainder leaves fp32's range below, x / scale is under 2^-40 and only whether it is zero counts.)  A block's scale is shared, so its
// reciprocal is taken once: 4 operations a value in place of a division's 11.
constexpr float SMALL_SCALE = 0x1p-60f, LARGE_SCALE = 0x1p100f;   // beyond these plain division
__device__ inline float quotient(float x, float scale, float inverse) {
  const float q = x * inverse, q1 = fmaf(fmaf(-q, scale, x), inverse, q);
  return fmaf(fmaf(-q1, scale, x), inverse, q1);
}
// One of the two neighbours of u = |x| / scale; `bits16` says which where the part cut off leaves a choice.
template <bool SIGNED>
__device__ inline uint32_t code_of(float x, float u, uint32_t bits16) {   // (u is at most 1.875 and a rounding)
  const int code = (int)((__float_as_uint(u) + (bits16 << 4)) >> 20) - ((SIGNED ? 112 : 96) << 3);
  if constexpr (SIGNED) {
    constexpr float LEAST = 1.125f * 0x1p-15f;
    const uint32_t c = u < LEAST ? (u * (65536.0f / LEAST) > (float)bits16 ? 1u : 0u) : (uint32_t)min(max(code, 1), 127);
    return x < 0.0f && c ? c + 128u : c;
  } else {
    return x != 0.0f ? (uint32_t)min(max(code, 1), 255) : 0u;   // (u is 0 or NaN beside, and of, a value that left the range: its scale is infinite, and all that is not 0 stays so)
  }
}

struct Step {
  const Entry* entries;
  const int32_t* map;
  const float *factor, *rate;
  const int64_t* step;
  int64_t desc_step;
  float desc_rate, beta1, beta2, rest1, rest2, eps, decay, log1, log2;   // rest1, log1: 1 - beta1 and beta1's logarithm, from 64 bits
  uint32_t seed;
};

template <typename T, bool VEC>
__device__ inline void read(const T* p, int64_t left, float (&v)[V]) {
  if constexpr (VEC) {
    if (left >= V) return load<V>(p, v);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < left ? (float)p[e] : 0.0f;
}
template <typename T, bool VEC>
__device__ inline void write(T* p, int64_t left, const float (&v)[V]) {
  if constexpr (VEC) {
    if (left >= V) return store<V>(p, v);
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < left) p[e] = (T)v[e];
}
template <bool SIGNED, bool VEC>
__device__ inline void read_codes(const uint8_t* p, int64_t left, float scale, float (&v)[V]) {
  if constexpr (VEC) {
    if (left >= V) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = value_of<SIGNED>((w[e / 4] >> (8 * (e % 4))) & 255u, scale);
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < left ? value_of<SIGNED>(p[e], scale) : 0.0f;
}
// New codes and scale of a block that SHARE threads hold.
template <bool SIGNED, bool VEC>
__device__ inline void write_codes(uint8_t* p, float* scale, int64_t left, bool first, const float (&v)[V], const uint32_t (&bits)[V]) {
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < V; ++e) top = max_or_nan(top, fabsf(v[e]));
#pragma unroll
  for (int m = SHARE / 2; m; m >>= 1) top = max_or_nan(top, __shfl_xor(top, m));
  const float s = top * (1.0f / 1.875f);
  if (left <= 0) return;
  if (first) *scale = s;
  const bool plain = !(s >= SMALL_SCALE && s <= LARGE_SCALE);
  const float inverse = 1.0f / s;
  uint32_t c[V];
  if (plain) {
#pragma unroll
    for (int e = 0; e < V; ++e) c[e] = code_of<SIGNED>(v[e], s > 0.0f ? fabsf(v[e]) / s : fabsf(v[e]), SIGNED ? bits[e] >> 16 : bits[e] & 0xFFFFu);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) c[e] = code_of<SIGNED>(v[e], quotient(fabsf(v[e]), s, inverse), SIGNED ? bits[e] >> 16 : bits[e] & 0xFFFFu);
  }
  if constexpr (VEC) {
    if (left >= V) {
      *reinterpret_cast<u32x2*>(p) = u32x2{c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24};
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < left) p[e] = (uint8_t)c[e];
}

struct Factors {
  float factor, rate, keep, inv1, inv2;
  uint32_t key;
};
// N chunks of V values of each thread, the first from value `start` on; every load stands before the first store.  WHOLE: all values exist.
// One rounding to an operation, so that codes do not depend on what a compiler joins.
#pragma clang fp contract(off)
template <int N, bool WHOLE, bool VEC, bool STATE8, typename TG>
__device__ inline void chunks_step(const Step& p, const Entry& t, int64_t start, const Factors& f) {
  float w[N][V], g[N][V], m[N][V], v[N][V];
  int64_t at[N], left[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t i = start + k * (THREADS * V) + (int64_t)threadIdx.x * V;
    left[k] = WHOLE ? V : t.n - i;
    at[k] = left[k] > 0 ? i : 0;
    read<TG, VEC>((const TG*)t.grad + at[k], left[k], g[k]);
    if constexpr (STATE8) {
      read_codes<true, VEC>((const uint8_t*)t.m + at[k], left[k], t.m_scale[at[k] / BLOCK], m[k]);
      read_codes<false, VEC>((const uint8_t*)t.v + at[k], left[k], t.v_scale[at[k] / BLOCK], v[k]);
    } else {
      read<float, VEC>((const float*)t.m + at[k], left[k], m[k]);
      read<float, VEC>((const float*)t.v + at[k], left[k], v[k]);
    }
    read<float, VEC>(t.param + at[k], left[k], w[k]);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      g[k][e] *= f.factor;
      m[k][e] = p.beta1 * m[k][e] + p.rest1 * g[k][e];
      v[k][e] = p.beta2 * v[k][e] + p.rest2 * (g[k][e] * g[k][e]);
      w[k][e] = w[k][e] * f.keep - f.rate * (m[k][e] * f.inv1) / (sqrtf(v[k][e] * f.inv2) + p.eps);
    }
    write<float, VEC>(t.param + at[k], left[k], w[k]);
    if (t.copy) write<__bf16, VEC>(t.copy + at[k], left[k], w[k]);
    if constexpr (STATE8) {
      const int64_t block = at[k] / BLOCK;
      const uint32_t key = mix(f.key + (uint32_t)(t.block + block) * 0x9E3779B9u);
      uint32_t bits[V];
#pragma unroll
      for (int e = 0; e < V; ++e) bits[e] = mix(key + (uint32_t)(threadIdx.x % SHARE * V + e) * 0x85157AF5u);
      const bool first = threadIdx.x % SHARE == 0;
      write_codes<true, VEC>((uint8_t*)t.m + at[k], t.m_scale + block, left[k], first, m[k], bits);
      write_codes<false, VEC>((uint8_t*)t.v + at[k], t.v_scale + block, left[k], first, v[k], bits);
    } else {
      write<float, VEC>((float*)t.m + at[k], left[k], m[k]);
      write<float, VEC>((float*)t.v + at[k], left[k], v[k]);
    }
  }
}
template <bool STATE8, typename TG>
__device__ inline void piece_step(const Step& p, const Entry& t, int64_t start, const Factors& f) {
  constexpr int N = PIECE / (THREADS * V);
  if (t.vec && start + PIECE <= t.n) return chunks_step<N, true, true, STATE8, TG>(p, t, start, f);
  for (int k = 0; k < N && start + k * (THREADS * V) < t.n; ++k) {   // (the same for the whole workgroup)
    if (t.vec) chunks_step<1, false, true, STATE8, TG>(p, t, start + k * (THREADS * V), f);
    else chunks_step<1, false, false, STATE8, TG>(p, t, start + k * (THREADS * V), f);
  }
}
__global__ __launch_bounds__(THREADS) void adamw_step_kernel(Step p, int64_t pieces) {
  Factors f;
  f.factor = p.factor ? *p.factor : 1.0f;
  if (!__builtin_isfinite(f.factor)) return;
  f.rate = p.rate ? *p.rate : p.desc_rate;
  const int64_t step = p.step ? (*p.step < 1 ? 1 : *p.step) : p.desc_step;
  f.inv1 = p.beta1 > 0.0f ? -1.0f / expm1f((float)step * p.log1) : 1.0f;
  f.inv2 = p.beta2 > 0.0f ? -1.0f / expm1f((float)step * p.log2) : 1.0f;
  f.key = p.seed + (uint32_t)step * 0x632BE5ABu;
  for (int64_t k = blockIdx.x; k < pieces; k += gridDim.x) {
    const Entry t = entry_of(p.entries, scalar<int32_t>(p.map, k));
    const int64_t start = (k - t.first) * PIECE;
    f.keep = 1.0f - (t.no_decay ? 0.0f : f.rate * p.decay);
    if (t.state8) t.grad_bf16 ? piece_step<true, __bf16>(p, t, start, f) : piece_step<true, float>(p, t, start, f);
    else t.grad_bf16 ? piece_step<false, __bf16>(p, t, start, f) : piece_step<false, float>(p, t, start, f);
  }
}
#pragma clang fp contract(fast)

// ---- norm ----------------------------------------------------------------------------------------------

__device__ inline double wave_sum64(double v) {
#pragma unroll
  for (int m = WAVE / 2; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ inline double group_sum64(double v, double* lds) {
  v = wave_sum64(v);
  if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < THREADS / WAVE; ++w) v += lds[w];
  return v;
}
__global__ __launch_bounds__(THREADS) void adamw_squares_kernel(const Entry* entries, const int32_t* map, int64_t pieces, double* parts) {
  __shared__ double lds[THREADS / WAVE];
  double sum = 0.0;   // squares of large gradients leave fp32's range
  for (int64_t k = blockIdx.x; k < pieces; k += gridDim.x) {
    const Entry t = entry_of(entries, scalar<int32_t>(map, k));
    const int64_t start = (k - t.first) * PIECE;
#pragma unroll
    for (int j = 0; j < PIECE; j += THREADS * V) {
      const int64_t i = start + j + (int64_t)threadIdx.x * V, left = t.n - i, at = left > 0 ? i : 0;
      float g[V];
      if (t.grad_bf16) t.vec ? read<__bf16, true>((const __bf16*)t.grad + at, left, g) : read<__bf16, false>((const __bf16*)t.grad + at, left, g);
      else t.vec ? read<float, true>((const float*)t.grad + at, left, g) : read<float, false>((const float*)t.grad + at, left, g);
#pragma unroll
      for (int e = 0; e < V; ++e) sum += (double)g[e] * g[e];
    }
  }
  sum = group_sum64(sum, lds);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}
__global__ __launch_bounds__(THREADS) void adamw_norm_kernel(const double* parts, int n, float max_norm, float* out) {
  __shared__ double lds[THREADS / WAVE];
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += THREADS) sum += parts[i];
  sum = group_sum64(sum, lds);
  if (threadIdx.x) return;
  const float norm = (float)sqrt(sum);
  out[0] = norm;
  out[1] = !__builtin_isfinite(norm) ? __builtin_nanf("") : norm > max_norm ? max_norm / norm : 1.0f;
}

// ---- values of codes -----------------------------------------------------------------------------------

template <typename T, bool SIGNED, bool VEC>
__global__ __launch_bounds__(THREADS) void adamw_unpack_kernel(const uint8_t* codes, const float* scale, int64_t n, T* out) {
  for (int64_t i = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * V; i < n; i += (int64_t)gridDim.x * THREADS * V) {
    float v[V];
    read_codes<SIGNED, VEC>(codes + i, n - i, scale[i / BLOCK], v);
    write<T, VEC>(out + i, n - i, v);
  }
}

// ---- checks --------------------------------------------------------------------------------------------

// Number of pieces, or a negative error code.
int64_t count_pieces(const mebptt_adamw_tensor* t, int32_t count) {
  if (count < 0 || count > MAX_TENSORS) return set_error(MEBPTT_EINVAL, "count must be 0 .. %lld", (long long)MAX_TENSORS);
  if (count && !t) return set_error(MEBPTT_EINVAL, "tensors is NULL");
  int64_t pieces = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].n < 0 || t[i].n > 1ll << 40) return set_error(MEBPTT_EINVAL, "n of tensor %d must be 0 .. 2^40", i);
    pieces += ceil_div(t[i].n, PIECE);
  }
  if (pieces > (1ll << 42) / PIECE) return set_error(MEBPTT_EINVAL, "tensors have over 2^42 values");
  return pieces;
}
int check_table(const void* table, size_t bytes, const mebptt_adamw_tensor* t, int32_t count, int64_t* pieces) {
  *pieces = count_pieces(t, count);
  if (*pieces < 0) return (int)*pieces;
  const size_t needed = map_at(count) + align_up((size_t)*pieces * 4);
  if (!table) return set_error(MEBPTT_EWORKSPACE, "table is NULL");
  if (bytes < needed) return set_error(MEBPTT_EWORKSPACE, "table has %zu bytes, %zu needed", bytes, needed);
  if (!aligned(table, ALIGN)) return set_error(MEBPTT_EWORKSPACE, "table must be 256-byte aligned");
  return MEBPTT_OK;
}
unsigned grid_of(int64_t pieces, int64_t most) { return (unsigned)std::min<int64_t>(pieces, most); }

}  // namespace

extern "C" {

size_t mebptt_adamw_table_bytes(const mebptt_adamw_tensor* tensors, int32_t count) {
  const int64_t pieces = count_pieces(tensors, count);
  return pieces < 0 ? 0 : std::max(ALIGN, map_at(count) + align_up((size_t)pieces * 4));
}

int mebptt_adamw_prepare(const mebptt_adamw_tensor* tensors, int32_t count, void* table, size_t table_bytes, void* stream) {
  int64_t pieces;
  int rc = check_table(table, table_bytes, tensors, count, &pieces);
  if (rc) return rc;
  for (int i = 0; i < count; ++i) {
    const mebptt_adamw_tensor& t = tensors[i];
    if (!float_dtype(t.grad_dtype) || (t.state_dtype != MEBPTT_FP32 && t.state_dtype != MEBPTT_INT8)) return set_error(MEBPTT_EINVAL, "unknown dtype in tensor %d", i);
    if ((t.flags & ~MEBPTT_ADAMW_NO_DECAY) || t.reserved) return set_error(MEBPTT_EINVAL, "unknown flags in tensor %d", i);
    if (!t.n) continue;
    if (!t.param || !t.grad || !t.m || !t.v) return set_error(MEBPTT_EINVAL, "param, grad, m and v of tensor %d are required", i);
    if (t.state_dtype == MEBPTT_INT8 && (!t.m_scale || !t.v_scale)) return set_error(MEBPTT_EINVAL, "m_scale and v_scale of tensor %d are required", i);
  }
  int64_t first = 0, block = 0;
  for (int i = 0; i < count; i += BATCH) {
    Batch b = {};
    b.first = i;
    b.count = std::min(BATCH, count - i);
    int64_t most = 1;
    for (int k = 0; k < b.count; ++k) {
      const mebptt_adamw_tensor& t = tensors[i + k];
      const size_t unit = t.state_dtype == MEBPTT_INT8 ? 8 : 16;
      const bool vec = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.m, unit) && aligned(t.v, unit) && aligned(t.copy, 16);
      b.e[k] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, (__bf16*)t.copy, t.n, first, block, t.grad_dtype == MEBPTT_BF16,
                t.state_dtype == MEBPTT_INT8, t.flags & MEBPTT_ADAMW_NO_DECAY, vec};
      const int64_t n = ceil_div(t.n, PIECE);
      first += n;
      block += ceil_div(t.n, BLOCK);
      most = std::max(most, n);
    }
    adamw_table_kernel<<<dim3(b.count, (unsigned)std::min<int64_t>(ceil_div(most, 256), 1024)), 256, 0, (hipStream_t)stream>>>(
        b, (Entry*)table, (int32_t*)((char*)table + map_at(count)));
    if ((rc = launched("mebptt_adamw_prepare"))) return rc;
  }
  return MEBPTT_OK;
}

size_t mebptt_adamw_workspace_bytes(const mebptt_adamw_tensor* tensors, int32_t count) {
  const int64_t pieces = count_pieces(tensors, count);
  return pieces < 0 ? 0 : align_up((size_t)std::max<int64_t>(std::min<int64_t>(pieces, NORM_GROUPS), 1) * 8);
}

int mebptt_adamw_norm(const mebptt_adamw_tensor* tensors, int32_t count, const void* table, size_t table_bytes, float max_norm, float* out,
                      void* workspace, size_t workspace_bytes, void* stream) {
  int64_t pieces;
  int rc = check_table(table, table_bytes, tensors, count, &pieces);
  if (rc) return rc;
  if (!(max_norm > 0.0f)) return set_error(MEBPTT_EINVAL, "max_norm must be above 0");
  if (!out) return set_error(MEBPTT_EINVAL, "out is required");
  if ((rc = check_workspace(workspace, workspace_bytes, mebptt_adamw_workspace_bytes(tensors, count)))) return rc;
  const unsigned grid = grid_of(pieces, NORM_GROUPS);
  if (grid) {
    adamw_squares_kernel<<<grid, THREADS, 0, (hipStream_t)stream>>>((const Entry*)table, (const int32_t*)((const char*)table + map_at(count)), pieces,
                                                                      (double*)workspace);
    if ((rc = launched("mebptt_adamw_norm"))) return rc;
  }
  adamw_norm_kernel<<<1, THREADS, 0, (hipStream_t)stream>>>((const double*)workspace, (int)grid, max_norm, out);
  return launched("mebptt_adamw_norm");
}

int mebptt_adamw_step(const mebptt_adamw_desc* d, const mebptt_adamw_tensor* tensors, int32_t count, const void* table, size_t table_bytes,
                      const float* factor, const float* rate, const int64_t* step, void* stream) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (!(d->beta1 >= 0.0 && d->beta1 < 1.0 && d->beta2 >= 0.0 && d->beta2 < 1.0)) return set_error(MEBPTT_EINVAL, "beta1 and beta2 must be 0 .. below 1");
  if (!(d->eps >= 0.0)) return set_error(MEBPTT_EINVAL, "eps must not be negative");
  if (!step && d->step < 1) return set_error(MEBPTT_EINVAL, "step must be at least 1");
  int64_t pieces;
  const int rc = check_table(table, table_bytes, tensors, count, &pieces);
  if (rc || !pieces) return rc;
  const Step p = {(const Entry*)table, (const int32_t*)((const char*)table + map_at(count)), factor, rate, step, d->step, (float)d->rate, (float)d->beta1, (float)d->beta2,
                  (float)(1.0 - d->beta1), (float)(1.0 - d->beta2), (float)d->eps, (float)d->decay, (float)log(d->beta1), (float)log(d->beta2), d->seed};
  adamw_step_kernel<<<grid_of(pieces, 1 << 22), THREADS, 0, (hipStream_t)stream>>>(p, pieces);
  return launched("mebptt_adamw_step");
}

int mebptt_adamw_unpack(const uint8_t* codes, const float* scale, int64_t n, int32_t is_signed, void* out, int32_t out_dtype, void* stream) {
  if (n < 0 || n > 1ll << 42) return set_error(MEBPTT_EINVAL, "n must be 0 .. 2^42");
  if (!float_dtype(out_dtype)) return set_error(MEBPTT_EINVAL, "unknown dtype");
  if (!n) return MEBPTT_OK;
  if (!codes || !scale || !out) return set_error(MEBPTT_EINVAL, "codes, scale and out are required");
  const bool vec = aligned(codes, 8) && aligned(out, 16);
  const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(n, THREADS * V), 1 << 20);
  auto go = [&](auto t, auto sign) {
    using T = decltype(t);
    constexpr bool S = decltype(sign)::value;
    if (vec) adamw_unpack_kernel<T, S, true><<<grid, THREADS, 0, (hipStream_t)stream>>>(codes, scale, n, (T*)out);
    else adamw_unpack_kernel<T, S, false><<<grid, THREADS, 0, (hipStream_t)stream>>>(codes, scale, n, (T*)out);
    return launched("mebptt_adamw_unpack");
  };
  auto at = [&](auto t) { return is_signed ? go(t, std::true_type{}) : go(t, std::false_type{}); };
  return out_dtype == MEBPTT_FP32 ? at(float{}) : at(__bf16{});
}

}  // extern "C"
