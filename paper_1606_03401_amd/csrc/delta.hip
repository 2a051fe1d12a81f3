// Gated delta rule: entry points, and single tokens.
#include "delta.h"

using namespace mebptt;
using namespace mebptt::delta;

namespace {

// Chunks whose records a forward call's workspace holds at once: 163 MB of them in bf16.
constexpr int64_t RECORDS = 4096;

int check(const mebptt_delta_desc* d) {
  if (!d) return set_error(MEBPTT_EINVAL, "desc is NULL");
  if (d->t < 0 || d->t > 1 << 30) return set_error(MEBPTT_EINVAL, "t must be 0 .. 2^30");
  if (d->B < 0 || d->B > 65535) return set_error(MEBPTT_EINVAL, "B must be 0 .. 65535");
  if (d->H < 1 || d->H > MAX_HEADS || d->Hk < 1 || d->H % d->Hk) return set_error(MEBPTT_EINVAL, "H must be 1 .. %d and a multiple of Hk", MAX_HEADS);
  if ((int64_t)d->B * d->H > 1 << 22) return set_error(MEBPTT_EINVAL, "B * H must be at most 2^22");
  if (d->dk < 1 || d->dk > MAX_DK) return set_error(MEBPTT_EINVAL, "dk must be 1 .. %d", MAX_DK);
  if (d->dv < 1 || d->dv > MAX_DV) return set_error(MEBPTT_EINVAL, "dv must be 1 .. %d", MAX_DV);
  if (!float_dtype(d->dtype)) return set_error(MEBPTT_EINVAL, "unknown dtype");
  if (!(d->eps >= 0.0f)) return set_error(MEBPTT_EINVAL, "eps must not be negative");
  return MEBPTT_OK;
}
int check_stretch(const mebptt_delta_desc* d) {
  if (d->stretch < C || d->stretch > 1 << 20 || d->stretch % C) return set_error(MEBPTT_EINVAL, "stretch must be a multiple of %d up to 2^20", C);
  return MEBPTT_OK;
}
int check_seq(const mebptt_seq& s, const mebptt_delta_desc* d, const char* what) {
  if (!s.data) return set_error(MEBPTT_EINVAL, "%s is required", what);
  if (d->t > 1 && (s.stride_t < 0 || s.stride_t > NEAR)) return set_error(MEBPTT_EINVAL, "stride_t of %s must be 0 .. %lld", what, (long long)NEAR);
  return MEBPTT_OK;
}
int check_output(const mebptt_seq& s, const mebptt_delta_desc* d, int64_t channels, const char* what) {
  const int rc = check_seq(s, d, what);
  if (rc) return rc;
  return rows_apart(s, d->t, d->B, channels) ? MEBPTT_OK : set_error(MEBPTT_EINVAL, "rows of %s overlap", what);
}
int check_inputs(const mebptt_delta_desc* d, const mebptt_delta_inputs* in, bool steps) {
  int rc;
  if (!in) return set_error(MEBPTT_EINVAL, "in is NULL");
  if (steps && ((rc = check_seq(in->q, d, "q")) || (rc = check_seq(in->k, d, "k")) || (rc = check_seq(in->v, d, "v")) || (rc = check_seq(in->b, d, "b")) ||
                (in->a.data && (rc = check_seq(in->a, d, "a")))))
    return rc;
  if (d->activate && in->a.data && !in->A) return set_error(MEBPTT_EINVAL, "A is required");
  return MEBPTT_OK;
}

int64_t chunks_of(const mebptt_delta_desc* d) { return ceil_div(d->t, C); }
size_t state_bytes(const mebptt_delta_desc* d) { return align_up((size_t)d->B * d->H * d->dk * d->dv * 4); }

int whole(const mebptt_delta_desc* d, int n) {
  const int V = d->dtype == MEBPTT_FP32 ? 4 : 8;
  return (int)ceil_div(n, V) * V;
}
// Room for rows of q, k, v and dy that are copied to whole vectors (any may be: it depends on their addresses).
size_t row_bytes(const mebptt_delta_desc* d, int64_t chunks, int heads, int n) {
  return align_up((size_t)std::min<int64_t>(chunks * C, d->t) * d->B * heads * whole(d, n) * elem_bytes(d->dtype));
}

struct Forward {
  int64_t slab, seg;           // chunks of a launch, and of its segments
  size_t records, carry, moves, ends, starts, total;
};
// Segments of a launch: as many as fill the chip with the workgroups that walk, of at least eight chunks, since what segments do to the state has to be
// found out first, which costs as much again as the walk (dk + dv columns instead of dv, without y).
int64_t segment_of(const mebptt_delta_desc* d, int64_t chunks) {
  const int64_t groups = std::max<int64_t>(1, (int64_t)d->B * d->H * ceil_div(d->dv, 64));
  const int64_t n = std::min<int64_t>(256 / groups, chunks / 8);
  return n < 3 ? std::max<int64_t>(chunks, 1) : ceil_div(chunks, n);
}
Forward forward_layout(const mebptt_delta_desc* d) {
  const int64_t BH = (int64_t)d->B * d->H, chunks = chunks_of(d), KD = padded(d->dk), dvp = ceil_div(d->dv, 32) * 32;
  Forward f = {};
  f.slab = std::min(std::max<int64_t>(1, RECORDS / std::max<int64_t>(BH, 1)), std::max<int64_t>(chunks, 1));
  f.seg = segment_of(d, f.slab);
  const int64_t segments = ceil_div(f.slab, f.seg);
  f.records = align_up((size_t)(std::min(f.slab, chunks) * BH) * record_bytes(d->dtype, false));
  f.carry = f.slab < chunks ? state_bytes(d) : 0;
  if (segments > 1) {
    f.moves = align_up((size_t)((segments - 1) * BH) * KD * KD * 4);
    f.ends = align_up((size_t)((segments - 1) * BH) * KD * dvp * 4);
    f.starts = align_up((size_t)(segments * BH) * KD * dvp * 4);
  }
  f.total = f.records + f.carry + f.moves + f.ends + f.starts + 2 * row_bytes(d, f.slab, d->Hk, d->dk) + row_bytes(d, f.slab, d->H, d->dv);
  return f;
}
struct Backward {
  int64_t slab, seg;
  size_t records, states, rows, carry, parts, total;
};
// A stretch after the other, or, where there is little in one, as many at a time as have 512 chunks in all.
Backward backward_layout(const mebptt_delta_desc* d) {
  const int64_t BH = (int64_t)d->B * d->H, chunks = chunks_of(d), dvp = ceil_div(d->dv, 32) * 32;
  Backward w = {};
  w.seg = d->stretch / C;
  w.slab = std::min(w.seg * std::max<int64_t>(1, 512 / std::max<int64_t>(w.seg * BH, 1)), std::max<int64_t>(chunks, 1));
  const size_t n = (size_t)(std::min(w.slab, chunks) * BH);
  w.records = align_up(n * record_bytes(d->dtype, true));
  w.states = align_up(n * padded(d->dk) * dvp * 4);
  w.rows = align_up(n * C * dvp * 4);
  w.carry = w.slab < chunks ? state_bytes(d) : 0;
  w.parts = align_up((size_t)chunks * d->B * 2 * d->H * 4);
  w.total = w.records + 2 * w.states + 2 * w.rows + w.carry + w.parts + 2 * row_bytes(d, w.slab, d->Hk, d->dk) + 2 * row_bytes(d, w.slab, d->H, d->dv);
  return w;
}

Args args_of(const mebptt_delta_desc* d, const mebptt_delta_inputs* in) {
  Args p = {};
  p.a = in->a, p.b = in->b;
  p.A = in->A, p.bias = in->a_bias, p.lengths = in->lengths;
  p.t = d->t, p.B = d->B, p.Hk = d->Hk, p.H = d->H, p.dk = d->dk, p.dv = d->dv, p.dvp = (int)ceil_div(d->dv, 32) * 32;
  p.activate = d->activate, p.normalise = d->normalise, p.scale = d->scale, p.eps = d->eps;
  return p;
}
// Rows of a launch's steps as the kernels read them: in place, or copied to `room`, which moves on.  Copies have a sequence's steps next to each other, however
// the caller's lie: offsets inside a chunk have 32 bits, and with all sequences between two steps they would leave them.
Rows rows_of(Padded& all, const Args& p, const mebptt_delta_desc* d, const mebptt_seq& from, int heads, int n, char*& room, int64_t slab) {
  const int width = whole(d, n), V = d->dtype == MEBPTT_FP32 ? 4 : 8;
  if (width == n && rows_aligned(from, d->dtype, V)) return {from.data, from.stride_t, from.stride_b, n, n};
  char* at = room;
  room += row_bytes(d, slab, heads, n);
  all.one[all.n++] = {from, at, heads, n, width};
  static_assert((int64_t)MAX_HEADS * MAX_DV <= NEAR && MAX_DK <= MAX_DV && MAX_DV % 8 == 0, "a copy's steps are near each other");
  const int64_t st = (int64_t)heads * width, sb = launch_steps(p) * st;
  return {at - (int64_t)p.c0 * C * st * (int64_t)elem_bytes(d->dtype), st, sb, width, width};    // (as if it held all steps)
}

// ---- single tokens -------------------------------------------------------------------------------------

struct Step {
  mebptt_seq q, k, v, a, b, y;
  const float *A, *bias, *in;
  float* out;
  const int32_t* index;
  int64_t slots;
  int B, Hk, H, dk, dv, activate, normalise;
  float scale, eps;
};

// A workgroup has 4 LC columns of one sequence's and head's state, a thread up to 128 LC / 256 of its rows in four columns: read once, all
// loads on their way before the first is waited for, and written once.  With kS and qS from the same pass, y = scale (alpha qS + beta (q.k) r).
// Bound: HBM.  256 x 16 heads of 128 x 128: 114 us, 537 MB of states at 4.7 TB/s; 4 x 4 heads of 64 x 64: 6.6, a launch and two dependent reads.
template <typename T, int LC, bool VEC>
__global__ __launch_bounds__(256) void delta_step_kernel(Step p) {
  constexpr int RG = 256 / LC, ROWS = MAX_DK / RG;
  __shared__ float k_[MAX_DK], q_[MAX_DK], sums[4][3];
  __shared__ __align__(16) float dots[2][RG][4 * LC];
  const int bh = blockIdx.x, b = bh / p.H, h = bh % p.H, hk = h / (p.H / p.Hk);
  const int c0 = blockIdx.y * 4 * LC, lc = threadIdx.x % LC, rg = threadIdx.x / LC;
  const int64_t slot = p.index ? p.index[b] : b;
  T* y = (T*)p.y.data + b * p.y.stride_b + h * p.dv;
  if (slot < 0 || slot >= p.slots) {
    for (int c = c0 + threadIdx.x; c < min(c0 + 4 * LC, p.dv); c += 256) y[c] = (T)0.0f;
    return;
  }
  const int64_t base = (slot * p.H + h) * p.dk * p.dv;
  const float* in = p.in + base;
  auto column = [&](int e) { return VEC ? c0 + 4 * lc + e : c0 + lc + LC * e; };
  float s[ROWS][4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int d = rg + RG * i;
    if constexpr (VEC) {
      f32x4 x = {};
      if (d < p.dk && column(0) < p.dv) x = *reinterpret_cast<const f32x4*>(in + d * p.dv + column(0));
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = d < p.dk && column(e) < p.dv ? in[d * p.dv + column(e)] : 0.0f;
    }
  }
  const T* vp = (const T*)p.v.data + b * p.v.stride_b + h * p.dv;
  {   // k, q and the sums of their products
    float k = 0.0f, q = 0.0f;
    if (threadIdx.x < p.dk) {
      k = (float)((const T*)p.k.data)[b * p.k.stride_b + hk * p.dk + threadIdx.x];
      q = (float)((const T*)p.q.data)[b * p.q.stride_b + hk * p.dk + threadIdx.x];
    }
    if (threadIdx.x < MAX_DK) {
      k_[threadIdx.x] = k;
      q_[threadIdx.x] = q;
    }
    const float kk = wave_sum(k * k), qq = wave_sum(q * q), qk = wave_sum(q * k);
    if (threadIdx.x % WAVE == 0) {
      float* to = sums[threadIdx.x / WAVE];
      to[0] = kk, to[1] = qq, to[2] = qk;
    }
  }
  const float bv = (float)((const T*)p.b.data)[b * p.b.stride_b + h];
  const float beta = p.activate ? 1.0f / (1.0f + expf(-bv)) : bv;
  float lg = 0.0f;
  if (p.a.data) {
    lg = (float)((const T*)p.a.data)[b * p.a.stride_b + h];
    if (p.activate) {
      lg += p.bias ? p.bias[h] : 0.0f;
      lg = p.A[h] * (fmaxf(lg, 0.0f) + log1pf(expf(-fabsf(lg))));
    }
  }
  const float alpha = expf(lg);
  __syncthreads();
  float ks[4] = {}, qs[4] = {};
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float k = k_[rg + RG * i], q = q_[rg + RG * i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ks[e] += k * s[i][e];
      qs[e] += q * s[i][e];
    }
  }
  *reinterpret_cast<f32x4*>(&dots[0][rg][4 * lc]) = f32x4{ks[0], ks[1], ks[2], ks[3]};
  *reinterpret_cast<f32x4*>(&dots[1][rg][4 * lc]) = f32x4{qs[0], qs[1], qs[2], qs[3]};
  const float kk = sums[0][0] + sums[1][0], qq = sums[0][1] + sums[1][1];
  const float rk = p.normalise ? 1.0f / sqrtf(kk + p.eps) : 1.0f, rq = p.normalise ? 1.0f / sqrtf(qq + p.eps) : 1.0f;
  const float qk = (sums[0][2] + sums[1][2]) * rk * rq;
  __syncthreads();
  f32x4 kS = {}, qS = {};
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    kS += *reinterpret_cast<const f32x4*>(&dots[0][i][4 * lc]);
    qS += *reinterpret_cast<const f32x4*>(&dots[1][i][4 * lc]);
  }
  float r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = column(e);
    r[e] = c < p.dv ? beta * ((float)vp[c] - alpha * rk * kS[e]) : 0.0f;
    if (rg == 0 && c < p.dv) y[c] = (T)(p.scale * (alpha * rq * qS[e] + qk * r[e]));
    r[e] *= rk;
  }
  float* out = p.out + base;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int d = rg + RG * i;
    const float k = k_[d];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][e] = alpha * s[i][e] + k * r[e];
    if (d < p.dk) {
      if constexpr (VEC) {
        if (column(0) < p.dv) *reinterpret_cast<f32x4*>(out + d * p.dv + column(0)) = f32x4{s[i][0], s[i][1], s[i][2], s[i][3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (column(e) < p.dv) out[d * p.dv + column(e)] = s[i][e];
      }
    }
  }
}

template <typename T, int LC>
int step(const Step& p, bool vec, hipStream_t stream) {
  const dim3 grid((unsigned)(p.B * p.H), (unsigned)ceil_div(p.dv, 4 * LC));
  if (vec) delta_step_kernel<T, LC, true><<<grid, 256, 0, stream>>>(p);
  else delta_step_kernel<T, LC, false><<<grid, 256, 0, stream>>>(p);
  return launched("mebptt_delta_step");
}

}  // namespace

extern "C" {

size_t mebptt_delta_state_bytes(const mebptt_delta_desc* d) {
  if (check(d) || check_stretch(d)) return 0;
  return (size_t)ceil_div(d->t, d->stretch) * d->B * d->H * d->dk * d->dv * 4;
}

size_t mebptt_delta_workspace_bytes(const mebptt_delta_desc* d, int32_t backward) {
  if (check(d) || (backward && check_stretch(d))) return 0;
  const size_t f = forward_layout(d).total;
  return backward ? std::max(f, backward_layout(d).total) : f;
}

int mebptt_delta_forward(const mebptt_delta_desc* d, const mebptt_delta_inputs* in, mebptt_seq y, float* h_out, void* states,
                         size_t states_bytes, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check(d)) || (states && (rc = check_stretch(d)))) return rc;
  const bool steps = d->t && d->B;
  if ((rc = check_inputs(d, in, steps)) || (steps && (rc = check_output(y, d, (int64_t)d->H * d->dv, "y")))) return rc;
  if (states && steps) {
    if (states_bytes < mebptt_delta_state_bytes(d)) return set_error(MEBPTT_EWORKSPACE, "states have %zu bytes, %zu needed", states_bytes, mebptt_delta_state_bytes(d));
    if (!aligned(states, ALIGN)) return set_error(MEBPTT_EWORKSPACE, "states must be 256-byte aligned");
  }
  const Forward f = forward_layout(d);
  if ((rc = check_workspace(workspace, workspace_bytes, f.total))) return rc;
  if (!d->B) return MEBPTT_OK;
  hipStream_t s = (hipStream_t)stream;
  Args p = args_of(d, in);
  p.y = y;
  p.vec_out = d->dv % 4 == 0 && rows_aligned(y, d->dtype, 4);
  p.records = (char*)workspace;
  p.states = (float*)states;
  p.keep = states ? d->stretch / C : 1;
  const int64_t chunks = chunks_of(d);
  float* carry = (float*)((char*)workspace + f.records);
  if (!chunks) {
    p.from = in->h0, p.to = h_out, p.seg = 1;
    return h_out ? walk(p, d->dtype, WALK, s) : MEBPTT_OK;
  }
  for (int64_t c = 0; c < chunks; c += f.slab) {
    p.c0 = (int)c, p.c1 = (int)std::min(c + f.slab, chunks), p.seg = (int)f.seg;
    p.from = c ? carry : in->h0;
    p.to = p.c1 < chunks ? carry : h_out;
    char* room = (char*)workspace + f.records + f.carry;
    p.moves = (float*)room, p.ends = (float*)(room + f.moves);
    p.starts = p.c1 - p.c0 > p.seg ? (float*)(room + f.moves + f.ends) : nullptr, p.start_rows = padded(d->dk), p.start_width = p.dvp;
    room += f.moves + f.ends + f.starts;
    Padded all = {};
    p.q = rows_of(all, p, d, in->q, d->Hk, d->dk, room, f.slab);
    p.k = rows_of(all, p, d, in->k, d->Hk, d->dk, room, f.slab);
    p.v = rows_of(all, p, d, in->v, d->H, d->dv, room, f.slab);
    if ((rc = pad_rows(all, p, d->dtype, s))) return rc;
    if ((rc = prepare(p, d->dtype, false, s))) return rc;
    if (p.starts && ((rc = walk(p, d->dtype, SURVEY, s)) || (rc = join_segments(p, d->dtype, s)))) return rc;
    if ((rc = walk(p, d->dtype, WALK, s))) return rc;
  }
  return MEBPTT_OK;
}

int mebptt_delta_backward(const mebptt_delta_desc* d, const mebptt_delta_inputs* in, mebptt_seq dy, const float* dh_out,
                          const void* states, size_t states_bytes, const mebptt_delta_grads* grads, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check(d)) || (rc = check_stretch(d))) return rc;
  const bool steps = d->t && d->B;
  if ((rc = check_inputs(d, in, steps))) return rc;
  if (!grads) return set_error(MEBPTT_EINVAL, "grads is NULL");
  const int64_t qk = (int64_t)d->Hk * d->dk;
  if (steps && ((rc = check_seq(dy, d, "dy")) || (rc = check_output(grads->dq, d, qk, "dq")) || (rc = check_output(grads->dk, d, qk, "dk")) ||
                (rc = check_output(grads->dv, d, (int64_t)d->H * d->dv, "dv")) || (rc = check_output(grads->db, d, d->H, "db")) ||
                (in->a.data && (rc = check_output(grads->da, d, d->H, "da")))))
    return rc;
  if (steps) {
    if (!states) return set_error(MEBPTT_EINVAL, "states are required");
    if (states_bytes < mebptt_delta_state_bytes(d)) return set_error(MEBPTT_EWORKSPACE, "states have %zu bytes, %zu needed", states_bytes, mebptt_delta_state_bytes(d));
    if (!aligned(states, ALIGN)) return set_error(MEBPTT_EWORKSPACE, "states must be 256-byte aligned");
  }
  const Backward w = backward_layout(d);
  if ((rc = check_workspace(workspace, workspace_bytes, w.total))) return rc;
  hipStream_t s = (hipStream_t)stream;
  Args p = args_of(d, in);
  p.dq = grads->dq, p.dkey = grads->dk, p.dval = grads->dv, p.da = grads->da, p.db = grads->db;
  p.vec_out = d->dv % 4 == 0 && rows_aligned(grads->dv, d->dtype, 4);
  char* at = (char*)workspace;
  auto take = [&](size_t n) {
    char* got = at;
    at += n;
    return (float*)got;
  };
  p.records = (char*)take(w.records);
  p.S = take(w.states), p.dS = take(w.states), p.R = take(w.rows), p.Z = take(w.rows);
  float *carry = take(w.carry), *parts = take(w.parts);
  const int64_t chunks = chunks_of(d), BH = (int64_t)d->B * d->H;
  if (d->B && !chunks && grads->dh0) {
    p.from = dh_out, p.to = grads->dh0;
    if ((rc = walk_back(p, d->dtype, s))) return rc;
  }
  for (int64_t slab = d->B ? ceil_div(chunks, w.slab) : 0; slab-- > 0;) {
    p.c0 = (int)(slab * w.slab), p.c1 = (int)std::min(p.c0 + w.slab, chunks);
    p.parts = parts + (int64_t)p.c0 * d->B * 2 * d->H;
    char* room = at;
    Padded all = {};
    p.q = rows_of(all, p, d, in->q, d->Hk, d->dk, room, w.slab);
    p.k = rows_of(all, p, d, in->k, d->Hk, d->dk, room, w.slab);
    p.v = rows_of(all, p, d, in->v, d->H, d->dv, room, w.slab);
    p.dy = rows_of(all, p, d, dy, d->H, d->dv, room, w.slab);
    if ((rc = pad_rows(all, p, d->dtype, s))) return rc;
    if ((rc = prepare(p, d->dtype, true, s))) return rc;
    const int64_t state = BH * d->dk * d->dv;
    p.seg = (int)w.seg;
    p.starts = (float*)states + p.c0 / p.seg * state, p.start_rows = d->dk, p.start_width = d->dv;   // (read only)
    p.to = nullptr;
    if ((rc = walk(p, d->dtype, AGAIN, s))) return rc;
    p.from = p.c1 == chunks ? dh_out : carry;
    p.to = slab ? carry : grads->dh0;
    if ((rc = walk_back(p, d->dtype, s)) || (rc = gradients(p, d->dtype, s))) return rc;
  }
  if (!grads->dA && !grads->da_bias) return MEBPTT_OK;   // (zeros without an a, which an a of no steps cannot be told from)
  const int64_t cols[2] = {d->H, d->H};
  float* const outs[2] = {grads->dA, grads->da_bias};
  return sum_parts(parts, chunks * d->B, 2, cols, outs, s);
}

int mebptt_delta_step(const mebptt_delta_desc* d, const mebptt_delta_inputs* in, const float* state_in, int64_t slots, const int32_t* index,
                      mebptt_seq y, float* state_out, void* stream) {
  int rc;
  if ((rc = check(d))) return rc;
  if (d->t != 1) return set_error(MEBPTT_EINVAL, "t must be 1");
  if ((rc = check_inputs(d, in, d->B > 0))) return rc;
  if (!d->B) return MEBPTT_OK;
  if ((rc = check_output(y, d, (int64_t)d->H * d->dv, "y"))) return rc;
  if (slots < 0 || slots > 1ll << 31) return set_error(MEBPTT_EINVAL, "slots must be 0 .. 2^31");
  if (slots && (!state_in || !state_out)) return set_error(MEBPTT_EINVAL, "state_in and state_out are required");
  const Step p = {in->q, in->k, in->v, in->a, in->b, y, in->A, in->a_bias, state_in, state_out, index, slots, d->B, d->Hk, d->H, d->dk, d->dv,
                  d->activate, d->normalise, d->scale, d->eps};
  const bool vec = d->dv % 4 == 0 && aligned(state_in, 16) && aligned(state_out, 16);
  hipStream_t s = (hipStream_t)stream;
  auto at = [&](auto t) {
    using T = decltype(t);
    return d->dv <= 32 ? step<T, 8>(p, vec, s) : d->dv <= 64 ? step<T, 16>(p, vec, s) : step<T, 32>(p, vec, s);
  };
  return d->dtype == MEBPTT_FP32 ? at(float{}) : at(__bf16{});
}

}  // extern "C"
