// What a served target's logits leave to train on, and the loss that is trained on it:
//   topk_logits   the k largest logits of every row, in order, with the row's log-sum-exp
//   distill       KL divergence of a student's logits from a teacher's top logits, and its gradient
// Both pass over [rows, vocab] arrays of logits that do not fit any cache: what bounds them is memory.
#include "kernels.h"
#include "prof.h"
#include "tide_common.h"

namespace tide {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Order of the logits: a key that ascends as the values do, with every NaN above +inf and one zero.  Together with the
// complement of the index it is unique in a row and says "larger value first, equal values by ascending index".
constexpr uint32_t kNanKey = 0xFFFFFFFEu;   // (a pair of all ones is larger than every element's)
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return kNanKey;
  const uint32_t b = __float_as_uint(v + 0.f);   // -0 + 0 = +0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == kNanKey) return __uint_as_float(0x7FC00000u);
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
__device__ __forceinline__ uint64_t order_pair(float v, int idx) { return ((uint64_t)order_key(v) << 32) | (uint32_t)~idx; }

// Running (max, sum of 2^(c (z - max))) over eight more values.  The difference comes first: it is 0 for the largest value whatever
// that is, also where c times it has no number (columns masked with the type's lowest value).
struct Online { float m, s; };
__device__ __forceinline__ void online_add8(Online& o, const float (&v)[8], float c) {
  float cm = v[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) cm = fmaxf(cm, v[j]);
  const float nm = fmaxf(o.m, cm);
  const float sh = nm == -INFINITY ? 0.f : nm;      // nothing but -inf so far: every term is 0
  float part = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) part += __builtin_amdgcn_exp2f((v[j] - sh) * c);
  o.s = (o.m == -INFINITY ? o.s : o.s * __builtin_amdgcn_exp2f((o.m - nm) * c)) + part;   // (before any number: 0, or NaN)
  o.m = nm;
}
__device__ __forceinline__ Online online_join(const Online& a, const Online& b, float c) {
  const float nm = fmaxf(a.m, b.m);
  const float sa = a.m == -INFINITY ? a.s : a.s * __builtin_amdgcn_exp2f((a.m - nm) * c);   // (a NaN in the sum stays)
  const float sb = b.m == -INFINITY ? b.s : b.s * __builtin_amdgcn_exp2f((b.m - nm) * c);
  return Online{nm, sa + sb};
}
// of a block of NT threads; every thread gets the result.  sm: NT / 64 pairs.  Two barriers.
template <int NT>
__device__ __forceinline__ Online online_block(Online o, float c, Online* sm) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const Online x{__shfl_xor(o.m, d, 64), __shfl_xor(o.s, d, 64)};
    o = online_join(o, x, c);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = o;
  __syncthreads();
  o = sm[0];
  for (int i = 1; i < NT / 64; ++i) o = online_join(o, sm[i], c);
  return o;
}
template <typename T>
__device__ __forceinline__ void load_tail8(const T* zr, int c, int V, float (&v)[8]) {
  if (c + 8 <= V) {
    ld8(zr, c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < V ? ldf(zr, c + j) : -INFINITY;
  }
}
// log-sum-exp of a row's values over the temperature, from their largest one and the sum beside it
__device__ __forceinline__ float row_lse(const Online& o, float tau) {
  if (o.m == -INFINITY || o.m == INFINITY) return o.s != o.s && o.m == -INFINITY ? o.s : o.m;
  return o.m / tau + logf(o.s);
}

}  // namespace

// ----------------------------------------------------------------------------------------------
// One block per row: the log-sum-exp, then the k largest one after the other, each the largest pair below the last.
// ----------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void topk_logits_kernel(const T* __restrict__ z, int64_t ldz, int V, int k, float tau,
                                                          int32_t* __restrict__ ids, float* __restrict__ values,
                                                          float* __restrict__ lse) {
  __shared__ Online sm[4];
  __shared__ uint64_t best[4];
  const size_t row = blockIdx.x;
  const T* zr = z + row * (size_t)ldz;
  const float c = kLog2e / tau;
  if (lse) {
    Online o{-INFINITY, 0.f};
    for (int i = threadIdx.x * 8; i < V; i += 256 * 8) {
      float v[8];
      load_tail8(zr, i, V, v);
      online_add8(o, v, c);
    }
    o = online_block<256>(o, c, sm);
    if (threadIdx.x == 0) lse[row] = row_lse(o, tau);
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < k; ++j) {
    uint64_t mine = 0;
    for (int i = threadIdx.x; i < V; i += 256) {
      const uint64_t p = order_pair(ldf(zr, i), i);
      if (p < last && p > mine) mine = p;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const uint64_t x = __shfl_xor((unsigned long long)mine, d, 64);
      mine = x > mine ? x : mine;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = mine;
    __syncthreads();
    last = best[0];
    for (int i = 1; i < 4; ++i) last = best[i] > last ? best[i] : last;
    if (threadIdx.x == 0) {
      ids[row * (size_t)k + j] = (int32_t)~(uint32_t)last;
      values[row * (size_t)k + j] = key_value((uint32_t)(last >> 32));
    }
  }
}

hipError_t launch_topk_logits(int64_t rows, int V, const void* z, int64_t ldz, int k, float tau, int32_t* ids, float* values, float* lse,
                              int dtype, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  ProfScope ps("topk_logits", 0, (double)rows * ((double)V * dtype_size(dtype) + 8.0 * k), s);
  const dim3 grid((unsigned)rows), blk(256);
  if (dtype == kBF16) hipLaunchKernelGGL(topk_logits_kernel<bf16_t>, grid, blk, 0, s, (const bf16_t*)z, ldz, V, k, tau, ids, values, lse);
  else hipLaunchKernelGGL(topk_logits_kernel<float>, grid, blk, 0, s, (const float*)z, ldz, V, k, tau, ids, values, lse);
  return hipGetLastError();
}

// ----------------------------------------------------------------------------------------------
// Distillation.  With a = t / tau over the teacher's valid entries, p = exp(a - L) (L their log-sum-exp, or the given one),
// P = sum p, q = softmax(z / tau):
//   loss = tau^2 sum_j p_j (log p_j - log q_{id_j})      dz_v = tau (P q_v - sum_{j: id_j = v} p_j)
// ----------------------------------------------------------------------------------------------
namespace {

// A row's teacher, in LDS: entry j's column (-1: none), probability and student logit.
struct Teacher {
  int id[kMaxTeacher];
  float p[kMaxTeacher], z[kMaxTeacher];
  float mass, loss;     // P, and sum_j p_j log p_j
  int any;              // whether an entry says anything
};

// By one wave: everything of the row's teacher that the student's statistics do not enter.  The student's logits at its
// columns are read here, before anything of the row can be overwritten.
template <typename T>
__device__ __forceinline__ void teacher_load(Teacher& te, const T* zr, int V, int k, const int32_t* ids, const float* t, const float* lse, size_t row,
                                             float tau, int lane) {
  constexpr int PER = kMaxTeacher / 64;
  int id[PER];
  float a[PER], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 64 * i;
    id[i] = j < k ? ids[row * (size_t)k + j] : -1;
    if (id[i] >= V) id[i] = -1;
    a[i] = id[i] >= 0 ? t[row * (size_t)k + j] / tau : -INFINITY;
    if (id[i] < 0) id[i] = -1;
    m = fmaxf(m, a[i]);
  }
  bool any = false, nan = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    any |= a[i] > -INFINITY;
    nan |= a[i] != a[i];
  }
  any = __any(any || nan);
  m = wave_max(m);
  float L;
  if (lse) {
    L = lse[row];
  } else {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) s += id[i] >= 0 && any ? expf(a[i] - m) : 0.f;
    L = m + logf(wave_sum(s));
  }
  float mass = 0.f, ent = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = lane + 64 * i;
    const float p = id[i] >= 0 && any ? expf(a[i] - L) : 0.f;
    mass += p;
    ent += p != 0.f ? p * (a[i] - L) : 0.f;
    te.id[j] = id[i];
    te.p[j] = p;
    te.z[j] = id[i] >= 0 ? ldf(zr, (size_t)id[i]) : 0.f;
  }
  mass = wave_sum(mass);
  ent = wave_sum(ent);
  if (lane == 0) { te.mass = mass; te.loss = ent; te.any = any ? 1 : 0; }
}
// by one wave: sum_j p_j (log p_j - log q_j), with log q_j = (z_j - M) / tau - log S
__device__ __forceinline__ float teacher_loss(const Teacher& te, int k, const Online& o, float tau, int lane) {
  const float log_s = logf(o.s);
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxTeacher / 64; ++i) {
    const int j = lane + 64 * i;
    if (j < k && te.p[j] != 0.f) x += te.p[j] * ((te.z[j] - o.m) / tau - log_s);
  }
  return te.loss - wave_sum(x);
}
// gradient at a teacher's column: all of the row's probability on it
__device__ __forceinline__ float teacher_grad(const Teacher& te, int k, int j, float q_mass, float tau) {
  float p = 0.f;
  for (int i = 0; i < k; ++i) p += te.id[i] == te.id[j] ? te.p[i] : 0.f;
  return tau * (q_mass - p);
}

}  // namespace

// A block owns a row and reads it twice, for the statistics and for the gradient.  The columns of the teacher's entries are
// written over by the thread that wrote their eight columns before.
template <typename T, bool GRAD>
__global__ __launch_bounds__(512) void distill_kernel(DistillArgs a) {
  constexpr int NT = 512;
  __shared__ Teacher te;
  __shared__ Online sm[NT / 64];
  const size_t row = blockIdx.x;
  const T* zr = (const T*)a.z + row * (size_t)a.ldz;
  const float c = kLog2e / a.tau;
  const int V = a.V, lane = threadIdx.x & 63;
  if (threadIdx.x < 64) teacher_load(te, zr, V, a.k, a.ids, a.t, a.tlse, row, a.tau, lane);
  Online o{-INFINITY, 0.f};
  for (int i = threadIdx.x * 8; i < V; i += NT * 8) {
    float v[8];
    load_tail8(zr, i, V, v);
    online_add8(o, v, c);
  }
  o = online_block<NT>(o, c, sm);
  const bool keep = a.mask[row] != 0 && te.any;
  if (threadIdx.x < 64) {
    const float loss = keep ? a.tau * a.tau * teacher_loss(te, a.k, o, a.tau, lane) : 0.f;
    if (lane == 0) { a.lse[row] = row_lse(o, a.tau); a.loss_rows[row] = loss; }
  }
  if constexpr (GRAD) {
    T* dr = (T*)a.dz + row * (size_t)a.ldz;
    const float f = te.mass / o.s;
    for (int i = threadIdx.x * 8; i < a.ldz; i += NT * 8) {
      float v[8];
      if (keep) {
        load_tail8(zr, i, V, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < V ? a.tau * f * __builtin_amdgcn_exp2f((v[j] - o.m) * c) : 0.f;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
      }
      st8(dr, i, v);
    }
    if (keep)
      for (int j = 0; j < a.k; ++j)
        if (te.id[j] >= 0 && (te.id[j] >> 3) % NT == (int)threadIdx.x)
          stf(dr, (size_t)te.id[j], teacher_grad(te, a.k, j, f * __builtin_amdgcn_exp2f((te.z[j] - o.m) * c), a.tau));
  }
}

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const bool grad = a.dz != nullptr;
  ProfScope ps(grad ? "distill_train" : "distill_eval", 0, (double)a.rows * dtype_size(dtype) * (a.V + (grad ? (double)a.ldz : 0.0)), s);
  const dim3 grid((unsigned)a.rows), blk(512);
  if (dtype == kBF16) {
    if (grad) hipLaunchKernelGGL((distill_kernel<bf16_t, true>), grid, blk, 0, s, a);
    else hipLaunchKernelGGL((distill_kernel<bf16_t, false>), grid, blk, 0, s, a);
  } else {
    if (grad) hipLaunchKernelGGL((distill_kernel<float, true>), grid, blk, 0, s, a);
    else hipLaunchKernelGGL((distill_kernel<float, false>), grid, blk, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace tide
