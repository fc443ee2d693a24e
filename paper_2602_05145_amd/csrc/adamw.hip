// AdamW over any list of tensors, moments in 32 bits or in 8: include/tide_draft.h has the formulas.
#include <cmath>

#include "../../include/tide_draft.h"
#include "kernels.h"
#include "loose.h"
#include "prof.h"

namespace tide {
namespace {

constexpr int kPerThread = 8;                       // consecutive elements
constexpr int kThreads = 256;
constexpr int kPerBlock = kPerThread * kThreads;    // 2048 elements of one tensor
constexpr int kScaled = 256;                        // elements that share a scale: 32 lanes
constexpr int kPerLaunch = 44;                      // tensors whose table fits the 4 KB of a launch's arguments
constexpr float kTop = 448.f;                       // the largest e4m3 number

struct Entry {
  void* param; float* master; const void* grad; void *m, *v; float *m_scale, *v_scale;
  int64_t n; float decay; uint32_t index, flags;    // index: place in the caller's list
};
enum : uint32_t { kParamBf16 = 1, kGradBf16 = 2, kEightBits = 4 };
struct Table {
  Entry t[kPerLaunch];
  uint32_t first[kPerLaunch];   // first block of each tensor, those behind the last: 2^32 - 1
  float beta1, beta2, eps, lr, inv_bc1, inv_sqrt_bc2;
  uint32_t key;
  const float* grad_scale;
  const AdamwSchedule* schedule;   // lr, the two corrections and the key from device memory
};
static_assert(sizeof(Table) <= 4096);

// 32 bits that look random from any 32: xor-shifts and odd multipliers (fractional digits of the roots of 2 and 3).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ uint32_t step_key(uint32_t seed, int64_t t) {
  return mix(mix(seed ^ (uint32_t)t) + (uint32_t)((uint64_t)t >> 32));
}

__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int count) {
  if (count >= 8) return LDX(u32x2_of_bytes, p);
  u32x2 c = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) c[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
  return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int count, const u32x2& c) {
  if (count >= 8) { STX(u32x2_of_bytes, p, c); return; }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) p[j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
}
// e4m3 codes times their scale; every code is exact in fp32
__device__ __forceinline__ void decode(const u32x2& c, float scale, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], true);
    x[4 * h] = lo[0] * scale, x[4 * h + 1] = lo[1] * scale, x[4 * h + 2] = hi[0] * scale, x[4 * h + 3] = hi[1] * scale;
  }
}
__device__ __forceinline__ float max_of_32(float v) {   // over the 32 lanes that hold a block
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// The codes of eight of a block's numbers.  x beside the block's largest magnitude (448 stands for it) is rounded to one of the two codes around it, up as
// often as it lies beyond the lower: `coin` holds 16 random bits for each.  (To the nearest, a second moment would stand still: a step moves it by up to
// 1 - beta2 of itself, and the codes lie 6 to 12 % apart.)  Numbers that are not finite become NaN and leave the others alone.
__device__ __forceinline__ u32x2 encode(const float (&x)[8], const uint32_t (&coin)[8], bool upper, float& scale) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]) < INFINITY ? fabsf(x[j]) : 0.f);
  top = max_of_32(top);
  if (!(top >= 0x1p-100f)) top = 0.f;   // (1 / top has to be a number)
  const float factor = top > 0.f ? (1.f / top) * kTop : 0.f;   // (what this rounds moves the largest by a few of the 2^20 that `coin` covers)
  scale = top * (1.f / kTop);
  u32x2 c = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = fminf(fabsf(x[j]) * factor, kTop);
    // below the smallest normal number, 2^-6, the codes are 2^-9 apart as they are up to 2^-5: one more in front makes them alike.  20 bits go.
    const bool low = y < 0x1p-6f;
    const uint32_t bits = __float_as_uint(low ? y + 0x1p-6f : y) + ((upper ? coin[j] >> 16 : coin[j] & 0xFFFFu) << 4) + 8;
    const bool fine = fabsf(x[j]) < INFINITY;
    const uint32_t code = fine ? ((bits >> 20) - (low ? 968 : 960)) | (x[j] < 0.f ? 0x80u : 0u) : 0x7Fu;
    c[j / 4] |= code << (8 * (j % 4));
  }
  return c;
}

// One element; every operation rounds by itself, so that the bits do not hang on how a compiler joins them.
struct Rate { float lr, decay, beta1, beta2, rest1, rest2, eps, inv_bc1, inv_sqrt_bc2; };
__device__ __forceinline__ void update(const Rate& r, float g, float& m, float& v, float& root, float& w) {
#pragma clang fp contract(off)
  m = r.beta1 * m + r.rest1 * g;
  v = r.beta2 * v + r.rest2 * g * g;
  root = sqrtf(v);
  w = w * r.decay - r.lr * (m * r.inv_bc1) / (root * r.inv_sqrt_bc2 + r.eps);
}

// Block b works on 2048 elements of the tensor its index falls in, a thread on 8 consecutive ones.
__global__ __launch_bounds__(kThreads) void adamw_list_kernel(const Table a) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63;
  const int at = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < kPerLaunch && a.first[min(lane, kPerLaunch - 1)] <= blockIdx.x)) - 1);
  const Entry& t = a.t[at];
  const int64_t i = (int64_t)(blockIdx.x - a.first[at]) * kPerBlock + threadIdx.x * kPerThread;
  const int count = (int)min(max(t.n - i, (int64_t)0), (int64_t)kPerThread);
  if (!(t.flags & kEightBits) && count == 0) return;   // (lanes of a shared scale stay)
  const bool dyn = a.schedule != nullptr;
  Rate r;
  r.lr = dyn ? a.schedule->lr : a.lr;
  r.inv_bc1 = dyn ? a.schedule->inv_bc1 : a.inv_bc1;
  r.inv_sqrt_bc2 = dyn ? a.schedule->inv_sqrt_bc2 : a.inv_sqrt_bc2;
  r.decay = 1.f - r.lr * t.decay;
  r.beta1 = a.beta1, r.beta2 = a.beta2, r.rest1 = 1.f - a.beta1, r.rest2 = 1.f - a.beta2, r.eps = a.eps;
  float g[8], w[8], m[8], v[8], root[8];
  if (count > 0 && (t.flags & kGradBf16)) load_some((const bf16_t*)t.grad + i, count, g);
  else load_some((const float*)t.grad + i, count, g);
  float* weights = (t.flags & kParamBf16) ? t.master : (float*)t.param;
  load_some(weights + i, count, w);
  if (t.flags & kEightBits) {
    const u32x2 cm = load_codes((const uint8_t*)t.m + i, count), cv = load_codes((const uint8_t*)t.v + i, count);
    const int64_t block = min(i, t.n - 1) / kScaled;
    decode(cm, t.m_scale[block], m);
    decode(cv, t.v_scale[block], v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * v[j];
  } else {
    load_some((const float*)t.m + i, count, m);
    load_some((const float*)t.v + i, count, v);
  }
  if (a.grad_scale) {
    const float s = *a.grad_scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= s;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) update(r, g[j], m[j], v[j], root[j], w[j]);
  store_some(weights + i, count, w);
  if (t.flags & kParamBf16) store_some((bf16_t*)t.param + i, count, w);
  if (!(t.flags & kEightBits)) {
    store_some((float*)t.m + i, count, m);
    store_some((float*)t.v + i, count, v);
    return;
  }
  const uint32_t key = mix((dyn ? a.schedule->key : a.key) + t.index) + (uint32_t)i + (uint32_t)((uint64_t)i >> 32) * 0x9E3779B9u;
  uint32_t coin[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) coin[j] = mix(key + j);   // (i is a multiple of 8: its upper half is the same for all)
  if (count < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= count) m[j] = root[j] = 0.f;
  }
  float sm, sv;
  const u32x2 cm = encode(m, coin, false, sm), cv = encode(root, coin, true, sv);
  store_codes((uint8_t*)t.m + i, count, cm);
  store_codes((uint8_t*)t.v + i, count, cv);
  if (count > 0 && (lane & 31) == 0) t.m_scale[i / kScaled] = sm, t.v_scale[i / kScaled] = sv;
}

__global__ void adamw_schedule_kernel(const float* __restrict__ lr, int64_t* __restrict__ step, float beta1, float beta2, uint32_t seed, AdamwSchedule* __restrict__ out) {
  const int64_t t = *step + 1;
  *out = AdamwSchedule{*lr, (float)(1.0 / (1.0 - pow_int((double)beta1, t))), (float)(1.0 / sqrt(1.0 - pow_int((double)beta2, t))), step_key(seed, t)};
  *step = t;
}

}  // namespace

hipError_t launch_adamw_list(const AdamwListArgs& a, hipStream_t s) {
  Table d{};
  d.beta1 = a.beta1, d.beta2 = a.beta2, d.eps = a.eps, d.lr = a.lr;
  d.grad_scale = a.grad_scale, d.schedule = a.schedule;
  if (a.schedule) {
    ProfScope ps("adamw_schedule", 0, 0, s);
    hipLaunchKernelGGL(adamw_schedule_kernel, dim3(1), dim3(1), 0, s, a.lr_dev, a.step_dev, a.beta1, a.beta2, a.seed, a.schedule);
    if (const hipError_t e = hipGetLastError()) return e;
  } else {
    const int64_t t = a.step + 1;
    d.inv_bc1 = (float)(1.0 / (1.0 - pow_int((double)a.beta1, t)));
    d.inv_sqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - pow_int((double)a.beta2, t)));
    d.key = step_key(a.seed, t);
  }
  for (int i = 0; i < a.n_tensors;) {
    int n = 0;
    int64_t blocks = 0;
    double bytes = 0;
    for (int k = 0; k < kPerLaunch; ++k) d.first[k] = 0xFFFFFFFFu;
    for (; i < a.n_tensors && n < kPerLaunch; ++i) {
      const tide_adamw_tensor& x = a.tensors[i];
      if (x.n == 0) continue;
      const int64_t need = (x.n + kPerBlock - 1) / kPerBlock;
      if (blocks + need >= (1 << 24)) break;   // (a launch holds fewer than 2^32 threads, and a tensor no more blocks than that)
      const bool bf16 = x.param_dtype == TIDE_DTYPE_BF16;
      const uint32_t flags = (bf16 ? kParamBf16 : 0u) | (x.grad_dtype == TIDE_DTYPE_BF16 ? kGradBf16 : 0u) | (x.state_bits == 8 ? kEightBits : 0u);
      d.t[n] = Entry{x.param, x.master, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.n, x.weight_decay, (uint32_t)i, flags};
      d.first[n++] = (uint32_t)blocks;
      blocks += need;
      bytes += (double)x.n * ((flags & kGradBf16 ? 2 : 4) + (bf16 ? 10 : 8) + (flags & kEightBits ? 4.0625 : 16));
    }
    if (n == 0) break;
    ProfScope ps("adamw_list", 0, bytes, s);
    hipLaunchKernelGGL(adamw_list_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, d);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace tide
