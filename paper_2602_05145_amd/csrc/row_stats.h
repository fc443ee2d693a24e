// Statistics of a softmax over rows of thousands of columns: the maximum and the sum of exponentials beside it, kept per lane, joined over
// a wave and a block.
#pragma once
#include "tide_common.h"

namespace tide {

constexpr float kLog2e = 1.4426950408889634f;

// Maximum and sum over a wave on the vector unit alone (a shuffle through LDS takes ten times as long, and a row's few blocks wait for each);
// every lane gets the result.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float v, float none) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float scalar(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }   // the same in every lane
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63)); }
__device__ __forceinline__ float fast_max(float v) {
  v = fmaxf(v, dpp<0x111, 0xf>(v, -INFINITY));   // from 1, 2, 4 and 8 lanes below in a row of 16
  v = fmaxf(v, dpp<0x112, 0xf>(v, -INFINITY));
  v = fmaxf(v, dpp<0x114, 0xf>(v, -INFINITY));
  v = fmaxf(v, dpp<0x118, 0xf>(v, -INFINITY));
  v = fmaxf(v, dpp<0x142, 0xa>(v, -INFINITY));   // the row below's last lane, in rows 1 and 3; then the lower half's, in the upper
  v = fmaxf(v, dpp<0x143, 0xc>(v, -INFINITY));
  return last_lane(v);
}
__device__ __forceinline__ float fast_sum(float v) {
  v += dpp<0x111, 0xf>(v, 0.f);
  v += dpp<0x112, 0xf>(v, 0.f);
  v += dpp<0x114, 0xf>(v, 0.f);
  v += dpp<0x118, 0xf>(v, 0.f);
  v += dpp<0x142, 0xa>(v, 0.f);
  v += dpp<0x143, 0xc>(v, 0.f);
  return last_lane(v);
}

// 2^(c (z - m)) of values z <= m as fix 2^(slope z + shift), one fused step and the power per value.  shift is -c m rounded, and what that
// rounding leaves of the exponent of the largest value, the same for all, goes into `fix`.  From |c m| = 2^30 on it would be 32 and more: there a power of
// two takes the place of c, so that slope m is exact; the largest value gives 1 and the next smaller fp32 number 0, which is less than 2^-64
// beside it.  (Difference first, (z - m) c, is one step more per value.)  A row of -inf gives 0, one with +inf +inf, one with NaN NaN.
struct Power { float slope, shift, fix; };
__device__ __forceinline__ Power power_of(float m, float c) {
  const float shift = -m * c;
  if (fabsf(shift) < 0x1p30f) return Power{c, shift, __builtin_amdgcn_exp2f(-fmaf(m, c, shift))};
  const uint32_t e = (__float_as_uint(m) >> 23) & 255;   // m is normal, infinite or NaN
  if (e == 255) return Power{1.f, 0.f, 1.f};
  const float slope = __uint_as_float((127 + 40 + 127 - e) << 23);   // slope m in 2^40 .. 2^41
  return Power{slope, -m * slope, 1.f};
}

// Running (max, sum of 2^(c (z - max))) over eight more values.  The difference comes first: it is 0 for the largest value whatever
// that is, also where c times it has no number (columns masked with the type's lowest value).
struct Online { float m, s; };
__device__ __forceinline__ void online_add8(Online& o, const float (&v)[8], float c) {
  float cm = v[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) cm = fmaxf(cm, v[j]);
  const float nm = fmaxf(o.m, cm);
  const float sh = fabsf(nm) == INFINITY ? 0.f : nm;
  float part = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) part += __builtin_amdgcn_exp2f((v[j] - sh) * c);
  o.s = (o.m == nm ? o.s : o.s * __builtin_amdgcn_exp2f((o.m - nm) * c)) + part;
  o.m = nm;
}
// of a block of NT threads; every thread gets the result.  sm: NT / 64 pairs.  Two barriers.
template <int NT>
__device__ __forceinline__ Online online_block(const Online& o, float c, Online* sm) {
  auto scaled = [&](const Online& x, float m) { return x.m == m ? x.s : x.s * __builtin_amdgcn_exp2f((x.m - m) * c); };   // (a NaN in the sum stays)
  const float wm = fast_max(o.m);
  const float ws = fast_sum(scaled(o, wm));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = Online{wm, ws};
  __syncthreads();
  const Online x = sm[threadIdx.x % (NT / 64)];
  const float m = fast_max(x.m);
  return Online{m, fast_sum((threadIdx.x & 63) < NT / 64 ? scaled(x, m) : 0.f)};
}

template <typename T> struct Raw8Once : Raw8<T> {   // loads past the caches: nothing is read again
  __device__ __forceinline__ void load_buffer(__amdgpu_buffer_rsrc_t rs, int at) {   // from byte `at`
    this->a = __builtin_bit_cast(decltype(this->a), __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 2));
    if constexpr (sizeof(T) == 4) this->b = __builtin_bit_cast(decltype(this->b), __builtin_amdgcn_raw_buffer_load_b128(rs, at + 16, 0, 2));
  }
  __device__ __forceinline__ void load_once(const T* p, size_t i) {
    typedef unsigned u32x4_nt __attribute__((ext_vector_type(4)));
    const u32x4_nt* q = reinterpret_cast<const u32x4_nt*>(p + i);
    if constexpr (sizeof(T) == 2) {
      const u32x4_nt x = __builtin_nontemporal_load(q);
      this->a = make_uint4(x.x, x.y, x.z, x.w);
    } else {
      const u32x4_nt x = __builtin_nontemporal_load(q), y = __builtin_nontemporal_load(q + 1);
      this->a = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
      this->b = make_float4(__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w));
    }
  }
};

// Of a thread of a block of NT, over columns 0 .. n of a row in memory, four chunks requested at a time.  The row is 16-byte aligned and what
// is behind its last column up to the next multiple of eight can be read.  ONCE: it is not read again.
template <typename T, int NT, bool ONCE = false>
__device__ __forceinline__ Online row_stats(const T* zr, int V, float c) {
  constexpr int U = sizeof(T) == 2 ? 4 : 2, STEP = NT * 8;
  const int last = (V - 1) / 8 * 8;
  Online o{-INFINITY, 0.f};
  for (int base = 0; base < V; base += U * STEP) {
    Raw8Once<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)min(base + u * STEP + (int)threadIdx.x * 8, last);
      if constexpr (ONCE) raw[u].load_once(zr, at); else raw[u].load(zr, at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = base + u * STEP + threadIdx.x * 8;
      float v[8];
      raw[u].get(v);
      if (base + U * STEP > V) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = col + j < V ? v[j] : -INFINITY;
      }
      online_add8(o, v, c);
    }
  }
  return o;
}

}  // namespace tide
