// Vector accesses at addresses that are aligned as one element is, for arrays that may begin anywhere (views of a flat buffer, rows of an odd width).
#pragma once
#include "tide_common.h"

namespace tide {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef f32x4 __attribute__((aligned(4))) f32x4_of_floats;
typedef u32x4 __attribute__((aligned(2))) u32x4_of_halves;
typedef u32x2 __attribute__((aligned(1))) u32x2_of_bytes;
#ifdef TIDE_NTL
#define LDX(T, p) __builtin_nontemporal_load(reinterpret_cast<const T*>(p))
#else
#define LDX(T, p) (*reinterpret_cast<const T*>(p))
#endif
#ifdef TIDE_NTS
#define STX(T, p, v) __builtin_nontemporal_store(v, reinterpret_cast<T*>(p))
#else
#define STX(T, p, v) (*reinterpret_cast<T*>(p) = (v))
#endif

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = LDX(f32x4_of_floats, p), b = LDX(f32x4_of_floats, p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  STX(f32x4_of_floats, p, (f32x4{x[0], x[1], x[2], x[3]}));
  STX(f32x4_of_floats, p + 4, (f32x4{x[4], x[5], x[6], x[7]}));
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) {
  const u32x4 a = LDX(u32x4_of_halves, p);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(a[j] << 16), x[2 * j + 1] = __uint_as_float(a[j] & 0xFFFF0000u);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {
  STX(u32x4_of_halves, p, (u32x4{f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(x[4], x[5]), f2bf2(x[6], x[7])}));
}
template <typename T> __device__ __forceinline__ void load_some(const T* p, int count, float (&x)[8]) {
  if (count >= 8) return load8(p, x);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j < count ? ldf(p, j) : 0.f;
}
template <typename T> __device__ __forceinline__ void store_some(T* p, int count, const float (&x)[8]) {
  if (count >= 8) return store8(p, x);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < count) stf(p, j, x[j]);
}

}  // namespace tide
