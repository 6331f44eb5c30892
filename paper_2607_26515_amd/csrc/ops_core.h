// Loads, stores and sums shared by the row kernels (norm.hip, logprob.hip).
//
// Rows may start at any element: eight elements move in one or two 16-byte accesses with the
// element's own alignment, which gfx950's memory system takes for global memory at any address
// (the compiler emits dwordx4 for these types), so there is no second path for odd row strides.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace resq {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(2))) Bf16x8 { u32x4 v; };
struct __attribute__((packed, aligned(4))) F32x4 { f32x4 v; };

__device__ __forceinline__ float bf16_value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// The nearest bf16, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_value(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = bf16_bits(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

__device__ __forceinline__ void load8(const uint16_t* p, float v[8]) {
  const u32x4 u = reinterpret_cast<const Bf16x8*>(p)->v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float v[8]) {
  const f32x4 a = reinterpret_cast<const F32x4*>(p)[0].v, b = reinterpret_cast<const F32x4*>(p)[1].v;
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void store8(uint16_t* p, const float v[8]) {
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
  reinterpret_cast<Bf16x8*>(p)->v = u;
}
__device__ __forceinline__ void store8(float* p, const float v[8]) {
  f32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
  reinterpret_cast<F32x4*>(p)[0].v = a;
  reinterpret_cast<F32x4*>(p)[1].v = b;
}

// Elements 0 .. n - 1 of eight (n <= 0: none), the others `fill`.
template <typename T>
__device__ __forceinline__ void load_upto8(const T* p, int n, float fill, float v[8]) {
  if (n >= 8) {
    load8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? load1(p + i) : fill;
  }
}
template <typename T>
__device__ __forceinline__ void store_upto8(T* p, int n, const float v[8]) {
  if (n >= 8) {
    store8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) store1(p + i, v[i]);
  }
}

}  // namespace resq
