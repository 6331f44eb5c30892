// Loads, stores and sums shared by the row kernels and the few-token products (norm.hip,
// logprob.hip, matvec.hip).
//
// Rows may start at any element: eight elements move in one or two 16-byte accesses with the
// element's own alignment, which gfx950's memory system takes for global memory at any address
// (the compiler emits dwordx4 for these types), so there is no second path for odd row strides.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_fp4.h"

namespace resq {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(2))) Bf16x8 { u32x4 v; };
struct __attribute__((packed, aligned(2))) Bf16x4 { u32x2 v; };
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

// E consecutive elements as loaded, to be taken apart later (a load in flight holds no more registers
// than its bytes).
template <typename T, int E>
struct Raw {
  T v[E];
};
template <>
struct Raw<uint16_t, 8> {
  u32x4 v;
};
template <>
struct Raw<uint16_t, 4> {
  u32x2 v;
};
template <>
struct Raw<float, 4> {
  f32x4 a;
};
template <>
struct Raw<float, 8> {
  f32x4 a, b;
};
template <typename T>
__device__ __forceinline__ void load_raw(const T* p, Raw<T, 1>& r) { r.v[0] = *p; }
__device__ __forceinline__ void load_raw(const uint16_t* p, Raw<uint16_t, 8>& r) {
  r.v = reinterpret_cast<const Bf16x8*>(p)->v;
}
__device__ __forceinline__ void load_raw(const uint16_t* p, Raw<uint16_t, 4>& r) {
  r.v = reinterpret_cast<const Bf16x4*>(p)->v;
}
__device__ __forceinline__ void load_raw(const float* p, Raw<float, 4>& r) {
  r.a = reinterpret_cast<const F32x4*>(p)->v;
}
__device__ __forceinline__ void load_raw(const float* p, Raw<float, 8>& r) {
  r.a = reinterpret_cast<const F32x4*>(p)[0].v;
  r.b = reinterpret_cast<const F32x4*>(p)[1].v;
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw<T, 1>& r, float v[1]) { v[0] = load1(&r.v[0]); }
__device__ __forceinline__ void unpack(const Raw<uint16_t, 8>& r, float v[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r.v[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw<uint16_t, 4>& r, float v[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[2 * i] = __uint_as_float(r.v[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw<float, 4>& r, float v[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = r.a[i];
}
__device__ __forceinline__ void unpack(const Raw<float, 8>& r, float v[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
}

__device__ __forceinline__ void load8(const uint16_t* p, float v[8]) {
  Raw<uint16_t, 8> r;
  load_raw(p, r);
  unpack(r, v);
}
__device__ __forceinline__ void load8(const float* p, float v[8]) {
  Raw<float, 8> r;
  load_raw(p, r);
  unpack(r, v);
}

__device__ __forceinline__ void store4(uint16_t* p, const float v[4]) {
  reinterpret_cast<Bf16x4*>(p)->v = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}
__device__ __forceinline__ void store4(float* p, const float v[4]) {
  reinterpret_cast<F32x4*>(p)->v = f32x4{v[0], v[1], v[2], v[3]};
}

// E consecutive elements (E = 8, 4 or 1).
template <int E, typename T>
__device__ __forceinline__ void load_n(const T* p, float v[E]) {
  Raw<T, E> r;
  load_raw(p, r);
  unpack(r, v);
}
template <int E, typename T>
__device__ __forceinline__ void store_n(T* p, const float v[E]) {
  if constexpr (E == 8) store8(p, v);
  else if constexpr (E == 4) store4(p, v);
  else store1(p, v[0]);
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

// A value from another lane of the same 16 (DPP; both halves of a double), and the sum with the
// lanes 16 or 32 away (gfx950's half swaps).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __uint_as_float(dpp_u32<CTRL>(__float_as_uint(v))); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, ((uint64_t)dpp_u32<CTRL>((uint32_t)(u >> 32)) << 32) | dpp_u32<CTRL>((uint32_t)u));
}
constexpr int kDppRor4 = 0x124, kDppRor8 = 0x128;  // lane i of 16 <- lane i - 4, i - 8 (mod 16)
template <bool HALF>
__device__ __forceinline__ u32x2 swap_rows(uint32_t v) {
  if constexpr (HALF) return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
  else return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
}
template <bool HALF>
__device__ __forceinline__ float add_swapped(float v) {
  const u32x2 r = swap_rows<HALF>(__float_as_uint(v));
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <bool HALF>
__device__ __forceinline__ double add_swapped(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const u32x2 lo = swap_rows<HALF>((uint32_t)u), hi = swap_rows<HALF>((uint32_t)(u >> 32));
  return __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) +
         __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
}

// Two sums in one: over the lanes 32 (16) apart, of a in the lower half (even rows of 16), of b in the other.
template <bool HALF>
__device__ __forceinline__ float add_pair(float a, float b) {
  u32x2 r;
  if constexpr (HALF) r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false));
  else r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false));
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace resq
