// FP4 values dequantized to bf16 in registers, exact, for the kernels that multiply 4-bit weights
// with bf16 activations on the bf16 MFMA (mixed.hip, matvec.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace resq {

// 2^E as float32 for an E8M0 code (E = code - 127; 2^-127 is a float32 subnormal).
__device__ __forceinline__ float e8m0_f32(uint32_t code) {
  return code ? __uint_as_float(code << 23) : __uint_as_float(0x00400000u);
}

// Eight MXFP4 elements (one 32-bit word of codes, element i in nibble i) dequantized to bf16
// bits, exact, two per output word: E2M1 magnitude times 2^E through gfx950's scaled
// conversion (v_cvt_scalef32_pk_bf16_fp4).
__device__ __forceinline__ void mx_dequant8(uint32_t w, uint32_t scale, uint32_t out[4]) {
  const float sc = e8m0_f32(scale);
  out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0));
  out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1));
  out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2));
  out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3));
}

// HiF4 decoding by table (the lane's 32 elements of a round lie in one 64-block).  Per round:
// the bf16 patterns L[k] of k (4+m) 2^(e-35) for k = 0..7 (exact, L[0] = 0), split into
// their low and high bytes, four entries per dword, and the lane's level-2 (4) and level-3
// (8) shift bits.  Per 8 elements: the magnitudes k spread to bytes select the bytes of
// their entries (v_perm), the signs go into the high bytes of nonzero elements, the bytes
// pair up into bf16 values, and a saturating 16-bit subtraction of b << 7 lowers the
// exponent by the element's shift b (nonzero values keep biased exponents far above 2, and
// zero stays zero).
struct Hif4Table {
  uint32_t lo03, lo47, hi03, hi47;  // low / high bytes of L[0..3], L[4..7]
  uint32_t l2, l3;                  // level-2 bits of the lane's 4 groups of 8, level-3 of its 8 of 4
};

__device__ __forceinline__ Hif4Table hif4_table(uint32_t scale, int h) {
  const uint32_t f = 4u + (scale & 3u);
  const int e = (int)((scale >> 2) & 63u) - 35;
  uint32_t L[8];
  L[0] = 0u;
#pragma unroll
  for (int k = 1; k < 8; ++k) L[k] = __float_as_uint(ldexpf((float)(k * f), e)) >> 16;  // exact
  const uint32_t p01 = L[0] | (L[1] << 16), p23 = L[2] | (L[3] << 16);
  const uint32_t p45 = L[4] | (L[5] << 16), p67 = L[6] | (L[7] << 16);
  Hif4Table t;
  t.lo03 = __builtin_amdgcn_perm(p23, p01, 0x06040200u);
  t.hi03 = __builtin_amdgcn_perm(p23, p01, 0x07050301u);
  t.lo47 = __builtin_amdgcn_perm(p67, p45, 0x06040200u);
  t.hi47 = __builtin_amdgcn_perm(p67, p45, 0x07050301u);
  t.l2 = (scale >> (8 + 4 * h)) & 0xFu;
  t.l3 = (scale >> (16 + 8 * h)) & 0xFFu;
  return t;
}

typedef unsigned short v2u16 __attribute__((ext_vector_type(2)));

// Four elements: their nibbles in the low nibbles of the four bytes of sp; out0/out1 receive
// elements 0,1 / 2,3 as bf16 pairs, shifted down by b.
__device__ __forceinline__ void hif4_decode4(uint32_t sp, uint32_t b, const Hif4Table& t, uint32_t& out0,
                                             uint32_t& out1) {
  const uint32_t k = sp & 0x07070707u;
  const uint32_t lo = __builtin_amdgcn_perm(t.lo47, t.lo03, k);
  uint32_t hi = __builtin_amdgcn_perm(t.hi47, t.hi03, k);
  hi |= (sp << 4) & (k + 0x7F7F7F7Fu) & 0x80808080u;  // the sign bit of each nonzero element
  const v2u16 sub = __builtin_bit_cast(v2u16, b * 0x00800080u);
  out0 = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(
                                          __builtin_bit_cast(v2u16, __builtin_amdgcn_perm(hi, lo, 0x05010400u)), sub));
  out1 = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(
                                          __builtin_bit_cast(v2u16, __builtin_amdgcn_perm(hi, lo, 0x07030602u)), sub));
}

// Eight elements of step kk (elements 8 kk .. 8 kk + 7 of the lane's 32): one level-2 group,
// two level-3 groups.
template <int KK>
__device__ __forceinline__ void hif4_decode8(uint32_t w, const Hif4Table& t, uint32_t out[4]) {
  const uint32_t b2 = (t.l2 >> KK) & 1u;
  const uint32_t ba = b2 + ((t.l3 >> (2 * KK)) & 1u), bb = b2 + ((t.l3 >> (2 * KK + 1)) & 1u);
  const uint32_t ta = __builtin_amdgcn_perm(w, w, 0x0C010C00u), tb = __builtin_amdgcn_perm(w, w, 0x0C030C02u);
  hif4_decode4(ta | (ta << 4), ba, t, out[0], out[1]);
  hif4_decode4(tb | (tb << 4), bb, t, out[2], out[3]);
}

}  // namespace resq
