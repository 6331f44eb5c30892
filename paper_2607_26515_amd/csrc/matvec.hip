// A few tokens (1 to 16) times 4-bit weights with group scales: Y = X Q(W)^T, the single-token
// form of the weight-only linear (mixed.hip).
//
// Bound by the read of the codes and scales (4.25 or 4.5 bits per weight).  The bf16 MFMA
// 16x16x32 takes 16 weight rows as its row operand and the tokens, padded to 16, as its column
// operand: the products cost the same for 1 to 16 tokens and stay exact in float32.  A workgroup
// owns 16 rows; its W waves take the K range in turns of 128 (a wave reads 64 contiguous bytes of
// codes of each row per turn) and add their tiles through LDS in wave order.
//
// K order: lane l holds row (token) l % 16 and, of a turn, the 32 consecutive elements
// 32 (l / 16) .. + 31; MFMA kk takes elements 8 kk .. 8 kk + 7 of them from weights and tokens
// alike.  Result: lane l register r is row 4 (l / 16) + r, token l % 16.
#include "kernels.h"
#include "fp4_bf16.h"
#include "ops_core.h"
#include "profiler.h"

namespace resq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int FMT, int W>
__global__ __launch_bounds__(64 * W) void matvec_kernel(const uint16_t* __restrict__ X, int m, int64_t d, int64_t ldx,
                                                        const uint8_t* __restrict__ codes,
                                                        const void* __restrict__ scales, int64_t n, void* Y,
                                                        int64_t ldy, bool out_bf16) {
  __shared__ f32x4 red[W][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, row = min(n0 + r, n - 1);
  const uint8_t* wrow = codes + row * (d / 2);
  const uint16_t* xrow = X + (int64_t)r * ldx;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int64_t k = (int64_t)wave * 128 + 32 * q; k - 32 * q < d; k += W * 128) {
    u32x4 w = {0u, 0u, 0u, 0u};
    uint32_t sc = 0u;
    u32x4 x[4] = {w, w, w, w};
    if (k < d) {
      w = *reinterpret_cast<const u32x4*>(wrow + k / 2);
      sc = FMT == 0 ? reinterpret_cast<const uint8_t*>(scales)[row * (d / 32) + k / 32]
                    : reinterpret_cast<const uint32_t*>(scales)[row * (d / 64) + k / 64];
      if (r < m)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) x[kk] = reinterpret_cast<const Bf16x8*>(xrow + k + 8 * kk)->v;
    }
    uint32_t b[4][4];
    if constexpr (FMT == 0) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) mx_dequant8(w[kk], sc, b[kk]);
    } else {
      const Hif4Table t = hif4_table(sc, (int)((k >> 5) & 1));
      hif4_decode8<0>(w[0], t, b[0]);
      hif4_decode8<1>(w[1], t, b[1]);
      hif4_decode8<2>(w[2], t, b[2]);
      hif4_decode8<3>(w[3], t, b[3]);
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const u32x4 a = {b[kk][0], b[kk][1], b[kk][2], b[kk][3]};
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, x[kk]),
                                                    acc, 0, 0, 0);
    }
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
  for (int w = 1; w < W; ++w) acc += red[w][lane];
  if (r >= m) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t j = n0 + 4 * q + i;
    if (j >= n) continue;
    if (out_bf16) reinterpret_cast<uint16_t*>(Y)[(int64_t)r * ldy + j] = bf16_bits(acc[i]);
    else reinterpret_cast<float*>(Y)[(int64_t)r * ldy + j] = acc[i];
  }
}

}  // namespace

void launch_matvec(int fmt, const uint16_t* X, int64_t m, int64_t d, int64_t ldx, const uint8_t* codes,
                   const void* scales, int64_t n, void* Y, int64_t ldy, bool out_bf16, hipStream_t s) {
  const dim3 grid((unsigned)((n + 15) / 16));
  if (fmt == 0)
    launch_timed(matvec_kernel<0, 8>, grid, dim3(512), 0u, s, X, (int)m, d, ldx, codes, scales, n, Y, ldy, out_bf16);
  else
    launch_timed(matvec_kernel<1, 8>, grid, dim3(512), 0u, s, X, (int)m, d, ldx, codes, scales, n, Y, ldy, out_bf16);
}

}  // namespace resq
