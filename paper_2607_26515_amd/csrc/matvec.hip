// A few tokens (1 to 16) times 4-bit weights with group scales: Y = X Q(W)^T, the single-token
// form of the weight-only linear (mixed.hip).
//
// Bound by the read of the codes and scales (4.25 or 4.5 bits per weight) once the decoding fits
// under it.  What decides is how that read is laid out: with the operand layouts of the 16 and 32 row
// MFMAs a load touches 16 or 32 rows for 32 to 64 bytes each, and the L1 takes about as many cycles as
// there are such pieces (4 tokens x 37888 x 3584 HiF4: 37 us, its L1 accesses alone 34).  The
// MFMA 4x4x4 of 16 blocks fits instead: its block b, lanes 4 b .. 4 b + 3, multiplies 4 tokens with 4
// weight rows over K elements of its own, so a wave's 16-byte loads take 256 contiguous bytes of codes
// (512 elements) of each of 4 rows, and lane 4 b + j holds 32 consecutive elements of row j: one MXFP4
// block, or half a HiF4 block, with its scale.  Result register r is token r, row j, of block b's
// elements; at the end the 16 blocks are added by lane exchange.
//
// Work split.  The quads of rows are dealt in contiguous ranges ("shares") to as many workgroups as
// there are CUs, and a share's steps (a quad's 512-element steps one after the other) in equal parts to
// the 16 waves of a workgroup: every CU and wave is busy to the end whatever the sizes.  A quad that
// several waves have a part of is added through LDS in wave order.  The order of additions depends on
// n and d alone, so a token's result is the same alone and among others.  (With whole quads to waves,
// 2.3 a wave at 4 x 37888 x 3584, the same loop took 23.0 us instead of 22.0.)
//
// Measured (a large copy runs at 5.08 TB/s, an empty kernel takes about 4 us of a graph): one token x 2560 x
// 2048 MXFP4 5.0 us, launch and first loads; 4 x 37888 x 3584 HiF4 18.2 us, 4.2 TB/s; 1 x 37888 x 3584
// MXFP4 18.9 us; 16 x 37888 x 3584 30.7 us HiF4, 25.6 us MXFP4, where four tokens' reads of X from LDS to
// each step, 512 cycles of a CU, stand beside the decoding.  16 x 2048 x 11008 HiF4 15.7 us: four batches,
// each decoding all weights.  The tile GEMM of mixed.hip takes 7.2, 55 and 40 us for the first, second and last.
//
// Data movement.  X lies in LDS.  Tokens that do not fit together are taken in B batches by B
// workgroups on one XCD, each with up to B shares (so that X is copied once per workgroup and the codes come
// from HBM once and from the L2 B - 1 times).  Codes and scales go straight into a ring of kAhead steps
// in each wave's own part of LDS (buffer loads with the LDS destination: a step waits for its own loads
// only; with loads to registers the compiler waited for all in flight).  Tokens past the last repeat
// it and are dropped; weight rows past the last read zeros.
//
// Decoding.  MXFP4: a half is one 32-block, so gfx950's scaled FP4 conversion gives exact bf16
// weights and the tile accumulates over all of K.  HiF4: an element is k/4 s1 2^-(b2+b3).  The byte
// sign | k is the FP8 E4M3 value +-k 2^-9 (a subnormal), which the scaled FP8 conversion turns into
// bf16 times 128 >> (b2 + b3), two elements per instruction; s1, constant over the block, multiplies
// the block's tile in float32.  About 2.3 instructions per weight, where
// a table of the block's eight values (mixed.hip) takes 5.4: at 4 tokens x 37888 x 3584 the decoding
// alone would take longer than the read.
#include <algorithm>

#include "fp4_bf16.h"
#include "kernels.h"
#include "ops_core.h"
#include "profiler.h"

namespace resq {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void* lds_ptr_t;

constexpr int kWaves = 16, kThreads = 64 * kWaves;
constexpr int kStep = 512;         // K elements of a step
constexpr int kAhead = 2;          // steps in a ring (1, 2, 3, 4: 24.0, 23.0, 23.8, 24.6 us at 4 x 37888 x 3584)
constexpr int kPad = 8;            // elements between X rows in LDS: four tokens' reads miss each other's banks
constexpr int kSlot = 1024 + 256;  // bytes of a step's codes and scales in the ring
constexpr int kLds = 160 * 1024;
constexpr int kRings = kWaves * kAhead * kSlot;
constexpr int kParts = kWaves * 16 * 16;  // bytes of the waves' parts of quads, 16 tokens x 4 rows each

struct MatvecParams {
  const uint16_t* X;
  int64_t ldx;
  const uint8_t* codes;
  const uint8_t* scales;
  void* Y;
  int64_t ldy, n;
  int m, d;
  int batch, batches;     // tokens in LDS at a time
  int shares, each, groups;  // shares of quads, of a workgroup; workgroups per batch, a multiple of 8 (one XCD per share)
  int quads, quads_left;  // quads per share; the first quads_left shares have one more
  int part_at, part_stride, part_flip;  // LDS of a wave's parts of quads; distance of two shares' (B > 1)
  bool out_bf16;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int64_t bytes) {
  const int64_t most = 0xFFFFFE00ll;  // a tile's offsets stay far below
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)(uint32_t)min(bytes, most), 0x00020000);
}
// 16 (4) bytes per lane from offset voff into LDS: lane l's land at lds + 16 l (4 l).
__device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t r, void* lds, uint32_t voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)lds, 16, voff, 0, 0, 0);
}
__device__ __forceinline__ void copy4(__amdgpu_buffer_rsrc_t r, void* lds, uint32_t voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)lds, 4, voff, 0, 0, 0);
}
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Barrier that leaves loads in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One byte 128 >> (b2 + b3) per group of four, for the four groups of 16 elements.
__device__ __forceinline__ uint32_t hif4_steps(uint32_t b2, uint32_t b3) {
  // bit i of b3 to byte i; bit i of b2 to bytes 2 i and 2 i + 1
  const uint32_t three = ((b3 & 0xFu) * 0x00204081u) & 0x01010101u;
  const uint32_t two = ((b2 & 3u) * 0x00808101u) & 0x01010101u;
  return __builtin_amdgcn_perm(0u, 0x00204080u, three + two);
}

template <int HI>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t v, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, HI));
}

// Eight HiF4 elements (one word of codes): +-k 2^-9 times the step 128 >> (b2 + b3) of their group
// of four, which is +-k/4 2^-(b2+b3); in the order 0 2 1 3 4 6 5 7 (low nibbles and high nibbles of a
// byte pair).
__device__ __forceinline__ void hif4_bf16(uint32_t w, float s0, float s1, uint32_t out[4]) {
  const uint32_t lo = (w & 0x07070707u) | ((w << 4) & 0x80808080u);
  const uint32_t hi = ((w >> 4) & 0x07070707u) | (w & 0x80808080u);
  out[0] = fp8_pair<0>(lo, s0);
  out[1] = fp8_pair<0>(hi, s0);
  out[2] = fp8_pair<1>(lo, s1);
  out[3] = fp8_pair<1>(hi, s1);
}

// TG: groups of four tokens in a batch.
template <int FMT, int TG>
__global__ __launch_bounds__(kThreads) void matvec_kernel(MatvecParams p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // rings, X, parts
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 3, blk = lane >> 2;
  const int turns = (p.d + kStep - 1) / kStep;
  const int t0 = (int)(blockIdx.x / p.groups) * p.batch, tokens = min(p.batch, p.m - t0);  // may be none
  const int share0 = (int)(blockIdx.x % p.groups) * p.each, share1 = min(p.shares, share0 + p.each);
  if (share0 >= share1 || tokens <= 0) return;

  // A share's steps, and those of a wave (parts that differ by one at most).
  auto quads_of = [&](int sh) { return p.quads + (sh < p.quads_left ? 1 : 0); };
  auto begin_of = [&](int sh, int v) {
    const uint32_t all = (uint32_t)quads_of(sh) * turns;
    return v * (all / kWaves) + min((uint32_t)v, all % kWaves);
  };
  auto first_quad = [&](int sh) { return sh * p.quads + min(sh, p.quads_left); };

  uint8_t* ring = lds + wave * (kAhead * kSlot);
  uint16_t* xs = reinterpret_cast<uint16_t*>(lds + kRings);
  const int width = turns * kStep, stride = width + kPad;  // a row of X, zeros past d
  const int per_row = width / 8, t_step = kThreads / per_row, c_step = kThreads % per_row;

  // Loads of the wave's steps, one after the other through its shares, into slot after slot.
  const int64_t code_row = p.d / 2, scale_row = FMT == 0 ? p.d / 32 : p.d / 64 * 4;
  const uint32_t mis = (uint32_t)(uintptr_t)p.scales & 3u;  // MXFP4: scales go as the aligned dwords around them
  const uint32_t code_at = (uint32_t)(j * code_row) + 16 * blk;
  const uint32_t scale_at = (uint32_t)(j * scale_row) + (FMT == 0 ? mis + blk : 4 * (blk >> 1));
  __amdgpu_buffer_rsrc_t code_buf, scale_buf;
  int load_share = share0 - 1, load_left = 0, load_quad = 0, load_turn = 0, load_slot = 0;
  auto seek = [&]() {  // a quad's four rows, as far as the matrix has them
    const int64_t row = 4 * (int64_t)load_quad, rows = min((int64_t)4, p.n - row);
    code_buf = buffer(p.codes + row * code_row, rows * code_row);
    scale_buf = buffer(p.scales + row * scale_row - mis, (rows * scale_row + mis + 3) & ~3ll);
  };
  auto more = [&]() {  // moves to the next share with steps left; false: none
    while (load_left == 0) {
      if (++load_share >= share1) return false;
      const uint32_t b = begin_of(load_share, wave);
      load_left = (int)(begin_of(load_share, wave + 1) - b);
      if (load_left == 0) continue;
      load_quad = first_quad(load_share) + (int)(b / (uint32_t)turns);
      load_turn = (int)(b % (uint32_t)turns);
      seek();
    }
    return true;
  };
  auto load = [&]() {
    const uint32_t k = load_turn * kStep;
    uint8_t* dst = ring + load_slot * kSlot;
    copy16(code_buf, dst, code_at + k / 2);
    const uint32_t at = scale_at + (FMT == 0 ? k / 32 : k / 16);
    copy4(scale_buf, dst + 1024, FMT == 0 ? at & ~3u : at);
    load_slot = load_slot + 1 == kAhead ? 0 : load_slot + 1;
    if (--load_left > 0 && ++load_turn == turns) {
      load_turn = 0;
      ++load_quad;
      seek();
    }
  };
  int in_flight = 0;
  while (in_flight < kAhead && more()) {
    load();
    ++in_flight;
  }

  // X of the batch into LDS, in pieces of eight elements: piece tid, tid + kThreads, ..
  int t = tid / per_row, c = tid - t * per_row;
  while (t < tokens) {
    u32x4 v[8];
    uint16_t* dst[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = u32x4{0u, 0u, 0u, 0u};
      dst[i] = t < tokens ? xs + t * stride + 8 * c : nullptr;
      if (t < tokens && 8 * c < p.d) v[i] = reinterpret_cast<const Bf16x8*>(p.X + (int64_t)(t0 + t) * p.ldx + 8 * c)->v;
      t += t_step;
      c += c_step;
      if (c >= per_row) {
        c -= per_row;
        ++t;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u32x4 o = v[i];
      if constexpr (FMT != 0)  // in the order hif4_bf16 gives: 0 2 1 3 4 6 5 7
        o = u32x4{__builtin_amdgcn_perm(o[1], o[0], 0x05040100u), __builtin_amdgcn_perm(o[1], o[0], 0x07060302u),
                  __builtin_amdgcn_perm(o[3], o[2], 0x05040100u), __builtin_amdgcn_perm(o[3], o[2], 0x07060302u)};
      if (dst[i]) *reinterpret_cast<u32x4*>(dst[i]) = o;
    }
  }
  lds_barrier();

  f32x4 sum[TG] = {};
  const uint16_t* xlane[TG];
#pragma unroll
  for (int g = 0; g < TG; ++g) xlane[g] = xs + min(4 * g + j, tokens - 1) * stride + 32 * blk;
  auto multiply = [&](int at, const u32x4& w, uint32_t sc) {
    uint32_t v[4][4];
    if constexpr (FMT == 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) mx_dequant8(w[q], sc, v[q]);
    } else {
      const uint32_t h = blk & 1, b2 = sc >> (8 + 4 * h), b3 = sc >> (16 + 8 * h);
      const uint32_t lo = hif4_steps(b2, b3), hi = hif4_steps(b2 >> 2, b3 >> 4);
      hif4_bf16(w[0], (float)(lo & 0xFFu), (float)((lo >> 8) & 0xFFu), v[0]);
      hif4_bf16(w[1], (float)((lo >> 16) & 0xFFu), (float)(lo >> 24), v[1]);
      hif4_bf16(w[2], (float)(hi & 0xFFu), (float)((hi >> 8) & 0xFFu), v[2]);
      hif4_bf16(w[3], (float)((hi >> 16) & 0xFFu), (float)(hi >> 24), v[3]);
    }
#pragma unroll
    for (int g = 0; g < TG; ++g) {
      f32x4 r = FMT == 0 ? sum[g] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(xlane[g] + at + 8 * q);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const u32x2 a = {x[2 * e], x[2 * e + 1]}, b = {v[q][2 * e], v[q][2 * e + 1]};
          r = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), r, 0, 0, 0);
        }
      }
      if constexpr (FMT == 0) {
        sum[g] = r;
      } else {
        // s1 = 2^(e-31) (1 + m/4) for code 4 e + m
        const float s1 = __uint_as_float(((sc & 0xFFu) << 21) + ((127u - 31u) << 23));
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[g][i] = fmaf(s1, r[i], sum[g][i]);
      }
    }
  };
  // The 16 blocks' sums added, the four tokens' in one go: lane 16 r + j (j < 4) gets token r of row j.
  // Clears them.
  auto reduce = [&](float out[TG]) {
#pragma unroll
    for (int g = 0; g < TG; ++g) {
      float v = add_pair<false>(add_pair<true>(sum[g][0], sum[g][2]), add_pair<true>(sum[g][1], sum[g][3]));
      v += dpp<kDppRor8>(v);
      out[g] = v + dpp<kDppRor4>(v);
      sum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  const bool holds = (blk & 3) == 0;  // this lane's sum is the one that is kept: of token 4 g + tok
  const int tok = lane >> 4;
  auto store = [&](int quad, const float v[TG]) {
    const int64_t row = 4 * (int64_t)quad + j;
    if (!holds || row >= p.n) return;
#pragma unroll
    for (int g = 0; g < TG; ++g) {
      const int tk = 4 * g + tok;
      if (tk >= tokens) continue;
      const int64_t at = (int64_t)(t0 + tk) * p.ldy + row;
      if (p.out_bf16) reinterpret_cast<uint16_t*>(p.Y)[at] = bf16_bits(v[g]);
      else reinterpret_cast<float*>(p.Y)[at] = v[g];
    }
  };

  int slot = 0;
  for (int sh = share0; sh < share1; ++sh) {
    const uint32_t begin = begin_of(sh, wave);
    const int q0 = first_quad(sh), count = (int)(begin_of(sh, wave + 1) - begin);
    int quad = q0 + (int)(begin / (uint32_t)turns), turn = (int)(begin % (uint32_t)turns);
    bool whole = turn == 0;  // this wave has the quad from its first step on
    float head[TG] = {};     // of a quad that an earlier wave began
    for (int s = 0; s < count; ++s) {
      if (in_flight == kAhead) wait_vm<2 * (kAhead - 1)>();
      else wait_vm<0>();
      const uint8_t* src = ring + slot * kSlot;
      const u32x4 w = *reinterpret_cast<const u32x4*>(src + 16 * lane);
      uint32_t sc = *reinterpret_cast<const uint32_t*>(src + 1024 + 4 * lane);
      if constexpr (FMT == 0) {
        sc = (sc >> (8 * (scale_at & 3u))) & 0xFFu;
        // past the row's end the code may be any row's: a finite one, against zeros of X
        if (turn == turns - 1 && turn * kStep + 32 * blk >= p.d) sc = 127u;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
      --in_flight;
      if (more()) {
        load();
        ++in_flight;
      }
      multiply(turn * kStep, w, sc);
      slot = slot + 1 == kAhead ? 0 : slot + 1;
      if (++turn == turns) {
        float v[TG];
        reduce(v);
        if (whole) {
          store(quad, v);
        } else {
#pragma unroll
          for (int g = 0; g < TG; ++g) head[g] = v[g];
        }
        whole = true;
        turn = 0;
        ++quad;
      }
    }
    // Shared quads: each wave leaves its part of a quad that an earlier wave began.  (Two shares' parts
    // lie apart: a wave may be in the next share's steps while another still adds.)
    float tail[TG];
    reduce(tail);
    const bool inside = count > 0 && !whole;  // its only quad neither begins nor ends here
    const int at = p.part_at + ((sh - share0) & 1) * p.part_flip;
    if (holds)
#pragma unroll
      for (int g = 0; g < TG; ++g)
        reinterpret_cast<float*>(lds + at + wave * p.part_stride)[g * 16 + 4 * tok + j] = inside ? tail[g] : head[g];
    lds_barrier();
    if (whole && turn > 0) {  // this wave began the quad: add the waves after it up to the quad's end
      const uint32_t end = (uint32_t)(quad - q0 + 1) * turns;
      for (int v = wave + 1; v < kWaves && begin_of(sh, v) < end; ++v)
        if (holds && begin_of(sh, v + 1) > begin_of(sh, v))
#pragma unroll
          for (int g = 0; g < TG; ++g)
            tail[g] += reinterpret_cast<const float*>(lds + at + v * p.part_stride)[g * 16 + 4 * tok + j];
      store(quad, tail);
    }
  }
}

// d = 0: sums of nothing.
__global__ __launch_bounds__(256) void matvec_zero_kernel(MatvecParams p) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.n) return;
  for (int t = 0; t < p.m; ++t) {
    if (p.out_bf16) reinterpret_cast<uint16_t*>(p.Y)[t * p.ldy + i] = 0;
    else reinterpret_cast<float*>(p.Y)[t * p.ldy + i] = 0.f;
  }
}

int64_t x_bytes(int64_t tokens, int64_t d) { return tokens * ((d + kStep - 1) / kStep * kStep + kPad) * 2; }

template <int FMT>
void launch_fmt(MatvecParams p, hipStream_t s) {
  const int64_t quads = (p.n + 3) / 4;
  p.shares = (int)std::min<int64_t>(quads, 256);
  p.quads = (int)(quads / p.shares);
  p.quads_left = (int)(quads % p.shares);
  const int fit = (int)((kLds - kRings - 2 * kParts) / x_bytes(1, p.d));
  p.batches = 1;  // a power of two: with 256 shares every CU gets one workgroup
  if (p.m * x_bytes(1, p.d) > kLds - kRings)
    while (p.batches * fit < p.m) p.batches *= 2;
  p.batch = (p.m + p.batches - 1) / p.batches;
  p.each = (p.shares * p.batches + 255) / 256;
  p.groups = p.batches == 1 ? p.shares : ((p.shares + p.each - 1) / p.each + 7) / 8 * 8;
  int64_t lds = kRings + x_bytes(p.batch, p.d);
  if (p.batches == 1) {  // one share: a wave's ring is free by the time its parts are written
    p.part_at = 0;
    p.part_stride = kAhead * kSlot;
  } else {
    p.part_at = (int)lds;
    p.part_stride = kParts / kWaves;
    p.part_flip = kParts;
    lds += 2 * kParts;
  }
  const dim3 grid((unsigned)(p.groups * p.batches));
  const int tg = (p.batch + 3) / 4;
  if (tg == 1) launch_timed(matvec_kernel<FMT, 1>, grid, dim3(kThreads), (uint32_t)lds, s, p);
  else if (tg == 2) launch_timed(matvec_kernel<FMT, 2>, grid, dim3(kThreads), (uint32_t)lds, s, p);
  else if (tg == 3) launch_timed(matvec_kernel<FMT, 3>, grid, dim3(kThreads), (uint32_t)lds, s, p);
  else launch_timed(matvec_kernel<FMT, 4>, grid, dim3(kThreads), (uint32_t)lds, s, p);
}

}  // namespace

bool matvec_supported(int64_t d) { return kRings + 2 * kParts + x_bytes(1, d) <= kLds; }

void launch_matvec(int fmt, const uint16_t* X, int64_t m, int64_t d, int64_t ldx, const uint8_t* codes,
                   const void* scales, int64_t n, void* Y, int64_t ldy, bool out_bf16, hipStream_t s) {
  MatvecParams p{};
  p.X = X; p.ldx = ldx; p.codes = codes; p.scales = (const uint8_t*)scales; p.Y = Y; p.ldy = ldy;
  p.n = n; p.m = (int)m; p.d = (int)d; p.out_bf16 = out_bf16;
  if (d == 0) launch_timed(matvec_zero_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0u, s, p);
  else if (fmt == 0) launch_fmt<0>(p, s);
  else launch_fmt<1>(p, s);
}

}  // namespace resq
