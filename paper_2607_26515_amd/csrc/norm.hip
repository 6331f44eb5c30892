// Norms before and after a block, fused with the block's gate, its residual scale and the
// residual addition, and their gradients (resq_block_norm_fwd / resq_block_norm_bwd):
//
//   t = y r_y gamma_post           r = 1 / sqrt(mean(row^2) + eps)
//   h' = h + alpha g t             g: none, per channel or per token
//   x = h' r_h gamma_pre           of the stored h'
//
// Both are bound by HBM: each row is read once and kept in registers between its statistics and
// its use.  A row belongs to L lanes of one workgroup, each holding C groups of eight consecutive
// elements; L <= 64 shares a workgroup between several rows.
#include <algorithm>

#include "kernels.h"
#include "ops_core.h"
#include "profiler.h"

namespace resq {
namespace {

constexpr int kMaxWaves = 16;

// Sum of N values per lane over the L lanes of a row (L a power of two up to 64, or a multiple of
// 64: then the whole workgroup is one row and lds holds N * kMaxWaves values).  Every lane gets
// the sum; the order is fixed.  Barriers: one (L > 64); lds must not be in use by an earlier call.
template <int N, typename T>
__device__ __forceinline__ void row_sum(T v[N], int L, T* lds) {
  const int width = L < 64 ? L : 64;
  for (int o = 1; o < width; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if (L > 64) {
    const int wave = threadIdx.x >> 6, waves = L >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[i * kMaxWaves + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      T t = lds[i * kMaxWaves];
      for (int w = 1; w < waves; ++w) t += lds[i * kMaxWaves + w];
      v[i] = t;
    }
  }
}

// 1 / sqrt(s / d + eps) with every step rounded to float32, as the RMSNorm producer of the
// forward computes it from its exact sum (so the two give one X).  A sum past float32's range is
// taken on in float64.
__device__ __forceinline__ float rms_factor(double s, int64_t d, float eps) {
  const float f = (float)s;
  if (f < INFINITY) return 1.f / sqrtf(f / (float)d + eps);
  return (float)(1.0 / sqrt(s / (double)d + (double)eps));
}

template <typename TH, typename TY, int C>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(NormFwd p, int L) {
  __shared__ double lds[2][kMaxWaves];
  const int lane = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / L) + threadIdx.x / L;
  const bool in = row < p.m;
  const TH* h = reinterpret_cast<const TH*>(p.h) + row * p.ldh;
  const TY* y = reinterpret_cast<const TY*>(p.y) + row * p.ldy;
  float v[C][8], t[C][8];
  int64_t col[C];
  int n[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = ((int64_t)c * L + lane) * 8;
    n[c] = in ? (int)max((int64_t)0, min((int64_t)8, p.d - col[c])) : 0;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) load_upto8(h + col[c], n[c], 0.f, v[c]);
  if (p.y) {
#pragma unroll
    for (int c = 0; c < C; ++c) load_upto8(y + col[c], n[c], 0.f, t[c]);
    if (p.gamma_post) {
      double s[1] = {0.0};
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fma((double)t[c][i], (double)t[c][i], s[0]);
      row_sum<1>(s, L, lds[0]);
      const float r = rms_factor(s[0], p.d, p.eps);
      if (p.rstd && in && lane == 0) p.rstd[row] = r;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float g[8];
        load_upto8(p.gamma_post + col[c], n[c], 0.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[c][i] = t[c][i] * r * g[i];
      }
    }
    float a = p.alpha;
    if (p.gate_mode == kGateToken && in)
      a *= p.gate_f32 ? reinterpret_cast<const float*>(p.gate)[row]
                      : bf16_value(reinterpret_cast<const uint16_t*>(p.gate)[row]);
    TH* ho = reinterpret_cast<TH*>(p.h_out) + row * p.ldho;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (p.gate_mode == kGateChannel) {
        float g[8];
        if (p.gate_f32) load_upto8(reinterpret_cast<const float*>(p.gate) + col[c], n[c], 0.f, g);
        else load_upto8(reinterpret_cast<const uint16_t*>(p.gate) + col[c], n[c], 0.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[c][i] *= g[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[c][i] = fmaf(a, t[c][i], v[c][i]);
        if constexpr (sizeof(TH) == 2) v[c][i] = bf16_value(bf16_bits(v[c][i]));
      }
      store_upto8(ho + col[c], n[c], v[c]);
    }
  }
  if (p.rstd && in && lane == 0 && !(p.y && p.gamma_post)) p.rstd[row] = 0.f;
  if (!p.gamma_pre) {
    if (p.rstd && in && lane == 0) p.rstd[p.m + row] = 0.f;
    return;
  }
  double s[1] = {0.0};
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = fma((double)v[c][i], (double)v[c][i], s[0]);
  row_sum<1>(s, L, lds[1]);
  const float r = rms_factor(s[0], p.d, p.eps);
  if (p.rstd && in && lane == 0) p.rstd[p.m + row] = r;
  uint16_t* x = p.x + row * p.ldx;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float g[8];
    load_upto8(p.gamma_pre + col[c], n[c], 0.f, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = v[c][i] * r * g[i];
    store_upto8(x + col[c], n[c], g);
  }
}

// Gradients, per row (hn = h r_h, yn = y r_y, or y itself without the norm):
//   e  = dh' + r_h (dx gamma_pre - hn c),  c = mean(dx gamma_pre hn)                -> dh
//   dt = alpha g e,  t = yn gamma_post
//   dy = r_y (dt gamma_post - yn k),  k = mean(dt gamma_post yn)   (dy = dt without the norm)
//   dg = sum of alpha e t over the axis that g is broadcast along
//   dgamma_pre = sum over rows of dx hn,  dgamma_post = sum over rows of dt yn
// With w = alpha gamma_post yn (times g of the channel) the second mean follows from sums that
// need no c: sum(w e) = sum(w (dh' + r_h dx gamma_pre)) - r_h c sum(w hn), so one reduction per
// row gives c, k and a token's dg.
// A workgroup walks over rows and keeps the column sums in registers; each of its row groups
// writes one row of partial sums, which norm_bwd_sum_kernel adds in a fixed order.
template <typename TH, typename TY, typename TX, int C>
__global__ __launch_bounds__(1024) void norm_bwd_kernel(NormBwd p, int L) {
  __shared__ float lds[2][3 * kMaxWaves];
  const int lane = threadIdx.x % L, groups = blockDim.x / L;
  const int64_t group = (int64_t)blockIdx.x * groups + threadIdx.x / L, n_groups = (int64_t)gridDim.x * groups;
  const bool pre = p.gamma_pre != nullptr, post = p.gamma_post != nullptr;
  const bool need_y = p.y != nullptr;
  int64_t col[C];
  int nc[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = ((int64_t)c * L + lane) * 8;
    nc[c] = (int)max((int64_t)0, min((int64_t)8, p.d - col[c]));
  }
  float s_pre[C][8] = {}, s_post[C][8] = {}, s_gate[C][8] = {};
  const int64_t trips = (p.m + n_groups - 1) / n_groups;
  for (int64_t k = 0; k < trips; ++k) {  // the same count for every lane: row_sum has a barrier
    const int64_t row = group + k * n_groups;
    const bool in = row < p.m;
    float h[C][8], u[C][8], e[C][8], yn[C][8];
    const float rh = pre && in ? p.rstd[p.m + row] : 0.f, ry = post && in ? p.rstd[row] : 1.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = in ? nc[c] : 0;
      if (pre) {
        load_upto8(reinterpret_cast<const TH*>(p.h) + row * p.ldh + col[c], n, 0.f, h[c]);
        load_upto8(reinterpret_cast<const TX*>(p.dx) + row * p.lddx + col[c], n, 0.f, u[c]);
      }
      if (p.dho) load_upto8(reinterpret_cast<const TH*>(p.dho) + row * p.lddho + col[c], n, 0.f, e[c]);
      else
        for (int i = 0; i < 8; ++i) e[c][i] = 0.f;
      if (need_y) load_upto8(reinterpret_cast<const TY*>(p.y) + row * p.ldy + col[c], n, 0.f, yn[c]);
    }
    float gt = 1.f;
    if (p.gate_mode == kGateToken && in)
      gt = p.gate_f32 ? reinterpret_cast<const float*>(p.gate)[row]
                      : bf16_value(reinterpret_cast<const uint16_t*>(p.gate)[row]);
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (pre) {
        float g[8];
        load_upto8(p.gamma_pre + col[c], nc[c], 0.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[c][i] *= rh;
          s_pre[c][i] = fmaf(u[c][i], h[c][i], s_pre[c][i]);
          u[c][i] *= g[i];
          s[0] = fmaf(u[c][i], h[c][i], s[0]);
          e[c][i] = fmaf(rh, u[c][i], e[c][i]);
        }
      }
      if (need_y) {
        float gp[8], gc[8];
        if (post) load_upto8(p.gamma_post + col[c], nc[c], 0.f, gp);
        if (p.gate_mode == kGateChannel) {
          if (p.gate_f32) load_upto8(reinterpret_cast<const float*>(p.gate) + col[c], nc[c], 0.f, gc);
          else load_upto8(reinterpret_cast<const uint16_t*>(p.gate) + col[c], nc[c], 0.f, gc);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          yn[c][i] *= ry;
          float w = p.alpha * yn[c][i];
          if (post) w *= gp[i];
          if (p.gate_mode == kGateChannel) w *= gc[i];
          s[1] = fmaf(w, e[c][i], s[1]);
          if (pre) s[2] = fmaf(w, h[c][i], s[2]);
        }
      }
    }
    row_sum<3>(s, L, lds[k & 1]);
    const float rc = rh * (s[0] / (float)p.d);
    const float we = s[1] - rc * s[2];
    if (p.gate_mode == kGateToken && p.dgate && in && lane == 0) p.dgate[row] = we;
    const float km = we * gt / (float)p.d, a = p.alpha * gt;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = in ? nc[c] : 0;
      if (pre)
#pragma unroll
        for (int i = 0; i < 8; ++i) e[c][i] = fmaf(-rc, h[c][i], e[c][i]);
      if (p.dh) store_upto8(reinterpret_cast<TH*>(p.dh) + row * p.lddh + col[c], n, e[c]);
      if (!need_y && !p.dy) continue;
      float gp[8], gc[8];
      if (post) load_upto8(p.gamma_post + col[c], nc[c], 0.f, gp);
      if (p.gate_mode == kGateChannel) {
        if (p.gate_f32) load_upto8(reinterpret_cast<const float*>(p.gate) + col[c], nc[c], 0.f, gc);
        else load_upto8(reinterpret_cast<const uint16_t*>(p.gate) + col[c], nc[c], 0.f, gc);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float dt = a * e[c][i];
        if (p.gate_mode == kGateChannel) {
          if (p.part_gate) s_gate[c][i] = fmaf(dt * (post ? gp[i] : 1.f), yn[c][i], s_gate[c][i]);
          dt *= gc[i];
        }
        if (post) {
          s_post[c][i] = fmaf(dt, yn[c][i], s_post[c][i]);
          dt = ry * (dt * gp[i] - yn[c][i] * km);
        }
        e[c][i] = dt;
      }
      if (p.dy) {
        if (p.dy_f32) store_upto8(reinterpret_cast<float*>(p.dy) + row * p.lddy + col[c], n, e[c]);
        else store_upto8(reinterpret_cast<uint16_t*>(p.dy) + row * p.lddy + col[c], n, e[c]);
      }
    }
  }
  // partial sums: [vector][group][d]
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (p.part_pre) store_upto8(p.part_pre + group * p.d + col[c], nc[c], s_pre[c]);
    if (p.part_post) store_upto8(p.part_post + group * p.d + col[c], nc[c], s_post[c]);
    if (p.part_gate) store_upto8(p.part_gate + group * p.d + col[c], nc[c], s_gate[c]);
  }
}

struct ColumnSums {
  const float* part[3];
  float* out[3];
};

// out[j] = sum over the n_groups partial rows of column j, in float64: a workgroup takes 64
// columns, its 16 waves every 16th row, and the waves' sums are added in order.
__global__ __launch_bounds__(1024) void norm_bwd_sum_kernel(ColumnSums q, int64_t n_groups, int64_t d) {
  __shared__ double lds[16][64];
  const float* part = q.part[blockIdx.y];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t j = (int64_t)blockIdx.x * 64 + lane;
  double s = 0.0;
  if (j < d)
#pragma unroll 4
    for (int64_t g = wave; g < n_groups; g += 16) s += (double)part[g * d + j];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && j < d) {
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    q.out[blockIdx.y][j] = (float)s;
  }
}

struct RowLanes {
  int L, threads, C;
};

// Lanes per row and groups of eight per lane: up to 64 lanes a power of two, several rows to a
// workgroup of 256; beyond, whole waves.
RowLanes row_lanes(int64_t d) {
  const int64_t g = (d + 7) / 8;
  RowLanes r{};
  r.C = g <= 256 ? 1 : 2;
  const int64_t lanes = (g + r.C - 1) / r.C;
  if (lanes <= 64) {
    r.L = 1;
    while (r.L < lanes) r.L *= 2;
    r.threads = 256;
  } else {
    r.L = (int)((lanes + 63) / 64 * 64);
    r.threads = r.L;
  }
  return r;
}

int64_t bwd_workgroups(int64_t m, int64_t d) {
  const RowLanes r = row_lanes(d);
  const int64_t rows = r.threads / r.L;
  return std::min<int64_t>((m + rows - 1) / rows, 512);
}

}  // namespace

size_t norm_bwd_ws_bytes(int64_t m, int64_t d) {
  if (m <= 0 || d <= 0 || d > kNormMaxD) return 0;
  const RowLanes r = row_lanes(d);
  return (size_t)bwd_workgroups(m, d) * (r.threads / r.L) * d * 3 * sizeof(float);
}

void launch_norm_fwd(const NormFwd& p, bool h_f32, bool y_f32, hipStream_t s) {
  const RowLanes r = row_lanes(p.d);
  const int64_t rows = r.threads / r.L;
  const dim3 grid((unsigned)((p.m + rows - 1) / rows)), block(r.threads);
#define RESQ_NF(H, Y, C) launch_timed(norm_fwd_kernel<H, Y, C>, grid, block, 0u, s, p, r.L)
#define RESQ_NF2(H, Y) do { if (r.C == 1) RESQ_NF(H, Y, 1); else RESQ_NF(H, Y, 2); } while (0)
  if (h_f32) { if (y_f32) RESQ_NF2(float, float); else RESQ_NF2(float, uint16_t); }
  else { if (y_f32) RESQ_NF2(uint16_t, float); else RESQ_NF2(uint16_t, uint16_t); }
#undef RESQ_NF2
#undef RESQ_NF
}

void launch_norm_bwd(NormBwd p, bool h_f32, bool y_f32, bool dx_f32, float* dgamma_post, float* dgamma_pre,
                     float* workspace, hipStream_t s) {
  const RowLanes r = row_lanes(p.d);
  const int64_t wgs = bwd_workgroups(p.m, p.d), n_groups = wgs * (r.threads / r.L);
  ColumnSums q{};
  int nv = 0;
  float* next = workspace;
  auto sums = [&](float* out) -> float* {
    if (!out) return nullptr;
    float* part = next;
    next += n_groups * p.d;
    q.part[nv] = part;
    q.out[nv++] = out;
    return part;
  };
  p.part_pre = sums(dgamma_pre);
  p.part_post = sums(dgamma_post);
  p.part_gate = sums(p.gate_mode == kGateChannel ? p.dgate : nullptr);
  const dim3 grid((unsigned)wgs), block(r.threads);
#define RESQ_NB(H, Y, X, C) launch_timed(norm_bwd_kernel<H, Y, X, C>, grid, block, 0u, s, p, r.L)
#define RESQ_NB2(H, Y, X) do { if (r.C == 1) RESQ_NB(H, Y, X, 1); else RESQ_NB(H, Y, X, 2); } while (0)
#define RESQ_NB3(H, Y) do { if (dx_f32) RESQ_NB2(H, Y, float); else RESQ_NB2(H, Y, uint16_t); } while (0)
  if (h_f32) { if (y_f32) RESQ_NB3(float, float); else RESQ_NB3(float, uint16_t); }
  else { if (y_f32) RESQ_NB3(uint16_t, float); else RESQ_NB3(uint16_t, uint16_t); }
#undef RESQ_NB3
#undef RESQ_NB2
#undef RESQ_NB
  if (nv > 0)
    launch_timed(norm_bwd_sum_kernel, dim3((unsigned)((p.d + 63) / 64), (unsigned)nv), dim3(1024), 0u, s, q, n_groups,
                 p.d);
}

}  // namespace resq
