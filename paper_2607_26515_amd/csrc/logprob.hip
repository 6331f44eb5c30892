// Log probabilities of given tokens with the entropy and the top alternatives, and the gradient of
// the logits (resq_token_logprobs / resq_token_logprobs_bwd).  Per row x of V logits, temperature T:
//
//   M = max x,  S = sum exp((x - M) / T),  log p_j = (x_j - M) / T - log S
//   H = -sum p log p = log S - sum(exp((x - M) / T) (x - M)) / (T S)
//   dx_j = (a (delta_jt - p_j) - b p_j (log p_j + H)) / T      a = dlogp, b = dentropy
//
// The forward reads the logits once: every lane keeps a running maximum, the sum and the weighted
// sum relative to it, and the largest group of eight it has seen.  Few rows are split over several
// workgroups, whose partial results a second kernel joins.
//
// Top k (k <= 32): the k-th largest of the lanes' largest elements bounds the k-th largest element
// of the row from below, and every element at or above that bound lies with one of the k lanes
// whose own largest is.  So only those lanes' elements are looked at again.  Elements are ranked by
// 64-bit keys (the value's order-preserving pattern, then the inverted index), so ties go to the
// lowest index and the result does not depend on the order of work.
#include <algorithm>

#include "kernels.h"
#include "ops_core.h"
#include "profiler.h"

namespace resq {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kGroup = 8;                            // elements per load
constexpr int64_t kStep = (int64_t)kThreads * kGroup;  // elements per trip of a workgroup

// Descending order of values as ascending-free unsigned keys: larger value, then lower index.
// -inf and NaN are no alternatives: key 0.
__device__ __forceinline__ uint64_t top_key(float v, uint32_t idx) {
  if (!(v > -INFINITY)) return 0ull;
  if (v == 0.f) v = 0.f;  // -0 ranks with +0
  const uint32_t u = __float_as_uint(v);
  const uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return ((uint64_t)o << 32) | (uint32_t)~idx;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o ^ ((uint32_t)((int32_t)~o >> 31) | 0x80000000u));
}

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t v, int o) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, o, 64), hi = (uint32_t)__shfl_xor((int)(v >> 32), o, 64);
  return ((uint64_t)hi << 32) | lo;
}

// The wave's 64 keys in descending order by lane (bitonic sort).
__device__ __forceinline__ uint64_t sort64(uint64_t v, int lane) {
#pragma unroll
  for (int k = 2; k <= 64; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const uint64_t o = shfl_xor_u64(v, j);
      const bool keep_max = ((lane & j) == 0) == ((lane & k) == 0);
      v = keep_max ? max(v, o) : min(v, o);
    }
  return v;
}
// Lanes 0..31 and, reversed, 32..63 hold descending lists: the 64 keys in descending order.
__device__ __forceinline__ uint64_t merge64(uint64_t v, int lane) {
#pragma unroll
  for (int j = 32; j > 0; j >>= 1) {
    const uint64_t o = shfl_xor_u64(v, j);
    v = (lane & j) == 0 ? max(v, o) : min(v, o);
  }
  return v;
}
// Takes 64 more keys into the descending list of 32 in lanes 0..31.
__device__ __forceinline__ uint64_t take64(uint64_t list, uint64_t more, int lane) {
  const uint64_t least = ((uint64_t)(uint32_t)__shfl((int)(list >> 32), 31, 64) << 32) |
                         (uint32_t)__shfl((int)(uint32_t)list, 31, 64);
  if (__ballot(more > least) == 0ull) return list;
  more = sort64(more, lane);
  // the 32 largest of them, reversed, in lanes 32..63
  const uint64_t rev = shfl_xor_u64(more, 63);
  return merge64(lane < 32 ? list : rev, lane);
}

// Joins the waves' lists (lanes 0..31 of each) in wave 0.  Every wave must call it.
__device__ __forceinline__ uint64_t join_waves(uint64_t list, uint64_t (*lds)[32], int lane, int wave) {
  for (int half = kWaves / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (wave >= half && wave < 2 * half && lane < 32) lds[wave - half][lane] = list;
    __syncthreads();
    if (wave < half) list = merge64(lane < 32 ? list : lds[wave][63 - lane], lane);
  }
  return list;
}

struct Sums {
  float M, S, W;  // maximum, sum of e = exp((x - M) / T), sum of e (x - M)
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }  // below 2^-126: 0

// The sums relative to a larger maximum M > -inf.  Where the factor is zero so is the weighted sum:
// at distances near the type's lowest value S (a.M - M) overflows.  An empty side (maximum -inf)
// holds zeros, or a NaN element's NaN, and keeps them.
__device__ __forceinline__ Sums rebase(const Sums& a, float M, float c) {
  if (a.M == -INFINITY) return {M, a.S, a.W};
  const float d = a.M - M, f = exp2_fast(d * c);
  return {M, a.S * f, f > 0.f ? (a.W + a.S * d) * f : 0.f};
}

// Two partial sums joined at their larger maximum.
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c) {
  const float M = fmaxf(a.M, b.M);
  if (M == -INFINITY) return {M, a.S + b.S, a.W + b.W};
  const Sums sa = rebase(a, M, c), sb = rebase(b, M, c);
  return {M, sa.S + sb.S, sa.W + sb.W};
}

__device__ __forceinline__ Sums wave_join(Sums s, float c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    s = join(s, Sums{__shfl_xor(s.M, o, 64), __shfl_xor(s.S, o, 64), __shfl_xor(s.W, o, 64)}, c);
  return s;
}

struct Args {
  LogprobFwd p;
  float c, inv_t;       // log2(e) / T, 1 / T
  int64_t splits, len;  // workgroups per row, elements each (a multiple of kStep)
  Sums* sums;           // [m][splits]
  uint64_t* keys;       // [m][splits][32]
};

__device__ __forceinline__ int64_t target_of(const LogprobFwd& p, int64_t row) { return p.targets ? p.targets[row] : 0; }

// The row's results from its sums (all lanes of wave 0 call it; list: the top keys).
template <typename T>
__device__ __forceinline__ void finish(const Args& a, int64_t row, const Sums& s, uint64_t list, int lane) {
  const LogprobFwd& p = a.p;
  const bool dead = p.targets && p.targets[row] < 0;
  const float log_s = s.M == -INFINITY && s.S == 0.f ? -INFINITY : logf(s.S);
  const bool none = s.M == -INFINITY;
  if (lane == 0) {
    float H = none ? s.S : log_s - s.W / s.S * a.inv_t;
    if (H < 0.f) H = 0.f;
    p.stats[row * 3] = dead ? 0.f : s.M;
    p.stats[row * 3 + 1] = dead ? 0.f : log_s;
    p.stats[row * 3 + 2] = dead ? 0.f : H;
    if (p.logp) {
      float lp = 0.f;
      if (!dead) {
        const int64_t t = p.targets[row];
        if (t >= p.V) lp = NAN;
        else if (none) lp = s.S == 0.f ? -INFINITY : NAN;
        else lp = (load1(reinterpret_cast<const T*>(p.logits) + row * p.ld + t) - s.M) * a.inv_t - log_s;
      }
      p.logp[row] = lp;
    }
  }
  if (lane < p.top_k) {
    const bool has = list != 0ull && !dead;
    p.top_index[row * p.top_k + lane] = has ? (int32_t)~(uint32_t)list : -1;
    p.top_logp[row * p.top_k + lane] = has ? (key_value(list) - s.M) * a.inv_t - log_s : -INFINITY;
  }
}

// One workgroup per row and split.
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_kernel(Args a) {
  __shared__ Sums wave_sums[kWaves];
  __shared__ uint64_t lists[kWaves][32];
  __shared__ uint64_t bound_key;
  __shared__ int n_owner;
  __shared__ int owner[32];
  const int64_t row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool dead = a.p.targets && a.p.targets[row] < 0;
  if (dead && a.splits > 1) return;
  const T* x = reinterpret_cast<const T*>(a.p.logits) + row * a.p.ld;
  const int64_t lo = split * a.len, hi = dead ? lo : min(a.p.V, lo + a.len);

  Sums s{-INFINITY, 0.f, 0.f};
  float best = -INFINITY;
  int64_t best_at = 0;
  for (int64_t i = lo + (int64_t)tid * kGroup; i < hi; i += kStep) {
    float v[8];
    load_upto8(x + i, (int)min((int64_t)8, hi - i), -INFINITY, v);
    float g = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) g = fmaxf(g, v[j]);
    if (g > best) { best = g; best_at = i; }
    const float M = fmaxf(s.M, g);
    const float base = M == -INFINITY ? 0.f : M;
    if (M > s.M) s = rebase(s, M, a.c);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float dj = v[j] - base, e = exp2_fast(dj * a.c);
      s.S += e;
      s.W = fmaf(e, fmaxf(dj, -3.4028234663852886e38f), s.W);
    }
  }
  uint64_t mine = 0ull;
  if constexpr (TOP) {
    if (best > -INFINITY) {
      float v[8];
      load_upto8(x + best_at, (int)min((int64_t)8, hi - best_at), -INFINITY, v);
      int at = 0;
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (v[j] == best) at = j;
      mine = top_key(best, (uint32_t)(best_at + at));
    }
  }
  s = wave_join(s, a.c);
  if (lane == 0) wave_sums[wave] = s;
  if (tid == 0) n_owner = 0;
  __syncthreads();
  if (wave == 0) {
    s = lane < kWaves ? wave_sums[lane] : Sums{-INFINITY, 0.f, 0.f};
    s = wave_join(s, a.c);
  }
  uint64_t list = 0ull;
  if constexpr (TOP) {
    list = join_waves(sort64(mine, lane), lists, lane, wave);
    if (wave == 0 && lane == a.p.top_k - 1) bound_key = list;
    __syncthreads();
    const uint64_t bound = bound_key;
    // the lanes whose largest element is among the k largest of them
    if (mine != 0ull && mine >= bound) owner[atomicAdd(&n_owner, 1)] = tid;
    __syncthreads();
    const int owners = n_owner;
    const int64_t trips = (hi - lo + kStep - 1) / kStep;
    list = 0ull;
    for (int o = wave; o < owners; o += kWaves) {
      const int64_t first = lo + (int64_t)owner[o] * kGroup;
      for (int64_t t = 0; t < trips; t += 64 / kGroup) {  // 64 elements: eight groups of this owner
        const int64_t i = first + (t + lane / kGroup) * kStep + lane % kGroup;
        uint64_t k = 0ull;
        if (t + lane / kGroup < trips && i < hi) k = top_key(load1(x + i), (uint32_t)i);
        list = take64(list, k >= bound ? k : 0ull, lane);
      }
    }
    list = join_waves(list, lists, lane, wave);
  }
  if (wave != 0) return;
  if (a.splits == 1) {
    finish<T>(a, row, s, list, lane);
  } else {
    if (lane == 0) a.sums[blockIdx.x] = s;
    if (TOP && lane < 32) a.keys[(int64_t)blockIdx.x * 32 + lane] = list;
  }
}

// Joins the splits of a row: one wave per row.
template <typename T, bool TOP>
__global__ __launch_bounds__(64) void logprob_join_kernel(Args a) {
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  Sums s{-INFINITY, 0.f, 0.f};
  uint64_t list = 0ull;
  if (!(a.p.targets && a.p.targets[row] < 0)) {
    for (int64_t i = lane; i < a.splits; i += 64) s = join(s, a.sums[row * a.splits + i], a.c);
    s = wave_join(s, a.c);
    if constexpr (TOP)
      for (int64_t i = 0; i < a.splits * 32; i += 64) {
        const uint64_t k = i + lane < a.splits * 32 ? a.keys[row * a.splits * 32 + i + lane] : 0ull;
        list = take64(list, k, lane);
      }
  }
  finish<T>(a, row, s, list, lane);
}

// Workgroups per row: enough to give every CU four, none with less than one trip.
int64_t splits_of(int64_t m, int64_t V) {
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(m, 1));
  const int64_t trips = (V + kStep - 1) / kStep;
  const int64_t per = (trips + want - 1) / want;
  return (trips + per - 1) / per;
}
int64_t split_len(int64_t V, int64_t splits) {
  const int64_t trips = (V + kStep - 1) / kStep;
  return (trips + splits - 1) / splits * kStep;
}
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

// The gradient: one pass, a workgroup per kBwdLen elements of a row.
constexpr int kBwdThreads = 256;
constexpr int64_t kBwdLen = (int64_t)kBwdThreads * 8 * 2;

template <typename T, typename O>
__global__ __launch_bounds__(kBwdThreads) void logprob_bwd_kernel(LogprobBwd p, int64_t parts, float inv_t) {
  const int64_t row = blockIdx.x / parts;
  const int64_t lo = (blockIdx.x % parts) * kBwdLen, hi = min(p.V, lo + kBwdLen);
  const T* x = reinterpret_cast<const T*>(p.logits) + row * p.ld;
  O* out = reinterpret_cast<O*>(p.dlogits) + row * p.ldd;
  const int64_t target = p.targets[row];
  const float M = p.stats[row * 3], log_s = p.stats[row * 3 + 1], H = p.stats[row * 3 + 2];
  const bool zero = target < 0 || M == -INFINITY;
  float a = p.dlogp ? p.dlogp[row] : 0.f;
  const float b = p.dentropy ? p.dentropy[row] : 0.f;
  if (target >= p.V) a = NAN;
  for (int64_t i = lo + (int64_t)threadIdx.x * 8; i < hi; i += kBwdThreads * 8) {
    const int n = (int)min((int64_t)8, hi - i);
    float v[8];
    if (!zero) load_upto8(x + i, n, -INFINITY, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float g = 0.f;
      if (!zero) {
        const float lp = (v[j] - M) * inv_t - log_s;
        const float q = exp2_fast(lp * 1.4426950408889634f);
        g = -q * (a + (q > 0.f ? b * (lp + H) : 0.f));
        if (i + j == target) g += a;
        g *= inv_t;
      }
      v[j] = g;
    }
    store_upto8(out + i, n, v);
  }
}

}  // namespace

size_t logprob_ws_bytes(int64_t m, int64_t V, int top_k) {
  if (m <= 0 || V <= 0) return 0;
  const int64_t sp = splits_of(m, V);
  if (sp == 1) return 0;
  return up256((size_t)(m * sp) * sizeof(Sums)) + (top_k > 0 ? (size_t)(m * sp) * 32 * 8 : 0);
}

void launch_logprob_fwd(const LogprobFwd& p, bool f32, void* workspace, hipStream_t s) {
  Args a{};
  a.p = p;
  a.c = (float)(1.4426950408889634 / p.temperature);
  a.inv_t = (float)(1.0 / p.temperature);
  a.splits = splits_of(p.m, p.V);
  a.len = split_len(p.V, a.splits);
  a.sums = (Sums*)workspace;
  a.keys = (uint64_t*)((char*)workspace + up256((size_t)(p.m * a.splits) * sizeof(Sums)));
  const dim3 grid((unsigned)(p.m * a.splits)), joins((unsigned)p.m);
#define RESQ_LP(T, K)                                                                          \
  do {                                                                                         \
    launch_timed(logprob_kernel<T, K>, grid, dim3(kThreads), 0u, s, a);                        \
    if (a.splits > 1) launch_timed(logprob_join_kernel<T, K>, joins, dim3(64), 0u, s, a);      \
  } while (0)
  if (f32) { if (p.top_k > 0) RESQ_LP(float, true); else RESQ_LP(float, false); }
  else { if (p.top_k > 0) RESQ_LP(uint16_t, true); else RESQ_LP(uint16_t, false); }
#undef RESQ_LP
}

bool logprob_bwd_supported(int64_t m, int64_t V) {
  return m <= INT32_MAX / std::max<int64_t>(1, (V + kBwdLen - 1) / kBwdLen);
}

void launch_logprob_bwd(const LogprobBwd& p, bool f32, bool out_f32, hipStream_t s) {
  const int64_t parts = (p.V + kBwdLen - 1) / kBwdLen;
  const dim3 grid((unsigned)(p.m * parts));
  const float inv_t = (float)(1.0 / p.temperature);
#define RESQ_LB(T, O) launch_timed(logprob_bwd_kernel<T, O>, grid, dim3(kBwdThreads), 0u, s, p, parts, inv_t)
  if (f32) { if (out_f32) RESQ_LB(float, float); else RESQ_LB(float, uint16_t); }
  else { if (out_f32) RESQ_LB(uint16_t, float); else RESQ_LB(uint16_t, uint16_t); }
#undef RESQ_LB
}

}  // namespace resq
