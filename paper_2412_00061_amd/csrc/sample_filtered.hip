// verify_sample_filtered: the target's token after every node, drawn from what temperature, top-k, top-p and min-p leave of its
// distribution.
//
// Tokens in the order of falling logits, equal ones by index: each filter keeps a beginning of that order, so all three together keep the
// tokens down to one threshold (logit, index).  One workgroup has a row and goes over it a few times, from memory once and from the caches
// then.  It finds the threshold by narrowing: a histogram over the distance from the largest logit, counts and weights, tells which bin holds
// the place where a filter ends; a bin of few tokens is listed and ranked, one of many is divided again - by logit and index, as one 64-bit
// number, so that equal logits divide too.  Then the kept weights are summed in vocabulary order and searched: wavefronts of a chunk,
// lanes of a wavefront, four elements of a lane.
//
// Weights are exp((z - z_max) / t) in 64 bits, relative to the largest: where they are compared with a border they are whole multiples of
// 2^-45, whose sums do not depend on their order; where the draw sums them they are doubles, in a fixed order.
#include "common.h"

namespace ctcspec {

constexpr int kFilterThreads = 1024;
constexpr int kFilterWaves = kFilterThreads / 64;
constexpr int kFilterMaxV = 1 << 18;  // so many whole weights fit 63 bits
constexpr int kFilterChunks = kFilterMaxV / 4 / kFilterThreads + 1;  // of a 16-byte group per thread, at any alignment
constexpr int kFilterBins = 1024;     // one for each thread
constexpr int kFilterList = 1024;     // tokens that are ranked one by one: one for each thread
constexpr float kFilterBinsPerNat = 32.f;

struct FilterParams {
  const float* logits;       // [B][N][V]
  const int32_t* n_nodes;    // [B]
  const float* uniforms;     // [B][N]
  const float* temperature;  // [B]
  const int32_t* top_k;      // [B] or null
  const float* top_p;        // [B] or null
  const float* min_p;        // [B] or null
  int N, V;
  int32_t* target;           // [B][N]
  int32_t* n_kept;           // [B][N] or null
  float* logp;               // [B][N] or null
};

typedef unsigned long long u64;

__device__ __forceinline__ double wave_scan_incl(double v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}
__device__ __forceinline__ u64 wave_scan_incl(u64 v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}

// 2^x, x <= 0, in 64 bits: 2^f = sum (f ln 2)^k / k! for |f| <= 1/2, whose first term left out is below 4e-16 of it
__device__ __forceinline__ double exp2_64(double x) {
  x = x > -1100.0 ? x : -1100.0;
  const double n = __builtin_rint(x), f = (x - n) * 0.693147180559945309417;
  double p = 1.0 / 479001600.0;
  p = __builtin_fma(p, f, 1.0 / 39916800.0);
  p = __builtin_fma(p, f, 1.0 / 3628800.0);
  p = __builtin_fma(p, f, 1.0 / 362880.0);
  p = __builtin_fma(p, f, 1.0 / 40320.0);
  p = __builtin_fma(p, f, 1.0 / 5040.0);
  p = __builtin_fma(p, f, 1.0 / 720.0);
  p = __builtin_fma(p, f, 1.0 / 120.0);
  p = __builtin_fma(p, f, 1.0 / 24.0);
  p = __builtin_fma(p, f, 1.0 / 6.0);
  p = __builtin_fma(p, f, 0.5);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_amdgcn_ldexp(p, (int)n);
}

// what the histogram's bins and the search among them leave behind
struct FilterShared {
  u64 weight[kFilterBins];
  u64 key[kFilterList];       // the listed tokens: larger key, earlier in the order
  u64 key_weight[kFilterList];
  unsigned int count[kFilterBins];
  double wave_total[kFilterChunks * kFilterWaves];
  u64 wave_u64[kFilterWaves];
  unsigned int wave_u32[kFilterWaves];
  u64 lo, hi;                 // the bin that holds the border: its keys
  u64 ahead_weight;           // of the tokens before the bin
  u64 threshold, mass;
  double rest, total;
  unsigned int ahead, listed, found;
  int entry, kept;
};

__global__ __launch_bounds__(kFilterThreads) void sample_filtered_kernel(FilterParams p) {
  __shared__ FilterShared sh;
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t row = (size_t)b * p.N + i;
  auto leave = [&](int token, int kept, float lp) {
    p.target[row] = token;
    if (p.n_kept) p.n_kept[row] = kept;
    if (p.logp) p.logp[row] = lp;
  };
  if (i >= p.n_nodes[b]) {
    if (tid == 0) leave(-1, 0, 0.f);
    return;
  }
  // ---- the row: it starts `lead` elements past a 16-byte boundary; group g, thread g % 1024 of chunk g / 1024, holds its elements
  // 4g - lead .. 4g - lead + 3.  What is no number, and what lies outside, counts as -infinity.
  const size_t row0 = row * p.V;
  const int lead = (int)(row0 & 3), chunks = (((lead + p.V + 3) >> 2) + kFilterThreads - 1) / kFilterThreads;
  const float* base = p.logits + (row0 - lead);
  auto load = [&](int k) __attribute__((always_inline)) -> f32x4 {
    const int e0 = 4 * (k * kFilterThreads + tid) - lead;
    f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (e0 >= 0 && e0 + 3 < p.V) {
      v = *(const f32x4*)(base + lead + e0);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (e0 + c >= 0 && e0 + c < p.V) v[c] = base[lead + e0 + c];
    }
    return v;
  };
  // each(f): f(chunk, element in the group, logit) for every logit above -infinity
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    f32x4 next = load(0);
    for (int k = 0; k < chunks; ++k) {
      const f32x4 v = next;
      if (k + 1 < chunks) next = load(k + 1);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (v[c] > -INFINITY) f(k, c, v[c]);
    }
  };
  auto index_of = [&](int k, int c) -> unsigned int { return (unsigned)(4 * (k * kFilterThreads + tid) - lead + c); };

  float mx = -INFINITY;
  constexpr int kAhead = 8;  // chunks under way: the row comes from memory here
  for (int k0 = 0; k0 < chunks; k0 += kAhead) {
    f32x4 v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = load(k0 + k);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) mx = fmaxf(fmaxf(fmaxf(mx, v[k][0]), fmaxf(v[k][1], v[k][2])), v[k][3]);  // (passes over NaN)
  }
  mx = wave_max_f32(mx);
  if (lane == 0) sh.wave_u32[wave] = __float_as_uint(mx);
  __syncthreads();
  mx = __uint_as_float(sh.wave_u32[0]);
  for (int w = 1; w < kFilterWaves; ++w) mx = fmaxf(mx, __uint_as_float(sh.wave_u32[w]));
  if (mx == -INFINITY) {  // nothing to draw
    if (tid == 0) leave(-1, 0, -INFINITY);
    return;
  }

  float t = p.temperature[b];
  const bool greedy = !(t > 0.f);
  const int top_k = greedy ? 1 : (p.top_k ? p.top_k[b] : 0);
  t = greedy ? 1.f : t;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;
  const bool by_k = top_k > 0 && top_k < p.V, by_p = !greedy && top_p < 1.f, by_min = !greedy && min_p > 0.f;
  // weights, relative to the largest; an infinite largest logit takes all
  const double per = 1.4426950408889634074 / (double)t;
  auto weight = [&](float v) -> double { return v == mx ? 1.0 : (mx == INFINITY ? 0.0 : exp2_64(((double)v - (double)mx) * per)); };
  auto whole = [&](double w) -> u64 { return (u64)(long long)(w * 35184372088832.0 + 0.5); };  // in units of 2^-45

  u64 threshold = 0ull;  // kept: key >= threshold
  u64 mass = 0ull;       // whole weights of the first top_k tokens
  // One filter after the other: stage 0 ends after top_k tokens, stage 1 with the token that brings the weights to top_p of those of stage 0.
  for (int stage = by_k ? 0 : 1; stage < (by_p ? 2 : 1); ++stage) {
    double need = 0.0;  // stage 1: the weight before a token that is kept is below this
    u64 lo = 0ull, hi = ~0ull;
    unsigned int ahead = 0u;
    u64 ahead_weight = 0ull;
    const float scale = fminf(kFilterBinsPerNat / t, 1e30f);
    for (int level = 0;; ++level) {
      int shift = 0;
      while (((hi - lo) >> shift) >= (u64)kFilterBins) ++shift;
      // the tokens with lo <= key <= hi, in bins: by distance first, then by key.  (Both grow along the order.)
      auto bin_of = [&](int k, int c, float v, u64& key) __attribute__((always_inline)) -> int {
        key = rank_key(v, index_of(k, c));
        if (level == 0) return v == mx ? 0 : (int)fminf((mx - v) * scale, (float)(kFilterBins - 1));
        return key >= lo && key <= hi ? (int)((hi - key) >> shift) : -1;
      };
      sh.weight[tid] = 0ull;
      sh.count[tid] = 0u;
      if (tid == 0) { sh.listed = 0u; sh.found = kFilterBins; }
      __syncthreads();
      each([&](int k, int c, float v) __attribute__((always_inline)) {
        u64 key;
        const int bin = bin_of(k, c, v, key);
        if (bin < 0) return;
        atomicAdd(&sh.count[bin], 1u);
        if (by_p) atomicAdd(&sh.weight[bin], whole(weight(v)));
      });
      __syncthreads();
      // -- sums over the bins, one to a thread; the first that reaches the border
      const unsigned int mine = sh.count[tid];
      const u64 mine_weight = sh.weight[tid];
      const u64 c_incl = wave_scan_incl((u64)mine, lane), w_incl = wave_scan_incl(mine_weight, lane);
      if (lane == 63) { sh.wave_u32[wave] = (unsigned int)c_incl; sh.wave_u64[wave] = w_incl; }
      __syncthreads();
      u64 c_before = ahead + c_incl - mine, w_before = ahead_weight + w_incl - mine_weight, w_all = 0ull;
      for (int w = 0; w < kFilterWaves; ++w) {
        if (w < wave) { c_before += sh.wave_u32[w]; w_before += sh.wave_u64[w]; }
        w_all += sh.wave_u64[w];
      }
      if (level == 0 && (stage == 0 || !by_k)) mass = w_all;
      if (stage == 1) need = fmax((double)top_p * (double)mass, 0.5);
      const bool reaches = stage == 0 ? c_before + mine >= (u64)top_k : (double)(w_before + mine_weight) >= need;
      if (reaches && mine > 0u) atomicMin(&sh.found, (unsigned int)tid);
      __syncthreads();
      const unsigned int found = sh.found;
      if (found == kFilterBins) break;  // (no more than top_k tokens: all of them)
      if (tid == (int)found) {
        sh.ahead = (unsigned int)c_before;
        sh.ahead_weight = w_before;
        sh.lo = ~0ull;
        sh.hi = 0ull;
      }
      const unsigned int in_bin = sh.count[found];
      __syncthreads();
      ahead = sh.ahead;
      ahead_weight = sh.ahead_weight;
      // -- its tokens: listed, or the range of their keys
      each([&](int k, int c, float v) __attribute__((always_inline)) {
        u64 key;
        if (bin_of(k, c, v, key) != (int)found) return;
        if (in_bin <= kFilterList) {
          const unsigned int at = atomicAdd(&sh.listed, 1u);
          sh.key[at] = key;
          sh.key_weight[at] = by_p ? whole(weight(v)) : 0ull;
        } else {
          atomicMin(&sh.lo, key);
          atomicMax(&sh.hi, key);
        }
      });
      __syncthreads();
      if (in_bin <= kFilterList) {
        if (tid < (int)in_bin) {
          const u64 key = sh.key[tid], w = sh.key_weight[tid];
          unsigned int rank = ahead;
          u64 before = ahead_weight;
          for (unsigned int j = 0; j < in_bin; ++j) {
            const bool earlier = sh.key[j] > key;
            rank += earlier ? 1u : 0u;
            before += earlier ? sh.key_weight[j] : 0ull;
          }
          const bool last = stage == 0 ? rank + 1 == (unsigned int)top_k : (double)before < need && (double)(before + w) >= need;
          if (last) {
            sh.threshold = key;
            sh.mass = before + w;
          }
        }
        __syncthreads();
        threshold = sh.threshold > threshold ? sh.threshold : threshold;
        if (stage == 0) mass = sh.mass;
        __syncthreads();
        break;
      }
      lo = sh.lo;
      hi = sh.hi;
      __syncthreads();
    }
  }

  // ---- what is kept, summed in vocabulary order ----------------------------------------------------------------------------------
  const float tv = threshold ? rank_key_value(threshold) : -INFINITY;
  const unsigned int ti = threshold ? rank_key_index(threshold) : 0xffffffffu;
  const double least = by_min ? (double)min_p : 0.0;
  // the weight of a kept token, -1 for others
  auto kept = [&](int k, int c, float v) __attribute__((always_inline)) -> double {
    if (!(v > -INFINITY) || v < tv || (v == tv && index_of(k, c) > ti)) return -1.0;
    const double w = weight(v);
    return w >= least || v == mx ? w : -1.0;
  };
  int mine = 0;
  {
    f32x4 next = load(0);
    for (int k = 0; k < chunks; ++k) {
      const f32x4 v = next;
      if (k + 1 < chunks) next = load(k + 1);
      double s = 0.0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const double w = kept(k, c, v[c]);
        if (w >= 0.0) { s += w; ++mine; }
      }
      double wt = 0.0;
      if (__ballot(s > 0.0)) wt = wave_scan_incl(s, lane);
      if (lane == 63) sh.wave_total[k * kFilterWaves + wave] = wt;
    }
  }
  mine = wave_sum_i32(mine);
  if (lane == 0) sh.wave_u32[wave] = (unsigned int)mine;  // (its readers above are behind a barrier)
  __syncthreads();
  const int entries = chunks * kFilterWaves, each_lane = (entries + 63) / 64;
  if (wave == 0) {
    double local = 0.0;
    for (int q = 0; q < each_lane; ++q) {
      const int j = lane * each_lane + q;
      local += j < entries ? sh.wave_total[j] : 0.0;
    }
    const double incl = wave_scan_incl(local, lane), total = __shfl(incl, 63, 64);
    const double want = fmax((double)p.uniforms[row] * total, 0.0);  // (a number below 0 counts as 0)
    double run = incl - local;
    int found = -1, last = -1;
    double rest = 0.0;
    for (int q = 0; q < each_lane; ++q) {
      const int j = lane * each_lane + q;
      const double v = j < entries ? sh.wave_total[j] : 0.0;
      if (found < 0 && v > 0.0 && run + v > want) { found = j; rest = want - run; }
      if (v > 0.0) last = j;
      run += v;
    }
    const u64 hit = __ballot(found >= 0), any = __ballot(last >= 0);
    if (hit) {
      const int src = __ffsll((long long)hit) - 1;
      found = __shfl(found, src, 64);
      rest = __shfl(rest, src, 64);
    } else {  // rounded up to the total: the last entry that has any weight
      found = __shfl(last, 63 - __clzll((long long)any), 64);
      rest = INFINITY;
    }
    if (lane == 0) {
      int n = 0;
      for (int w = 0; w < kFilterWaves; ++w) n += (int)sh.wave_u32[w];
      sh.entry = found;
      sh.rest = rest;
      sh.total = total;
      sh.kept = n;
    }
  }
  __syncthreads();
  const int chunk = sh.entry / kFilterWaves;
  if (wave != sh.entry % kFilterWaves) return;
  const f32x4 v = load(chunk);
  double w[4], s = 0.0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    w[c] = fmax(kept(chunk, c, v[c]), 0.0);
    s += w[c];
  }
  const double rest = sh.rest, incl = wave_scan_incl(s, lane);
  const u64 cross = __ballot(s > 0.0 && incl > rest), some = __ballot(s > 0.0);
  const int src = cross ? __ffsll((long long)cross) - 1 : 63 - __clzll((long long)some);
  if (lane != src) return;
  const double left = cross ? rest - (incl - s) : INFINITY;
  int pick = -1;
  double run = 0.0, chosen = 0.0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    run += w[c];
    if (pick < 0 && w[c] > 0.0 && run > left) { pick = c; chosen = w[c]; }
  }
  if (pick < 0) {  // (rounding: the last one with any weight)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (w[c] > 0.0) { pick = c; chosen = w[c]; }
  }
  leave((int)index_of(chunk, pick), sh.kept, (float)log(chosen / sh.total));
}

// code of this translation unit loaded onto the current device (context creation calls this: a stage call never
// triggers a load, so it can be the first thing a stream capture records)
hipError_t prepare_sample_filtered() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)sample_filtered_kernel);
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" int verify_sample_filtered(ctcspec_ctx* ctx, const float* logits, const int32_t* n_nodes, const float* uniforms,
                                      const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int B,
                                      int max_nodes, int V, int32_t* target_sampled, int32_t* n_kept, float* logp) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, logits && n_nodes && uniforms && temperature && target_sampled, CTCSPEC_EINVAL, "verify_sample_filtered: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && max_nodes > 0 && V > 0, CTCSPEC_EINVAL, "verify_sample_filtered: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, aligned16(logits), CTCSPEC_EINVAL, "verify_sample_filtered: logits must be 16-byte aligned");
  CTCSPEC_REQUIRE(ctx, V <= kFilterMaxV && B <= 65535, CTCSPEC_EUNSUPPORTED, "verify_sample_filtered: V <= %d, B <= 65535", kFilterMaxV);
  FilterParams p;
  p.logits = logits; p.n_nodes = n_nodes; p.uniforms = uniforms; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.N = max_nodes; p.V = V; p.target = target_sampled; p.n_kept = n_kept; p.logp = logp;
  hipLaunchKernelGGL(sample_filtered_kernel, dim3((unsigned)max_nodes, (unsigned)B), dim3(kFilterThreads), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}
