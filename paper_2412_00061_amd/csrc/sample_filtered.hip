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
// Bound: 8 rows of 32000 logits take 9 (min-p) to 20 us (top-p alone), 8 x 64 rows 22 to 44 (66 MB, 1.5 to 3 TB/s): dependent passes of
// one workgroup a row, and the exponentials in 64 bits - without a filter 7 us of 14.5 for the 32 of each thread.
//
// Weights are exp((z - z_max) / t) in 64 bits, relative to the largest: where they are compared with a border they are whole multiples of
// 2^-45, whose sums do not depend on their order; where the draw sums them they are doubles, in a fixed order.
#include <type_traits>

#include "common.h"
#include "filter_plan.h"

namespace ctcspec {

constexpr int kFilterThreads = 1024;
constexpr int kFilterWaves = kFilterThreads / 64;
constexpr int kFilterMaxV = 1 << 18;  // so many whole weights fit 63 bits
constexpr int kFilterChunks = kFilterMaxV / 4 / kFilterThreads + 1;  // of a 16-byte group per thread, at any alignment
constexpr int kFilterBins = 1024;     // one for each thread
constexpr int kFilterList = 1024;     // tokens that are ranked one by one: one for each thread
constexpr float kFilterBinsPerNat = 32.f;  // (8 rows of 128000 broad logits, top-p 0.9, us with 8 / 32 / 128: 296 / 225 / 1718)

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

// Inclusive sums over the lanes of a wavefront: within the rows of 16 lanes, then each row's end into the next and that of the second into
// the upper half - all without the LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned int dpp_shift(unsigned int v) {  // (lanes without a source: 0)
  return (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
#define CTCSPEC_SCAN_STEPS(STEP) STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)
__device__ __forceinline__ unsigned int wave_scan_incl(unsigned int v) {
#define CTCSPEC_STEP(CTRL, ROWS) v += dpp_shift<CTRL, ROWS>(v);
  CTCSPEC_SCAN_STEPS(CTCSPEC_STEP)
#undef CTCSPEC_STEP
  return v;
}
__device__ __forceinline__ u64 wave_scan_incl(u64 v) {
#define CTCSPEC_STEP(CTRL, ROWS) v += (u64)dpp_shift<CTRL, ROWS>((unsigned int)(v >> 32)) << 32 | dpp_shift<CTRL, ROWS>((unsigned int)v);
  CTCSPEC_SCAN_STEPS(CTCSPEC_STEP)
#undef CTCSPEC_STEP
  return v;
}
__device__ __forceinline__ double wave_scan_incl(double v) {
#define CTCSPEC_STEP(CTRL, ROWS)                                                                                                     \
  {                                                                                                                                  \
    const u64 u = (u64)__double_as_longlong(v);                                                                                      \
    v += __longlong_as_double((long long)((u64)dpp_shift<CTRL, ROWS>((unsigned int)(u >> 32)) << 32 | dpp_shift<CTRL, ROWS>((unsigned int)u))); \
  }
  CTCSPEC_SCAN_STEPS(CTCSPEC_STEP)
#undef CTCSPEC_STEP
  return v;
}
#undef CTCSPEC_SCAN_STEPS
__device__ __forceinline__ u64 readlane_u64(u64 v, int lane) {
  return (u64)readlane_u32((unsigned int)(v >> 32), lane) << 32 | readlane_u32((unsigned int)v, lane);
}

// p f + c.  (Left to itself the compiler keeps the polynomial's coefficients in vector registers and copies each into place first.)
__device__ __forceinline__ double fma_scalar(double p, double f, double c) {
#if defined(__HIP_DEVICE_COMPILE__)
  double r;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(p), "v"(f), "s"(c));
  return r;
#else
  return p * f + c;
#endif
}
// 2^x for x <= 0 in 64 bits: 2^f for |f| <= 1/2 by the polynomial that meets it at the ten Chebyshev nodes, within 2.1e-14 of it; its
// constant, 1.4e-14 above 1, is 1 here, so that 2^0 is.  (x less its integer is formed of the rounded x: beyond 2^53 it is 0, where the product that x
// comes from may be off from it by more than a polynomial has room for.)
__device__ __forceinline__ double exp2_64(double x) {
#pragma clang fp contract(off)
  const double n = __builtin_rint(x), f = x - n;
  double p = __builtin_fma(f, 1.0213253744950635e-07, 1.3259724569891773e-06);
  p = fma_scalar(p, f, 1.5252635829510196e-05);
  p = fma_scalar(p, f, 0.00015403433277607625);
  p = fma_scalar(p, f, 0.0013333558257234673);
  p = fma_scalar(p, f, 0.00961812919485203);
  p = fma_scalar(p, f, 0.0555041086644319);
  p = fma_scalar(p, f, 0.2402265069563423);
  p = fma_scalar(p, f, 0.6931471805599428);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_amdgcn_ldexp(p, (int)n);  // (an n beyond the integers' range is their smallest: 0)
}

// A weight up to 1 in whole units of 2^-45: the low bits of its sum with 2^7 units of 2^45.
__device__ __forceinline__ u64 whole(double w) {
  return (u64)__double_as_longlong(__builtin_fma(w, 35184372088832.0, 4503599627370496.0)) - 0x4330000000000000ull;
}

// a sum of weights
__device__ __forceinline__ u64 whole_sum(double w) { return (u64)(w * 35184372088832.0); }

// What the temperature and the filters of a sequence ask for.
struct Filters {
  int top_k;
  float t, top_p, min_p;
  bool by_k, by_p, by_min;
  __device__ __forceinline__ Filters(const FilterParams& p, int b) {
    t = p.temperature[b];
    const bool greedy = !(t > 0.f);
    top_k = greedy ? 1 : (p.top_k ? p.top_k[b] : 0);
    t = greedy ? 1.f : t;
    top_p = p.top_p ? p.top_p[b] : 1.f;
    min_p = p.min_p ? p.min_p[b] : 0.f;
    by_k = top_k > 0 && top_k < p.V;
    by_p = !greedy && top_p < 1.f;
    by_min = !greedy && min_p > 0.f;
  }
};
// Weights of logits above -infinity, relative to the largest.
struct Weights {
  double mx, per;
  __device__ __forceinline__ double operator()(float v) const {
#pragma clang fp contract(off)
    return exp2_64(((double)v - mx) * per);
  }
};
// Where the largest logit is infinite it takes all: it counts as 0, all others as -infinity.
__device__ __forceinline__ f32x4 of_infinite(f32x4 v) {
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = v[c] == INFINITY ? 0.f : -INFINITY;
  return v;
}
__device__ __forceinline__ void leave(const FilterParams& p, size_t row, int token, int kept, float lp) {
  p.target[row] = token;
  if (p.n_kept) p.n_kept[row] = kept;
  if (p.logp) p.logp[row] = lp;
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

// A row that goes by as often as it takes: of any length, with any number of tokens kept.
__device__ __forceinline__ void sample_streamed(const FilterParams& p, FilterShared& sh) {
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t row = (size_t)b * p.N + i;
  // ---- the row: it starts `lead` elements past a 16-byte boundary; group g, thread g % 1024 of chunk g / 1024, holds its elements
  // 4g - lead .. 4g - lead + 3.  What is no number, and what lies outside, counts as -infinity.
  const size_t row0 = row * p.V;
  const int lead = (int)(row0 & 3), chunks = (((lead + p.V + 3) >> 2) + kFilterThreads - 1) / kFilterThreads;
  const float* base = p.logits + (row0 - lead);
  bool infinite = false;
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
    return infinite ? of_infinite(v) : v;
  };
  // each(f): f(chunk, element in the group, logit) for every logit above -infinity
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    f32x4 next = load(0);
    for (int k = 0; k < chunks; ++k) {
      const f32x4 v = next;
      if (k + 1 < chunks) next = load(k + 1);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (v[c] > -INFINITY) f(k, c, v[c]);
        __builtin_amdgcn_sched_barrier(0);
      }
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
    if (tid == 0) leave(p, row, -1, 0, -INFINITY);
    return;
  }
  if (mx == INFINITY) {
    infinite = true;
    mx = 0.f;
  }

  const Filters want(p, b);
  const int top_k = want.top_k;
  const bool by_k = want.by_k, by_p = want.by_p;
  const Weights weight = {(double)mx, 1.4426950408889634074 / (double)want.t};

  u64 threshold = 0ull;  // kept: key >= threshold
  u64 mass = 0ull;       // whole weights of the first top_k tokens
  // One filter after the other: stage 0 ends after top_k tokens, stage 1 with the token that brings the weights to top_p of those of stage 0.
  for (int stage = by_k ? 0 : 1; stage < (by_p ? 2 : 1); ++stage) {
    double need = 0.0;  // stage 1: the weight before a token that is kept is below this
    u64 lo = 0ull, hi = ~0ull;
    unsigned int ahead = 0u;
    u64 ahead_weight = 0ull;
    const float scale = fminf(kFilterBinsPerNat / want.t, 1e30f);
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
      const u64 c_incl = wave_scan_incl((u64)mine), w_incl = wave_scan_incl(mine_weight);
      if (lane == 63) { sh.wave_u32[wave] = (unsigned int)c_incl; sh.wave_u64[wave] = w_incl; }
      __syncthreads();
      u64 c_before = ahead + c_incl - mine, w_before = ahead_weight + w_incl - mine_weight, w_all = 0ull;
      for (int w = 0; w < kFilterWaves; ++w) {
        if (w < wave) { c_before += sh.wave_u32[w]; w_before += sh.wave_u64[w]; }
        w_all += sh.wave_u64[w];
      }
      if (level == 0 && (stage == 0 || !by_k)) mass = w_all;
      if (stage == 1) need = fmax((double)want.top_p * (double)mass, 0.5);
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
  const double least = want.by_min ? (double)want.min_p : 0.0;
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
      if (__ballot(s > 0.0)) wt = wave_scan_incl(s);
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
    const double incl = wave_scan_incl(local), total = __shfl(incl, 63, 64);
    const double target = fmax((double)p.uniforms[row] * total, 0.0);  // (a number below 0 counts as 0)
    double run = incl - local;
    int found = -1, last = -1;
    double rest = 0.0;
    for (int q = 0; q < each_lane; ++q) {
      const int j = lane * each_lane + q;
      const double v = j < entries ? sh.wave_total[j] : 0.0;
      if (found < 0 && v > 0.0 && run + v > target) { found = j; rest = target - run; }
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
  const double rest = sh.rest, incl = wave_scan_incl(s);
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
  leave(p, row, (int)index_of(chunk, pick), sh.kept, (float)log(chosen / sh.total));
}

// ---- rows of which few tokens may be kept ---------------------------------------------------------------------------------------------
constexpr int kFilterCandidates = 14336;  // what the LDS holds (half as many are no faster where they suffice)
constexpr int kFilterMembers = 512;     // of a bin, ranked one by one
// Parts of a thread's logits, the largest of each of which helps to choose the candidates.  (8 rows of 32000, us with 2 / 4 / 8: top-k 50
// 11.7 / 11.9 / 12.3, top-k 1000 14.8 / 14.8 / 15.2, top-p 0.9 of broad rows 28.7 / 31.2 / 24.8; of 128000 244 / 225 / 228.)
constexpr int kFilterParts = 4;

struct ListShared {
  unsigned int count[kFilterBins];
  u64 bin_weight[kFilterBins];
  unsigned int part_count[kFilterBins];
  float logit[kFilterCandidates];
  unsigned int index[kFilterCandidates];
  u64 key[kFilterMembers], key_weight[kFilterMembers];
  // a word for each wavefront: every one of them is written once (block_sum's in turn)
  double plain_sum[kFilterWaves];
  u64 bin_sum[kFilterWaves], draw_sum[kFilterWaves], block_sum[2][kFilterWaves];
  float largest[kFilterWaves], lowest[kFilterWaves];
  unsigned int part_sum[kFilterWaves], count_sum[kFilterWaves], kept[kFilterWaves];
  u64 ahead_weight, threshold, mass;
  unsigned int candidates, ahead, found, members, certain;
};

__device__ __forceinline__ double dpp_f64(double v, int which) {
  const u64 u = (u64)__double_as_longlong(v);
  unsigned int lo = (unsigned int)u, hi = (unsigned int)(u >> 32);
  switch (which) {
    case 1: lo = dpp_row_ror<1>(lo); hi = dpp_row_ror<1>(hi); break;
    case 2: lo = dpp_row_ror<2>(lo); hi = dpp_row_ror<2>(hi); break;
    case 4: lo = dpp_row_ror<4>(lo); hi = dpp_row_ror<4>(hi); break;
    default: lo = dpp_row_ror<8>(lo); hi = dpp_row_ror<8>(hi); break;
  }
  return __longlong_as_double((long long)((u64)hi << 32 | lo));
}
__device__ __forceinline__ double readlane_f64(double v, int lane) {
  const u64 u = (u64)__double_as_longlong(v);
  return __longlong_as_double((long long)((u64)readlane_u32((unsigned int)(u >> 32), lane) << 32 | readlane_u32((unsigned int)u, lane)));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v += dpp_f64(v, 1);
  v += dpp_f64(v, 2);
  v += dpp_f64(v, 4);
  v += dpp_f64(v, 8);
  return (readlane_f64(v, 0) + readlane_f64(v, 16)) + (readlane_f64(v, 32) + readlane_f64(v, 48));
}

// Sums over the threads before this one, and over all: of counts, and of whole weights.  waves: a word for each wavefront; nothing else may
// be under way with it.  (One barrier: whoever writes to it next has one between.)
__device__ __forceinline__ void sums_before(unsigned int own, unsigned int& before, unsigned int& all, unsigned int* waves, int lane, int wave) {
  static_assert(kFilterWaves == 16, "a row of lanes");
  const unsigned int incl = wave_scan_incl(own);
  if (lane == 63) waves[wave] = incl;
  __syncthreads();
  const unsigned int of_waves = wave_scan_incl(waves[lane & 15]);  // (the first row's are those of the wavefronts)
  all = readlane_u32(of_waves, 15);
  before = incl - own + (wave > 0 ? readlane_u32(of_waves, wave > 0 ? wave - 1 : 0) : 0u);
}
__device__ __forceinline__ void sums_before(u64 own, u64& before, u64& all, u64* waves, int lane, int wave) {
  const u64 incl = wave_scan_incl(own);
  if (lane == 63) waves[wave] = incl;
  __syncthreads();
  const u64 of_waves = wave_scan_incl(waves[lane & 15]);
  all = readlane_u64(of_waves, 15);
  before = incl - own + (wave > 0 ? readlane_u64(of_waves, wave > 0 ? wave - 1 : 0) : 0ull);
}

// Top-p's share of all tokens is first taken of a sum in float: exponents whole in 64 bits, their fractions off by 2^-25, the exponential by
// 2^-23, sums of four by 2^-23, then 64 bits again; together below 2.7e-7 of the sum, 2^-21 = 4.8e-7.  Where the tokens that top-p keeps are
// not the same for both ends of that, the sum is formed in 64 bits.
constexpr double kFilterRough = 4.76837158203125e-07;

// The tokens that may be kept are few, mostly, and a bound below them all is easily had: among the first top_k tokens' logits is none below
// the top_k-th of any top_k and more logits - such as the largest logits of the threads' parts of the row -, min-p is a distance from the
// largest logit, and for top-p a guess is good whose tokens weigh enough, or else a lower one.  The tokens above it are listed, and all the
// rest is done on the list; where it would be too long, or too many tokens share the bin where a filter ends, the row is done again by
// sample_streamed.
//
// NV: 16-byte groups of the row that a thread keeps in registers; 0: any number, fetched again for every pass.  Returns whether the row
// is still to be done.
template <int NV>
__device__ __forceinline__ bool sample_listed(const FilterParams& p, ListShared& sh) {
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t row = (size_t)b * p.N + i;
  // Each wavefront has a stretch of the row, 64 groups at a time.  (The row starts `lead` elements past a 16-byte boundary; group g holds
  // its elements 4g - lead .. 4g - lead + 3; what is no number, and what lies outside, counts as -infinity.)
  const size_t row0 = row * p.V;
  const int lead = (int)(row0 & 3), nv = ((lead + p.V + 3) / 4 + kFilterThreads - 1) / kFilterThreads;
  const float* base = p.logits + (row0 - lead);
  const int first = 4 * (wave * nv * 64 + lane) - lead;  // this lane's first element; its j-th group is 256 j behind
  bool infinite = false;
  auto load = [&](int j) __attribute__((always_inline)) -> f32x4 {
    const int e0 = first + 256 * j;
    f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (j < nv) {
      if (e0 >= 0 && e0 + 3 < p.V) {
        v = *(const f32x4*)(base + lead + e0);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (e0 + c >= 0 && e0 + c < p.V) v[c] = base[lead + e0 + c];
      }
    }
    return infinite ? of_infinite(v) : v;
  };
  f32x4 x[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) x[j] = load(j);
  }
  // f(j, group) for this lane's groups, in their order
  auto groups = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (NV > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (j < nv) f(j, x[j]);
        __builtin_amdgcn_sched_barrier(0);  // (group by group: what all of them need at once does not fit the registers)
      }
    } else {
      f32x4 next = load(0);
      for (int j = 0; j < nv; ++j) {
        const f32x4 v = next;
        next = load(j + 1);
        f(j, v);
      }
    }
  };
  const Filters want(p, b);
  const float uniform_number = p.uniforms[row];
  sh.count[tid] = 0u;
  sh.part_count[tid] = 0u;
  sh.bin_weight[tid] = 0ull;
  if (tid == 0) { sh.candidates = sh.members = 0u; sh.found = kFilterBins; }
  float part[kFilterParts], mx = -INFINITY;  // (the largest of numbers: fmaxf passes over NaN)
  if constexpr (NV > 0) {
#pragma unroll
    for (int q = 0; q < kFilterParts; ++q) {
      part[q] = -INFINITY;
#pragma unroll
      for (int j = q * NV / kFilterParts; j < (q + 1) * NV / kFilterParts; ++j)
        part[q] = fmaxf(fmaxf(fmaxf(part[q], x[j][0]), fmaxf(x[j][1], x[j][2])), x[j][3]);
    }
  } else {
    constexpr int kAhead = 8;  // groups under way: the row comes from memory here
#pragma unroll
    for (int q = 0; q < kFilterParts; ++q) part[q] = -INFINITY;
    for (int j0 = 0; j0 < nv; j0 += kAhead) {
      f32x4 v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) v[j] = load(j0 + j);
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        part[j % kFilterParts] = fmaxf(fmaxf(fmaxf(part[j % kFilterParts], v[j][0]), fmaxf(v[j][1], v[j][2])), v[j][3]);
    }
  }
  float low = INFINITY;
#pragma unroll
  for (int q = 0; q < kFilterParts; ++q) {
    mx = fmaxf(mx, part[q]);
    low = part[q] > -INFINITY ? fminf(low, part[q]) : low;
  }
  mx = wave_max_f32(mx);
  low = -wave_max_f32(-low);
  if (lane == 0) { sh.largest[wave] = mx; sh.lowest[wave] = low; }
  __syncthreads();  // (and the bins are cleared)
  mx = wave_max_f32(sh.largest[lane & 15]);
  low = -wave_max_f32(-sh.lowest[lane & 15]);
  if (mx == -INFINITY) {  // nothing to draw
    if (tid == 0) leave(p, row, -1, 0, -INFINITY);
    return false;
  }
  if (mx == INFINITY) {
    infinite = true;
    mx = 0.f;
    if constexpr (NV > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) x[j] = of_infinite(x[j]);
    }
#pragma unroll
    for (int q = 0; q < kFilterParts; ++q) part[q] = part[q] == INFINITY ? 0.f : -INFINITY;
    low = 0.f;
  }
  const Weights weight = {(double)mx, 1.4426950408889634074 / (double)want.t};

  if (!want.by_k && !want.by_p && !want.by_min) {
    // ---- every token: sums of the lanes, of the wavefronts, then the search in the opposite order -------------------------------------
    double s = 0.0;
    int n = 0;
    groups([&](int, const f32x4& v) __attribute__((always_inline)) {
      double w[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool there = v[c] > -INFINITY;
        const double y = weight(v[c]);
        w[c] = there ? y : 0.0;
        n += there;
      }
      s += ((w[0] + w[1]) + w[2]) + w[3];
    });
    s = wave_sum_f64(s);
    n = wave_sum_i32(n);
    if (lane == 0) { sh.plain_sum[wave] = s; sh.kept[wave] = (unsigned)n; }
    __syncthreads();
    double total = 0.0;
    int kept = 0, last = 0, at = -1;
#pragma unroll 4
    for (int w = 0; w < kFilterWaves; ++w) {
      total += sh.plain_sum[w];
      kept += (int)sh.kept[w];
      last = sh.plain_sum[w] > 0.0 ? w : last;
    }
    const double target = fmax((double)uniform_number * total, 0.0);  // (a number below 0 counts as 0)
    double run = 0.0, rest = INFINITY;
#pragma unroll 4
    for (int w = 0; w < kFilterWaves; ++w) {
      const double v = sh.plain_sum[w];
      if (at < 0 && v > 0.0 && run + v > target) { at = w; rest = target - run; }
      run += v;
    }
    if (wave != (at < 0 ? last : at)) return false;  // (rounded up to the total: the last one that has any weight)
    // group after group of 64 lanes; then the lanes of the one that reaches it, then its four elements
    double before = 0.0, chosen = 0.0;
    int pick = -1;
    bool done = false;
    groups([&](int j, const f32x4& v) __attribute__((always_inline)) {
      if (done) return;
      double w[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const double y = weight(v[c]);
        w[c] = v[c] > -INFINITY ? y : 0.0;
      }
      const double mine = ((w[0] + w[1]) + w[2]) + w[3];
      const double incl = before + wave_scan_incl(mine);
      const u64 cross = __ballot(mine > 0.0 && incl > rest), some = __ballot(mine > 0.0);
      if (some) {  // the token if the row ended here: the last one with any weight; the one that is looked for, where it is
        const int src = cross ? __ffsll((long long)cross) - 1 : 63 - __clzll((long long)some);
        double sum = incl - mine, best = 0.0;
        int c_at = 0;
        bool have = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          sum += w[c];
          if (w[c] > 0.0 && !have) { c_at = c; best = w[c]; have = cross && sum > rest; }
        }
        pick = __shfl(first + 256 * j + c_at, src, 64);
        chosen = __shfl(best, src, 64);
        done = cross != 0ull;
      }
      before = readlane_f64(incl, 63);
    });
    if (lane == 0) leave(p, row, pick, kept, (float)log(chosen / total));
    return false;
  }

  // ---- the bound: every candidate's logit is at least `bound` -----------------------------------------------------------------------------
  auto bin_of = [&](float v, float scale) __attribute__((always_inline)) -> int { return (int)fminf((mx - v) * scale, (float)(kFilterBins - 1)); };
  // the parts' largest logits, in bins of the distance up to the smallest (but of no more than 64 in all: masked logits may be far away)
  unsigned int parts_here = 0u, parts_before = 0u, parts = 0u;
  const float part_reach = fminf(mx - low, 64.f), part_scale = part_reach > 0.f ? (float)(kFilterBins - 1) / part_reach : 0.f;
  if (want.by_k || want.by_p) {
#pragma unroll
    for (int q = 0; q < kFilterParts; ++q)
      if (part[q] > -INFINITY) atomicAdd(&sh.part_count[bin_of(part[q], part_scale)], 1u);
    __syncthreads();
    parts_here = sh.part_count[tid];
    sums_before(parts_here, parts_before, parts, sh.part_sum, lane, wave);
  }
  // a bound that at least `wanted` of them lie above
  auto below_parts = [&](unsigned int wanted) __attribute__((always_inline)) -> float {
    if (tid == 0) sh.found = kFilterBins;
    __syncthreads();
    if (parts_before < wanted && parts_before + parts_here >= wanted) sh.found = tid;
    __syncthreads();
    const unsigned int found = sh.found;
    __syncthreads();
    // (one bin further: what rounding moves across a bin's end)
    return found + 2 < (unsigned)kFilterBins && part_scale > 0.f ? mx - (float)(found + 2) / part_scale : -INFINITY;
  };
  // The candidates, in any order: those with from <= logit, and for more of them logit < to.  Marked group by group, then counted and written a batch of groups at a
  // time, so that a wavefront asks for its places once a batch.
  constexpr int kBatch = NV > 0 ? NV : 8;
  auto list_batch = [&](int j0, const f32x4 (&v)[kBatch], float from, float to, auto&& also, auto more) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
    unsigned int marks = 0u;  // bit 4 j + c
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        bool in = v[j][c] >= from;
        if constexpr (MORE) in = in && v[j][c] < to;
        marks |= in ? 1u << (4 * j + c) : 0u;
      }
      if (j0 + j < nv) also(v[j]);
      __builtin_amdgcn_sched_barrier(0);  // (group by group: what all of them need at once does not fit the registers)
    }
    if (__ballot(marks != 0u) == 0ull) return;
    const unsigned int incl = wave_scan_incl((unsigned)__popc(marks));
    unsigned int place = 0u;
    if (lane == 63) place = atomicAdd(&sh.candidates, incl);
    place = readlane_u32(place, 63) + incl - (unsigned)__popc(marks);
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if ((marks >> (4 * j)) & 15u) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if ((marks >> (4 * j + c)) & 1u) {
            if (place < (unsigned)kFilterCandidates) {
              sh.logit[place] = v[j][c];
              sh.index[place] = (unsigned)(first + 256 * (j0 + j) + c);
            }
            ++place;
          }
      }
  };
  auto list = [&](float from, float to, auto&& also, auto more) __attribute__((always_inline)) {
    from = fmaxf(from, -3.402823466e38f);  // (no -infinity)
    if constexpr (NV > 0) {
      list_batch(0, x, from, to, also, more);
    } else {
      for (int j0 = 0; j0 < nv; j0 += kBatch) {
        f32x4 v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) v[j] = load(j0 + j);
        list_batch(j0, v, from, to, also, more);
      }
    }
    __syncthreads();
  };
  const bool of_all = want.by_p && !want.by_k;  // top-p's share is of all tokens
  float bound = want.by_k ? below_parts((unsigned)want.top_k) : (want.by_p ? below_parts(filter_parts_above(parts, 0)) : -INFINITY);
  float distance = -INFINITY;  // every token that min-p keeps is above this
  if (want.by_min && !(want.by_k && want.by_p)) {  // (top-p's share is of all top-k tokens)
    const float nats = -__logf(fminf(fmaxf(want.min_p, 1e-37f), 1.f));
    if (want.min_p >= 1e-37f) distance = mx - (nats * 1.0001f + 1e-3f) * want.t - fabsf(mx) * 1e-6f;
  }
  bound = fmaxf(bound, distance);
  u64 mass = 0ull;
  double rough = 0.0;
  list(bound, INFINITY, [&](const f32x4& v) __attribute__((always_inline)) {
    if (of_all) {
      float w[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const double x = fmax(((double)v[c] - weight.mx) * weight.per, -1000.0), n = __builtin_rint(x);  // (what is no number: a weight of 0)
        w[c] = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((float)(x - n)), (int)n);
      }
      rough += (double)((w[0] + w[1]) + (w[2] + w[3]));
    }
  }, std::false_type{});
  unsigned int listed = sh.candidates;
  int turn = 0;
  auto block_sum = [&](u64 v) __attribute__((always_inline)) -> u64 {
    u64 before, all;
    sums_before(v, before, all, sh.block_sum[turn], lane, wave);
    turn ^= 1;
    return all;
  };
  if (of_all) {
    // as many candidates as it takes to weigh enough: a quarter of the parts, three quarters, nearly all
    mass = block_sum(whole_sum(rough));
    const double enough = (double)want.top_p * (double)mass * (1.0 + kFilterRough);
    u64 weighs = 0ull;
    unsigned int weighed = 0u;
    for (int round = 1;; ++round) {
      if (listed > (unsigned)kFilterCandidates) return true;
      u64 more = 0ull;
      for (unsigned int e = weighed + tid; e < listed; e += kFilterThreads) more += whole(weight(sh.logit[e]));
      weighs += block_sum(more);
      weighed = listed;
      if ((double)weighs >= enough || bound == -INFINITY || bound == distance) break;
      const float upto = bound;
      bound = filter_next_bound(upto, round < kFilterPartRounds ? below_parts(filter_parts_above(parts, round)) : -INFINITY, distance);
      list(bound, upto, [](const f32x4&) {}, std::true_type{});
      listed = sh.candidates;
    }
  }
  if (listed > (unsigned)kFilterCandidates) return true;
  const int n = (int)listed;
  // ---- their weights, and bins of them -----------------------------------------------------------------------------------------------
  const float reach = bound > -INFINITY ? mx - bound : fminf(2.f * (mx - low), 64.f);
  const float scale = reach > 0.f && reach < INFINITY ? (float)(kFilterBins - 1) / reach : 0.f;
  auto key_at = [&](int e) __attribute__((always_inline)) -> u64 { return rank_key(sh.logit[e], sh.index[e]); };
  u64 threshold = 0ull;  // kept: key >= threshold
  if (want.by_k || want.by_p) {
    for (int e = tid; e < n; e += kFilterThreads) {
      const float v = sh.logit[e];
      const int bin = bin_of(v, scale);
      atomicAdd(&sh.count[bin], 1u);
      if (want.by_p) atomicAdd(&sh.bin_weight[bin], whole(weight(v)));
    }
    __syncthreads();
    const unsigned int own = sh.count[tid];
    const u64 own_weight = sh.bin_weight[tid];
    unsigned int before = 0u, all = 0u;
    u64 before_weight = 0ull, all_weight = 0ull;
    if (want.by_k) sums_before(own, before, all, sh.count_sum, lane, wave);
    if (want.by_p) sums_before(own_weight, before_weight, all_weight, sh.bin_sum, lane, wave);
    // f(key, weight, tokens of the bin before it, their weight) for the tokens of a bin
    auto rank = [&](unsigned int bin, auto&& f) __attribute__((always_inline)) {
      for (int e = tid; e < n; e += kFilterThreads)
        if ((unsigned)bin_of(sh.logit[e], scale) == bin) {
          const unsigned int to = atomicAdd(&sh.members, 1u);
          sh.key[to] = key_at(e);
          sh.key_weight[to] = whole(weight(sh.logit[e]));
        }
      __syncthreads();
      const unsigned int members = sh.members;
      if (tid < (int)members) {
        const u64 key = sh.key[tid];
        unsigned int ahead = 0u;
        u64 ahead_weight = 0ull;
        for (unsigned int m = 0; m < members; ++m) {
          const bool earlier = sh.key[m] > key;
          ahead += earlier ? 1u : 0u;
          ahead_weight += earlier ? sh.key_weight[m] : 0ull;
        }
        f(key, sh.key_weight[tid], ahead, ahead_weight);
      }
      __syncthreads();
    };
    unsigned int last_bin = kFilterBins;  // where top-k ends
    if (want.by_k && all >= (unsigned)want.top_k) {
      if (before < (unsigned)want.top_k && before + own >= (unsigned)want.top_k) {
        sh.found = tid;
        sh.ahead = before;
        sh.ahead_weight = before_weight;
        sh.members = 0u;
      }
      __syncthreads();
      last_bin = sh.found;
      const unsigned int ahead = sh.ahead;
      const u64 base_weight = sh.ahead_weight;
      if (sh.count[last_bin] > kFilterMembers) return true;
      rank(last_bin, [&](u64 key, u64 w, unsigned int a, u64 aw) __attribute__((always_inline)) {
        if (ahead + a + 1 == (unsigned)want.top_k) {
          sh.threshold = key;
          sh.mass = base_weight + aw + w;
        }
      });
      threshold = sh.threshold;
      all_weight = sh.mass;
      __syncthreads();
    } else if (want.by_k && bound > distance) {
      return true;  // (a candidate lost to rounding)
    }
    if (want.by_p) {
      if (want.by_k) mass = all_weight;
      for (double slack = of_all ? kFilterRough : 0.0;;) {
        // the weight before a token that is kept is below the share, which lies between these two
        const double share = (double)want.top_p * (double)mass, need = fmax(share * (1.0 + slack), 0.5), least_need = fmax(share * (1.0 - slack), 0.5);
        bool certain = (double)all_weight < least_need;
        if ((double)all_weight >= need) {
          // (in the bin where top-k ends its last tokens bring the weights there, if none before did)
          const bool here = (double)before_weight < need && (tid < (int)last_bin ? (double)(before_weight + own_weight) >= need : tid == (int)last_bin);
          if (here) {
            sh.found = tid;
            sh.ahead_weight = before_weight;
            sh.members = 0u;
          }
          __syncthreads();
          const unsigned int bin = sh.found;
          const u64 base_weight = sh.ahead_weight;
          if (sh.count[bin] > kFilterMembers) return true;
          rank(bin, [&](u64 key, u64 w, unsigned int, u64 aw) __attribute__((always_inline)) {
            if ((double)(base_weight + aw) < need && (double)(base_weight + aw + w) >= need) {
              sh.threshold = key;
              sh.certain = (double)(base_weight + aw) < least_need ? 1u : 0u;
            }
          });
          threshold = sh.threshold;
          certain = sh.certain != 0u;
        }  // (else all candidates: the tokens that min-p keeps, or all)
        if (certain || slack == 0.0) break;
        mass = 0ull;
        for (int j = 0; j < nv; ++j) {  // (fetched again: kept until here, the row would not fit the registers)
          const f32x4 v = load(j);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const u64 y = whole(weight(v[c]));
            mass += v[c] > -INFINITY ? y : 0ull;
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        mass = block_sum(mass);
        slack = 0.0;
      }
    }
    __syncthreads();
  }
  // ---- the draw: weights by stretches of the vocabulary, then the tokens of the one that the number falls into ------------------------------
  sh.bin_weight[tid] = 0ull;
  if (tid == 0) sh.members = 0u;
  int shift = 0;
  while ((p.V - 1) >> shift >= kFilterBins) ++shift;
  __syncthreads();
  const double least = want.by_min ? (double)want.min_p : 0.0;
  // (a whole weight of a kept token is at least 1: the number 0 takes the first that has any)
  constexpr u64 none = ~0ull;
  auto drawn_weight = [&](int e, float v, double y) __attribute__((always_inline)) -> u64 {
    if (key_at(e) < threshold || !(y >= least || v == mx)) return none;
    const u64 w = whole(y);
    return y == 0.0 ? 0ull : (w > 0ull ? w : 1ull);
  };
  int kept = 0;
  for (int e = tid; e < n; e += kFilterThreads) {
    const float v = sh.logit[e];
    const double y = weight(v);
    const u64 w = drawn_weight(e, v, y);
    kept += w != none;
    if (w != none && w > 0ull) atomicAdd(&sh.bin_weight[sh.index[e] >> shift], w);
  }
  kept = wave_sum_i32(kept);
  if (lane == 0) sh.kept[wave] = (unsigned)kept;
  __syncthreads();
  const u64 own = sh.bin_weight[tid];
  u64 before, total;
  sums_before(own, before, total, sh.draw_sum, lane, wave);
  const double wanted = fmax((double)uniform_number * (double)total, 0.0);  // (a number below 0 counts as 0)
  u64 target = total - 1;
  if (wanted < (double)total && (u64)wanted < target) target = (u64)wanted;
  if (before <= target && before + own > target) {
    sh.found = tid;
    sh.ahead_weight = before;
  }
  __syncthreads();
  const unsigned int stretch = sh.found;
  for (int e = tid; e < n; e += kFilterThreads)
    if (sh.index[e] >> shift == stretch) {
      const float v = sh.logit[e];
      const u64 w = drawn_weight(e, v, weight(v));
      if (w == none || w == 0ull) continue;
      const unsigned int to = atomicAdd(&sh.members, 1u);
      sh.key[to] = (u64)sh.index[e] << 32 | __float_as_uint(v);
      sh.key_weight[to] = w;
    }
  __syncthreads();
  const unsigned int members = sh.members;
  if (tid < (int)members) {
    const u64 key = sh.key[tid];
    u64 ahead = sh.ahead_weight;
    for (unsigned int m = 0; m < members; ++m) ahead += sh.key[m] < key ? sh.key_weight[m] : 0ull;
    if (ahead <= target && ahead + sh.key_weight[tid] > target) {
      int n_kept = 0;
#pragma unroll 4
      for (int w = 0; w < kFilterWaves; ++w) n_kept += (int)sh.kept[w];
      leave(p, row, (int)(key >> 32), n_kept, (float)log(weight(__uint_as_float((unsigned)key)) / ((double)total * 0x1p-45)));
    }
  }
  return false;
}

template <int NV>
__global__ __launch_bounds__(kFilterThreads) void sample_filtered_kernel(FilterParams p) {
  __shared__ union { ListShared list; FilterShared filter; } shared;
  if ((int)blockIdx.x >= p.n_nodes[blockIdx.y]) {
    if (threadIdx.x == 0) leave(p, (size_t)blockIdx.y * p.N + blockIdx.x, -1, 0, 0.f);
    return;
  }
  if (!sample_listed<NV>(p, shared.list)) return;
  __syncthreads();  // (all threads come here or none)
  sample_streamed(p, shared.filter);
}

// code of this translation unit loaded onto the current device (context creation calls this: a stage call never
// triggers a load, so it can be the first thing a stream capture records)
hipError_t prepare_sample_filtered() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)sample_filtered_kernel<0>);
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
  CTCSPEC_REQUIRE(ctx, V <= kFilterMaxV && B <= 65535 && max_nodes < 1 << 22, CTCSPEC_EUNSUPPORTED,
                  "verify_sample_filtered: V <= %d, B <= 65535, max_nodes < 2^22", kFilterMaxV);
  FilterParams p;
  p.logits = logits; p.n_nodes = n_nodes; p.uniforms = uniforms; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
  p.N = max_nodes; p.V = V; p.target = target_sampled; p.n_kept = n_kept; p.logp = logp;
  const dim3 grid((unsigned)max_nodes, (unsigned)B), block(kFilterThreads);
  hipStream_t st = ctx->stream;
  const int nv = ((V + 6) / 4 + kFilterThreads - 1) / kFilterThreads;  // groups of a row that starts 3 past a boundary
  // (rows of 32000 in registers / fetched again for every pass, us for 8: top-k 50 11.9 / 14.6, no filter 14.5 / 18.7)
  if (nv <= 2) hipLaunchKernelGGL(sample_filtered_kernel<2>, grid, block, 0, st, p);
  else if (nv <= 8) hipLaunchKernelGGL(sample_filtered_kernel<8>, grid, block, 0, st, p);
  else hipLaunchKernelGGL(sample_filtered_kernel<0>, grid, block, 0, st, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}
