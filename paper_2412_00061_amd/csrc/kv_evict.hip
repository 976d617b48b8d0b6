// kv_evict: the cache of a layer brought down to `budget` rows per sequence and key head - the first positions, the last ones and,
// of the others, those that have gathered the most attention weight.
//
// Keys carry their position in themselves and attention does not ask for an order, so nothing has to move but the kept rows
// behind the budget, into the places of the rows that go: the j-th such row into the j-th such place.  Sources lie behind the budget and
// places before it, so the moves need no order among each other, and the call reads and writes only what moves.
//   * kv_evict_select_kernel - one workgroup per (sequence, key head): the budget-th largest weight by a radix search, then
//                              which row of the old cache every row of the new one is
//   * kv_evict_move_kernel   - the moves, and the kept rows' weights and positions
#include "common.h"

namespace ctcspec {

struct KvEvictParams {
  unsigned char* k_cache;
  unsigned char* v_cache;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const float* weight;      // [B][H_kv][kv_cap]
  const int32_t* pos;       // [B][H_kv][kv_cap] or null
  const int32_t* next_pos;  // [B] or null
  int32_t* kept;            // [B][H_kv][budget]
  float* weight_out;        // [B][H_kv][kv_cap]
  int32_t* pos_out;         // [B][H_kv][kv_cap] or null
  int32_t* ctx_len_out;     // [B]
  int kv_cap, H_kv, budget, sink, recent;
  int row_bytes, elem_bytes;
};

constexpr int kEvWaves = 16, kEvThreads = 64 * kEvWaves;
constexpr int kEvBits = 11, kEvBins = 1 << kEvBits;  // three digits: the upper 11 bits, the next 11, the last 10
constexpr int kEvList = 8192;                        // moved rows per round

// Order of the rows: larger weight first, then smaller index; rows that stay in any case before all others; a weight that is not
// a number behind all others.
__device__ __forceinline__ unsigned int evict_key(const KvEvictParams& p, const float* w, const int32_t* pos, int j, int fresh) {
  const float v = w[j];
  unsigned int key = v != v ? 0u : float_to_ordered(v);
  if (pos) {
    const int at = pos[j];
    key = at < p.sink || at >= fresh ? 0xffffffffu : key;
  }
  return key;
}

__global__ __launch_bounds__(kEvThreads) void kv_evict_select_kernel(KvEvictParams p) {
  __shared__ unsigned int hist[kEvBins];
  __shared__ int list[kEvList];
  __shared__ int wsum[2][kEvWaves];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kh = blockIdx.x, b = blockIdx.y;
  int L = __builtin_amdgcn_readfirstlane(p.ctx_len[b]);
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int n = L < p.budget ? L : p.budget;
  const size_t head = (size_t)b * p.H_kv + kh;
  int32_t* kept = p.kept + head * p.budget;
  if (kh == 0 && tid == 0) p.ctx_len_out[b] = n;
  for (int j = n + tid; j < p.budget; j += kEvThreads) kept[j] = -1;
  if (L <= p.budget) {
    for (int j = tid; j < n; j += kEvThreads) kept[j] = j;
    return;
  }
  const float* w = p.weight + head * p.kv_cap;
  const int32_t* pos = p.pos ? p.pos + head * p.kv_cap : nullptr;
  const int fresh = p.recent > 0 ? p.next_pos[b] - p.recent : 0x7fffffff;
  // every wavefront has a range of rows of its own, so that ranks follow from counts
  const int range = (L + kEvThreads - 1) / kEvThreads * 64, j0 = wave * range, j1 = j0 + range < L ? j0 + range : L;

  // ---- the n-th largest key, digit by digit: `above` keys are larger than all that begin with `prefix`, `want` of those stay --------
  unsigned int prefix = 0u;
  int want = n;
  for (int d = 0; d < 3; ++d) {
    const int shift = d == 0 ? 21 : (d == 1 ? 10 : 0), bits = d == 2 ? 10 : 11;
    for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0u;
    __syncthreads();
    for (int j = j0 + lane; j < j1; j += 64) {
      const unsigned int key = evict_key(p, w, pos, j, fresh);
      if (d == 0 || (key >> (shift + bits)) == prefix) {
        const unsigned int bin = (key >> shift) & ((1u << bits) - 1u);
        atomicAdd(&hist[bin], 1u);
      }
    }
    __syncthreads();
    // thread t: bins 2 t' and 2 t' + 1 from the top; how many keys lie in the bins above
    const int hi = kEvBins - 1 - 2 * tid;
    const int c1 = (int)hist[hi], c0 = (int)hist[hi - 1];
    int sum = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int other = __shfl_up(sum, o, 64);
      if (lane >= o) sum += other;
    }
    if (lane == 63) wsum[0][wave] = sum;
    __syncthreads();
    int above = sum - c0 - c1;
    for (int v = 0; v < wave; ++v) above += wsum[0][v];
    if (above < want && want <= above + c1) { found[0] = hi; found[1] = above; }
    else if (above + c1 < want && want <= above + c1 + c0) { found[0] = hi - 1; found[1] = above + c1; }
    __syncthreads();
    prefix = (prefix << bits) | (unsigned)found[0];
    want -= found[1];
    __syncthreads();
  }
  // keys > prefix stay, and the first `want` that equal it
  auto count = [&](int x, int slot) __attribute__((always_inline)) {  // of the wavefronts before this one; x: this wavefront's
    if (lane == 0) wsum[slot][wave] = x;
    __syncthreads();
    int before = 0;
    for (int v = 0; v < wave; ++v) before += wsum[slot][v];
    return before;
  };
  int equal = 0;
  for (int j = j0; j < j1; j += 64) {
    const bool eq = j + lane < j1 && evict_key(p, w, pos, j + lane, fresh) == prefix;
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(eq));
  }
  const int equal0 = count(equal, 0);
  const unsigned long long below = (1ull << lane) - 1ull;
  // f(j, which of rows j .. j + 63 exist, which stay)
  auto rows = [&](auto&& f) __attribute__((always_inline)) {
    int eqs = equal0;
    for (int j = j0; j < j1; j += 64) {
      const bool there = j + lane < j1;
      const unsigned int key = there ? evict_key(p, w, pos, j + lane, fresh) : 0u;
      const bool eq = there && key == prefix;
      const unsigned long long em = __builtin_amdgcn_ballot_w64(eq);
      const bool stays = there && (key > prefix || (eq && eqs + __builtin_popcountll(em & below) < want));
      eqs += __builtin_popcountll(em);
      f(j, there, stays);
    }
  };
  int holes = 0, moving = 0;
  rows([&](int j, bool there, bool stays) __attribute__((always_inline)) {
    holes += __builtin_popcountll(__builtin_amdgcn_ballot_w64(there && !stays && j + lane < n));
    moving += __builtin_popcountll(__builtin_amdgcn_ballot_w64(stays && j + lane >= n));
  });
  const int hole0 = count(holes, 1);
  __syncthreads();
  const int move0 = count(moving, 0);
  int total = 0;
  for (int v = 0; v < kEvWaves; ++v) total += wsum[0][v];
  // ---- the j-th moving row into the j-th free place, kEvList of them at a time ---------------------------------------------------------
  for (int from = 0; from == 0 || from < total; from += kEvList) {
    __syncthreads();
    int at = move0;
    rows([&](int j, bool, bool stays) __attribute__((always_inline)) {
      const bool moves = stays && j + lane >= n;
      const unsigned long long mm = __builtin_amdgcn_ballot_w64(moves);
      const int rank = at + __builtin_popcountll(mm & below) - from;
      if (moves && rank >= 0 && rank < kEvList) list[rank] = j + lane;
      at += __builtin_popcountll(mm);
    });
    __syncthreads();
    at = hole0;
    rows([&](int j, bool there, bool stays) __attribute__((always_inline)) {
      const bool hole = there && !stays && j + lane < n;
      const unsigned long long hm = __builtin_amdgcn_ballot_w64(hole);
      const int rank = at + __builtin_popcountll(hm & below) - from;
      if (hole && rank >= 0 && rank < kEvList) kept[j + lane] = list[rank];
      if (from == 0 && stays && j + lane < n) kept[j + lane] = j + lane;
      at += __builtin_popcountll(hm);
    });
  }
}

// a wavefront per 64 rows of the new cache
__global__ __launch_bounds__(256) void kv_evict_move_kernel(KvEvictParams p) {
  __shared__ int todo[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kh = blockIdx.y, b = blockIdx.z;
  int L = p.ctx_len[b];
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int n = L < p.budget ? L : p.budget;
  const int j = (blockIdx.x * 4 + wave) * 64 + lane;
  const size_t head = (size_t)b * p.H_kv + kh;
  int src = j;
  if (j < n) {
    src = p.kept[head * p.budget + j];
    p.weight_out[head * p.kv_cap + j] = p.weight[head * p.kv_cap + src];
    if (p.pos) p.pos_out[head * p.kv_cap + j] = p.pos[head * p.kv_cap + src];
  }
  const bool moves = src != j;
  const unsigned long long m = __builtin_amdgcn_ballot_w64(moves);
  if (m == 0ull) return;
  if (moves) todo[wave][__builtin_popcountll(m & ((1ull << lane) - 1ull))] = lane;
  const int count = __builtin_popcountll(m), chunks = p.row_bytes / 16;
  const int first = j - lane;
  unsigned char* kc = p.k_cache + (size_t)p.kv_off[b] * p.elem_bytes + (size_t)kh * p.kv_cap * p.row_bytes;
  unsigned char* vc = p.v_cache + (size_t)p.kv_off[b] * p.elem_bytes + (size_t)kh * p.kv_cap * p.row_bytes;
  __builtin_amdgcn_wave_barrier();
  for (int x0 = 0; x0 < count * chunks; x0 += 64) {
    const int x = x0 + lane, i = x / chunks, row = i < count ? todo[wave][i] : 0;
    const int from = __shfl(src, row, 64);
    if (i < count) {
      const size_t s = (size_t)from * p.row_bytes + (x - i * chunks) * 16, d = (size_t)(first + row) * p.row_bytes + (x - i * chunks) * 16;
      const u32x4 k = *(const u32x4*)(kc + s), v = *(const u32x4*)(vc + s);
      *(u32x4*)(kc + d) = k;
      *(u32x4*)(vc + d) = v;
    }
  }
}

hipError_t prepare_kv_evict() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)kv_evict_select_kernel);
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" int kv_evict(ctcspec_ctx* ctx, ctcspec_dtype dt, void* k_cache, void* v_cache, const int64_t* kv_off,
                        const int32_t* ctx_len, int kv_cap, const float* weight, const int32_t* pos, const int32_t* next_pos, int B,
                        int H_kv, int dh, int budget, int sink, int recent, int32_t* kept, float* weight_out, int32_t* pos_out,
                        int32_t* ctx_len_out) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, k_cache && v_cache && kv_off && ctx_len && weight && kept && weight_out && ctx_len_out, CTCSPEC_EINVAL,
                  "kv_evict: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && H_kv > 0 && dh > 0 && kv_cap > 0 && budget > 0, CTCSPEC_EINVAL, "kv_evict: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "kv_evict: unknown element type");
  CTCSPEC_REQUIRE(ctx, sink >= 0 && recent >= 0 && (long long)sink + recent <= budget, CTCSPEC_EINVAL,
                  "kv_evict: sink and recent must not be negative and fit the budget together");
  CTCSPEC_REQUIRE(ctx, (pos != nullptr) == (pos_out != nullptr) && (pos || sink + recent == 0) && (next_pos || recent == 0),
                  CTCSPEC_EINVAL, "kv_evict: sink and recent need pos and pos_out, recent needs next_pos");
  CTCSPEC_REQUIRE(ctx, weight_out != weight && (!pos || pos_out != pos) && ctx_len_out != ctx_len, CTCSPEC_EINVAL,
                  "kv_evict: weight_out, pos_out and ctx_len_out must not be the inputs");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && B <= ctx->lim.max_batch && H_kv <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim && B <= 65535 && H_kv <= 65535,
                  CTCSPEC_EUNSUPPORTED, "kv_evict: dh must be a multiple of 8 and <= %d, the shape within the context's limits",
                  CTCSPEC_MAX_HEAD_DIM);
  CTCSPEC_REQUIRE(ctx, aligned16(k_cache) && aligned16(v_cache), CTCSPEC_EINVAL, "kv_evict: the caches must be 16-byte aligned");
  KvEvictParams p;
  p.k_cache = (unsigned char*)k_cache; p.v_cache = (unsigned char*)v_cache; p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.weight = weight; p.pos = pos; p.next_pos = next_pos; p.kept = kept; p.weight_out = weight_out; p.pos_out = pos_out;
  p.ctx_len_out = ctx_len_out; p.kv_cap = kv_cap; p.H_kv = H_kv; p.budget = budget; p.sink = sink; p.recent = recent;
  p.elem_bytes = dt == CTCSPEC_F32 ? 4 : 2;
  p.row_bytes = dh * p.elem_bytes;
  hipLaunchKernelGGL(kv_evict_select_kernel, dim3((unsigned)H_kv, (unsigned)B), dim3(kEvThreads), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  const int rows = budget < kv_cap ? budget : kv_cap;
  hipLaunchKernelGGL(kv_evict_move_kernel, dim3((unsigned)((rows + 255) / 256), (unsigned)H_kv, (unsigned)B), dim3(256), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}
