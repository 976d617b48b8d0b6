// kv_weight_update: what the accepted rows of a step looked at, added to the weight that every cached key has gathered.
//
//   weight[b,hk,j] += sum over the heads of hk's group and the accepted rows of exp(scale q . k_j - lse)
//
// With the rows' lse at hand (prefix_verify_attn) one read of K is all it takes: at most nine rows per head, so the call is bound by
// that read.  S = Q K^T goes through matrix instructions with the rows of the group (up to 32 at a time) on one side and 32 keys on
// the other; a lane then holds 16 rows of ONE key, and their sum is 16 additions and one exchange.
#include <type_traits>

#include "common.h"

namespace ctcspec {

typedef __attribute__((ext_vector_type(16))) float f32x16;

struct KvWeightParams {
  const unsigned char* q;        // [B][H][max_nodes][dh]
  const float* lse;              // [B][H][max_nodes]
  const unsigned char* k_cache;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const unsigned char* k_tree;   // [B][H_kv][max_nodes][dh]
  const int32_t* accept_len;
  const int32_t* accept_nodes;   // [B][T + 1]
  float* weight;                 // [B][H_kv][kv_cap]
  int32_t* pos;                  // [B][H_kv][kv_cap] or null
  const int32_t* next_pos;       // [B] or null
  int T, kv_cap, H, H_kv, group, dh, max_nodes;
  float sl2;                     // scale * log2(e)
};

constexpr int kKwTiles = 4;                       // key tiles of a wavefront
constexpr int kKwKeys = 4 * 32 * kKwTiles;        // keys of a workgroup
constexpr int kKwMaxRows = 9 * 256;               // rows of a group: (T + 1) heads

// DHP: dh padded.  ONE: the rows fit one block of 32 and stay in registers.
template <bool F32, int DHP, bool ONE>
__global__ __launch_bounds__(256) void kv_weight_kernel(KvWeightParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int ES = F32 ? 4 : 2, QU = DHP * ES / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h2 = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kh = blockIdx.y, b = blockIdx.z, rb = p.dh * ES;
  int L = __builtin_amdgcn_readfirstlane(p.ctx_len[b]);
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int key0 = blockIdx.x * kKwKeys;
  if (key0 >= L && blockIdx.x != 0) return;  // (the first workgroup also has the new rows)
  int len = __builtin_amdgcn_readfirstlane(p.accept_len[b]);
  len = len < 0 ? 0 : (len > p.T ? p.T : len);
  const int32_t* path = p.accept_nodes + (size_t)b * (p.T + 1);
  const int rows = (len + 1) * p.group, blocks = (rows + 31) / 32;

  // ---- the rows: row r is head r % group of path entry r / group; its lse in the log2 domain (infinite: counts for nothing) and
  // where its query begins -------------------------------------------------------------------------------------------------------
  float* row_lse = (float*)smem;
  int* row_at = (int*)smem + blocks * 32;
  const size_t head0 = (size_t)b * p.H + (size_t)kh * p.group;
  for (int r = tid; r < blocks * 32; r += 256) {
    float v = INFINITY;
    int at = -1;
    if (r < rows) {
      const int i = r / p.group, node = path[i];
      if (node >= 0 && node < p.max_nodes) {
        const int row = (r - i * p.group) * p.max_nodes + node;
        const float s = p.lse[head0 * p.max_nodes + row];
        at = row;
        v = s == -INFINITY ? INFINITY : s * 1.4426950408889634f;
      }
    }
    row_lse[r] = v;
    row_at[r] = at;
  }
  __syncthreads();

  const unsigned char* q = p.q + head0 * p.max_nodes * rb;
  u32x4 qf[QU];
  f32x4 lse[4];
  auto load_rows = [&](int blk) __attribute__((always_inline)) {
    const int at = row_at[blk * 32 + c];
#pragma unroll
    for (int i = 0; i < QU; ++i) {
      const int o = (2 * i + h2) * 16;
      qf[i] = u32x4{0u, 0u, 0u, 0u};
      if (at >= 0 && o < rb) qf[i] = *(const u32x4*)(q + (size_t)at * rb + o);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) lse[j] = *(const f32x4*)(row_lse + blk * 32 + 8 * j + 4 * h2);  // registers 4 j .. 4 j + 3
  };
  // the rows' weights of this lane's key, added up; rows below `from` do not see it
  auto gathered = [&](const u32x4 (&kf)[QU], int from) __attribute__((always_inline)) {
    float sum = 0.f;
    for (int blk = 0; blk < (ONE ? 1 : blocks); ++blk) {
      if constexpr (!ONE) load_rows(blk);
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(qf[i][e]), __uint_as_float(kf[i][e]), s, 0, 0, 0);
        } else {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, qf[i]), __builtin_bit_cast(bf16x8, kf[i]), s, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[i], p.sl2, -lse[i / 4][i % 4]));
        const int r = blk * 32 + 8 * (i / 4) + 4 * h2 + i % 4;
        // (a row that counts for nothing: its score may be anything, the query of a row that is none is zero)
        sum += lse[i / 4][i % 4] < INFINITY || lse[i / 4][i % 4] != lse[i / 4][i % 4] ? (r >= from ? w : 0.f) : 0.f;
      }
    }
    return sum + __shfl_xor(sum, 32, 64);
  };
  if constexpr (ONE) load_rows(0);

  float* weight = p.weight + ((size_t)b * p.H_kv + kh) * p.kv_cap;
  const unsigned char* kc = p.k_cache + ((size_t)p.kv_off[b] + (size_t)kh * p.kv_cap * p.dh) * ES;
  auto load_keys = [&](int k0, u32x4 (&kf)[QU]) __attribute__((always_inline)) {
    int left = L - k0;  // rows behind the last key: zeros, nothing is read
    left = left < 0 ? 0 : (left > 32 ? 32 : left);
    const long long at = (long long)(uintptr_t)(kc + (size_t)(left ? k0 : 0) * rb);
    const long long base = (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 |
                                       (unsigned)__builtin_amdgcn_readfirstlane((int)at));
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (unsigned)__builtin_amdgcn_readfirstlane(left * rb), 0x00020000);
#pragma unroll
    for (int i = 0; i < QU; ++i) {
      const int o = (2 * i + h2) * 16;
      kf[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, o < rb ? c * rb + o : 0x40000000, 0, 0));
    }
  };
  if (key0 < L) {
    u32x4 kf[2][QU];
    int k = key0 + wave * 32;
    load_keys(k, kf[0]);
#pragma unroll
    for (int t = 0; t < kKwTiles; ++t, k += 128) {
      if (k >= L) break;
      const int j = k + c;
      float old = 0.f;
      if (h2 == 0 && j < L) old = weight[j];
      if (t + 1 < kKwTiles) load_keys(k + 128, kf[(t + 1) & 1]);
      const float sum = gathered(kf[t & 1], 0);
      if (h2 == 0 && j < L) weight[j] = old + sum;
    }
  }
  // ---- the rows that kv_commit appends: path entry m becomes row L + m, seen by entries m and later --------------------------------
  if (blockIdx.x == 0 && wave == 0) {
    const int node = c <= len ? path[c] : -1, j = L + c;
    const bool there = node >= 0 && node < p.max_nodes && j < p.kv_cap;
    const unsigned char* kt = p.k_tree + (((size_t)b * p.H_kv + kh) * p.max_nodes + (there ? node : 0)) * rb;
    u32x4 kf[QU];
#pragma unroll
    for (int i = 0; i < QU; ++i) {
      const int o = (2 * i + h2) * 16;
      kf[i] = u32x4{0u, 0u, 0u, 0u};
      if (there && o < rb) kf[i] = *(const u32x4*)(kt + o);
    }
    const float sum = gathered(kf, c * p.group);
    if (there && h2 == 0) {
      weight[j] = sum;
      if (p.pos) p.pos[((size_t)b * p.H_kv + kh) * p.kv_cap + j] = p.next_pos[b] + c;
    }
  }
#endif
}

template <bool F32, int DHP>
static hipError_t launch_kv_weight(const KvWeightParams& p, dim3 grid, bool one, size_t lds, hipStream_t stream) {
  if (one) hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, true>), grid, dim3(256), lds, stream, p);
  else hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, false>), grid, dim3(256), lds, stream, p);
  return hipGetLastError();
}

hipError_t prepare_kv_weight() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)kv_weight_kernel<false, 128, true>);
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" int kv_weight_update(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* q, const float* lse, const void* k_cache,
                                const int64_t* kv_off, const int32_t* ctx_len, int kv_cap, const void* k_tree,
                                const int32_t* accept_len, const int32_t* accept_nodes, int T, int B, int H, int H_kv, int dh,
                                int max_nodes, float scale, float* weight, int32_t* pos, const int32_t* next_pos) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, q && lse && k_cache && kv_off && ctx_len && k_tree && accept_len && accept_nodes && weight, CTCSPEC_EINVAL,
                  "kv_weight_update: null pointer");
  CTCSPEC_REQUIRE(ctx, !pos || next_pos, CTCSPEC_EINVAL, "kv_weight_update: pos needs next_pos");
  CTCSPEC_REQUIRE(ctx, T > 0 && B > 0 && H > 0 && H_kv > 0 && dh > 0 && max_nodes > 0 && kv_cap > 0, CTCSPEC_EINVAL,
                  "kv_weight_update: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, H % H_kv == 0, CTCSPEC_EINVAL, "kv_weight_update: H must be a multiple of H_kv");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "kv_weight_update: unknown element type");
  CTCSPEC_REQUIRE(ctx, scale > 0.f && scale <= 3.0e38f, CTCSPEC_EINVAL, "kv_weight_update: the scale must be positive and finite");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && max_nodes <= CTCSPEC_MAX_NODES && T <= CTCSPEC_MAX_SLOTS &&
                           (T + 1) * (long long)(H / H_kv) <= kKwMaxRows && H_kv <= 65535,
                  CTCSPEC_EUNSUPPORTED, "kv_weight_update: dh must be a multiple of 8 and <= %d, max_nodes <= %d, T <= %d, (T+1)*H/H_kv <= %d",
                  CTCSPEC_MAX_HEAD_DIM, CTCSPEC_MAX_NODES, CTCSPEC_MAX_SLOTS, kKwMaxRows);
  CTCSPEC_REQUIRE(ctx, B <= ctx->lim.max_batch && B <= 65535 && max_nodes <= ctx->lim.max_nodes && H <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim,
                  CTCSPEC_EUNSUPPORTED, "kv_weight_update: shape exceeds the context's limits");
  for (const void* a : {q, k_cache, k_tree})
    CTCSPEC_REQUIRE(ctx, aligned16(a), CTCSPEC_EINVAL, "kv_weight_update: q, k_cache and k_tree must be 16-byte aligned");
  KvWeightParams p;
  p.q = (const unsigned char*)q; p.lse = lse; p.k_cache = (const unsigned char*)k_cache; p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.k_tree = (const unsigned char*)k_tree; p.accept_len = accept_len; p.accept_nodes = accept_nodes;
  p.weight = weight; p.pos = pos; p.next_pos = next_pos;
  p.T = T; p.kv_cap = kv_cap; p.H = H; p.H_kv = H_kv; p.group = H / H_kv; p.dh = dh; p.max_nodes = max_nodes;
  p.sl2 = scale * 1.4426950408889634f;
  const int rows = (T + 1) * p.group, blocks = (rows + 31) / 32;
  const dim3 grid((unsigned)(((long long)kv_cap + kKwKeys - 1) / kKwKeys), (unsigned)H_kv, (unsigned)B);
  const size_t lds = (size_t)blocks * 32 * 8;
  const bool one = blocks == 1;
  hipError_t e;
  if (dt == CTCSPEC_F32) e = dh <= 64 ? launch_kv_weight<true, 64>(p, grid, one, lds, ctx->stream) : launch_kv_weight<true, 128>(p, grid, one, lds, ctx->stream);
  else e = dh <= 64 ? launch_kv_weight<false, 64>(p, grid, one, lds, ctx->stream) : launch_kv_weight<false, 128>(p, grid, one, lds, ctx->stream);
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
