// kv_weight_update: what the accepted rows of a step looked at, added to the weight that every cached key has gathered.
//
//   weight[b,hk,j] += sum over the heads of hk's group and the accepted rows of exp(scale q . k_j - lse)
//
// With the rows' lse at hand (prefix_verify_attn) one read of K is all it takes: at most nine rows per head, so the call is bound by
// that read (8 sequences x 32 heads of 256 to 2048 keys, 79 MB: 18 to 21 us from card to card, 3.8 to 4.4 TB/s; 4 x 8 key heads of 16384
// to 65536, 346 MB: 69 to 78 us, 4.4 to 5.0 TB/s).  S = Q K^T goes through matrix instructions with 16 rows of the group on one side and 16 keys on the other; a
// lane then holds four rows of ONE key, and a key's sum is three additions and two exchanges.  (32 x 32 tiles: twice the
// exponentials for nine rows, and loads of 32 bytes of a key instead of 64.)
#include <type_traits>

#include "common.h"

namespace ctcspec {

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
  int T, kv_cap, H, H_kv, group, dh, max_nodes, tiles;
  float scale;
};

constexpr int kKwMaxRows = 9 * 256;  // rows of a group: (T + 1) heads

// Tiles of 32 keys that a wavefront takes one after the other, each requested under the products of the one before: several where
// there are enough wavefronts for the chip all the same.  (bf16, 128 wide, us with one for every 4096 / 16384 / 32768 tiles there
// are / with one always: 8 sequences x 32 key heads of 256 to 2048 keys 19.7 / 18.2 / 18.2 / 18.2, of 4096 62.5 / 55.3 / 59.3 / 59.2,
// of 1000 to 8000 53.0 / 50.4 / 69.5 / 69.6; 4 x 8 of 16384 to 65536 73.8 / 68.9 / 71.5 / 82.8.)  The tiles are those of the capacity, as the
// host does not know the lengths: in a cache with much room few wavefronts take many tiles each (8 x 32 heads of 500 keys: 11.0 us with
// room for 516, 11.9 for 4096, 15.8 for 16384; of 2000: 28.9 with room for 2016, 33.6 for 16384).
inline int weight_tiles(long long tiles) {
  const long long most = tiles / 16384;
  return most < 1 ? 1 : (most > 8 ? 8 : (int)most);
}

// DHP: dh padded.  NB: blocks of 16 rows that stay in registers; 0: as many as there are, read again for every tile.  (The smallest
// that holds them, as few registers as possible: 9 rows a key head 19.7 us with one block, 22.4 with room for five, 25.7 read again; 36
// rows 73.8 with three, 80.3 with five, 111 read again.)
template <bool F32, int DHP, int NB>
__global__ __launch_bounds__(256, 2) void kv_weight_kernel(KvWeightParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int ES = F32 ? 4 : 2, QS = DHP * ES / 64;  // steps of 64 bytes of a row
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kh = blockIdx.y, b = blockIdx.z, rb = p.dh * ES;
  const bool fresh = blockIdx.x == gridDim.x - 1;  // the last workgroup: the rows that kv_commit appends
  int L = __builtin_amdgcn_readfirstlane(p.ctx_len[b]);
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int key0 = blockIdx.x * p.tiles * 128 + wave * 32, step = 128;
  if (!fresh && (int)(blockIdx.x * p.tiles * 128) >= L) return;
  if (fresh && L >= p.kv_cap) return;  // no room for any

  // ---- keys: lane (c, g) has 16 bytes of key c of a half tile, chunk 4 u + g -------------------------------------------------------
  const unsigned char* kc = p.k_cache + ((size_t)p.kv_off[b] + (size_t)kh * p.kv_cap * p.dh) * ES;
  auto load_keys = [&](int k0, u32x4 (&kf)[2][QS]) __attribute__((always_inline)) {
    int left = L - k0;  // rows behind the last key: zeros, nothing is read
    left = left < 0 ? 0 : (left > 32 ? 32 : left);
    const unsigned long long at = (unsigned long long)(kc + (size_t)(left ? k0 : 0) * rb);
    const unsigned long long base = (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 |
                                    (unsigned)__builtin_amdgcn_readfirstlane((int)at);
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (unsigned)__builtin_amdgcn_readfirstlane(left * rb), 0x00020000);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < QS; ++u) {
        const int o = u * 64 + g * 16;
        kf[h][u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, o < rb ? (16 * h + c) * rb + o : 0x40000000, 0, 0));
      }
  };
  u32x4 kf[2][QS];
  if (!fresh) load_keys(key0, kf);  // (first of all: nothing else is as far away)

  // ---- the rows: row r is head r % group of path entry r / group; its lse (infinite: counts for nothing) and
  // where its query begins -------------------------------------------------------------------------------------------------------
  int len = __builtin_amdgcn_readfirstlane(p.accept_len[b]);
  len = len < 0 ? 0 : (len > p.T ? p.T : len);
  const int32_t* path = p.accept_nodes + (size_t)b * (p.T + 1);
  const int rows = (len + 1) * p.group, blocks = (rows + 15) / 16;
  float* row_lse = (float*)smem;
  int* row_at = (int*)smem + blocks * 16;
  const size_t head0 = (size_t)b * p.H + (size_t)kh * p.group;
  for (int r = tid; r < blocks * 16; r += 256) {
    float v = INFINITY;
    int at = -1;
    if (r < rows) {
      const int i = r / p.group, node = path[i];
      if (node >= 0 && node < p.max_nodes) {
        at = (r - i * p.group) * p.max_nodes + node;
        const float s = p.lse[head0 * p.max_nodes + at];
        v = s == -INFINITY ? INFINITY : s;
      }
    }
    row_lse[r] = v;
    row_at[r] = at;
  }
  __syncthreads();

  const unsigned char* q = p.q + head0 * p.max_nodes * rb;
  auto load_rows = [&](int blk, u32x4 (&qf)[QS], f32x4& lse) __attribute__((always_inline)) {
    const int at = row_at[blk * 16 + c];
#pragma unroll
    for (int u = 0; u < QS; ++u) {
      const int o = u * 64 + g * 16;
      const u32x4 x = *(const u32x4*)(q + (size_t)(at < 0 ? 0 : at) * rb + (o < rb ? o : 0));
      qf[u] = at >= 0 && o < rb ? x : u32x4{0u, 0u, 0u, 0u};
    }
    lse = *(const f32x4*)(row_lse + blk * 16 + 4 * g);  // registers 0 .. 3 of the products
  };
  // a block's weights of this lane's key; rows below `from` do not see it
  auto weigh = [&](const u32x4 (&qf)[QS], f32x4 lse, const u32x4 (&kf)[QS], int row0, int from) __attribute__((always_inline)) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
      // (sums side by side: a long one's every addition is rounded at the size of the whole)
      f32x4 part[4] = {s, s, s, s};
#pragma unroll
      for (int u = 0; u < QS; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          part[u % 4] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(qf[u][e]), __uint_as_float(kf[u][e]), part[u % 4], 0, 0, 0);
      s = (part[0] + part[1]) + (part[2] + part[3]);
    } else {
#pragma unroll
      for (int u = 0; u < QS; ++u)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qf[u]), __builtin_bit_cast(bf16x8, kf[u]), s, 0, 0, 0);
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // (the difference first, rounded once: score and lse are large against it, and so are their roundings)
      const float w = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale, -lse[i]) * 1.4426950408889634f);
      // (a row that counts for nothing: its score may be anything)
      sum += lse[i] == INFINITY || row0 + 4 * g + i < from ? 0.f : w;
    }
    return sum;
  };
  auto over_lanes = [&](float sum) __attribute__((always_inline)) {
    sum += __shfl_xor(sum, 16, 64);
    return sum + __shfl_xor(sum, 32, 64);
  };
  u32x4 qf[NB ? NB : 1][QS];
  f32x4 lse[NB ? NB : 1];
#pragma unroll
  for (int i = 0; i < NB; ++i)
    if (i < blocks) load_rows(i, qf[i], lse[i]);
  // what the rows give the 16 keys of a half tile
  auto gathered = [&](const u32x4 (&kf)[QS], int from) __attribute__((always_inline)) {
    float sum = 0.f;
    if constexpr (NB > 0) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
        if (i < blocks) sum += weigh(qf[i], lse[i], kf, 16 * i, from);
    } else {
      for (int i = 0; i < blocks; ++i) {
        load_rows(i, qf[0], lse[0]);
        sum += weigh(qf[0], lse[0], kf, 16 * i, from);
      }
    }
    return over_lanes(sum);
  };

  float* weight = p.weight + ((size_t)b * p.H_kv + kh) * p.kv_cap;
  if (!fresh) {
    for (int t = 0, k = key0; t < p.tiles && k < L; ++t, k += step) {
      u32x4 next[2][QS];
      const int j = k + (lane & 31);
      float old = 0.f;
      if (lane < 32 && j < L) old = weight[j];
      if (t + 1 < p.tiles) load_keys(k + step, next);
      const float first = gathered(kf[0], 0), second = gathered(kf[1], 0);
      if (lane < 32 && j < L) weight[j] = old + (lane < 16 ? first : second);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < QS; ++u) kf[h][u] = next[h][u];
    }
  } else if (wave == 0) {
    // path entry m becomes row L + m, seen by entries m and later
    const int node = c <= len ? path[c] : -1, j = L + c;
    const bool there = node >= 0 && node < p.max_nodes && j < p.kv_cap;
    const unsigned char* kt = p.k_tree + (((size_t)b * p.H_kv + kh) * p.max_nodes + (there ? node : 0)) * rb;
#pragma unroll
    for (int u = 0; u < QS; ++u) {
      const int o = u * 64 + g * 16;
      const u32x4 x = *(const u32x4*)(kt + (o < rb ? o : 0));
      kf[0][u] = o < rb ? x : u32x4{0u, 0u, 0u, 0u};
    }
    const float sum = gathered(kf[0], c * p.group);
    if (there && g == 0) {
      weight[j] = sum;
      if (p.pos) p.pos[((size_t)b * p.H_kv + kh) * p.kv_cap + j] = p.next_pos[b] + c;
    }
  }
#endif
}

template <bool F32, int DHP>
static hipError_t launch_kv_weight(const KvWeightParams& p, dim3 grid, int blocks, hipStream_t stream) {
  const size_t lds = (size_t)blocks * 16 * 8;
  // rows of 256 and 512 bytes: five blocks and one are what the registers hold beside two tiles of keys
  constexpr int kMost = F32 ? (DHP == 64 ? 3 : 1) : 5;
  if (blocks == 1) hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, 1>), grid, dim3(256), lds, stream, p);
  else if (blocks <= 3 && kMost >= 3) hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, kMost >= 3 ? 3 : 1>), grid, dim3(256), lds, stream, p);
  else if (blocks <= kMost) hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, kMost>), grid, dim3(256), lds, stream, p);
  else hipLaunchKernelGGL((kv_weight_kernel<F32, DHP, 0>), grid, dim3(256), lds, stream, p);
  return hipGetLastError();
}

hipError_t prepare_kv_weight() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)kv_weight_kernel<false, 128, 1>);
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
  CTCSPEC_REQUIRE(ctx, kv_cap <= (1 << 30), CTCSPEC_EUNSUPPORTED, "kv_weight_update: kv_cap must be <= 2^30");
  for (const void* a : {q, k_cache, k_tree})
    CTCSPEC_REQUIRE(ctx, aligned16(a), CTCSPEC_EINVAL, "kv_weight_update: q, k_cache and k_tree must be 16-byte aligned");
  KvWeightParams p;
  p.q = (const unsigned char*)q; p.lse = lse; p.k_cache = (const unsigned char*)k_cache; p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.k_tree = (const unsigned char*)k_tree; p.accept_len = accept_len; p.accept_nodes = accept_nodes;
  p.weight = weight; p.pos = pos; p.next_pos = next_pos;
  p.T = T; p.kv_cap = kv_cap; p.H = H; p.H_kv = H_kv; p.group = H / H_kv; p.dh = dh; p.max_nodes = max_nodes;
  p.scale = scale;
  p.tiles = weight_tiles((long long)B * H_kv * ((kv_cap + 31LL) / 32));
  const int blocks = ((T + 1) * p.group + 15) / 16;
  const dim3 grid((unsigned)(((long long)kv_cap + 128 * p.tiles - 1) / (128 * p.tiles)) + 1, (unsigned)H_kv, (unsigned)B);
  hipError_t e;
  if (dt == CTCSPEC_F32) e = dh <= 64 ? launch_kv_weight<true, 64>(p, grid, blocks, ctx->stream) : launch_kv_weight<true, 128>(p, grid, blocks, ctx->stream);
  else e = dh <= 64 ? launch_kv_weight<false, 64>(p, grid, blocks, ctx->stream) : launch_kv_weight<false, 128>(p, grid, blocks, ctx->stream);
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
