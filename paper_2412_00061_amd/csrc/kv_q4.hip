// kv_append_q4, kv_commit_q4, kv_read_q4: rows of keys and values into a cache held in 4 bits (q4_format.h) - a prompt's in their order,
// an accepted path's by its nodes - and back out of it.
//
// Eight elements to a lane: 16 bytes of a bf16 row, four lanes to a block of 32, whose largest magnitude goes round among them; 4 bytes of
// codes go out, and of the first of the four lanes the scale.  Both directions are bound by their bytes: K and V of 4096 rows of 32 heads of 128
// in bf16, 85 MB either way, go in within 15.4 us (5.5 TB/s) and out again in 14.6; the accepted rows of eight sequences in 3.1.
#include "q4_format.h"

namespace ctcspec {

struct Q4StoreParams {
  const unsigned char* rows[2];   // K, V: [B][H_kv][max_rows][dh]
  const int32_t* count;           // [B]
  const int32_t* nodes;           // [B][T + 1]: the rows' places, count[b] + 1 of them; or null: count[b] rows in their order
  unsigned char* codes[2];
  unsigned char* scales[2];
  const int64_t* kv_off;
  const int32_t* ctx_len;
  int32_t* ctx_len_out;           // or null
  int T, max_rows, kv_cap, H_kv, dh;
};

constexpr int kQ4Threads = 256;
constexpr int q4_rows_per_group(int blocks) { return kQ4Threads / (4 * blocks); }

template <bool F32, int NB>
__global__ __launch_bounds__(kQ4Threads) void q4_store_kernel(Q4StoreParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = 4 * NB, RPG = q4_rows_per_group(NB);
  const int kh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  int L = p.ctx_len[b], n = p.count[b];
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int most = p.nodes ? p.T : p.max_rows;
  n = (n < 0 ? 0 : (n > most ? most : n)) + (p.nodes ? 1 : 0);
  const int room = p.kv_cap - L;
  if (p.ctx_len_out && blockIdx.x == 0 && kh == 0 && tid == 0) p.ctx_len_out[b] = L + (n < room ? n : room);
  n = n < room ? n : room;
  const int j = blockIdx.x * RPG + tid / LPR, part = tid % LPR;
  // (a block's four lanes go or stay together)
  if (tid >= RPG * LPR || j >= n) return;
  int from = j;
  if (p.nodes) {
    from = p.nodes[(size_t)b * (p.T + 1) + j];
    if (from < 0 || from >= p.max_rows) return;
  }
  const size_t src = (((size_t)b * p.H_kv + kh) * p.max_rows + from) * p.dh + part * 8;
  const size_t dst = (size_t)p.kv_off[b] + (size_t)kh * p.kv_cap + L + j;
  const bool there = part * 8 < p.dh;
  float x[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if constexpr (F32) {
      const f32x4* at = (const f32x4*)((const float*)p.rows[t] + src);
      const f32x4 a = there ? at[0] : f32x4{0.f, 0.f, 0.f, 0.f}, c = there ? at[1] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[t][i] = a[i]; x[t][4 + i] = c[i]; }
    } else {
      const u32x4 a = there ? *(const u32x4*)((const unsigned short*)p.rows[t] + src) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[t][2 * i] = __uint_as_float(a[i] << 16); x[t][2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    unsigned int amax = 0u;  // (bits of magnitudes: infinities and NaN are above all numbers)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned int a = __float_as_uint(x[t][i]) & 0x7fffffffu;
      amax = a > amax ? a : amax;
    }
    const unsigned int a1 = (unsigned)__builtin_amdgcn_update_dpp(0, (int)amax, 0xb1, 0xf, 0xf, false);  // lanes 1 0 3 2 of four
    amax = a1 > amax ? a1 : amax;
    const unsigned int a2 = (unsigned)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4e, 0xf, 0xf, false);  // lanes 2 3 0 1
    amax = a2 > amax ? a2 : amax;
    const int s = q4_scale(amax);
    *(unsigned int*)(p.codes[t] + dst * (NB * kQ4BlockBytes) + part * 4) = q4_encode(x[t], s);
    if (part % 4 == 0) p.scales[t][dst * NB + part / 4] = (unsigned char)s;
  }
#endif
}

struct Q4ReadParams {
  const unsigned char* codes[2];
  const unsigned char* scales[2];
  const int64_t* kv_off;
  const int32_t* first;
  const int32_t* count;
  unsigned char* rows[2];   // [B][H_kv][max_rows][dh]
  int max_rows, kv_cap, H_kv, dh;
};

template <bool F32, int NB>
__global__ __launch_bounds__(kQ4Threads) void q4_read_kernel(Q4ReadParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = 4 * NB, RPG = q4_rows_per_group(NB);
  const int kh = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  int n = p.count[b];
  n = n > p.max_rows ? p.max_rows : n;
  const int j = blockIdx.x * RPG + tid / LPR, part = tid % LPR;
  const long long row = (long long)p.first[b] + j;
  if (tid >= RPG * LPR || j >= n || row < 0 || row >= p.kv_cap || part * 8 >= p.dh) return;
  const size_t src = (size_t)p.kv_off[b] + (size_t)kh * p.kv_cap + (size_t)row;
  const size_t dst = (((size_t)b * p.H_kv + kh) * p.max_rows + j) * p.dh + part * 8;
  unsigned int w[2], s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    w[t] = *(const unsigned int*)(p.codes[t] + src * (NB * kQ4BlockBytes) + part * 4);
    s[t] = p.scales[t][src * NB + part / 4];
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const u32x4 v = q4_decode(w[t], q4_scale_value((int)s[t]));
    if constexpr (F32) {
      f32x4* at = (f32x4*)((float*)p.rows[t] + dst);
      at[0] = f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u), __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
      at[1] = f32x4{__uint_as_float(v[2] << 16), __uint_as_float(v[2] & 0xffff0000u), __uint_as_float(v[3] << 16), __uint_as_float(v[3] & 0xffff0000u)};
    } else {
      *(u32x4*)((unsigned short*)p.rows[t] + dst) = v;
    }
  }
#endif
}

// code of this translation unit loaded onto the current device (context creation calls this: a stage call never
// triggers a load, so it can be the first thing a stream capture records)
hipError_t prepare_kv_q4() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, (const void*)q4_store_kernel<false, 4>);
}

template <template <bool, int> class K>
static auto q4_kernel(bool f32, int blocks) {
  switch (blocks) {
    case 1: return f32 ? K<true, 1>::at : K<false, 1>::at;
    case 2: return f32 ? K<true, 2>::at : K<false, 2>::at;
    case 3: return f32 ? K<true, 3>::at : K<false, 3>::at;
    default: return f32 ? K<true, 4>::at : K<false, 4>::at;
  }
}
template <bool F32, int NB> struct Q4Store { static constexpr auto at = q4_store_kernel<F32, NB>; };
template <bool F32, int NB> struct Q4Read { static constexpr auto at = q4_read_kernel<F32, NB>; };

// what the three calls ask of their arguments
static int q4_check(ctcspec_ctx* ctx, const char* call, ctcspec_dtype dt, const ctcspec_q4_cache* cache, const void* k_rows, const void* v_rows,
                    int kv_cap, int B, int H_kv, int dh, int rows) {
  CTCSPEC_REQUIRE(ctx, cache && cache->k_codes && cache->k_scales && cache->v_codes && cache->v_scales && k_rows && v_rows, CTCSPEC_EINVAL,
                  "%s: null pointer", call);
  CTCSPEC_REQUIRE(ctx, B > 0 && H_kv > 0 && dh > 0 && rows > 0 && kv_cap > 0, CTCSPEC_EINVAL, "%s: sizes must be positive", call);
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "%s: unknown element type", call);
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM, CTCSPEC_EUNSUPPORTED, "%s: dh must be a multiple of 8 and <= %d", call,
                  CTCSPEC_MAX_HEAD_DIM);
  CTCSPEC_REQUIRE(ctx, B <= ctx->lim.max_batch && B <= 65535 && dh <= ctx->lim.max_head_dim && H_kv <= ctx->lim.max_heads && H_kv <= 65535 && kv_cap <= 1 << 30 &&
                           rows <= 1 << 27,  // (16 to 64 rows a workgroup: below 2^32 threads)
                  CTCSPEC_EUNSUPPORTED, "%s: shape exceeds the context's limits, kv_cap beyond 2^30 or max_rows beyond 2^27", call);
  CTCSPEC_REQUIRE(ctx, aligned16(cache->k_codes) && aligned16(cache->v_codes) && aligned16(k_rows) && aligned16(v_rows) &&
                           q4_scales_aligned(cache),
                  CTCSPEC_EINVAL, "%s: codes and rows must be 16-byte aligned, scales 4-byte aligned", call);
  return CTCSPEC_OK;
}

static int q4_store(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* k_rows, const void* v_rows, int max_rows, const int32_t* count,
                    const int32_t* nodes, int T, const ctcspec_q4_cache* cache, const int64_t* kv_off, const int32_t* ctx_len, int kv_cap, int B,
                    int H_kv, int dh, int32_t* ctx_len_out) {
  Q4StoreParams p;
  p.rows[0] = (const unsigned char*)k_rows; p.rows[1] = (const unsigned char*)v_rows;
  p.count = count; p.nodes = nodes; p.T = T; p.max_rows = max_rows;
  p.codes[0] = (unsigned char*)cache->k_codes; p.codes[1] = (unsigned char*)cache->v_codes;
  p.scales[0] = (unsigned char*)cache->k_scales; p.scales[1] = (unsigned char*)cache->v_scales;
  p.kv_off = kv_off; p.ctx_len = ctx_len; p.ctx_len_out = ctx_len_out; p.kv_cap = kv_cap; p.H_kv = H_kv; p.dh = dh;
  const int blocks = q4_blocks(dh), per = q4_rows_per_group(blocks), most = nodes ? T + 1 : max_rows;
  hipLaunchKernelGGL(q4_kernel<Q4Store>(dt == CTCSPEC_F32, blocks), dim3((unsigned)((most + per - 1) / per), (unsigned)H_kv, (unsigned)B),
                     dim3(kQ4Threads), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" int kv_append_q4(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* k_rows, const void* v_rows, const int32_t* n_rows, int max_rows,
                            const ctcspec_q4_cache* cache, const int64_t* kv_off, const int32_t* ctx_len, int kv_cap, int B, int H_kv, int dh,
                            int32_t* ctx_len_out) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, n_rows && kv_off && ctx_len, CTCSPEC_EINVAL, "kv_append_q4: null pointer");
  if (const int bad = q4_check(ctx, "kv_append_q4", dt, cache, k_rows, v_rows, kv_cap, B, H_kv, dh, max_rows)) return bad;
  // (one workgroup of a sequence writes it, others may still have to read these)
  CTCSPEC_REQUIRE(ctx, ctx_len_out != ctx_len && ctx_len_out != n_rows, CTCSPEC_EINVAL,
                  "kv_append_q4: ctx_len_out must not be the ctx_len or n_rows buffer");
  return q4_store(ctx, dt, k_rows, v_rows, max_rows, n_rows, nullptr, 0, cache, kv_off, ctx_len, kv_cap, B, H_kv, dh, ctx_len_out);
}

extern "C" int kv_commit_q4(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* k_tree, const void* v_tree, const int32_t* accept_len,
                            const int32_t* accept_nodes, int T, const ctcspec_q4_cache* cache, const int64_t* kv_off, const int32_t* ctx_len,
                            int kv_cap, int B, int H_kv, int dh, int max_nodes, int32_t* ctx_len_out) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, accept_len && accept_nodes && kv_off && ctx_len, CTCSPEC_EINVAL, "kv_commit_q4: null pointer");
  if (const int bad = q4_check(ctx, "kv_commit_q4", dt, cache, k_tree, v_tree, kv_cap, B, H_kv, dh, max_nodes)) return bad;
  CTCSPEC_REQUIRE(ctx, T > 0, CTCSPEC_EINVAL, "kv_commit_q4: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, T <= CTCSPEC_MAX_SLOTS && max_nodes <= CTCSPEC_MAX_NODES && max_nodes <= ctx->lim.max_nodes, CTCSPEC_EUNSUPPORTED,
                  "kv_commit_q4: T <= %d, max_nodes <= %d and within the context's limits", CTCSPEC_MAX_SLOTS, CTCSPEC_MAX_NODES);
  CTCSPEC_REQUIRE(ctx, ctx_len_out != ctx_len && ctx_len_out != accept_len && ctx_len_out != accept_nodes, CTCSPEC_EINVAL,
                  "kv_commit_q4: ctx_len_out must not be the ctx_len, accept_len or accept_nodes buffer");
  return q4_store(ctx, dt, k_tree, v_tree, max_nodes, accept_len, accept_nodes, T, cache, kv_off, ctx_len, kv_cap, B, H_kv, dh, ctx_len_out);
}

extern "C" int kv_read_q4(ctcspec_ctx* ctx, const ctcspec_q4_cache* cache, const int64_t* kv_off, const int32_t* first, const int32_t* n_rows,
                          int max_rows, int kv_cap, int B, int H_kv, int dh, ctcspec_dtype out_dt, void* k_rows, void* v_rows) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, kv_off && first && n_rows, CTCSPEC_EINVAL, "kv_read_q4: null pointer");
  if (const int bad = q4_check(ctx, "kv_read_q4", out_dt, cache, k_rows, v_rows, kv_cap, B, H_kv, dh, max_rows)) return bad;
  Q4ReadParams p;
  p.codes[0] = (const unsigned char*)cache->k_codes; p.codes[1] = (const unsigned char*)cache->v_codes;
  p.scales[0] = (const unsigned char*)cache->k_scales; p.scales[1] = (const unsigned char*)cache->v_scales;
  p.kv_off = kv_off; p.first = first; p.count = n_rows; p.rows[0] = (unsigned char*)k_rows; p.rows[1] = (unsigned char*)v_rows;
  p.max_rows = max_rows; p.kv_cap = kv_cap; p.H_kv = H_kv; p.dh = dh;
  const int blocks = q4_blocks(dh), per = q4_rows_per_group(blocks);
  hipLaunchKernelGGL(q4_kernel<Q4Read>(out_dt == CTCSPEC_F32, blocks), dim3((unsigned)((max_rows + per - 1) / per), (unsigned)H_kv, (unsigned)B),
                     dim3(kQ4Threads), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}
