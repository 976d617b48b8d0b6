// prefix_verify_attn: verification attention of a batch whose sequences continue one common prefix, one layer.
//
//   out[b,h,i] = sum_j p_j v_j,  p = softmax over the prefix's keys, the sequence's cached keys and the tree nodes it sees
//
// Softmax parts over disjoint keys join exactly: (O, m, l) with O = sum exp2(s - m) v, l = sum exp2(s - m).  So the prefix is a
// pass of its own in which the rows of ALL sequences (and of the heads that share a key head) stand side by side against
// each key tile - read and multiplied once for the batch -, the sequences' own keys are a second pass, and a third kernel joins
// what the two left.
//
// Both passes run prefix_attn_kernel.  The work is cut into units - one iteration over the keys (KP * KT tiles of 32) for one
// block of R rows - and the units of a pass, in the order (key head, row block, keys), are dealt to the workgroups in equal
// consecutive shares: lengths, node counts and prefix length are read on the device, and no workgroup waits for a longer one.  A
// workgroup whose share crosses from one block of rows into the next leaves a partial result for each.  Partial results are
// numbered workgroup + block: consecutive ones differ in either, so no two share a number (prefix_plan.h).
#include <type_traits>
#include <utility>

#include "common.h"
#include "prefix_plan.h"

namespace ctcspec {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

struct PrefixAttnParams {
  const unsigned char* q;         // [B][H][max_nodes][dh]
  const unsigned char* k_prefix;  // [H_kv][prefix_cap][dh]
  const unsigned char* v_prefix;
  const int32_t* prefix_len;      // [1]
  const unsigned char* k_cache;
  const unsigned char* v_cache;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const unsigned char* k_tree;    // [B][H_kv][max_nodes][dh]
  const unsigned char* v_tree;
  const int32_t* n_nodes;
  const unsigned long long* anc_mask;
  int prefix_cap, kv_cap, B, H, H_kv, group, dh, max_nodes;  // group: heads that share a key head
  float sl2;                      // scale * log2(e)
  float* po;                      // partial O of the pass: [slot][R / 32][DHP / 32][4][64 lanes][4]
  float* pml;                     // [slot][2][R]: maximum in the log2 domain, sum
};

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uniform(long long v) {
  return (long long)((unsigned long long)(unsigned)uniform((int)(v >> 32)) << 32 | (unsigned)uniform((int)v));
}

__device__ __forceinline__ const unsigned char* uniform(const unsigned char* p) {
  return (const unsigned char*)uniform((long long)p);
}

// what a pass or the join knows about the batch: lane b holds sequence b's (the limits allow 64 sequences)
struct Batch {
  int n, first;  // nodes, nodes of the sequences before it
  int ctx;       // cached rows
  int all;       // nodes of all sequences (uniform)
};
__device__ __forceinline__ Batch read_batch(const PrefixAttnParams& p) {
  const int lane = threadIdx.x & 63;
  Batch t{0, 0, 0, 0};
  if (lane < p.B) {
    const int n = p.n_nodes[lane], L = p.ctx_len[lane];
    t.n = n < 0 ? 0 : (n > p.max_nodes ? p.max_nodes : n);
    t.ctx = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  }
  int sum = t.n;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int below = __shfl_up(sum, d, 64);
    if (lane >= d) sum += below;
  }
  t.first = sum - t.n;
  t.all = __builtin_amdgcn_readlane(sum, 63);
  return t;
}

// the blocks of rows of a pass
template <bool OWN, int R, int TPI>
struct Blocks {
  // prefix: the same for all; own: lane b's sequence
  int blocks, iters;   // row blocks of a key head, iterations over the keys
  long long unit0;     // first unit of the sequence
  int block0;          // first block of the sequence, over its key heads
  long long units;     // of the pass (uniform)
  __device__ __forceinline__ static Blocks make(const PrefixAttnParams& p, const Batch& t) {
    Blocks k;
    if constexpr (!OWN) {
      int P = uniform(*p.prefix_len);
      P = P < 0 ? 0 : (P > p.prefix_cap ? p.prefix_cap : P);
      k.blocks = (t.all * p.group + R - 1) / R;
      k.iters = ((P + 31) / 32 + TPI - 1) / TPI;
      k.unit0 = 0;
      k.block0 = 0;
      k.units = (long long)p.H_kv * k.blocks * k.iters;
    } else {
      const int lane = threadIdx.x & 63;
      k.blocks = (t.n * p.group + R - 1) / R;
      k.iters = t.n ? ((t.ctx + 31) / 32 + (t.n + 31) / 32 + TPI - 1) / TPI : 0;
      const int mine = p.H_kv * k.blocks;
      int b = mine;
      long long u = (long long)mine * k.iters;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int bb = __shfl_up(b, d, 64);
        const long long ub = __shfl_up(u, d, 64);
        if (lane >= d) { b += bb; u += ub; }
      }
      k.block0 = b - mine;
      k.unit0 = u - (long long)mine * k.iters;
      k.units = uniform(__shfl(u, 63, 64));
    }
    return k;
  }
};

// R = 32 CW rows, CW * KP wavefronts: wavefront w has rows [32 rg, 32 rg + 32), rg = w % CW, and of an iteration's KP * KT key
// tiles the KT from kp * KT on, kp = w / CW; the KP parts are joined through LDS at the end.  Tiles (32 keys, K and V) go
// through registers into one of two LDS stages.  FINE: P as two bf16 numbers (16 bits of mantissa).
template <bool F32_, int DHP_, int CW_, int KP_, int KT_, bool FINE_>
struct PrefixShape {
  static constexpr bool F32 = F32_, FINE = FINE_;
  static constexpr int DHP = DHP_, CW = CW_, KP = KP_, KT = KT_, NW = CW * KP, R = 32 * CW, TPI = KP * KT;
  static constexpr int ES = F32 ? 4 : 2, ROWB = DHP * ES, TILE = 32 * ROWB, STAGE = TPI * 2 * TILE;
  static constexpr int RQ = TILE / 1024, NREQ = TPI * 2 * RQ / NW;  // requests of 1 KB per tile, per wavefront and stage
  static constexpr int DT = DHP / 32, QU = ROWB / 32;               // dh tiles of O; 32-byte steps of a row
  static constexpr int PART = (DT * 16 + 2) * 64 * 4;               // O, m, l of a wavefront
  static constexpr int JOIN = (KP - 1) * CW * PART;
  static constexpr int LDS = 2 * STAGE > JOIN ? 2 * STAGE : JOIN;
  static_assert(TPI * 2 * RQ % NW == 0 && LDS <= 160 * 1024, "requests in equal shares; fits the LDS");
  // 16-byte chunk c of row r lies at chunk c ^ f(r).  K: the LDS serves lanes l .. l+7 with l+16 .. l+23 together, which read
  // the same chunk of rows r .. r+7 and r+16 .. r+23 - 16 places of 16 bytes.  V, bf16: 32 lanes read 8 bytes each of four
  // chunks of four consecutive rows; float: 32 lanes read a row's 128 bytes, the others those of the row four further.
  static __device__ __forceinline__ int fk(int r) {
    return ROWB == 128 ? ((r >> 1) & 3) | (((r >> 4) & 1) << 2) : (r & 7) | (((r >> 4) & 1) << 3);
  }
  static __device__ __forceinline__ int fv(int r) {
    return F32 ? ((r >> 2) & 1) << 3 : (ROWB == 128 ? ((r >> 1) & 1) << 2 : (r & 3) << 2);
  }
};

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((address_space(3))) unsigned char lds_byte;
template <typename T>
__device__ __forceinline__ T lds_read(unsigned int at) { return *(const __attribute__((address_space(3))) T*)at; }
__device__ __forceinline__ s16x4 lds_read_tr(unsigned int at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
}
#endif

template <typename SH, bool OWN>
__global__ __launch_bounds__(64 * SH::NW) void prefix_attn_kernel(PrefixAttnParams p) {
#if defined(__HIP_DEVICE_COMPILE__)  // (buffer descriptors exist on the device only)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int R = SH::R, ROWB = SH::ROWB, TILE = SH::TILE, NREQ = SH::NREQ, DT = SH::DT, QU = SH::QU, TPI = SH::TPI;
  constexpr unsigned int kOutside = 0x40000000u;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave % SH::CW, kp = wave / SH::CW;
  const int c = lane & 31, h2 = lane >> 5;
  const int rb = p.dh * SH::ES;  // bytes of a row

  const Batch t = read_batch(p);
  const Blocks<OWN, R, TPI> blocks = Blocks<OWN, R, TPI>::make(p, t);
  const Deal d = prefix_deal(blocks.units);
  // Workgroups go to the 8 XCDs in turn, each with an L2 of its own: consecutive shares - the row blocks of a key head, which
  // read the same keys - go to the same one.
  static_assert(kPrefixGroups % 8 == 0);
  const int per = (d.groups + 7) / 8, w = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || w >= d.groups) return;
  long long u = uniform(d.begin(w));
  const long long u1 = uniform(d.begin(w + 1));

  // ---- loads: number x of a stage is tile x / (2 RQ), K then V, 1 KB after 1 KB; its place in the tile in memory and in LDS --
  unsigned int voff[NREQ], wplace[NREQ];
#pragma unroll
  for (int j = 0; j < NREQ; ++j) {
    const int x = wave * NREQ + j, part = x % SH::RQ;
    const bool is_v = x / SH::RQ & 1;
    const int row = part * (1024 / ROWB) + lane / (ROWB / 16), chunk = lane % (ROWB / 16);
    voff[j] = chunk * 16 < rb ? (unsigned)(row * rb + chunk * 16) : kOutside;
    wplace[j] = x / SH::RQ * TILE + row * ROWB + ((chunk ^ (is_v ? SH::fv(row) : SH::fk(row))) << 4);
  }
  const unsigned int lds0 = (unsigned)(size_t)(lds_byte*)smem;
  // this lane's place in a K tile (row c, first half of a 32-byte step) and in a V tile
  const unsigned int kplace = c * ROWB + ((h2 ^ SH::fk(c)) << 4);
  unsigned int vplace;
  if constexpr (SH::F32) {
    vplace = 4 * h2 * ROWB + (((c >> 2) ^ (h2 << 3)) << 4) + (c & 3) * 4;  // key 4 h2 (+ 8 (i / 4) + i % 4), dh c (+ 32 t)
  } else {
    // the transposing read: 16 lanes fetch 4 rows x 16 dh, 8 bytes each, and lane s of them receives dh s of the four rows
    const int s = lane & 15, row = 4 * h2 + (s >> 2), chunk = ((c >> 4) << 1) + ((s & 3) >> 1);
    vplace = row * ROWB + ((chunk ^ SH::fv(row)) << 4) + (s & 1) * 8;
  }

  while (u < u1) {
    // ---- which block of rows, which keys -------------------------------------------------------------------------------
    int b = 0, kh, blk, it0, iters, slot;
    if constexpr (OWN) {
      // (sequences without nodes have no units: the last sequence that starts at or before u and has some)
      const unsigned long long some = __builtin_amdgcn_ballot_w64(lane < p.B && blocks.iters > 0 && blocks.blocks > 0 && blocks.unit0 <= u);
      b = 63 - __builtin_clzll(some);
      iters = __builtin_amdgcn_readlane(blocks.iters, b);
      const int nb = __builtin_amdgcn_readlane(blocks.blocks, b);
      const long long rel = u - uniform(__shfl(blocks.unit0, b, 64));
      const int item = uniform((int)(rel / iters));
      it0 = uniform((int)(rel - (long long)item * iters));
      kh = uniform(item / nb);
      blk = item - kh * nb;
      slot = w + __builtin_amdgcn_readlane(blocks.block0, b) + item;
    } else {
      iters = blocks.iters;
      const int item = uniform((int)(u / iters));
      it0 = uniform((int)(u - (long long)item * iters));
      kh = uniform(item / blocks.blocks);
      blk = item - kh * blocks.blocks;
      slot = w + item;
    }
    const long long room = u1 - u;
    const int niter = uniform((int)(iters - it0 < room ? iters - it0 : room));
    u += niter;

    const int n = OWN ? __builtin_amdgcn_readlane(t.n, b) : t.all;  // nodes behind the rows
    int L;
    const unsigned char *kc, *vc, *kt = nullptr, *vt = nullptr;
    if constexpr (OWN) {
      L = __builtin_amdgcn_readlane(t.ctx, b);
      const size_t at = ((size_t)uniform((long long)p.kv_off[b]) + (size_t)kh * p.kv_cap * p.dh) * SH::ES;
      kc = p.k_cache + at;
      vc = p.v_cache + at;
      const size_t ta = ((size_t)b * p.H_kv + kh) * p.max_nodes * rb;
      kt = p.k_tree + ta;
      vt = p.v_tree + ta;
    } else {
      L = uniform(*p.prefix_len);
      L = L > p.prefix_cap ? p.prefix_cap : L;
      kc = p.k_prefix + (size_t)kh * p.prefix_cap * rb;
      vc = p.v_prefix + (size_t)kh * p.prefix_cap * rb;
    }
    kc = uniform(kc); vc = uniform(vc); kt = uniform(kt); vt = uniform(vt);
    const int ctx_tiles = (L + 31) / 32;

    // ---- this lane's query row -------------------------------------------------------------------------------------------
    const int r = blk * R + rg * 32 + c;
    const bool live = r < n * p.group;
    const bool live_wave = blk * R + rg * 32 < n * p.group;
    u32x4 qf[QU];
    unsigned long long mw0 = 0, mw1 = 0;
    {
      int node = r / p.group, bq = b;
      const int hg = r - node * p.group;
      if constexpr (!OWN) {
        bq = 0;
        for (int i = 1; i < p.B; ++i) bq += node >= __builtin_amdgcn_readlane(t.first, i) ? 1 : 0;
        // (sequences without nodes begin where the next one does: the last of them that begins here has the node)
        node -= __shfl(t.first, bq, 64);
      }
      const unsigned char* qrow = p.q + (((size_t)bq * p.H + kh * p.group + hg) * p.max_nodes + node) * rb;
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int at = (2 * i + h2) * 16;
        qf[i] = u32x4{0u, 0u, 0u, 0u};
        if (live && at < rb) qf[i] = *(const u32x4*)(qrow + at);
      }
      if (OWN && live) {
        const int W = (p.max_nodes + 63) >> 6;
        const unsigned long long* m = p.anc_mask + ((size_t)b * p.max_nodes + node) * W;
        mw0 = m[0];
        if (W > 1) mw1 = m[1];
      }
    }

    // ---- the tiles of iteration i of this segment into registers, and from there into a stage ------------------------------
    // (The bases are parameters: captured, the choice between them becomes one between their addresses, in scratch memory.
    // Loads straight into LDS are not an option: the compiler lets every transposing read wait for all of them.)
    u32x4 ld[NREQ];
    auto load = [&](int i, const unsigned char* kc, const unsigned char* vc, const unsigned char* kt, const unsigned char* vt)
        __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NREQ; ++j) {
        const int x = wave * NREQ + j, tile = x / (2 * SH::RQ);
        const bool is_v = x / SH::RQ & 1;
        const int k = (it0 + (i < niter ? i : niter - 1)) * TPI + tile;  // (behind the last iteration: the last one again)
        const bool tree = OWN && k >= ctx_tiles;
        const int row0 = (tree ? k - ctx_tiles : k) * 32;
        int left = (tree ? n : L) - row0;  // rows behind the last key: zeros, nothing is read
        left = left < 0 ? 0 : (left > 32 ? 32 : left);  // (a vector instruction: hence uniform() below)
        const unsigned char* base = is_v ? (tree ? vt : vc) : (tree ? kt : kc);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)row0 * rb), 0, (unsigned)uniform(left * rb), 0x00020000);
        ld[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff[j], 0, 0));
      }
    };
    auto commit = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NREQ; ++j) *(__attribute__((address_space(3))) u32x4*)(lds0 + stage * SH::STAGE + wplace[j]) = ld[j];
    };

    f32x16 o[DT];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

    // one tile: S^T = K Q^T with the keys as rows - a lane then holds 16 scores of one query row, its neighbour 32 lanes away
    // the other 16 -, P in the same registers is the right operand of O^T += V^T P
    auto compute = [&](int k, unsigned int tile, unsigned long long mw0, unsigned long long mw1) __attribute__((always_inline)) {
      const bool tree = OWN && k >= ctx_tiles;
      const int left = (tree ? n - (k - ctx_tiles) * 32 : L - k * 32);
      if (left <= 0) return;
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
      const unsigned int ka = tile + kplace, va = tile + TILE + vplace;
      // (the fragments of up to 8 steps are requested together)
#pragma unroll
      for (int i0 = 0; i0 < QU; i0 += 8) {
        u32x4 a[QU < 8 ? QU : 8];
#pragma unroll
        for (int i = 0; i < 8 && i < QU; ++i) a[i] = lds_read<u32x4>(ka ^ ((i0 + i) << 5));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 8 && i < QU; ++i) {
          if constexpr (SH::F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i][e]), __uint_as_float(qf[i0 + i][e]), s, 0, 0, 0);
          } else {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, qf[i0 + i]), s, 0, 0, 0);
          }
        }
      }
      // V^T fragments: requested under the softmax
      s16x8 v[SH::F32 ? 1 : DT][2];
      if constexpr (!SH::F32) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const s16x4 v0 = lds_read_tr((va ^ (dt << 6)) + 16 * kb * ROWB), v1 = lds_read_tr((va ^ (dt << 6)) + (16 * kb + 8) * ROWB);
            v[dt][kb] = s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      // register i, half h2: key 8 (i / 4) + 4 h2 + i % 4
      unsigned int vis = 0xffffffffu;
      if (tree || left < 32) {
        vis = left >= 32 ? 0xffffffffu : ((1u << left) - 1u);
        if (tree) {
          const int row0 = (k - ctx_tiles) * 32;
          vis &= (unsigned int)((row0 < 64 ? mw0 : mw1) >> (row0 & 63));
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (vis >> (8 * (i / 4) + 4 * h2 + i % 4)) & 1u ? s[i] : -INFINITY;
      }
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      // The reference only has to be near the maximum: it is moved when a score exceeds it by more than 2^8, so that P stays
      // below 256; the two lanes of a row then agree on the larger.
      if (__builtin_amdgcn_ballot_w64((mx - m_run) * p.sl2 > 8.0f) != 0ull) {
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if ((mx - m_run) * p.sl2 > 8.0f) {
          const float alpha = __builtin_amdgcn_exp2f((m_run - mx) * p.sl2);  // 0 on first use
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
          m_run = mx;
        }
      }
      const float ms = (m_run > -INFINITY ? m_run : 0.f) * p.sl2;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], p.sl2, -ms));
        sum += s[i];
      }
      l_run += sum;
      // A value that is no number or infinite must not reach the rows that do not see its key, and 0 times it is no number: in
      // a tile of tree nodes such values take part as 0 and are added afterwards where they are seen.
      bool odd = false;
      if constexpr (SH::F32) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float a = lds_read<float>((va ^ (dt << 7)) + (8 * (i / 4) + i % 4) * ROWB);
            if (tree) {
              const bool bad = (__float_as_uint(a) & 0x7f800000u) == 0x7f800000u;
              odd |= bad;
              a = bad ? 0.f : a;
            }
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, s[i], o[dt], 0, 0, 0);
          }
      } else {
        u32x4 hi[2], lo[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p0 = s[2 * i], p1 = s[2 * i + 1];
          if constexpr (SH::FINE) {
            // P = hi + lo: hi is P cut to its upper 16 bits, lo the rounded rest
            const unsigned int u0 = __float_as_uint(p0), u1b = __float_as_uint(p1);
            hi[i / 4][i % 4] = __builtin_amdgcn_perm(u1b, u0, 0x07060302u);
            lo[i / 4][i % 4] = __builtin_bit_cast(
                unsigned int, bf16x2{(__bf16)(p0 - __uint_as_float(u0 & 0xffff0000u)), (__bf16)(p1 - __uint_as_float(u1b & 0xffff0000u))});
          } else {
            // rounded to bf16, as the values are and as the result will be
            hi[i / 4][i % 4] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)p0, (__bf16)p1});
          }
        }
        if (tree) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const bool bad = (v[dt][kb][e] & 0x7f80) == 0x7f80;
                odd |= bad;
                v[dt][kb][e] = bad ? (short)0 : v[dt][kb][e];
              }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[dt][kb]), __builtin_bit_cast(bf16x8, hi[kb]), o[dt], 0, 0, 0);
        if constexpr (SH::FINE) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
              o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[dt][kb]), __builtin_bit_cast(bf16x8, lo[kb]), o[dt], 0, 0, 0);
        }
      }
      if (tree && __builtin_amdgcn_ballot_w64(odd) != 0ull) {
        for (int key = 0; key < (left < 32 ? left : 32); ++key) {
          const bool seen = (vis >> key) & 1u;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int at = (32 * dt + 8 * (i / 4) + 4 * h2 + i % 4) * SH::ES;
              const unsigned int place = tile + TILE + key * ROWB + (((at >> 4) ^ SH::fv(key)) << 4) + (at & 15);
              float v;
              if constexpr (SH::F32) v = lds_read<float>(place);
              else v = bf16_bits_to_float(lds_read<unsigned short>(place));
              if (seen && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[dt][i] += v;
            }
        }
      }
    };

    // ---- the loop: two stages; the next iteration's tiles are in registers, and in LDS behind the first of this one's ------
    load(0, kc, vc, kt, vt);
    commit(0);
    load(1, kc, vc, kt, vt);
    lds_barrier();
    for (int i = 0; i < niter; ++i) {
      const int stage = i & 1;
#pragma unroll
      for (int q = 0; q < SH::KT; ++q) {
        if (live_wave)
          compute((it0 + i) * TPI + kp * SH::KT + q, lds0 + stage * SH::STAGE + (kp * SH::KT + q) * 2 * TILE, mw0, mw1);
        if (q == 0) {
          commit(stage ^ 1);
          load(i + 2, kc, vc, kt, vt);
        }
      }
      lds_barrier();  // (not __syncthreads(): the loads stay in flight)
    }

    // ---- the key parts of a row group joined ------------------------------------------------------------------------------
    if constexpr (SH::KP > 1) {
      float* part = (float*)smem;
      if (kp > 0) {
        float* mine = part + ((kp - 1) * SH::CW + rg) * (SH::PART / 4) + lane * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) *(f32x4*)(mine + (dt * 4 + i) * 256) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        float* ml = part + ((kp - 1) * SH::CW + rg) * (SH::PART / 4) + DT * 16 * 64;
        ml[lane] = m_run;
        ml[64 + lane] = l_run;
      }
      __syncthreads();
      if (kp == 0) {
        for (int q = 0; q < SH::KP - 1; ++q) {
          const float* its = part + (q * SH::CW + rg) * (SH::PART / 4);
          const float mo = its[DT * 16 * 64 + lane], lo = its[DT * 16 * 64 + 64 + lane];
          const float m = fmaxf(m_run, mo), base = m > -INFINITY ? m : 0.f;
          const float a0 = __builtin_amdgcn_exp2f((m_run - base) * p.sl2), a1 = __builtin_amdgcn_exp2f((mo - base) * p.sl2);
          l_run = l_run * a0 + lo * a1;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 v = *(const f32x4*)(its + lane * 4 + (dt * 4 + i) * 256);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[dt][4 * i + e] = o[dt][4 * i + e] * a0 + v[e] * a1;
            }
          m_run = m;
        }
      }
      __syncthreads();  // (the next segment's requests write there)
    }
    // ---- what the segment leaves, in the order of the registers -------------------------------------------------------------
    if (kp == 0 && live_wave) {
      l_run += __shfl_xor(l_run, 32, 64);
      float* po = p.po + ((size_t)slot * SH::CW + rg) * (DT * 1024) + lane * 4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) *(f32x4*)(po + (dt * 4 + i) * 256) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
      if (h2 == 0) {
        float* ml = p.pml + (size_t)slot * 2 * R + rg * 32 + c;
        ml[0] = m_run * p.sl2;
        ml[R] = l_run;
      }
    }
  }
#endif
}

// ---- the join ------------------------------------------------------------------------------------------------------------
struct PrefixJoinParams {
  PrefixAttnParams a;
  const float *prefix_o, *prefix_ml, *own_o, *own_ml;
  int out_bf16;
  void* out;   // [B][H][max_nodes][dh]
  float* lse;  // [B][H][max_nodes] or null
};

// One workgroup of DHP / 32 wavefronts per (32 rows of a sequence, key head): every wavefront weighs the rows' partial results
// and adds up 32 components of them, in ascending order of the slots.
template <int DHP, int RP, int RO, int TPIP, int TPIO>
__global__ __launch_bounds__(2 * DHP) void prefix_join_kernel(PrefixJoinParams p) {
  constexpr int DT = DHP / 32;
  const int lane = threadIdx.x & 63, dt = threadIdx.x >> 6, c = lane & 31, h2 = lane >> 5;
  const int kh = blockIdx.y, b = blockIdx.z, r = blockIdx.x * 32 + c;
  const Batch t = read_batch(p.a);
  const auto pb = Blocks<false, RP, TPIP>::make(p.a, t);
  const auto ob = Blocks<true, RO, TPIO>::make(p.a, t);
  const int n = __builtin_amdgcn_readlane(t.n, b);
  if ((int)blockIdx.x * 32 >= n * p.a.group) return;
  const bool live = r < n * p.a.group;
  const Deal pd = prefix_deal(pb.units), od = prefix_deal(ob.units);
  // this row's place among all rows of the key head and in its sequence; the slots of its blocks
  const int rr = live ? r : 0;
  const int rp = __builtin_amdgcn_readlane(t.first, b) * p.a.group + rr;
  int w0 = 0, w1 = -1, item = 0;
  if (pb.iters > 0) {
    item = kh * pb.blocks + rp / RP;
    w0 = pd.owner((long long)item * pb.iters);
    w1 = pd.owner((long long)item * pb.iters + pb.iters - 1);
  }
  const int oi = __builtin_amdgcn_readlane(ob.iters, b), onb = __builtin_amdgcn_readlane(ob.blocks, b);
  const int oitem = kh * onb + rr / RO;
  const long long ou = __shfl(ob.unit0, b, 64) + (long long)oitem * oi;
  const int x0 = od.owner(ou), x1 = od.owner(ou + oi - 1), oslot = __builtin_amdgcn_readlane(ob.block0, b) + oitem;
  const float* pml = p.prefix_ml + (size_t)item * 2 * RP + rp % RP;
  const float* oml = p.own_ml + (size_t)oslot * 2 * RO + rr % RO;
  float m = -INFINITY;
  for (int w = w0; w <= w1; ++w) m = fmaxf(m, pml[(size_t)w * 2 * RP]);
  for (int w = x0; w <= x1; ++w) m = fmaxf(m, oml[(size_t)w * 2 * RO]);
  const float base = m > -INFINITY ? m : 0.f;
  const float* po = p.prefix_o + ((size_t)item * (RP / 32) + rp % RP / 32) * (DT * 1024) + dt * 1024 + (h2 * 32 + rp % 32) * 4;
  const float* oo = p.own_o + ((size_t)oslot * (RO / 32) + rr % RO / 32) * (DT * 1024) + dt * 1024 + (h2 * 32 + rr % 32) * 4;
  float l = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int w = w0; w <= w1; ++w) {
    const float a = __builtin_amdgcn_exp2f(pml[(size_t)w * 2 * RP] - base);
    l += a * pml[(size_t)w * 2 * RP + RP];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += a * *(const f32x4*)(po + (size_t)w * (RP / 32) * (DT * 1024) + i * 256);
  }
  for (int w = x0; w <= x1; ++w) {
    const float a = __builtin_amdgcn_exp2f(oml[(size_t)w * 2 * RO] - base);
    l += a * oml[(size_t)w * 2 * RO + RO];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += a * *(const f32x4*)(oo + (size_t)w * (RO / 32) * (DT * 1024) + i * 256);
  }
  if (!live) return;
  const int node = r / p.a.group, hg = r - node * p.a.group;
  const size_t row = ((size_t)b * p.a.H + kh * p.a.group + hg) * p.a.max_nodes + node;
  const bool none = m == -INFINITY && l == 0.f;  // no key at all
  const float inv = none ? 0.f : 1.0f / l;
  if (p.lse && dt == 0 && h2 == 0) p.lse[row] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = 32 * dt + 8 * i + 4 * h2;
    if (at >= p.a.dh) continue;
    const f32x4 v = o[i] * inv;
    if (p.out_bf16) {
      *(u32x2*)((unsigned short*)p.out + row * p.a.dh + at) = u32x2{__builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[0], (__bf16)v[1]}),
                                                                    __builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[2], (__bf16)v[3]})};
    } else {
      *(f32x4*)((float*)p.out + row * p.a.dh + at) = v;
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
template <bool F32, int DHP, int R, bool FINE>
struct ShapeFor;
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 256, FINE> { using type = PrefixShape<false, DHP, 8, 1, 2, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 128, FINE> { using type = PrefixShape<false, DHP, 4, 2, 1, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 64, FINE> { using type = PrefixShape<false, DHP, 2, 4, 1, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 32, FINE> { using type = PrefixShape<false, DHP, 1, 4, 1, FINE>; };
template <int DHP> struct ShapeFor<true, DHP, 128, true> { using type = PrefixShape<true, DHP, 4, 1, 1, true>; };
template <int DHP> struct ShapeFor<true, DHP, 32, true> { using type = PrefixShape<true, DHP, 1, 2, 1, true>; };

// f(shape tag) for the shape that R, dh, the type and the precision of P ask for
template <bool F32, int DHP, bool FINE, typename F>
static hipError_t with_rows(int rows, F&& f) {
  if constexpr (F32) {
    return rows == 32 ? f(typename ShapeFor<true, DHP, 32, true>::type{}) : f(typename ShapeFor<true, DHP, 128, true>::type{});
  } else {
    switch (rows) {
      case 32: return f(typename ShapeFor<false, DHP, 32, FINE>::type{});
      case 64: return f(typename ShapeFor<false, DHP, 64, FINE>::type{});
      case 128: return f(typename ShapeFor<false, DHP, 128, FINE>::type{});
      default: return f(typename ShapeFor<false, DHP, 256, FINE>::type{});
    }
  }
}
template <typename F>
static hipError_t with_shape(bool f32, int dhp, bool fine, int rows, F&& f) {
  if (f32) return dhp == 64 ? with_rows<true, 64, true>(rows, f) : with_rows<true, 128, true>(rows, f);
  if (dhp == 64) return fine ? with_rows<false, 64, true>(rows, f) : with_rows<false, 64, false>(rows, f);
  return fine ? with_rows<false, 128, true>(rows, f) : with_rows<false, 128, false>(rows, f);
}

hipError_t prepare_prefix_attn() {
  hipError_t e = hipSuccess;
  for (int f32 = 0; f32 < 2; ++f32)
    for (int dhp = 64; dhp <= 128; dhp += 64)
      for (int fine = f32; fine < 2; ++fine)
        for (int rows = 32; rows <= 256; rows *= 2) {
          if (e != hipSuccess || (f32 && rows != 32 && rows != 128)) continue;
          e = with_shape(f32, dhp, fine, rows, [](auto shape) {
            using SH = decltype(shape);
            const hipError_t e1 = hipFuncSetAttribute((const void*)prefix_attn_kernel<SH, false>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
            return e1 != hipSuccess ? e1 : hipFuncSetAttribute((const void*)prefix_attn_kernel<SH, true>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
          });
        }
  return e;
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" size_t prefix_verify_attn_workspace_bytes(int B, int H, int H_kv, int dh, int max_nodes) {
  if (B < 1 || H < 1 || H_kv < 1 || H % H_kv || dh < 1 || max_nodes < 1) return 0;
  const size_t a = prefix_workspace(B, H, H_kv, dh, max_nodes, false).total, f = prefix_workspace(B, H, H_kv, dh, max_nodes, true).total;
  return a > f ? a : f;
}

extern "C" int prefix_verify_attn(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* q, const void* k_prefix, const void* v_prefix,
                                  const int32_t* prefix_len, int prefix_cap, const void* k_cache, const void* v_cache,
                                  const int64_t* kv_off, const int32_t* ctx_len, int kv_cap, const void* k_tree, const void* v_tree,
                                  const int32_t* n_nodes, const uint64_t* anc_mask, int B, int H, int H_kv, int dh, int max_nodes,
                                  float scale, void* workspace, size_t workspace_bytes, ctcspec_dtype out_dt, void* out, float* lse) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, q && k_prefix && v_prefix && prefix_len && k_cache && v_cache && kv_off && ctx_len && k_tree && v_tree &&
                           n_nodes && anc_mask && workspace && out,
                  CTCSPEC_EINVAL, "prefix_verify_attn: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && H > 0 && H_kv > 0 && dh > 0 && max_nodes > 0 && prefix_cap >= 0 && kv_cap >= 0, CTCSPEC_EINVAL,
                  "prefix_verify_attn: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, H % H_kv == 0, CTCSPEC_EINVAL, "prefix_verify_attn: H must be a multiple of H_kv");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "prefix_verify_attn: unknown element type");
  CTCSPEC_REQUIRE(ctx, out_dt == CTCSPEC_F32 || (out_dt == CTCSPEC_BF16 && dt == CTCSPEC_BF16), CTCSPEC_EINVAL,
                  "prefix_verify_attn: the output is float, or bf16 with bf16 operands");
  CTCSPEC_REQUIRE(ctx, scale > 0.f && scale <= 3.0e38f, CTCSPEC_EINVAL, "prefix_verify_attn: the scale must be positive and finite");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && max_nodes <= CTCSPEC_MAX_NODES, CTCSPEC_EUNSUPPORTED,
                  "prefix_verify_attn: dh must be a multiple of 8 and <= %d, max_nodes <= %d", CTCSPEC_MAX_HEAD_DIM, CTCSPEC_MAX_NODES);
  CTCSPEC_REQUIRE(ctx, B <= ctx->lim.max_batch && B <= 64 && max_nodes <= ctx->lim.max_nodes && H <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim && H_kv <= 65535,
                  CTCSPEC_EUNSUPPORTED, "prefix_verify_attn: shape exceeds the context's limits");
  for (const void* a : {q, k_prefix, v_prefix, k_cache, v_cache, k_tree, v_tree, (const void*)workspace, (const void*)out})
    CTCSPEC_REQUIRE(ctx, aligned16(a), CTCSPEC_EINVAL, "prefix_verify_attn: pointers must be 16-byte aligned");
  const bool f32 = dt == CTCSPEC_F32, fine = out_dt == CTCSPEC_F32;
  const PrefixWorkspace ws = prefix_workspace(B, H, H_kv, dh, max_nodes, f32);
  CTCSPEC_REQUIRE(ctx, workspace_bytes >= ws.total, CTCSPEC_EINVAL, "prefix_verify_attn: workspace of %zu bytes needed, %zu given",
                  ws.total, workspace_bytes);

  unsigned char* base = (unsigned char*)workspace;
  PrefixJoinParams j;
  PrefixAttnParams& p = j.a;
  p.q = (const unsigned char*)q;
  p.k_prefix = (const unsigned char*)k_prefix; p.v_prefix = (const unsigned char*)v_prefix; p.prefix_len = prefix_len;
  p.k_cache = (const unsigned char*)k_cache; p.v_cache = (const unsigned char*)v_cache; p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.k_tree = (const unsigned char*)k_tree; p.v_tree = (const unsigned char*)v_tree; p.n_nodes = n_nodes;
  p.anc_mask = (const unsigned long long*)anc_mask;
  p.prefix_cap = prefix_cap; p.kv_cap = kv_cap; p.B = B; p.H = H; p.H_kv = H_kv; p.group = H / H_kv; p.dh = dh; p.max_nodes = max_nodes;
  p.sl2 = scale * 1.4426950408889634f;
  j.prefix_o = (float*)(base + ws.prefix_o); j.prefix_ml = (float*)(base + ws.prefix_ml);
  j.own_o = (float*)(base + ws.own_o); j.own_ml = (float*)(base + ws.own_ml);
  j.out_bf16 = out_dt == CTCSPEC_BF16; j.out = out; j.lse = lse;
  const int dhp = prefix_padded_dim(dh);
  hipStream_t st = ctx->stream;
  const hipError_t e = with_shape(f32, dhp, fine, ws.prefix_rows, [&](auto prefix_shape) {
    using SP = decltype(prefix_shape);
    p.po = (float*)(base + ws.prefix_o);
    p.pml = (float*)(base + ws.prefix_ml);
    hipLaunchKernelGGL((prefix_attn_kernel<SP, false>), dim3(kPrefixGroups), dim3(64 * SP::NW), SP::LDS, st, p);
    if (const hipError_t e1 = hipGetLastError(); e1 != hipSuccess) return e1;
    return with_rows<SP::F32, SP::DHP, SP::FINE>(ws.own_rows, [&](auto own_shape) {
      using SO = decltype(own_shape);
      if constexpr (SO::R > SP::R) {
        return hipErrorInvalidValue;  // (one sequence's rows are among all rows)
      } else {
        p.po = (float*)(base + ws.own_o);
        p.pml = (float*)(base + ws.own_ml);
        hipLaunchKernelGGL((prefix_attn_kernel<SO, true>), dim3(kPrefixGroups), dim3(64 * SO::NW), SO::LDS, st, p);
        if (const hipError_t e1 = hipGetLastError(); e1 != hipSuccess) return e1;
        hipLaunchKernelGGL((prefix_join_kernel<SP::DHP, SP::R, SO::R, SP::TPI, SO::TPI>),
                           dim3((unsigned)((max_nodes * p.group + 31) / 32), (unsigned)H_kv, (unsigned)B), dim3(2 * SP::DHP), 0, st, j);
        return hipGetLastError();
      }
    });
  });
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
