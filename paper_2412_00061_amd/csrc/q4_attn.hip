// q4_verify_attn: verification attention over a cache held in 4 bits (q4_format.h), with or without a sliding window, one layer.
//
//   out[b,h,i] = sum_j p_j v_j,  p = softmax over the cached keys and the tree nodes that row i sees
//
// What the codes stand for is exact in bf16, so a tile of keys becomes operands of the matrix instructions by conversions alone: a lane
// has 32 elements of a block, one scale, and its keys need no way through the LDS - which elements of a row form which step of a product is
// free, as long as the query's lanes hold the same.  Values are needed by columns: they are converted, written to the LDS a row at a time
// and fetched by transposing reads, each wavefront its own tile, so the loop has no barriers.
//
// The work - iterations of four tiles, one for each wavefront, of a block of rows - is dealt to the workgroups in equal shares
// (prefix_plan.h); the four wavefronts' results are joined in the LDS, the shares' by a second kernel.
#include <type_traits>

#include "q4_format.h"
#include "q4_plan.h"

namespace ctcspec {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

struct Q4AttnParams {
  const unsigned char* q;         // [B][H][max_nodes][dh]
  const unsigned char* k_codes;
  const unsigned char* k_scales;
  const unsigned char* v_codes;
  const unsigned char* v_scales;
  const int64_t* kv_off;          // in rows
  const int32_t* ctx_len;
  const unsigned char* k_tree;    // [B][H_kv][max_nodes][dh]
  const unsigned char* v_tree;
  const int32_t* n_nodes;
  const int32_t* depth;           // [B][max_nodes]; null without a window
  const unsigned long long* anc_mask;
  int kv_cap, B, H, H_kv, group, dh, blocks, max_nodes, window, sink;  // group: heads that share a key head; blocks: of 32 elements, of a row
  float sl2;                      // scale * log2(e)
  float* po;                      // partial O: [slot][rows / 32][DT][4][64 lanes][4]
  float* pml;                     // [slot][2][rows]: maximum in the log2 domain, sum
  int* odd;                       // [slot]: a value of a tree node is infinite or not a number
  int out_bf16;
  void* out;                      // [B][H][max_nodes][dh]
  float* lse;                     // [B][H][max_nodes] or null
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// QT: blocks of 32 rows; DT: blocks of 32 components (at least 2).  FINE: weights in three bf16 parts.
template <int QT_, int DT_, bool FINE_>
struct Q4Shape {
  static constexpr int QT = QT_, DT = DT_, R = 32 * QT, NW = kQ4Tiles;
  static constexpr bool FINE = FINE_;
  static constexpr int KB = (DT + 1) / 2, QU = 4 * KB;        // blocks of a key in a lane; steps of 16 elements of a product
  static constexpr int VB = (DT + 1) / 2;                     // blocks of values in a lane: 32 DT of them in 64 lanes
  static constexpr int ROWB = DT <= 2 ? 128 : 256, TILE = 32 * ROWB;  // values in the LDS
  static constexpr int PART = (DT * 16 + 2) * 64 * 4;         // O, m, l of 32 rows
  static constexpr int STAGE = NW * TILE > 2 * QT * PART ? NW * TILE : 2 * QT * PART;
  static constexpr int LDS = STAGE + 6 * 64 * 4;              // and the sequences' table: behind the tiles, whose places are formed by xor
  static constexpr int WPE = QT == 1 ? 2 : 1, GROUPS = QT == 1 ? 512 : 256;
  static_assert(2 * LDS <= 160 * 1024 && GROUPS <= kPrefixMaxGroups && GROUPS % 8 == 0);
  // 16-byte chunk c of row r lies at chunk c ^ place(r).  A transposing read of 32 lanes takes four chunks of each of four consecutive
  // rows: these differ in the chunk's upper bits (rows of 128 bytes: in every second row).  A write of eight lanes takes the same chunk of
  // a block from rows that are four apart: these differ in its lower bits.
  static __device__ __forceinline__ int place(int r) { return (ROWB == 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2) ^ ((r >> 2) & 3); }
  // the block of values that a lane converts as its u-th: row and block of the row
  static __device__ __forceinline__ int v_row(int x) {
    if constexpr (DT == 2) {
      const int a = x >> 1;
      return (a & 1) | ((a >> 1) & 7) << 2 | ((a >> 4) & 1) << 1;
    } else {
      const int a = x / DT;
      return (a & 7) << 2 | a >> 3;
    }
  }
  static __device__ __forceinline__ int v_block(int x) { return x % DT; }
};

// What both kernels know about the work: lane b holds sequence b's part (the limits allow 64 sequences), the rest is uniform.
struct Q4Work {
  int n, ctx, iters, blocks;     // lane: nodes, cached rows, iterations over its keys, blocks of its rows
  int unit0, block0;             // lane: units and blocks of the sequences before it, for one key head
  int head_units, head_blocks;   // of a key head
  int units;                     // of all key heads
};
template <typename SH>
__device__ __forceinline__ Q4Work q4_read_work(const Q4AttnParams& p) {
  const int lane = threadIdx.x & 63;
  Q4Work t{};
  if (lane < p.B) {
    const int n = p.n_nodes[lane], L = p.ctx_len[lane];
    t.n = n < 0 ? 0 : (n > p.max_nodes ? p.max_nodes : n);
    t.ctx = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  }
  t.blocks = (t.n * p.group + SH::R - 1) / SH::R;
  t.iters = t.n ? (q4_tiles(t.ctx, p.window, p.sink).count + (t.n + 31) / 32 + kQ4Tiles - 1) / kQ4Tiles : 0;
  const int mine = t.blocks * q4_units(t.iters);
  int b = t.blocks, u = mine;
  for (int d = 1; d < p.B; d *= 2) {
    const int bb = __shfl_up(b, d, 64), ub = __shfl_up(u, d, 64);
    if (lane >= d) { b += bb; u += ub; }
  }
  t.block0 = b - t.blocks;
  t.unit0 = u - mine;
  t.head_blocks = __builtin_amdgcn_readlane(b, p.B - 1);
  t.head_units = __builtin_amdgcn_readlane(u, p.B - 1);
  t.units = p.H_kv * t.head_units;
  return t;
}

// Row `node`'s depth, and the nodes that it sees: its mask row's, of these with a window those near enough or in the sink.
__device__ __forceinline__ int q4_depth(const Q4AttnParams& p, int b, int node) {
  const int d = p.depth[(size_t)b * p.max_nodes + node];
  return d < 0 ? 0 : (d >= p.max_nodes ? p.max_nodes - 1 : d);
}
struct Q4Mask {
  unsigned long long low, high;  // nodes 0 to 63, 64 to 127
  __device__ __forceinline__ unsigned int tile(int i) const { return (unsigned int)((i < 2 ? low : high) >> (32 * (i & 1))); }
  __device__ __forceinline__ bool node(int j) const { return ((j < 64 ? low : high) >> (j & 63)) & 1ull; }
};
__device__ __forceinline__ Q4Mask q4_tree_mask(const Q4AttnParams& p, int b, int node, int n, int L, int depth) {
  const int W = (p.max_nodes + 63) >> 6;
  const unsigned long long* row = p.anc_mask + ((size_t)b * p.max_nodes + node) * W;
  Q4Mask m = {row[0], W > 1 ? row[1] : 0ull};
  m.low &= n >= 64 ? ~0ull : (1ull << n) - 1;
  m.high &= n >= 128 ? ~0ull : (n > 64 ? (1ull << (n - 64)) - 1 : 0ull);
  // (no node is max_nodes deep: a longer window holds every node for every row)
  if (p.window > 0 && p.window < p.max_nodes) {
    for (int j = 0; j < n; ++j) {
      const int dj = q4_depth(p, b, j);
      const unsigned long long out = depth - dj >= p.window && L + dj >= p.sink ? 1ull << (j & 63) : 0ull;
      m.low &= j < 64 ? ~out : ~0ull;
      m.high &= j < 64 ? ~0ull : ~out;
    }
  }
  return m;
}

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((address_space(3))) unsigned char lds_byte;
__device__ __forceinline__ s16x4 lds_read_tr(unsigned int at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
}
#endif

template <typename SH>
__global__ __launch_bounds__(64 * SH::NW, SH::WPE) void q4_attn_kernel(Q4AttnParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int R = SH::R, QT = SH::QT, DT = SH::DT, KB = SH::KB, VB = SH::VB, QU = SH::QU, ROWB = SH::ROWB;
  const int lane = threadIdx.x & 63, c = lane & 31, h2 = lane >> 5;
  const int wave = uniform(threadIdx.x >> 6);
  const Q4Work t = q4_read_work<SH>(p);
  const Deal d = prefix_deal(t.units, SH::GROUPS);
  // (consecutive shares - neighbouring keys - to the same of the 8 XCDs)
  const int per = (d.groups + 7) / 8, w = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || w >= d.groups) return;
  int u = uniform(d.begin(w));
  const int u1 = uniform(d.begin(w + 1));

  // What the lanes know about the sequences, out of the registers while the keys go by; and a flag.
  int(*table)[64] = (int(*)[64])(smem + SH::STAGE);
  enum { kNodes, kCtx, kIters, kUnit0, kBlock0, kOdd };
  if (wave == 0) {
    table[kNodes][lane] = t.n;
    table[kCtx][lane] = t.ctx;
    table[kIters][lane] = t.iters;
    table[kUnit0][lane] = t.unit0;
    table[kBlock0][lane] = t.block0;
  }
  __syncthreads();
  const int head_units = t.head_units, head_blocks = t.head_blocks;
  unsigned char* vtile = smem + wave * SH::TILE;
  const unsigned int vbase = (unsigned int)(size_t)(lds_byte*)vtile;
  // the transposing read: 16 lanes fetch 4 rows x 16 components, 8 bytes each, and lane s of them receives component s of the four rows
  unsigned int vread;
  {
    const int s = lane & 15, row = 4 * h2 + (s >> 2), ch = ((c >> 4) << 1) + ((s & 3) >> 1);
    vread = vbase + row * ROWB + ((ch ^ SH::place(row)) << 4) + (s & 1) * 8;
  }

  while (u < u1) {
    // ---- which block of rows, which keys -------------------------------------------------------------------------------
    int seg_lane = lane;  // (as something new: addresses that only a segment's ends need are formed there)
    asm volatile("" : "+v"(seg_lane));
    const int kh = uniform(u / head_units), in_head = u - kh * head_units;
    // (sequences without nodes have no units: the last sequence that starts at or before the unit and has some)
    const int b = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(table[kIters][seg_lane] > 0 && table[kUnit0][seg_lane] <= in_head));
    const int n = uniform(table[kNodes][b]), L = uniform(table[kCtx][b]);
    const int units = q4_units(uniform(table[kIters][b]));
    const int in_seq = in_head - uniform(table[kUnit0][b]), blk = uniform(in_seq / units), at_unit = in_seq - blk * units;
    const int slot = w + kh * head_blocks + uniform(table[kBlock0][b]) + blk;
    const int share = uniform(units - at_unit < u1 - u ? units - at_unit : u1 - u);
    u += share;
    const int it0 = uniform(prefix_iterations(at_unit, kPrefixOwnWeight, false));
    const int niter = uniform(prefix_iterations(at_unit + share, kPrefixOwnWeight, false)) - it0;
    if (niter <= 0) continue;
    const Q4Tiles tiles = q4_tiles(L, p.window, p.sink);
    const int total = tiles.count + (n + 31) / 32;
    const size_t row0 = (size_t)p.kv_off[b] + (size_t)kh * p.kv_cap;
    const unsigned char* kc = p.k_codes + row0 * (size_t)(p.blocks * kQ4BlockBytes);
    const unsigned char* ks = p.k_scales + row0 * (size_t)p.blocks;
    const unsigned char* vc = p.v_codes + row0 * (size_t)(p.blocks * kQ4BlockBytes);
    const unsigned char* vs = p.v_scales + row0 * (size_t)p.blocks;
    const size_t tree0 = ((size_t)b * p.H_kv + kh) * p.max_nodes * (size_t)(p.dh * 2);

    // ---- this lane's query rows: step i of a product has elements 32 (KB h2 + i / 4) + 8 (i % 4) .. + 7 -----------------------------
    const int c = seg_lane & 31, h2 = seg_lane >> 5;
    u32x4 qf[QT][QU];
    Q4Mask mw[QT];
    int low[QT];  // the first position of the window
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = blk * R + qt * 32 + c;
      // (rows that are none do as row 0 does: nobody reads what comes of it)
      const int live = r < n * p.group ? r : 0, node = live / p.group, hg = live - node * p.group;
      const unsigned char* row = p.q + (((size_t)b * p.H + kh * p.group + hg) * p.max_nodes + node) * (size_t)(p.dh * 2);
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int at = 32 * (KB * h2 + i / 4) + 8 * (i % 4);
        qf[qt][i] = at < p.dh ? *(const u32x4*)(row + at * 2) : u32x4{0u, 0u, 0u, 0u};
      }
      const int depth = p.window > 0 ? q4_depth(p, b, node) : 0;
      low[qt] = L + depth - p.window + 1;
      mw[qt] = q4_tree_mask(p, b, node, n, L, depth);
    }
    f32x16 o[QT][DT];
    float m_run[QT], l_run[QT];
    bool odd = false;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m_run[qt] = -INFINITY;
      l_run[qt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[qt][dt][i] = 0.f;
    }

    // codes and scales of a cached tile: of key c the blocks KB h2 .., of the values blocks lane, lane + 64 (rows behind the last one: the last)
    u32x4 kraw[KB], vraw[VB];
    unsigned int kscale[KB], vscale[VB];
    auto fetch = [&](int x) __attribute__((always_inline)) {
      const int tile = x < tiles.lead ? x : x + tiles.gap, last = L - 1 - 32 * tile;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const int row = 32 * tile + (c < last ? c : last), blk = KB * h2 + k < p.blocks ? KB * h2 + k : p.blocks - 1;
        const size_t at = (size_t)row * p.blocks + blk;
        kraw[k] = *(const u32x4*)(kc + at * kQ4BlockBytes);
        kscale[k] = ks[at];
      }
#pragma unroll
      for (int k = 0; k < VB; ++k) {
        const int y = lane + 64 * k < 32 * DT ? lane + 64 * k : 0, key = SH::v_row(y);
        const int row = 32 * tile + (key < last ? key : last), blk = SH::v_block(y) < p.blocks ? SH::v_block(y) : p.blocks - 1;
        const size_t at = (size_t)row * p.blocks + blk;
        vraw[k] = *(const u32x4*)(vc + at * kQ4BlockBytes);
        vscale[k] = vs[at];
      }
    };

    const int first = it0 * kQ4Tiles + wave, end = (it0 + niter) * kQ4Tiles < total ? (it0 + niter) * kQ4Tiles : total;
    if (first < tiles.count && first < end) fetch(first);
    for (int x = first; x < end; x += kQ4Tiles) {
      const bool tree = x >= tiles.count;
      const int tile = tree ? x - tiles.count : (x < tiles.lead ? x : x + tiles.gap);
      u32x4 a[QU];
      if (!tree) {
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) a[4 * k + e] = q4_decode(kraw[k][e], q4_scale_value((int)kscale[k]));
        // values: block by block into this wavefront's tile
#pragma unroll
        for (int k = 0; k < VB; ++k) {
          const int y = lane + 64 * k, row = SH::v_row(y < 32 * DT ? y : 0), blk = SH::v_block(y < 32 * DT ? y : 0);
          if (y < 32 * DT) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *(u32x4*)(vtile + row * ROWB + (((4 * blk + e) ^ SH::place(row)) << 4)) = q4_decode(vraw[k][e], q4_scale_value((int)vscale[k]));
          }
        }
        if (x + kQ4Tiles < tiles.count && x + kQ4Tiles < end) fetch(x + kQ4Tiles);
      } else {
        // tree nodes: keys as they are, values into the tile as they are (nodes that are none: the last one).  (The lane's number, as
        // something new: what only these tiles need is then formed here, not kept in registers all the way.)
        int fresh = lane;
        asm volatile("" : "+v"(fresh));
        const int c = fresh & 31, h2 = fresh >> 5, key = 32 * tile + c < n ? 32 * tile + c : n - 1;
        const unsigned char* kt = p.k_tree + tree0 + (size_t)key * (p.dh * 2);
        const unsigned char* vt = p.v_tree + tree0;
#pragma unroll
        for (int i = 0; i < QU; ++i) {
          const int at = 32 * (KB * h2 + i / 4) + 8 * (i % 4);
          a[i] = at < p.dh ? *(const u32x4*)(kt + at * 2) : u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {  // 128 DT chunks of 8 components
          const int y = fresh + 64 * i, row = y / (4 * DT), ch = y % (4 * DT), from = 32 * tile + row < n ? 32 * tile + row : n - 1;
          *(u32x4*)(vtile + row * ROWB + ((ch ^ SH::place(row)) << 4)) =
              8 * ch < p.dh ? *(const u32x4*)(vt + (size_t)from * (p.dh * 2) + ch * 16) : u32x4{0u, 0u, 0u, 0u};
        }
      }
      asm volatile("" ::: "memory");

      // S^T = K Q^T: a lane then holds 16 scores of one query row, its neighbour 32 lanes away the other 16 - register i: key
      // 8 (i / 4) + 4 h2 + i % 4 -, and P in the same registers is the right operand of O^T += V^T P
      f32x16 s[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[qt][i] = 0.f;
#pragma unroll
        for (int i = 0; i < QU; ++i)
          s[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, qf[qt][i]), s[qt], 0, 0, 0);
      }
      // ---- keys that are not there or not seen ----------------------------------------------------------------------------
      const bool mixed = tree || 32 * tile + 32 > L || (p.window > 0 && 32 * tile <= L + p.max_nodes - 1 - p.window);
      unsigned int vis[QT];
      if (mixed) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          if (tree) {
            vis[qt] = mw[qt].tile(tile);
          } else {
            const int left = L - 32 * tile;
            vis[qt] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
            if (p.window > 0) {
              const int from = low[qt] - 32 * tile, sunk = p.sink - 32 * tile;
              vis[qt] &= (from <= 0 ? 0xffffffffu : (from >= 32 ? 0u : 0xffffffffu << from)) |
                         (sunk >= 32 ? 0xffffffffu : (sunk <= 0 ? 0u : (1u << sunk) - 1u));
            }
          }
          vis[qt] >>= 4 * h2;  // register i: bit 8 (i / 4) + i % 4
#pragma unroll
          for (int i = 0; i < 16; ++i) s[qt][i] = (vis[qt] >> (8 * (i / 4) + i % 4)) & 1u ? s[qt][i] : -INFINITY;
        }
      }

      // ---- the reference, in the log2 domain, only has to be near the maximum: it is moved when a score exceeds it by more than 2^8 -----
      bool far = false;
      float mx[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = s[qt][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx[qt] = fmaxf(mx[qt], s[qt][i]);
        far |= fmaf(mx[qt], p.sl2, -m_run[qt]) > 8.0f;
      }
      if (__builtin_amdgcn_ballot_w64(far) != 0ull) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const float m = fmaxf(mx[qt], __shfl_xor(mx[qt], 32, 64));
          if (fmaf(m, p.sl2, -m_run[qt]) > 8.0f) {
            const float top = m * p.sl2, alpha = __builtin_amdgcn_exp2f(m_run[qt] - top);  // 0 on first use
            l_run[qt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[qt][dt] *= alpha;
            m_run[qt] = top;
          }
        }
      }
      // ---- weights, and the products with the values ---------------------------------------------------------------------------
      u32x4 hi[QT][2], lo[QT][2], rest[QT][2];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const float ms = m_run[qt] > -INFINITY ? m_run[qt] : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[qt][2 * j], p.sl2, -ms)), p1 = __builtin_amdgcn_exp2f(fmaf(s[qt][2 * j + 1], p.sl2, -ms));
          const unsigned int h = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)p0, (__bf16)p1});
          hi[qt][j / 4][j % 4] = h;
          if constexpr (SH::FINE) {
            const float h0 = __uint_as_float(h << 16), h1 = __uint_as_float(h & 0xffff0000u);
            const unsigned int r = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)(p0 - h0), (__bf16)(p1 - h1)});
            lo[qt][j / 4][j % 4] = r;
            const float r0 = (p0 - h0) - __uint_as_float(r << 16), r1 = (p1 - h1) - __uint_as_float(r & 0xffff0000u);
            rest[qt][j / 4][j % 4] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)r0, (__bf16)r1});
          }
          sum += p0 + p1;
        }
        l_run[qt] += sum;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        u32x4 vr[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const s16x4 v0 = lds_read_tr((vread ^ (dt << 6)) + 16 * kb * ROWB), v1 = lds_read_tr((vread ^ (dt << 6) ^ 32) + (16 * kb + 8) * ROWB);
          vr[dt] = __builtin_bit_cast(u32x4, s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
        }
        if (mixed) {
          // A value that is no number must not reach the rows that do not see its key, and 0 times it is no number: such values take part
          // as 0.  A cached one is NaN and makes the rows that see it NaN: those that a product of marks finds.  What tree nodes have, which
          // may be infinite, is added by the join.
          unsigned int all = 0u;  // exponents of nothing but ones carry into the sign's place
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) all |= (vr[dt][e] & 0x7f807f80u) + 0x00800080u;
          if (__builtin_amdgcn_ballot_w64((all & 0x80008000u) != 0u) != 0ull) {
            odd |= tree;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              u32x4 mark;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const unsigned int t = ((vr[dt][e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                mark[e] = (t >> 15) * 0x3f80u;  // 1 in bf16
                vr[dt][e] &= ~((t >> 15) * 0xffffu);
              }
#pragma unroll
              for (int qt = 0; qt < QT; ++qt) {
                if (tree) continue;
                u32x4 sees;
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // registers 8 kb + 2 e, + 1
                  const int i = 8 * kb + 2 * e, bit = 8 * (i / 4) + i % 4;
                  sees[e] = ((vis[qt] >> bit) & 1u) * 0x3f80u + ((vis[qt] >> (bit + 1)) & 1u) * 0x3f800000u;
                }
                f32x16 count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.f;
                count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, mark), __builtin_bit_cast(bf16x8, sees), count, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[qt][dt][i] = count[i] > 0.f ? __uint_as_float(0x7fc00000u) : o[qt][dt][i];
              }
            }
          }
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, vr[dt]);
            o[qt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, hi[qt][kb]), o[qt][dt], 0, 0, 0);
            if constexpr (SH::FINE) {
              o[qt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, lo[qt][kb]), o[qt][dt], 0, 0, 0);
              o[qt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, rest[qt][kb]), o[qt][dt], 0, 0, 0);
            }
          }
      }
      asm volatile("" ::: "memory");  // (the next tile's values go where these were read)
    }

    // ---- the four wavefronts' parts joined: 2 to 0 and 3 to 1, then 1 to 0 -------------------------------------------------------
    if (threadIdx.x == 0) table[kOdd][0] = 0;
    __syncthreads();  // every tile is consumed: the LDS is free
    if (__builtin_amdgcn_ballot_w64(odd) != 0ull) table[kOdd][0] = 1;
    float* part = (float*)smem;
    asm volatile("" : "+v"(seg_lane));
    const int el = seg_lane;
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float* its = part + ((wave - half) * QT + qt) * (SH::PART / 4);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4*)(its + el * 4 + (dt * 4 + i) * 256) = f32x4{o[qt][dt][4 * i], o[qt][dt][4 * i + 1], o[qt][dt][4 * i + 2], o[qt][dt][4 * i + 3]};
          its[DT * 1024 + el] = m_run[qt];
          its[DT * 1024 + 64 + el] = l_run[qt];
        }
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const float* its = part + (wave * QT + qt) * (SH::PART / 4);
          const float mo = its[DT * 1024 + el], lother = its[DT * 1024 + 64 + el];
          const float m = fmaxf(m_run[qt], mo), base = m > -INFINITY ? m : 0.f;
          const float a0 = __builtin_amdgcn_exp2f(m_run[qt] - base), a1 = __builtin_amdgcn_exp2f(mo - base);
          l_run[qt] = l_run[qt] * a0 + lother * a1;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            __builtin_amdgcn_sched_barrier(0);  // (32 components at a time: all reads ahead do not fit the registers)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 x = *(const f32x4*)(its + el * 4 + (dt * 4 + i) * 256);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[qt][dt][4 * i + e] = o[qt][dt][4 * i + e] * a0 + x[e] * a1;
            }
          }
          m_run[qt] = m;
        }
      }
      __syncthreads();
    }
    if (threadIdx.x == 0) p.odd[slot] = table[kOdd][0];
    // ---- what the segment leaves, in the order of the registers -------------------------------------------------------------
    if (wave == 0) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        l_run[qt] += __shfl_xor(l_run[qt], 32, 64);
        if (blk * R + qt * 32 + (el & 31) < n * p.group) {
          float* po = p.po + ((size_t)slot * QT + qt) * (DT * 1024) + el * 4;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4*)(po + (dt * 4 + i) * 256) = f32x4{o[qt][dt][4 * i], o[qt][dt][4 * i + 1], o[qt][dt][4 * i + 2], o[qt][dt][4 * i + 3]};
          if (el < 32) {
            float* ml = p.pml + (size_t)slot * 2 * R + qt * 32 + el;
            ml[0] = m_run[qt];
            ml[R] = l_run[qt];
          }
        }
      }
    }
  }
#endif
}

// ---- the join ------------------------------------------------------------------------------------------------------------
// One workgroup of DT wavefronts per (32 rows of a sequence, key head): every wavefront weighs the rows' partial results and adds up 32
// components of them, in the order of their keys, four at a time under way.
template <typename SH>
__global__ __launch_bounds__(64 * SH::DT) void q4_join_kernel(Q4AttnParams p) {
  constexpr int DT = SH::DT, R = SH::R;
  const int lane = threadIdx.x & 63, dt = threadIdx.x >> 6, c = lane & 31, h2 = lane >> 5;
  const int kh = blockIdx.y, b = blockIdx.z, r = blockIdx.x * 32 + c;
  const Q4Work t = q4_read_work<SH>(p);
  const int n = __builtin_amdgcn_readlane(t.n, b), L = __builtin_amdgcn_readlane(t.ctx, b);
  if ((int)blockIdx.x * 32 >= n * p.group) return;
  const Deal d = prefix_deal(t.units, SH::GROUPS);
  const int iters = __builtin_amdgcn_readlane(t.iters, b), blk = uniform(blockIdx.x * 32 / R);
  const int first = kh * t.head_units + __builtin_amdgcn_readlane(t.unit0, b) + blk * q4_units(iters) + prefix_block_units(false);
  const int item = kh * t.head_blocks + __builtin_amdgcn_readlane(t.block0, b) + blk;
  const int w0 = d.owner(first), w1 = d.owner(first + (iters - 1) * kPrefixOwnWeight);
  if (r >= n * p.group) return;
  float m = -INFINITY, l = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float* ml = p.pml + (size_t)item * 2 * R + r % R;
  const float* po = p.po + ((size_t)item * (R / 32) + r % R / 32) * (DT * 1024) + dt * 1024 + lane * 4;
  constexpr int kBatch = 4;
  int odd = 0;
  for (int w = w0; w <= w1; w += kBatch) {
    float pm[kBatch], pl[kBatch];
    f32x4 x[kBatch][4];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {  // (behind the last one: the last one again, with no weight)
      const size_t s = w + q < w1 ? w + q : w1;
      pm[q] = ml[s * 2 * R];
      pl[q] = ml[s * 2 * R + R];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[q][i] = *(const f32x4*)(po + s * (R / 32) * (DT * 1024) + i * 256);
      odd |= p.odd[s + item];
    }
    float top = m;
#pragma unroll
    for (int q = 0; q < kBatch; ++q) top = fmaxf(top, pm[q]);
    const float base = top > -INFINITY ? top : 0.f, old = __builtin_amdgcn_exp2f(m - base);
    l *= old;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= old;
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (w + q > w1) continue;
      const float a = __builtin_amdgcn_exp2f(pm[q] - base);
      l += a * pl[q];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += a * x[q][i];
    }
    m = top;
  }
  const int node = r / p.group, hg = r - node * p.group;
  if (odd) {  // values of tree nodes that are infinite or not a number, left out so far: into the rows that see them
    const Q4Mask mask = q4_tree_mask(p, b, node, n, L, p.window > 0 ? q4_depth(p, b, node) : 0);
    const unsigned short* vt = (const unsigned short*)p.v_tree + ((size_t)b * p.H_kv + kh) * p.max_nodes * p.dh;
    for (int j = 0; j < n; ++j) {
      if (!mask.node(j)) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = 32 * dt + 8 * i + 4 * h2 + e;
          if (at >= p.dh) continue;
          const float v = bf16_bits_to_float(vt[(size_t)j * p.dh + at]);
          if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[i][e] += v;
        }
    }
  }
  const size_t row = ((size_t)b * p.H + kh * p.group + hg) * p.max_nodes + node;
  const bool none = m == -INFINITY && l == 0.f;  // no key at all
  const float inv = none ? 0.f : 1.0f / l;
  if (p.lse && dt == 0 && h2 == 0) p.lse[row] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = 32 * dt + 8 * i + 4 * h2;
    if (at >= p.dh) continue;
    const f32x4 v = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[i] * inv;
    if (p.out_bf16) {
      *(u32x2*)((unsigned short*)p.out + row * p.dh + at) = u32x2{__builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[0], (__bf16)v[1]}),
                                                                  __builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[2], (__bf16)v[3]})};
    } else {
      *(f32x4*)((float*)p.out + row * p.dh + at) = v;
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
template <int QT, int DT, typename F>
static hipError_t q4_with_precision(bool fine, F&& f) {
  return fine ? f(Q4Shape<QT, DT, true>{}) : f(Q4Shape<QT, DT, false>{});
}
template <int QT, typename F>
static hipError_t q4_with_dim(int blocks, bool fine, F&& f) {
  return blocks <= 2 ? q4_with_precision<QT, 2>(fine, f) : (blocks == 3 ? q4_with_precision<QT, 3>(fine, f) : q4_with_precision<QT, 4>(fine, f));
}
template <typename F>
static hipError_t q4_with_shape(int rows, int blocks, bool fine, F&& f) {
  return rows == 32 ? q4_with_dim<1>(blocks, fine, f) : q4_with_dim<2>(blocks, fine, f);
}

hipError_t prepare_q4_attn() {
  hipError_t e = hipSuccess;
  for (int rows = 32; rows <= 64; rows *= 2)
    for (int blocks = 2; blocks <= 4; ++blocks)
      for (int fine = 0; fine < 2; ++fine)
        if (e == hipSuccess)
          e = q4_with_shape(rows, blocks, fine, [](auto shape) {
            using SH = decltype(shape);
            return hipFuncSetAttribute((const void*)q4_attn_kernel<SH>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
          });
  return e;
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" size_t q4_verify_attn_workspace_bytes(int B, int H, int H_kv, int dh, int max_nodes) {
  if (B < 1 || H < 1 || H_kv < 1 || H % H_kv || dh < 1 || max_nodes < 1) return 0;
  return q4_workspace(B, H, H_kv, dh, max_nodes).total;
}

extern "C" int q4_verify_attn(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* q, const ctcspec_q4_cache* cache, const int64_t* kv_off,
                              const int32_t* ctx_len, int kv_cap, const void* k_tree, const void* v_tree, const int32_t* n_nodes,
                              const int32_t* node_depth, const uint64_t* anc_mask, int B, int H, int H_kv, int dh, int max_nodes, float scale,
                              int window, int sink, void* workspace, size_t workspace_bytes, ctcspec_dtype out_dt, void* out, float* lse) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, q && cache && kv_off && ctx_len && k_tree && v_tree && n_nodes && anc_mask && workspace && out, CTCSPEC_EINVAL,
                  "q4_verify_attn: null pointer");
  CTCSPEC_REQUIRE(ctx, (cache->k_codes && cache->k_scales && cache->v_codes && cache->v_scales) || kv_cap == 0, CTCSPEC_EINVAL,
                  "q4_verify_attn: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && H > 0 && H_kv > 0 && dh > 0 && max_nodes > 0 && kv_cap >= 0, CTCSPEC_EINVAL, "q4_verify_attn: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, H % H_kv == 0, CTCSPEC_EINVAL, "q4_verify_attn: H must be a multiple of H_kv");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_BF16, CTCSPEC_EUNSUPPORTED, "q4_verify_attn: queries and tree rows are bf16");
  CTCSPEC_REQUIRE(ctx, out_dt == CTCSPEC_F32 || out_dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "q4_verify_attn: unknown element type");
  CTCSPEC_REQUIRE(ctx, scale > 0.f && scale <= 2.0e38f, CTCSPEC_EINVAL, "q4_verify_attn: the scale must be positive and at most 2e38");
  CTCSPEC_REQUIRE(ctx, window >= 0 && sink >= 0, CTCSPEC_EINVAL, "q4_verify_attn: window and sink must not be negative");
  CTCSPEC_REQUIRE(ctx, window == 0 || node_depth, CTCSPEC_EINVAL, "q4_verify_attn: a window needs node_depth");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && max_nodes <= CTCSPEC_MAX_NODES, CTCSPEC_EUNSUPPORTED,
                  "q4_verify_attn: dh must be a multiple of 8 and <= %d, max_nodes <= %d", CTCSPEC_MAX_HEAD_DIM, CTCSPEC_MAX_NODES);
  CTCSPEC_REQUIRE(ctx, B <= ctx->lim.max_batch && B <= 64 && max_nodes <= ctx->lim.max_nodes && H <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim && H_kv <= 65535,
                  CTCSPEC_EUNSUPPORTED, "q4_verify_attn: shape exceeds the context's limits");
  const long long seq_rows = (long long)max_nodes * (H / H_kv);
  CTCSPEC_REQUIRE(ctx, q4_units_fit(B, H_kv, seq_rows, kv_cap, max_nodes), CTCSPEC_EUNSUPPORTED,
                  "q4_verify_attn: capacities or rows beyond 2^30, or work of more than 2^31 units");
  for (const void* a : {q, (const void*)cache->k_codes, (const void*)cache->v_codes, k_tree, v_tree, (const void*)workspace, (const void*)out})
    CTCSPEC_REQUIRE(ctx, aligned16(a), CTCSPEC_EINVAL, "q4_verify_attn: pointers must be 16-byte aligned");
  const Q4Workspace ws = q4_workspace(B, H, H_kv, dh, max_nodes);
  CTCSPEC_REQUIRE(ctx, workspace_bytes >= ws.total, CTCSPEC_EINVAL, "q4_verify_attn: workspace of %zu bytes needed, %zu given", ws.total,
                  workspace_bytes);
  unsigned char* base = (unsigned char*)workspace;
  Q4AttnParams p;
  p.q = (const unsigned char*)q;
  p.k_codes = (const unsigned char*)cache->k_codes; p.k_scales = (const unsigned char*)cache->k_scales;
  p.v_codes = (const unsigned char*)cache->v_codes; p.v_scales = (const unsigned char*)cache->v_scales;
  p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.k_tree = (const unsigned char*)k_tree; p.v_tree = (const unsigned char*)v_tree; p.n_nodes = n_nodes; p.depth = window ? node_depth : nullptr;
  p.anc_mask = (const unsigned long long*)anc_mask;
  p.kv_cap = kv_cap; p.B = B; p.H = H; p.H_kv = H_kv; p.group = H / H_kv; p.dh = dh; p.blocks = q4_blocks(dh); p.max_nodes = max_nodes;
  // (positions stay below 2^30 + 128: a longer window or sink is one that holds them all)
  p.window = window < (1 << 30) + 256 ? window : (1 << 30) + 256;
  p.sink = sink < (1 << 30) + 256 ? sink : (1 << 30) + 256;
  p.sl2 = scale * 1.4426950408889634f;
  p.po = (float*)(base + ws.o); p.pml = (float*)(base + ws.ml); p.odd = (int*)(base + ws.odd);
  p.out_bf16 = out_dt == CTCSPEC_BF16; p.out = out; p.lse = lse;
  hipStream_t st = ctx->stream;
  const hipError_t e = q4_with_shape(ws.rows, p.blocks, out_dt == CTCSPEC_F32, [&](auto shape) {
    using SH = decltype(shape);
    hipLaunchKernelGGL(q4_attn_kernel<SH>, dim3(SH::GROUPS), dim3(64 * SH::NW), SH::LDS, st, p);
    if (const hipError_t e1 = hipGetLastError(); e1 != hipSuccess) return e1;
    hipLaunchKernelGGL(q4_join_kernel<SH>, dim3((unsigned)((seq_rows + 31) / 32), (unsigned)H_kv, (unsigned)B), dim3(64 * SH::DT), 0, st, p);
    return hipGetLastError();
  });
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
