// q4_verify_attn: verification attention over a cache held in 4 bits (q4_format.h), with or without a sliding window, one layer.
//
//   out[b,h,i] = sum_j p_j v_j,  p = softmax over the cached keys and the tree nodes that row i sees
//
// What the codes stand for is exact in bf16, so a tile of keys becomes operands of the matrix instructions by conversions alone: a lane
// has 32 elements of a block, one scale, and its keys need no way through the LDS - which elements of a row form which step of a product is
// free, as long as the query's lanes hold the same.  Values are needed by columns: they are converted, written to the LDS a row at a time
// and fetched by transposing reads, each wavefront its own tile, so the loop has no barriers.
//
// The work - iterations of four tiles, one for each wavefront, of a block of rows - is dealt to the workgroups in pieces of blocks, or in equal
// shares that go across them (q4_plan.h, prefix_plan.h); the four wavefronts' results are joined in the LDS, the shares' by a second kernel.  Short
// caches and windows need neither: a workgroup has a block of rows whole.
//
// What bounds it.  Four single tokens behind 16384 to 65536 rows (8 key heads of 128): the cache's bytes, 178 MB in 37 to 39 us (4.7 TB/s), and the join,
// 5 us.  64 rows a sequence and key head behind 32768 rows (four sequences, 32 heads, 577 MB, 1.05 times that from HBM, 121 GFLOP): 170 to 183 us, the
// matrix units busy for 0.43 of them, the vector units for about half, and the two overlap only in part: a tile takes a wavefront 174 vector instructions
// beside its 16 matrix ones, 64 of them conversions (every block of 32 rows converts every key and value), 16 exponentials.  Short calls (8 single
// tokens behind 256 to 2048 rows 19 to 22 us, 64-node trees 31 us with weights in three parts): the way in - lengths, shares, first tile -, segments of
// a few iterations, and their joins.
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
  int kv_cap, B, H, H_kv, group, dh, max_nodes, window, sink;  // group: heads that share a key head
  float sl2;                      // scale * log2(e)
  float* po;                      // partial O: [slot][DT][4][64 lanes][4]
  float* pml;                     // [slot][2][32]: maximum in the log2 domain, sum
  int* odd;                       // [slot]: a value of a tree node is infinite or not a number
  int* span;                      // [key head][B][blocks of rows][4]: the workgroups from the first to the last one with keys of a block, and
  int blocks;                     // the block's number; blocks of max_nodes nodes
  int out_bf16;
  void* out;                      // [B][H][max_nodes][dh]
  float* lse;                     // [B][H][max_nodes] or null
};

// Up to here a weight's exponent - a scaled score less the rounded reference, in one rounding - is off by 16 at the most, by the same for all of a row.
constexpr float kQ4Far = 536870912.f;  // 2^29

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// DT: blocks of 32 components, of a row of the cache too.  FINE: weights in three bf16 parts, 24 bits together, for a float result; for a bf16 one
// they are one bf16 each, off by 2^-8 of themselves at most, as the result itself (against 64 bits the result is off by 1.8e-3 of its norm, 1.7e-3 with float
// weights), and a tile has 16 products instead of 32.  The sum that they are divided by, from which lse is formed, has 24 bits in both.
// ALONE: a workgroup has a block of rows whole, there is neither a deal nor a join.
template <int DT_, bool FINE_, bool ALONE_>
struct Q4Shape {
  static constexpr int DT = DT_, NW = kQ4Tiles;
  static constexpr bool FINE = FINE_, ALONE = ALONE_;
  static constexpr int KB = (DT + 1) / 2, QU = 4 * KB;        // blocks of a key in a lane; steps of 16 elements of a product
  static constexpr int VB = (DT + 1) / 2;                     // blocks of values in a lane: 32 DT of them in 64 lanes
  // Values in the LDS: a row has 64 bytes a block and as many more as make an odd number of them, four rows have 16 bytes more.  A transposing
  // read of 32 lanes takes 64 bytes of each of four consecutive rows, which then lie in different banks; a write of 16 lanes (0 to 7 with 16
  // to 23) the same 16 bytes of their blocks, which do if the lanes' rows are of four such groups, two of each (v_row).  (The document above
  // took 201 us so and 217 with a lane pair's rows in their order, 192 cycles of conflicts a tile instead of 64.)
  static constexpr int ROWB = 64 * (DT | 1), FOURB = 4 * ROWB + 16, TILE = 8 * FOURB;
  static __device__ __forceinline__ int place(int row) { return (row >> 2) * FOURB + (row & 3) * ROWB; }
  static constexpr int PART = (DT * 16 + 2) * 64 * 4;         // O, m, l of 32 rows
  static constexpr int STAGE = NW * TILE > 2 * PART ? NW * TILE : 2 * PART;
  static constexpr int LDS = STAGE + 8 * 64 * 4;              // and the sequences' table
  static_assert(kQ4Waves * LDS <= 160 * 1024 && kQ4Groups % 8 == 0);
  // The blocks of values that a lane converts: row and block of the row of its k-th.  (Four blocks a row: two neighbours of a row; else
  // those 64 further.)
  static constexpr bool PAIRS = DT == 4;
  static __device__ __forceinline__ int v_row(int lane, int k) {
    const int a = PAIRS ? lane >> 1 : (int)((unsigned)(lane + 64 * k) / DT);
    return PAIRS ? (a & 25) | (a & 2) << 1 | (a & 4) >> 1 : (DT == 2 ? (a & 24) | (a & 1) << 1 | (a & 2) << 1 | (a & 4) >> 2 : a);
  }
  static __device__ __forceinline__ int v_block(int lane, int k) { return PAIRS ? 2 * (lane & 1) + k : (int)((unsigned)(lane + 64 * k) % DT); }
  static __device__ __forceinline__ bool v_there(int lane, int k) { return DT % 2 == 0 || lane + 64 * k < 32 * DT; }
};

// What both kernels know about the work: lane b holds sequence b's part (the limits allow 64 sequences), the rest is uniform.
struct Q4Work {
  int n, ctx, iters, blocks;     // lane: nodes, cached rows, iterations over its keys, blocks of its rows
  int unit0, block0;             // lane: units and blocks of the sequences before it, for one key head
  int head_units, head_blocks;   // of a key head
  int units;                     // of all key heads
  int most;                      // iterations of a piece: then units are pieces, a share each; or 0
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
  t.blocks = (t.n * p.group + kQ4Rows - 1) / kQ4Rows;
  t.iters = t.n ? q4_iterations(t.n, t.ctx, p.window, p.sink) : 0;
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
  // Where little balance is lost, every share is a piece of one block, and no workgroup has parts of two: lane by lane the pieces' size, from the
  // ideal one on, and the first that makes no more pieces than there are workgroups.
  if (p.H_kv * t.head_blocks <= kQ4Groups && t.head_blocks > 0) {
    const int all = p.H_kv * ((t.head_units - t.head_blocks * q4_units(0)) / kPrefixOwnWeight);
    int ideal = (all - 1) / kQ4Groups + 1;
    ideal = ideal < kQ4LeastPiece ? kQ4LeastPiece : ideal;
    const int most = ideal + lane * (ideal < 64 ? 1 : ideal / 32);
    const float inv = __builtin_amdgcn_rcpf((float)most);
    int pieces = 0;
    for (int x = 0; x < p.B; ++x) {  // q4_pieces, the division by a product and what it may be off by
      const int n = __builtin_amdgcn_readlane(t.iters, x) - 1, blocks = __builtin_amdgcn_readlane(t.blocks, x);
      int q = (int)((float)n * inv);
      const int r = n - q * most;
      q += r >= most ? 1 : (r < 0 ? -1 : 0);
      pieces += n < 0 ? 0 : blocks * (q + 1);
    }
    const unsigned long long fits = __builtin_amdgcn_ballot_w64(p.H_kv * pieces <= kQ4Groups);
    const int first = fits ? __builtin_ctzll(fits) : 0, size = __builtin_amdgcn_readlane(most, first);
    if (fits && size <= ideal + ideal / 2 + kQ4PieceSlack) {
      t.most = size;
      const int own = t.blocks * q4_pieces(t.iters, size);
      int s = own;
      for (int d = 1; d < p.B; d *= 2) {
        const int sb = __shfl_up(s, d, 64);
        if (lane >= d) s += sb;
      }
      t.unit0 = s - own;
      t.head_units = __builtin_amdgcn_readlane(s, p.B - 1);
      t.units = p.H_kv * t.head_units;
    }
  }
  return t;
}

// Row `node`'s depth, and the nodes that it sees: its mask row's, of these with a window those near enough or in the sink.
__device__ __forceinline__ int q4_depth(const Q4AttnParams& p, int b, int node) {
  const int d = p.depth[(size_t)b * p.max_nodes + node];
  return d < 0 ? 0 : (d >= p.max_nodes ? p.max_nodes - 1 : d);
}
struct Q4Mask {
  unsigned long long low, high;  // nodes 0 to 63, 64 to 127
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

// Values of tree nodes that are infinite or not a number, left out so far: into the rows that see them.  (o: as in q4_write.)
template <int N>
__device__ __forceinline__ void q4_add_odd(const Q4AttnParams& p, int b, int kh, int node, int n, int at, f32x4 (&o)[N]) {
  const int len = p.ctx_len[b], L = len < 0 ? 0 : (len > p.kv_cap ? p.kv_cap : len);
  const Q4Mask mask = q4_tree_mask(p, b, node, n, L, p.window > 0 ? q4_depth(p, b, node) : 0);
  const unsigned short* vt = (const unsigned short*)p.v_tree + ((size_t)b * p.H_kv + kh) * p.max_nodes * p.dh;
  for (int j = 0; j < n; ++j) {
    if (!mask.node(j)) continue;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (at + 8 * i + e >= p.dh) continue;
        const float v = bf16_bits_to_float(vt[(size_t)j * p.dh + at + 8 * i + e]);
        if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[i][e] += v;
      }
  }
}
// Four components from `at` on, and those 8, 16 .. behind, of a row of the result: its weighted values o, the maximum m and the sum l of its weights.
template <int N>
__device__ __forceinline__ void q4_write(const Q4AttnParams& p, size_t row, bool with_lse, int at, const f32x4 (&o)[N], float m, float l) {
  const bool none = m == -INFINITY && l == 0.f;  // no key at all
  const float inv = none ? 0.f : 1.0f / l;
  if (p.lse && with_lse) p.lse[row] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (at + 8 * i >= p.dh) continue;
    const f32x4 v = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[i] * inv;
    if (p.out_bf16) {
      *(u32x2*)((unsigned short*)p.out + row * p.dh + at + 8 * i) = u32x2{__builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[0], (__bf16)v[1]}),
                                                                          __builtin_bit_cast(unsigned int, bf16x2{(__bf16)v[2], (__bf16)v[3]})};
    } else {
      *(f32x4*)((float*)p.out + row * p.dh + at + 8 * i) = v;
    }
  }
}

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((address_space(3))) unsigned char lds_byte;
// of a value of lanes 32 apart, in both
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// a descriptor of `bytes` bytes at p, both the same in every lane
__device__ __forceinline__ auto buffer(const unsigned char* p, int bytes) {
  const unsigned long long at = (unsigned long long)p;
  const unsigned long long base = (unsigned long long)(unsigned)uniform((int)(at >> 32)) << 32 | (unsigned)uniform((int)at);
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (unsigned)uniform(bytes), 0x00020000);
}
__device__ __forceinline__ s16x4 lds_read_tr(unsigned int at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
}
#endif

template <typename SH>
__global__ __launch_bounds__(64 * SH::NW, kQ4Waves) void q4_attn_kernel(Q4AttnParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int DT = SH::DT, KB = SH::KB, VB = SH::VB, QU = SH::QU;
  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  int(*table)[64] = (int(*)[64])(smem + SH::STAGE);
  enum { kNodes, kCtx, kIters, kUnit0, kBlock0, kOffLow, kOffHigh, kOdd };
  int u = 0, u1 = 1, w = 0, most = 0, head_units = 0, head_blocks = 0;
  Deal d{};
  if constexpr (!SH::ALONE) {
    const long long my_off = lane < p.B ? p.kv_off[lane] : 0;
    const Q4Work t = q4_read_work<SH>(p);
    d = prefix_deal(t.units, kQ4Groups);
    most = t.most;
    if (most) d = Deal{t.units, t.units, 1, 0};
    // (consecutive shares - neighbouring keys - to the same of the 8 XCDs)
    const int per = (d.groups + 7) / 8;
    w = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || w >= d.groups) return;
    u = uniform(d.begin(w));
    u1 = uniform(d.begin(w + 1));
    // What the lanes know about the sequences, out of the registers while the keys go by; and a flag.
    if (wave == 0) {
      table[kNodes][lane] = t.n;
      table[kCtx][lane] = t.ctx;
      table[kIters][lane] = t.iters;
      table[kUnit0][lane] = t.unit0;
      table[kBlock0][lane] = t.block0;
      table[kOffLow][lane] = (int)my_off;
      table[kOffHigh][lane] = (int)(my_off >> 32);
    }
    __syncthreads();
    head_units = t.head_units;
    head_blocks = t.head_blocks;
  }
  unsigned char* vtile = smem + wave * SH::TILE;
  const unsigned int vbase = (unsigned int)(size_t)(lds_byte*)vtile;
  // the transposing read: 16 lanes fetch 4 rows x 16 components, 8 bytes each, and lane s of them receives component s of the four rows
  unsigned int vread;
  {
    const int s = lane & 15, row = 4 * (lane >> 5) + (s >> 2), ch = (((lane & 31) >> 4) << 1) + ((s & 3) >> 1);
    vread = vbase + SH::place(row) + ch * 16 + (s & 1) * 8;
  }
  // where this lane's k-th block of values goes in the tile
  auto vwrite = [&](int k) __attribute__((always_inline)) -> unsigned int {
    const int row = SH::v_there(lane, k) ? SH::v_row(lane, k) : 0, blk = SH::v_there(lane, k) ? SH::v_block(lane, k) : 0;
    return vbase + SH::place(row) + blk * 64;
  };
  const unsigned int vwrite0 = vwrite(0);

  while (u < u1) {
    // ---- which block of rows, which keys -------------------------------------------------------------------------------
    int seg_lane = lane;  // (as something new: addresses that only a segment's ends need are formed there)
    asm volatile("" : "+v"(seg_lane));
    int kh, b, n, L, blk, slot = 0, iters, it0 = 0, niter;
    long long off;
    if constexpr (SH::ALONE) {
      blk = blockIdx.x;
      kh = blockIdx.y;
      b = blockIdx.z;
      n = p.n_nodes[b];
      L = p.ctx_len[b];
      off = p.kv_off[b];
      n = n > p.max_nodes ? p.max_nodes : n;
      if (n * p.group <= blk * kQ4Rows) return;
      L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
      iters = niter = q4_iterations(n, L, p.window, p.sink);
      u = u1;
    } else {
      int per_head = head_units;  // (and what divisions by it take)
      asm volatile("" : "+s"(per_head));
      kh = uniform(u / per_head);
      const int in_head = u - kh * per_head;
      // (sequences without nodes have no units: the last sequence that starts at or before the unit and has some)
      b = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(table[kIters][seg_lane] > 0 && table[kUnit0][seg_lane] <= in_head));
      n = uniform(table[kNodes][b]);
      L = uniform(table[kCtx][b]);
      off = (long long)((unsigned long long)(unsigned)uniform(table[kOffHigh][b]) << 32 | (unsigned)uniform(table[kOffLow][b]));
      iters = uniform(table[kIters][b]);
      const int units = uniform(most ? q4_pieces(iters, most) : q4_units(iters));
      const int in_seq = in_head - uniform(table[kUnit0][b]);
      blk = uniform(in_seq / units);
      const int at_unit = in_seq - blk * units;
      slot = w + kh * head_blocks + uniform(table[kBlock0][b]) + blk;
      const int share = uniform(units - at_unit < u1 - u ? units - at_unit : u1 - u);
      u += share;
      it0 = uniform(most ? q4_piece_begin(iters, units, at_unit) : prefix_iterations(at_unit, kPrefixOwnWeight, false));
      niter = uniform(most ? q4_piece_begin(iters, units, at_unit + 1) : prefix_iterations(at_unit + share, kPrefixOwnWeight, false)) - it0;
      if (niter <= 0) continue;
    }
    const bool whole = SH::ALONE || (it0 == 0 && niter == iters);  // (then there is nothing to join)
    if (threadIdx.x == 0 && !whole) {  // (the join need not deal the work once more)
      int* span = p.span + (((size_t)kh * p.B + b) * p.blocks + blk) * 4;
      if (it0 == 0) *(u32x2*)span = u32x2{(unsigned)(slot - w), (unsigned)w};
      if (it0 + niter == iters) span[2] = w;
    }
    const Q4Tiles tiles = q4_tiles(L, p.window, p.sink);
    const int total = tiles.count + (n + 31) / 32;
    const size_t row0 = (size_t)off + (size_t)kh * p.kv_cap;
    // codes and scales of cached tile x of the segment: of key c blocks KB h2 .., of the values blocks lane, lane + 64.  (Rows behind the last
    // one, and blocks behind a row's last, lie outside what the descriptors hold: zeros.)
    u32x4 kraw[KB], vraw[VB];
    unsigned int kscale[KB], vscale[VB];  // (two bytes in the first, where a lane's blocks are neighbours)
    auto fetch = [&](int x) __attribute__((always_inline)) {
      const int tile = x < tiles.lead ? x : x + tiles.gap, left = L - 32 * tile < 32 ? L - 32 * tile : 32;
      const size_t at = (row0 + 32 * (size_t)tile) * DT;
      const auto kc = buffer(p.k_codes + at * kQ4BlockBytes, left * DT * kQ4BlockBytes), ks = buffer(p.k_scales + at, left * DT);
      const auto vc = buffer(p.v_codes + at * kQ4BlockBytes, left * DT * kQ4BlockBytes), vs = buffer(p.v_scales + at, left * DT);
      constexpr int kOutside = 0x1000000;
      int fl = lane;  // (as something new: places in a tile are formed here, not kept in registers all the way)
      asm volatile("" : "+v"(fl));
      const int kfrom = (fl & 31) * DT + KB * (fl >> 5), vfrom = SH::v_row(fl, 0) * DT + SH::v_block(fl, 0);
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const int from = DT % 2 == 0 || KB * (fl >> 5) + k < DT ? kfrom : kOutside;
        kraw[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kc, from * kQ4BlockBytes, k * kQ4BlockBytes, 0));
        if constexpr (!SH::PAIRS) kscale[k] = __builtin_amdgcn_raw_buffer_load_b8(ks, from, k, 0);
      }
#pragma unroll
      for (int k = 0; k < VB; ++k) {
        const int from = SH::PAIRS ? vfrom : (SH::v_there(fl, k) ? SH::v_row(fl, k) * DT + SH::v_block(fl, k) : kOutside);
        vraw[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vc, from * kQ4BlockBytes, SH::PAIRS ? k * kQ4BlockBytes : 0, 0));
        if constexpr (!SH::PAIRS) vscale[k] = __builtin_amdgcn_raw_buffer_load_b8(vs, from, 0, 0);
      }
      if constexpr (SH::PAIRS) {
        kscale[0] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(ks, kfrom, 0, 0);
        vscale[0] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(vs, vfrom, 0, 0);
      }
    };
    auto scale_byte = [&](const auto& scales, int k) __attribute__((always_inline)) -> int {
      return (int)(SH::PAIRS ? (scales[0] >> (8 * k)) & 255u : scales[k]);
    };
    auto scale_of = [&](const auto& scales, int k) __attribute__((always_inline)) -> float { return q4_scale_value(scale_byte(scales, k)); };
    const int first = it0 * kQ4Tiles + wave, end = (it0 + niter) * kQ4Tiles < total ? (it0 + niter) * kQ4Tiles : total;
    // Of the cached tiles those from x_all on, up to x_part, are seen by every row in full.
    int x_all = p.window > 0 ? L + p.max_nodes - 1 - p.window : -1;
    x_all = x_all < 0 ? 0 : x_all / 32 + 1 - tiles.gap;
    const int x_part = L / 32 - tiles.gap, cached_end = end < tiles.count ? end : tiles.count;
    if (first < cached_end) fetch(first);

    // ---- this lane's query row: step i of a product has elements 32 (KB h2 + i / 4) + 8 (i % 4) .. + 7 ------------------------------
    u32x4 qf[QU];
    int low;  // the first position of the window
    {
      int fresh = lane, heads = p.group;
      asm volatile("" : "+v"(fresh), "+s"(heads));
      // (rows that are none do as row 0 does: nobody reads what comes of it)
      const int r = blk * kQ4Rows + (fresh & 31), at_row = r < n * heads ? r : 0, node = at_row / heads, hg = at_row - node * heads;
      const unsigned char* row = p.q + (((size_t)b * p.H + kh * heads + hg) * p.max_nodes + node) * (size_t)(p.dh * 2);
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int at = 32 * (KB * (fresh >> 5) + i / 4) + 8 * (i % 4);
        qf[i] = *(const u32x4*)(row + (at < p.dh ? at * 2 : 0));
        if (p.dh < 64 * KB) qf[i] = at < p.dh ? qf[i] : u32x4{0u, 0u, 0u, 0u};
      }
      low = p.window > 0 ? L + q4_depth(p, b, node) - p.window + 1 : 0;
    }
    f32x16 o[DT];
    float m_run = -INFINITY, l_run = 0.f;
    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float zero = 0.f;
        asm volatile("" : "+v"(zero));  // (one zero for all would stay in registers of its own)
        o[dt][i] = zero;
      }

    // S^T = K Q^T: a lane then holds 16 scores of one query row, its neighbour 32 lanes away the other 16 - register i: key
    // 8 (i / 4) + 4 h2 + i % 4 -, and P in the same registers is the right operand of O^T += V^T P.
    // What follows the scores s of a tile whose values lie in the LDS.
    auto weigh = [&](f32x16& s) __attribute__((always_inline)) {
      // the reference, in the log2 domain, only has to be near the maximum: it is moved when a score exceeds it by more than 2^8
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      if (__builtin_amdgcn_ballot_w64(fmaf(mx, p.sl2, -m_run) > 8.0f) != 0ull) {
        const float m = half_max(mx);
        float top = m * p.sl2;
        asm volatile("" : "+v"(top));  // (rounded for the factor below as for the weights: left to itself the compiler may form one exponent from the product)
        if (fmaf(m, p.sl2, -m_run) > 8.0f && top > m_run) {  // (not above where scaling takes every score to -infinity)
          const float alpha = __builtin_amdgcn_exp2f(m_run - top);  // 0 on first use
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
          m_run = top;
        }
      }
      float ms = m_run > -INFINITY ? m_run : 0.f;
      // Far from 0 the reference is off by more than an exponential has room for.  There a score is rounded as the reference was: it is the same, with a
      // weight of 1, or below it by 32 at the least, with none.
      if (__builtin_amdgcn_ballot_w64(fabsf(ms) >= kQ4Far) != 0ull) {
        const bool far = fabsf(ms) >= kQ4Far;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float scaled = s[i] * p.sl2;
          s[i] = far ? (scaled < ms ? -INFINITY : scaled * 0.f) : s[i];  // (what is no number stays none)
        }
        ms = far ? 0.f : ms;
      }
      u32x4 hi, lo, rest;
      auto weights = [&](int kb) __attribute__((always_inline)) {  // of 16 keys
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[8 * kb + 2 * j], p.sl2, -ms)), p1 = __builtin_amdgcn_exp2f(fmaf(s[8 * kb + 2 * j + 1], p.sl2, -ms));
          hi[j] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)p0, (__bf16)p1});
          if constexpr (SH::FINE) {
            const float h0 = __uint_as_float(hi[j] << 16), h1 = __uint_as_float(hi[j] & 0xffff0000u);
            lo[j] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)(p0 - h0), (__bf16)(p1 - h1)});
            const float r0 = (p0 - h0) - __uint_as_float(lo[j] << 16), r1 = (p1 - h1) - __uint_as_float(lo[j] & 0xffff0000u);
            rest[j] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)r0, (__bf16)r1});
          }
          l_run += p0 + p1;
        }
      };
      // the values of step i: 16 keys i / DT, 32 components i % DT; each is read a step ahead
      auto values = [&](int i) __attribute__((always_inline)) -> u32x4 {
        const int kb = i / DT, dt = i % DT;
        const s16x4 v0 = lds_read_tr(vread + dt * 64 + 4 * kb * SH::FOURB), v1 = lds_read_tr(vread + dt * 64 + (4 * kb + 2) * SH::FOURB);
        return __builtin_bit_cast(u32x4, s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
      };
      u32x4 next = values(0);
#pragma unroll
      for (int i = 0; i < 2 * DT; ++i) {
        const int kb = i / DT, dt = i % DT;
        const u32x4 vr = next;
        if (i + 1 < 2 * DT) next = values(i + 1);
        if (dt == 0) weights(kb);
        const bf16x8 v = __builtin_bit_cast(bf16x8, vr);
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, hi), o[dt], 0, 0, 0);
        if constexpr (SH::FINE) {
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, lo), o[dt], 0, 0, 0);
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, rest), o[dt], 0, 0, 0);
        }
        // (step by step: what all of them need at once does not fit the registers)
        asm volatile("" : "+v"(o[dt]) : : "memory");
      }
      asm volatile("" ::: "memory");  // (the next tile's values go where these were read)
    };

    auto cached_scores = [&](f32x16& s) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const float scale = scale_of(kscale, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q4_decode(kraw[k][e], scale)), __builtin_bit_cast(bf16x8, qf[4 * k + e]), s, 0, 0, 0);
          asm volatile("" : "+v"(s), "+v"(kraw[k]));  // (this product before the next conversions: all of them do not fit the registers)
        }
      }
    };
    auto cached_values = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < VB; ++k) {
        if (!SH::v_there(lane, k)) continue;
        const float scale = scale_of(vscale, k);
        const unsigned int to = SH::PAIRS || k == 0 ? vwrite0 + 64 * k : vwrite(k);
#pragma unroll
        for (int e = 0; e < 4; ++e) *(__attribute__((address_space(3))) u32x4*)(to + 16 * e) = q4_decode(vraw[k][e], scale);
        __builtin_amdgcn_sched_barrier(0);
      }
      asm volatile("" ::: "memory");
    };
    // A row that does not see a key has no part of it: a score of -infinity, and a value that is a number (0 times another is none).
    auto hide = [&](f32x16& s, unsigned int vis) __attribute__((always_inline)) {  // vis: the keys of the tile that this lane's row sees
      vis >>= 4 * (lane >> 5);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = (vis >> (8 * (i / 4) + i % 4)) & 1u ? s[i] : -INFINITY;
    };
    // ---- cached tiles -------------------------------------------------------------------------------------------------------------------
    for (int x = first; x < cached_end; x += kQ4Tiles) {
      // A SIMD serves its oldest wavefront first: three that began together ended after 118, 163 and 209 us of a document's attention, and the
      // last one alone is slow.  So a wavefront's priority falls with every quarter of its way.  (187 us -> 181; shorter ones leave it.)
      if (cached_end - first >= 16 * kQ4Tiles) {
        const int left = 4 * (cached_end - x), all = cached_end - first;
        if (left > 3 * all) __builtin_amdgcn_s_setprio(3);
        else if (left > 2 * all) __builtin_amdgcn_s_setprio(2);
        else if (left > all) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
      }
      f32x16 s;
      cached_scores(s);
      if (x < x_all || x >= x_part) {  // not every row sees every key
        const int at = 32 * (x < tiles.lead ? x : x + tiles.gap), left = L - at;
        unsigned int vis = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
        if (p.window > 0) {
          const int from = low - at, sunk = p.sink - at;
          vis &= (from <= 0 ? 0xffffffffu : (from >= 32 ? 0u : 0xffffffffu << from)) | (sunk >= 32 ? 0xffffffffu : (sunk <= 0 ? 0u : (1u << sunk) - 1u));
        }
        hide(s, vis);
        // blocks of values that are NaN: of the rows that see them here, and zeros for the product
#pragma unroll
        for (int k = 0; k < VB; ++k) {
          const bool nan = SH::v_there(lane, k) && scale_byte(vscale, k) == kQ4NoNumber;
          unsigned long long lanes = __builtin_amdgcn_ballot_w64(nan);
          while (lanes != 0ull) {
            const int from = __builtin_ctzll(lanes), row = SH::v_row(from, k), block = SH::v_block(from, k);
            lanes &= lanes - 1;
            const float add = (vis >> row) & 1u ? __builtin_nanf("") : 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
              if (block == dt) o[dt] += add;
          }
          vraw[k] = nan ? u32x4{0u, 0u, 0u, 0u} : vraw[k];
          if (nan) vscale[SH::PAIRS ? 0 : k] &= ~(SH::PAIRS ? 255u << (8 * k) : 255u);
        }
      }
      cached_values();
      if (x + kQ4Tiles < cached_end) fetch(x + kQ4Tiles);
      weigh(s);
    }
    // ---- a tile of the tree, of which a wavefront has one at the most: keys as they are, values into the LDS (nodes that are none: zeros) -----
    static_assert(kQ4Tiles * 32 >= 128);
    const int x_tree = first + (tiles.count <= first ? 0 : (tiles.count - first + kQ4Tiles - 1) / kQ4Tiles * kQ4Tiles);
    if (x_tree < end) {
      int fresh = lane;  // (as something new: what only this tile needs is formed here, not kept in registers all the way)
      asm volatile("" : "+v"(fresh));
      const int c = fresh & 31, h2 = fresh >> 5, tile = x_tree - tiles.count;
      const size_t tree0 = ((size_t)b * p.H_kv + kh) * p.max_nodes * (size_t)(p.dh * 2);
      const auto kt = buffer(p.k_tree + tree0, n * p.dh * 2), vt = buffer(p.v_tree + tree0, n * p.dh * 2);
      constexpr int kOutside = 0x1000000;
      // (everything fetched ahead of its use, as far as the registers hold it: keys and mask, and half of the values for half of the keys)
      u32x4 kf[QU], vf[DT];
      unsigned int strange = 0u;
      auto fetch_values = [&](int half) __attribute__((always_inline)) {  // of 128 DT chunks of 8 components
        int own = lane;
        asm volatile("" : "+v"(own));
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const int y = own + 64 * (half * DT + i), row = y / (4 * DT), ch = y % (4 * DT);
          vf[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vt, 8 * ch < p.dh ? ((32 * tile + row) * p.dh + 8 * ch) * 2 : kOutside, 0, 0));
        }
      };
      // values that are infinite or no numbers: left out, and added by the join to the rows that see them
      auto take_values = [&](int half) __attribute__((always_inline)) {
        int own = lane;
        asm volatile("" : "+v"(own));
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const int y = own + 64 * (half * DT + i), row = y / (4 * DT), ch = y % (4 * DT);
#pragma unroll
          for (int e = 0; e < 4; ++e) {  // (exponents of nothing but ones carry into the sign's place)
            const unsigned int bad = (((vf[i][e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15;
            strange |= bad;
            vf[i][e] &= ~(bad * 0xffffu);
          }
          *(__attribute__((address_space(3))) u32x4*)(vbase + SH::place(row) + ch * 16) = vf[i];
        }
        asm volatile("" : : : "memory");
      };
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int at = 32 * (KB * h2 + i / 4) + 8 * (i % 4);
        kf[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kt, at < p.dh ? ((32 * tile + c) * p.dh + at) * 2 : kOutside, 0, 0));
      }
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[i]), __builtin_bit_cast(bf16x8, qf[i]), s, 0, 0, 0);
        if (i % 4 == 3) {
          asm volatile("" : "+v"(s) : : "memory");
          if (i == 3) fetch_values(0);
        }
      }
      int heads = p.group, node = blk * kQ4Rows + c;
      asm volatile("" : "+s"(heads));
      node = node < n * heads ? node / heads : 0;
      // which nodes of the tile the row sees, as q4_tree_mask has it
      const int nodes = n - 32 * tile;  // (at least one)
      unsigned int vis = (unsigned int)(p.anc_mask[((size_t)b * p.max_nodes + node) * ((p.max_nodes + 63) >> 6) + (tile >> 1)] >> (32 * (tile & 1)));
      vis &= nodes >= 32 ? 0xffffffffu : (1u << nodes) - 1u;
      if (p.window > 0 && p.window < p.max_nodes) {  // (lane j has node j's depth: fetched one after the other they would take 0.2 us each)
        const int depth = q4_depth(p, b, node), theirs = q4_depth(p, b, 32 * tile + (c < nodes ? c : 0));
        for (int j = 0; j < 32; ++j) {
          const int dj = __builtin_amdgcn_readlane(theirs, j);
          vis &= depth - dj >= p.window && L + dj >= p.sink ? ~(1u << j) : 0xffffffffu;
        }
      }
      take_values(0);
      fetch_values(1);
      take_values(1);
      odd = __builtin_amdgcn_ballot_w64(strange != 0u) != 0ull;
      hide(s, vis);
      weigh(s);
    }

    // ---- the four wavefronts' parts joined: 2 to 0 and 3 to 1, then 1 to 0 -------------------------------------------------------
    if (threadIdx.x == 0) table[kOdd][0] = 0;
    __syncthreads();  // every tile is consumed: the LDS is free
    if (odd) table[kOdd][0] = 1;
    float* part = (float*)smem;
    asm volatile("" : "+v"(seg_lane));
    const int el = seg_lane;
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
      if (wave >= half && wave < 2 * half) {
        float* its = part + (wave - half) * (SH::PART / 4);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(f32x4*)(its + el * 4 + (dt * 4 + i) * 256) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        its[DT * 1024 + el] = m_run;
        its[DT * 1024 + 64 + el] = l_run;
      }
      __syncthreads();
      if (wave < half) {
        const float* its = part + wave * (SH::PART / 4);
        const float mo = its[DT * 1024 + el], lother = its[DT * 1024 + 64 + el];
        const float m = fmaxf(m_run, mo), base = m > -INFINITY ? m : 0.f;
        const float a0 = __builtin_amdgcn_exp2f(m_run - base), a1 = __builtin_amdgcn_exp2f(mo - base);
        l_run = l_run * a0 + lother * a1;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          __builtin_amdgcn_sched_barrier(0);  // (32 components at a time: all reads ahead do not fit the registers)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 x = *(const f32x4*)(its + el * 4 + (dt * 4 + i) * 256);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][4 * i + e] = o[dt][4 * i + e] * a0 + x[e] * a1;
          }
        }
        m_run = m;
      }
      __syncthreads();
    }
    if (!SH::ALONE && threadIdx.x == 0) p.odd[slot] = table[kOdd][0];
    // ---- what the segment leaves, in the order of the registers -------------------------------------------------------------
    if (wave == 0) {
      l_run = half_sum(l_run);
      // A block that one workgroup has whole is written by it, unless the join has infinite values of the tree, or such that are no numbers, to
      // add.  (8 sequences x 64 nodes x 32 heads behind 0, 224, 480 rows, us: 16.2, 18.9, 23.3; by way of the join 22.1, 23.3, 25.7.)
      const bool infinite = uniform(table[kOdd][0]) != 0, direct = whole && (SH::ALONE || !infinite);
      if (!SH::ALONE && threadIdx.x == 0 && whole) {
        int* span = p.span + (((size_t)kh * p.B + b) * p.blocks + blk) * 4;
        *(u32x2*)span = u32x2{(unsigned)(slot - w), direct ? 1u : (unsigned)w};
        span[2] = direct ? 0 : w;
      }
      int heads = p.group;
      asm volatile("" : "+s"(heads));
      const int r = blk * kQ4Rows + (el & 31), node = r / heads, hg = r - node * heads;
      if (r < n * heads && direct) {
        const size_t row = ((size_t)b * p.H + kh * heads + hg) * p.max_nodes + node;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          f32x4 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
          if (SH::ALONE && infinite) q4_add_odd(p, b, kh, node, n, 32 * dt + 4 * (el >> 5), x);
          q4_write(p, row, dt == 0 && el < 32, 32 * dt + 4 * (el >> 5), x, m_run, l_run);
        }
      } else if (!SH::ALONE && r < n * heads) {
        float* po = p.po + (size_t)slot * (DT * 1024) + el * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(f32x4*)(po + (dt * 4 + i) * 256) = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        if (el < 32) {
          float* ml = p.pml + (size_t)slot * (2 * kQ4Rows) + el;
          ml[0] = m_run;
          ml[kQ4Rows] = l_run;
        }
      }
    }
  }
#endif
}

// ---- the join ------------------------------------------------------------------------------------------------------------
// Workgroups of DT wavefronts, PARTS of them per (32 rows of a sequence, key head): every wavefront weighs the rows' partial results and adds
// up its components of them, 32 / PARTS.  Where there are 16 rows or fewer, lanes share a row: `shares` of them take every shares-th partial
// result, and what they have is added up in an order that the number of shares gives.  (4 single tokens with 8 key heads, 32 blocks of up
// to 39 partial results, us: 10.4 with neither, 6.8 with lanes that share, 5.2 with 4 parts as well.)
//
// Up to kQ4JoinFew blocks have 4 parts.  (us with 4 / 1: 32 blocks 5.2 / 6.8, 256 5.2 / 5.2 and 8.5 / 5.9, 416 5.9 / 5.1, 512 9.7 / 7.0.)
constexpr int kQ4JoinFew = 128;
template <typename SH, int PARTS>
__global__ __launch_bounds__(64 * SH::DT) void q4_join_kernel(Q4AttnParams p) {
  constexpr int DT = SH::DT, OWN = 4 / PARTS;
  const int lane = threadIdx.x & 63, dt = threadIdx.x >> 6, h2 = lane >> 5;
  const int kh = blockIdx.y, b = blockIdx.z, blk = blockIdx.x / PARTS, part = blockIdx.x % PARTS * OWN;
  const int* span = p.span + (((size_t)kh * p.B + b) * p.blocks + blk) * 4;
  const int item = span[0], w0 = span[1], w1 = span[2];  // (of a block without rows whatever was there)
  const int n = p.n_nodes[b] < p.max_nodes ? p.n_nodes[b] : p.max_nodes, rows = n * p.group - blk * 32;
  if (rows <= 0 || w0 > w1) return;  // (one workgroup had the whole block and has written the rows)
  int shares = 1;
  while (shares < 32 && shares <= w1 - w0 && 32 / (2 * shares) >= rows) shares *= 2;
  const int of = 32 / shares, c = lane & (of - 1), share = (lane & 31) / of, r = blk * 32 + c;
  float m = -INFINITY, l = 0.f;
  f32x4 o[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float* ml = p.pml + (size_t)item * (2 * kQ4Rows) + c;
  const float* po = p.po + (size_t)item * (DT * 1024) + (dt * 4 + part) * 256 + (h2 * 32 + c) * 4;
  auto add = [&](float pm, float pl, const f32x4 (&x)[OWN]) __attribute__((always_inline)) {
    const float top = fmaxf(m, pm), base = top > -INFINITY ? top : 0.f;
    const float old = __builtin_amdgcn_exp2f(m - base), a = __builtin_amdgcn_exp2f(pm - base);
    l = l * old + a * pl;
#pragma unroll
    for (int i = 0; i < OWN; ++i) o[i] = o[i] * old + a * x[i];
    m = top;
  };
  constexpr int kBatch = 4;
  int odd = 0;
  for (int w = w0 + share; w <= w1; w += kBatch * shares) {
    float pm[kBatch], pl[kBatch];
    f32x4 x[kBatch][OWN];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {  // (behind the last one: the last one again, with no weight)
      const int at = w + q * shares;
      const size_t s = at <= w1 ? at : w1;
      pm[q] = ml[s * (2 * kQ4Rows)];
      pl[q] = ml[s * (2 * kQ4Rows) + kQ4Rows];
#pragma unroll
      for (int i = 0; i < OWN; ++i) x[q][i] = *(const f32x4*)(po + s * (DT * 1024) + i * 256);
      odd |= p.odd[s + item];
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (w + q * shares <= w1) add(pm[q], pl[q], x[q]);
  }
  for (int d = of; d < 32; d *= 2) {
    const float pm = __shfl_xor(m, d, 64), pl = __shfl_xor(l, d, 64);
    f32x4 x[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) x[i] = f32x4{__shfl_xor(o[i][0], d, 64), __shfl_xor(o[i][1], d, 64), __shfl_xor(o[i][2], d, 64), __shfl_xor(o[i][3], d, 64)};
    add(pm, pl, x);
    odd |= __shfl_xor(odd, d, 64);
  }
  if (c >= rows || share) return;
  const int node = r / p.group, hg = r - node * p.group;
  if (odd) q4_add_odd(p, b, kh, node, n, 32 * dt + 8 * part + 4 * h2, o);
  const size_t row = ((size_t)b * p.H + kh * p.group + hg) * p.max_nodes + node;
  q4_write(p, row, dt == 0 && part == 0 && h2 == 0, 32 * dt + 8 * part + 4 * h2, o, m, l);
}

// ---- host side -----------------------------------------------------------------------------------------------------------
template <int DT, typename F>
static hipError_t q4_with_kind(bool fine, bool alone, F&& f) {
  if (alone) return fine ? f(Q4Shape<DT, true, true>{}) : f(Q4Shape<DT, false, true>{});
  return fine ? f(Q4Shape<DT, true, false>{}) : f(Q4Shape<DT, false, false>{});
}
template <typename F>
static hipError_t q4_with_shape(int blocks, bool fine, bool alone, F&& f) {
  switch (blocks) {
    case 1: return q4_with_kind<1>(fine, alone, f);
    case 2: return q4_with_kind<2>(fine, alone, f);
    case 3: return q4_with_kind<3>(fine, alone, f);
    default: return q4_with_kind<4>(fine, alone, f);
  }
}

hipError_t prepare_q4_attn() {
  hipError_t e = hipSuccess;
  for (int blocks = 1; blocks <= 4; ++blocks)
    for (int kind = 0; kind < 4; ++kind)
      if (e == hipSuccess)
        e = q4_with_shape(blocks, kind & 1, kind & 2, [](auto shape) {
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
  CTCSPEC_REQUIRE(ctx, q4_scales_aligned(cache), CTCSPEC_EINVAL, "q4_verify_attn: scales must be 4-byte aligned");
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
  p.kv_cap = kv_cap; p.B = B; p.H = H; p.H_kv = H_kv; p.group = H / H_kv; p.dh = dh; p.max_nodes = max_nodes;
  // (positions stay below 2^30 + 128: a longer window or sink is one that holds them all)
  p.window = window < (1 << 30) + 256 ? window : (1 << 30) + 256;
  p.sink = sink < (1 << 30) + 256 ? sink : (1 << 30) + 256;
  p.sl2 = scale * 1.4426950408889634f;
  p.po = (float*)(base + ws.o); p.pml = (float*)(base + ws.ml); p.odd = (int*)(base + ws.odd); p.span = (int*)(base + ws.span);
  p.blocks = (int)((seq_rows + kQ4Rows - 1) / kQ4Rows);
  p.out_bf16 = out_dt == CTCSPEC_BF16; p.out = out; p.lse = lse;
  hipStream_t st = ctx->stream;
  const hipError_t e = q4_with_shape(q4_blocks(dh), out_dt == CTCSPEC_F32, q4_alone(B, H_kv, seq_rows, kv_cap, max_nodes, window, sink), [&](auto shape) {
    using SH = decltype(shape);
    if constexpr (SH::ALONE) {
      hipLaunchKernelGGL(q4_attn_kernel<SH>, dim3((unsigned)p.blocks, (unsigned)H_kv, (unsigned)B), dim3(64 * SH::NW), SH::LDS, st, p);
    } else {
      hipLaunchKernelGGL(q4_attn_kernel<SH>, dim3(kQ4Groups), dim3(64 * SH::NW), SH::LDS, st, p);
      if (const hipError_t e1 = hipGetLastError(); e1 != hipSuccess) return e1;
      const bool few = (long long)p.blocks * H_kv * B <= kQ4JoinFew;
      const dim3 grid((unsigned)(p.blocks * (few ? 4 : 1)), (unsigned)H_kv, (unsigned)B), block(64 * SH::DT);
      if (few) hipLaunchKernelGGL((q4_join_kernel<SH, 4>), grid, block, 0, st, p);
      else hipLaunchKernelGGL((q4_join_kernel<SH, 1>), grid, block, 0, st, p);
    }
    return hipGetLastError();
  });
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
