// prefix_verify_attn: verification attention of a batch whose sequences continue one common prefix, one layer.
//
//   out[b,h,i] = sum_j p_j v_j,  p = softmax over the prefix's keys, the sequence's cached keys and the tree nodes it sees
//
// Softmax parts over disjoint keys join exactly: (O, m, l) with O = sum exp2(s - m) v, l = sum exp2(s - m).  So the rows of ALL
// sequences (and of the heads that share a key head) stand side by side against each tile of the prefix's keys - read and
// multiplied once for the batch -, every sequence's rows against its own keys, and a second kernel joins what they left.
//
// prefix_attn_kernel: the work is cut into units - one iteration over the keys (KP * KT tiles of 32) for one block of R rows, and
// some for the block itself - and the units, in the order (prefix: key head, row block, keys), (own: key head, sequence, row block, keys), are dealt to the
// workgroups in equal consecutive shares: lengths, node counts and prefix length are read on the device, and no workgroup waits
// for a longer one.  A workgroup whose share crosses from one block of rows into the next leaves a partial result for each, in a
// place of its own (prefix_plan.h).
//
// What bounds it.  Many rows over a long prefix: the products - 8 x 64 nodes, 32 heads of 128, behind 32768 keys, bf16: 332 us, 0.41 of
// the matrix units' cycles (0.75 PFLOP/s of the call's own products, 0.94 of those on whole blocks); a tile's exponentials take as long
// as its products and only partly run beside them.  Long histories: their bytes where a sequence's rows fill a block; where more rows
// share a prefix, a block has more than a sequence's rows, and on own keys only the wavefronts that have rows multiply - two of eight for
// 64 nodes: 8 x 64 nodes, 32 heads, each further 2048 own keys (268 MB) take 47 us (5.7 TB/s) in blocks of 64 rows, without a prefix,
// and 57 us (4.7 TB/s) in blocks of 256, behind one of a single key.  Short calls: the first keys' way in (about 6 k cycles for 64 KB a
// compute unit, all at once) and the second kernel (6 us, most of it latency).  8 x 64 nodes behind 2048 keys with 256 to 2048 of their
// own: 95 to 102 us, 203 MB; one token for each of 8 sequences behind 2048: 30 us, 52 MB.
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
  float* po;                      // partial O: [slot][R / 32][DHP / 32][4][64 lanes][4]
  float* pml;                     // [slot][2][R]: maximum in the log2 domain, sum
  int* odd;                       // [slot]: a value of a tree node is infinite or not a number
};

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uniform(long long v) {
  return (long long)((unsigned long long)(unsigned)uniform((int)(v >> 32)) << 32 | (unsigned)uniform((int)v));
}

__device__ __forceinline__ const unsigned char* uniform(const unsigned char* p) {
  return (const unsigned char*)uniform((long long)p);
}

// What both kernels know about the work: lane b holds sequence b's part (the limits allow 64 sequences), the rest is uniform.
struct Work {
  int n, first, ctx;          // lane: nodes, nodes of the sequences before it, cached rows
  int blocks, iters;          // lane: blocks of the sequence's rows, iterations over its own keys
  int unit0, block0;          // lane: units and blocks of the sequences before it, for one key head
  long long off;              // lane: kv_off
  int all, prefix;            // nodes of all sequences, rows of the prefix
  int pblocks, piters;        // blocks of all rows, iterations over the prefix
  int head_units, head_blocks;  // own units and blocks of a key head
  int punits, pitems, units;  // units and blocks of the prefix over all key heads; all units
};
// units of a block of rows
template <typename SH>
__device__ __forceinline__ int own_units(int iters) { return prefix_block_units(SH::F32) + iters * kPrefixOwnWeight; }
template <typename SH>
__device__ __forceinline__ int prefix_units(int iters) { return prefix_block_units(SH::F32) + iters * prefix_shared_weight(SH::R); }
template <typename SH>
__device__ __forceinline__ Work read_work(const PrefixAttnParams& p) {
  constexpr int R = SH::R, TPI = SH::TPI;
  const int lane = threadIdx.x & 63;
  Work t{};
  const int P = *p.prefix_len;
  if (lane < p.B) {
    t.off = p.kv_off[lane];
    const int n = p.n_nodes[lane], L = p.ctx_len[lane];
    t.n = n < 0 ? 0 : (n > p.max_nodes ? p.max_nodes : n);
    t.ctx = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  }
  t.blocks = (t.n * p.group + R - 1) / R;
  t.iters = t.n ? ((t.ctx + 31) / 32 + (t.n + 31) / 32 + TPI - 1) / TPI : 0;
  const int mine = t.blocks * own_units<SH>(t.iters);
  int n = t.n, b = t.blocks, u = mine;
  for (int d = 1; d < p.B; d *= 2) {
    const int nb = __shfl_up(n, d, 64), bb = __shfl_up(b, d, 64), ub = __shfl_up(u, d, 64);
    if (lane >= d) { n += nb; b += bb; u += ub; }
  }
  t.first = n - t.n;
  t.block0 = b - t.blocks;
  t.unit0 = u - mine;
  t.all = __builtin_amdgcn_readlane(n, p.B - 1);
  t.head_blocks = __builtin_amdgcn_readlane(b, p.B - 1);
  t.head_units = __builtin_amdgcn_readlane(u, p.B - 1);
  t.prefix = uniform(P < 0 ? 0 : (P > p.prefix_cap ? p.prefix_cap : P));
  t.piters = ((t.prefix + 31) / 32 + TPI - 1) / TPI;
  t.pblocks = uniform((t.all * p.group + R - 1) / R);
  t.pitems = t.piters ? p.H_kv * t.pblocks : 0;
  t.punits = t.pitems * prefix_units<SH>(t.piters);
  t.units = t.punits + p.H_kv * t.head_units;
  return t;
}

constexpr int kPrefixTable = 10 * 64 * 4;
template <bool F32_, int DHP_, int QT_, int CW_, int KP_, int KT_, int NS_, int WPE_, bool FINE_>
struct PrefixShape {
  static constexpr bool F32 = F32_, FINE = FINE_;
  static constexpr int DHP = DHP_, QT = QT_, CW = CW_, KP = KP_, KT = KT_, NS = NS_, WPE = WPE_;
  static constexpr int NW = CW * KP, R = 32 * QT * CW, TPI = KP * KT;
  static constexpr int ES = F32 ? 4 : 2, ROWB = DHP * ES, TILE = 32 * ROWB, STAGE = TPI * 2 * TILE;
  static constexpr int RQ = TILE / 1024, NREQ = TPI * 2 * RQ / NW;  // requests of 1 KB per tile, per wavefront and stage
  static constexpr int RPR = 1024 / ROWB;                           // rows of a request
  static constexpr int DT = DHP / 32, QU = ROWB / 32;               // dh tiles of O; 32-byte steps of a row
  static constexpr int PART = (DT * 16 + 2) * 64 * 4;               // O, m, l of 32 rows
  static constexpr int JOIN = (KP - 1) * CW * QT * PART;
  static constexpr int LDS = (NS * STAGE > JOIN ? NS * STAGE : JOIN) + kPrefixTable;
  // what 256 compute units hold at once
  static constexpr int GROUPS = WPE * 4 >= 2 * NW && 2 * LDS <= 160 * 1024 ? 512 : 256;
  static_assert(TPI == prefix_tiles(R, DHP, F32));
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

template <typename SH>
__global__ __launch_bounds__(64 * SH::NW, SH::WPE) void prefix_attn_kernel(PrefixAttnParams p) {
#if defined(__HIP_DEVICE_COMPILE__)  // (buffer descriptors exist on the device only)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  // Behind the stages (whose places are formed by xor: they begin at a multiple of a row's bytes): what the lanes know about the
  // sequences, out of the registers while the keys go by, and a flag.
  int(*table)[64] = (int(*)[64])(smem + SH::LDS - kPrefixTable);
  enum { kNodes, kCtx, kOff, kOffHigh, kFirst, kBlocks, kIters, kUnit0, kBlock0, kOdd };
  constexpr int R = SH::R, QT = SH::QT, ROWB = SH::ROWB, TILE = SH::TILE, NREQ = SH::NREQ, DT = SH::DT, QU = SH::QU, TPI = SH::TPI, KT = SH::KT;
  constexpr unsigned int kOutside = 0x40000000u;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave % SH::CW, kp = wave / SH::CW;
  const int c = lane & 31, h2 = lane >> 5;
  const int rb = p.dh * SH::ES;  // bytes of a row

  const Work t = read_work<SH>(p);
  const Deal d = prefix_deal(t.units, SH::GROUPS);
  // Workgroups go to the 8 XCDs in turn, each with an L2 of its own: consecutive shares - the row blocks of a key head, which
  // read the same keys - go to the same one.
  static_assert(SH::GROUPS % 8 == 0 && SH::GROUPS <= kPrefixMaxGroups);
  const int per = (d.groups + 7) / 8, w = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || w >= d.groups) return;
  int u = uniform(d.begin(w));
  const int u1 = uniform(d.begin(w + 1));
  if (wave == 0) {
    const int own[9] = {t.n, t.ctx, (int)t.off, (int)(t.off >> 32), t.first, t.blocks, t.iters, t.unit0, t.block0};
#pragma unroll
    for (int i = 0; i < 9; ++i) table[i][lane] = own[i];
  }
  __syncthreads();
  auto of = [&](int what, int b) __attribute__((always_inline)) { return uniform(table[what][b]); };
  const int all = t.all, prefix = t.prefix, pblocks = t.pblocks, piters = t.piters, punits = t.punits, pitems = t.pitems;
  const int head_units = t.head_units, head_blocks = t.head_blocks;

  // ---- requests: number x of a stage is tile x / (2 RQ), K then V, 1 KB (RPR rows) after 1 KB; this wavefront has NREQ in a
  // row, of one operand tile or of several whole ones.  Lane l of a request fills the l-th 16 bytes of its kilobyte: with the
  // chunk of the row that belongs there.
  constexpr int kRun = NREQ < SH::RQ ? NREQ : SH::RQ, kOperands = NREQ / kRun;  // requests of an operand tile, operand tiles
  static_assert(SH::RQ % kRun == 0 && NREQ % kRun == 0 && kOperands <= 2 && (kOperands == 1 || kRun == SH::RQ), "requests of a wavefront");
  unsigned int voff[NREQ];
#pragma unroll
  for (int j = 0; j < NREQ; ++j) {
    const int x = wave * NREQ + j, row = x % SH::RQ * SH::RPR + lane / (ROWB / 16);
    const int chunk = lane % (ROWB / 16) ^ (x / SH::RQ & 1 ? SH::fv(row) : SH::fk(row));
    voff[j] = chunk * 16 < rb ? (unsigned)(row * rb + chunk * 16) : kOutside;
  }
  const unsigned int lds0 = (unsigned)(size_t)(lds_byte*)smem;
  // this lane's place in a K tile (row c, first half of a 32-byte step) and in a V tile
  const unsigned int kplace = c * ROWB + ((h2 ^ SH::fk(c)) << 4);
  unsigned int vplace;
  if constexpr (SH::F32) {
    vplace = 4 * h2 * ROWB + (((c >> 2) ^ (h2 << 3)) << 4) + (c & 3) * 4;  // key 4 h2 (+ 8 (i / 4) + i % 4), dh c (+ 32 t)
  } else {
    // the transposing read: 16 lanes fetch 4 rows x 16 dh, 8 bytes each, and lane s of them receives dh s of the four rows
    const int s = lane & 15, row = 4 * h2 + (s >> 2), ch = ((c >> 4) << 1) + ((s & 3) >> 1);
    vplace = row * ROWB + ((ch ^ SH::fv(row)) << 4) + (s & 1) * 8;
  }

  while (u < u1) {
    // (The lane's number, as something new: addresses that only a segment's ends need are then formed there, not kept in registers
    // all the way - with them the kernels for one sequence's rows did not fit.)
    int seg_lane = lane;
    asm volatile("" : "+v"(seg_lane));
    const int sc = seg_lane & 31, sh = seg_lane >> 5;
    // ---- which block of rows, which keys -------------------------------------------------------------------------------
    const bool own = u >= punits;
    int b = 0, kh, blk, at_unit, units, weight, slot, n, L;  // at_unit: in the block's units, the first of which are no iterations
    const unsigned char *kc, *vc, *kt, *vt;
    if (own) {
      const int rel = u - punits;
      kh = uniform(rel / head_units);
      const int in_head = rel - kh * head_units;
      // (sequences without nodes have no units: the last sequence that starts at or before the unit and has some)
      b = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(table[kIters][seg_lane] > 0 && table[kUnit0][seg_lane] <= in_head));
      units = own_units<SH>(of(kIters, b));
      weight = kPrefixOwnWeight;
      const int in_seq = in_head - of(kUnit0, b);
      blk = uniform(in_seq / units);
      at_unit = in_seq - blk * units;
      slot = w + pitems + kh * head_blocks + of(kBlock0, b) + blk;
      n = of(kNodes, b);
      L = of(kCtx, b);
      const long long off = (long long)((unsigned long long)(unsigned)of(kOffHigh, b) << 32 | (unsigned)of(kOff, b));
      const size_t at = ((size_t)off + (size_t)kh * p.kv_cap * p.dh) * SH::ES;
      const size_t ta = ((size_t)b * p.H_kv + kh) * p.max_nodes * rb;
      kc = p.k_cache + at; vc = p.v_cache + at;
      kt = p.k_tree + ta; vt = p.v_tree + ta;
    } else {
      units = prefix_units<SH>(piters);
      weight = prefix_shared_weight(R);
      const int item = uniform(u / units);
      at_unit = u - item * units;
      kh = uniform(item / pblocks);
      blk = item - kh * pblocks;
      slot = w + item;
      n = all;
      L = prefix;
      kc = p.k_prefix + (size_t)kh * p.prefix_cap * rb;
      vc = p.v_prefix + (size_t)kh * p.prefix_cap * rb;
      kt = kc; vt = vc;
    }
    const int share = uniform(units - at_unit < u1 - u ? units - at_unit : u1 - u);
    u += share;
    // the iterations that begin in the share
    const int it0 = uniform(prefix_iterations(at_unit, weight, SH::F32));
    const int niter = uniform(prefix_iterations(at_unit + share, weight, SH::F32)) - it0;
    if (niter <= 0) continue;
    kc = uniform(kc); vc = uniform(vc); kt = uniform(kt); vt = uniform(vt);
    const int ctx_tiles = own ? (L + 31) / 32 : 0x7fffffff;  // the tiles from here on are tree nodes

    // ---- the tiles of iteration i of this segment into their stage -----------------------------------------------------------
    // (The bases are parameters: captured, the choice between them becomes one between their addresses, in scratch memory.  The
    // instruction is written out because the compiler would let every transposing read wait for all requests that it knows of;
    // it has no register for a result, and the loop below waits for it.  The compiler counts no wait states for what is written
    // out, so they stand inside: a vector instruction that writes a scalar register - v_readfirstlane for the descriptor, v_readlane
    // where it comes back from a spill - has to lie five wait states before the load that reads it: one for s_mov, four for s_nop 3.
    // m0 needs one of them.)
    auto request = [&](int i, const unsigned char* kc, const unsigned char* vc, const unsigned char* kt, const unsigned char* vt)
        __attribute__((always_inline)) {
      const unsigned int stage = lds0 + i % SH::NS * SH::STAGE + wave * NREQ * 1024;
#pragma unroll
      for (int q = 0; q < kOperands; ++q) {
        const int operand = wave * NREQ / SH::RQ + q, k = (it0 + i) * TPI + operand / 2;
        const bool tree = k >= ctx_tiles;
        const int row0 = (tree ? k - ctx_tiles : k) * 32;
        int left = (tree ? n : L) - row0;  // rows behind the last key, and all behind the last iteration: zeros, nothing is read
        left = left < 0 || i >= niter ? 0 : (left > 32 ? 32 : left);
        const unsigned char* base = operand & 1 ? (tree ? vt : vc) : (tree ? kt : kc);
        const int from = left > 0 ? row0 : 0;
        const unsigned long long at = (unsigned long long)base + (size_t)from * rb;
        const u32x4 rsrc = {(unsigned)uniform((int)at), (unsigned)uniform((int)(at >> 32)) & 0xffffu, (unsigned)uniform(left * rb), 0x00020000u};
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (that m0 is reserved: nothing else here uses it)
#pragma unroll
        for (int j = q * kRun; j < (q + 1) * kRun; ++j)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(stage + j * 1024), "v"(voff[j]), "s"(rsrc)
                       : "memory", "m0");
#pragma clang diagnostic pop
      }
    };
    constexpr int kEarly = SH::NS > 2 ? 2 : 1;  // stages in front of the rows, which everything waits for together
#pragma unroll
    for (int i = 0; i < kEarly; ++i) request(i, kc, vc, kt, vt);
    if (threadIdx.x == 0) table[kOdd][0] = 0;

    // ---- this lane's query rows ------------------------------------------------------------------------------------------
    const int row_first = blk * R + rg * 32 * QT;
    const bool live_wave = row_first < n * p.group;
    u32x4 qf[QT][QU];
    unsigned long long mw0[QT], mw1[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      const int r = row_first + qt * 32 + sc;
      const bool live = r < n * p.group;
      int node = r / p.group, bq = b;
      const int hg = r - node * p.group;
      if (!own) {
        // (sequences without nodes begin where the next one does: the last of those that begin here has the node)
        bq = 0;
        for (int i = 1; i < p.B; ++i) bq += node >= table[kFirst][i] ? 1 : 0;
        node -= table[kFirst][bq];
      }
      // (rows that are none read some row's query: nobody reads what comes of it)
      if (!live) { node = 0; bq = 0; }
      const unsigned char* qrow = p.q + (((size_t)bq * p.H + kh * p.group + hg) * p.max_nodes + node) * rb;
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        const int at = (2 * i + sh) * 16;
        qf[qt][i] = *(const u32x4*)(qrow + (at < rb ? at : 0));
        if (rb < ROWB) qf[qt][i] = at < rb ? qf[qt][i] : u32x4{0u, 0u, 0u, 0u};
      }
      mw0[qt] = mw1[qt] = 0ull;
      if (own && live) {
        const int W = (p.max_nodes + 63) >> 6;
        const unsigned long long* m = p.anc_mask + ((size_t)b * p.max_nodes + node) * W;
        mw0[qt] = m[0];
        if (W > 1) mw1[qt] = m[1];
      }
    }

    // (Here, for all wavefronts: a load that the compiler knows of and that may be under way in the loop would have it wait there
    // for everything.)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
      for (int i = 0; i < QU; ++i) asm volatile("" : "+v"(qf[qt][i]));
      asm volatile("" : "+v"(mw0[qt]), "+v"(mw1[qt]));
    }
#pragma unroll
    for (int i = kEarly; i < SH::NS - 1; ++i) request(i, kc, vc, kt, vt);

    f32x16 o[QT][DT], s[QT], s2[QT];
    float m_run[QT], l_run[QT];
    bool odd = false;  // values that are no numbers were met (below)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      m_run[qt] = -INFINITY;
      l_run[qt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[qt][dt][i] = 0.f;
    }

    // S^T = K Q^T of a tile, the keys as rows: a lane then holds 16 scores of one query row, its neighbour 32 lanes away the other
    // 16 - register i, half h2: key 8 (i / 4) + 4 h2 + i % 4 -, and P in the same registers is the right operand of O^T += V^T P.
    // A tile is a step of three parts: the products of the NEXT tile's scores with most of this tile's exponentials, the products of
    // the first half of its values with the rest of them, those of the second half with the search for the next tile's maximum.
    // Product by product, some of each: left alone, the scheduler puts all products at one end.
    constexpr int kAhead = QU < 4 ? QU : 4;  // keys' fragments that are read ahead of their products
    constexpr int kPairsA = 6;               // of the 8 pairs of exponentials, those of the first part
    u32x4 a[kAhead];
    auto read_keys = [&](unsigned int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) a[i] = lds_read<u32x4>((tile + kplace) ^ (i << 5));
    };
    auto score = [&](int i, f32x16 (&s)[QT]) __attribute__((always_inline)) {  // product i of a tile's scores
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        if constexpr (SH::F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            s[qt] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i % kAhead][e]), __uint_as_float(qf[qt][i][e]), s[qt], 0, 0, 0);
        } else {
          s[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i % kAhead]), __builtin_bit_cast(bf16x8, qf[qt][i]), s[qt], 0, 0, 0);
        }
      }
    };
    // scores of keys that are not there or not seen
    auto hide = [&](int k, bool any, f32x16 (&s)[QT], const unsigned long long (&mw0)[QT], const unsigned long long (&mw1)[QT])
        __attribute__((always_inline)) {
      const bool tree = k >= ctx_tiles;
      const int row0 = (tree ? k - ctx_tiles : k) * 32;
      const int left = any ? (tree ? n : L) - row0 : 0;
      if (tree || left < 32) {
        const unsigned int there = left >= 32 ? 0xffffffffu : (left > 0 ? (1u << left) - 1u : 0u);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const unsigned int vis = there & (tree ? (unsigned int)((row0 < 64 ? mw0[qt] : mw1[qt]) >> (row0 & 63)) : 0xffffffffu);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[qt][i] = (vis >> (8 * (i / 4) + 4 * h2 + i % 4)) & 1u ? s[qt][i] : -INFINITY;
        }
      }
    };
    // The reference (in the log2 domain) only has to be near the maximum: it is moved when a score exceeds it by more than 2^8, so that
    // P stays below 256; the two lanes of a row then agree on the larger.  What weights, factors and joins take is this one rounded
    // number, so that its rounding is in all of them alike; and where it is the maximum, the weight 1 is exact in bf16.
    auto reference = [&](const float (&mx)[QT]) __attribute__((always_inline)) {
      bool far = false;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) far |= fmaf(mx[qt], p.sl2, -m_run[qt]) > 8.0f;
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
    };

    // Tile k at `tile`, its scores in s and the reference set for them; the next tile k1 at `next` (any1: it is part of the
    // segment), whose scores go to sn; read_next() requests the first fragments of the tile behind it.
    auto step = [&](int k, unsigned int tile, int k1, bool any1, unsigned int next, f32x16 (&s)[QT], f32x16 (&sn)[QT], auto&& read_next,
                    const unsigned long long (&mw0)[QT], const unsigned long long (&mw1)[QT]) __attribute__((always_inline)) {
      const bool tree = k >= ctx_tiles;
      const unsigned int ka = next + kplace, va = tile + TILE + vplace;
      float ms[QT], sum[QT], mx[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        ms[qt] = m_run[qt] > -INFINITY ? m_run[qt] : 0.f;
        sum[qt] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sn[qt][i] = 0.f;
      }
      // A value that is no number or infinite must not reach the rows that do not see its key, and 0 times it is no number: in a
      // tile of tree nodes such values take part as 0, and the join adds them where they are seen.
      if constexpr (SH::F32) {
        constexpr int kGroups = 2 * DT;  // of eight values, read one group ahead
        float x[2][8];
        auto read_values = [&](int g) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[g % 2][i] = lds_read<float>((va ^ (g / 2 << 7)) + (16 * (g % 2) + 8 * (i / 4) + i % 4) * ROWB);
        };
#pragma unroll
        for (int i = 0; i < QU; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          score(i, sn);
          if (i + kAhead < QU) a[i % kAhead] = lds_read<u32x4>(ka ^ ((i + kAhead) << 5));
          if (i == QU - 1) read_values(0);
#pragma unroll
          for (int j = i * 16 / QU; j < (i + 1) * 16 / QU; ++j)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
              s[qt][j] = __builtin_amdgcn_exp2f(fmaf(s[qt][j], p.sl2, -ms[qt]));
              sum[qt] += s[qt][j];
              asm volatile("" : "+v"(sum[qt]));  // (here, not at the end of the tile)
            }
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          __builtin_amdgcn_sched_barrier(0);
          if (g + 1 < kGroups) read_values(g + 1);
          if (tree) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const bool bad = (__float_as_uint(x[g % 2][i]) & 0x7f800000u) == 0x7f800000u;
              odd |= bad;
              x[g % 2][i] = bad ? 0.f : x[g % 2][i];
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              o[qt][g / 2] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[g % 2][i], s[qt][8 * (g % 2) + i], o[qt][g / 2], 0, 0, 0);
          if (g == 0) {
            __builtin_amdgcn_sched_barrier(0);
            read_next();
            hide(k1, any1, sn, mw0, mw1);
          } else {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
#pragma unroll
              for (int i = (g - 1) * 16 / (kGroups - 1); i < g * 16 / (kGroups - 1); ++i) mx[qt] = i == 0 ? sn[qt][0] : fmaxf(mx[qt], sn[qt][i]);
              asm volatile("" : "+v"(mx[qt]));
            }
          }
        }
      } else {
        u32x4 hi[QT][2], lo[QT][2], rest[QT][2];
        s16x4 vr[DT][2][2];
        auto exponentials = [&](int from, int to) __attribute__((always_inline)) {  // pairs of registers
#pragma unroll
          for (int j = from; j < to; ++j)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
              // P is rounded to bf16, as the values are and as the result will be: 8 x 64 nodes behind 32768 keys 350 us, off from the
              // exact result by 1.88e-3 of it; with another part 440 us and 1.66e-3, which is the result's own rounding.  FINE: P = hi + lo
              // + rest, within 2^-24 of it.  (Two parts, within 2^-16, where 256 rows share a prefix: 8 x 64 nodes behind 2048 keys
              // 89 to 101 us instead of 95 to 102, and a weight off by up to 2^-17 as soon as more than 128 rows are in the batch.)
              const float p0 = __builtin_amdgcn_exp2f(fmaf(s[qt][2 * j], p.sl2, -ms[qt]));
              const float p1 = __builtin_amdgcn_exp2f(fmaf(s[qt][2 * j + 1], p.sl2, -ms[qt]));
              const unsigned int h = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)p0, (__bf16)p1});
              hi[qt][j / 4][j % 4] = h;
              if constexpr (SH::FINE) {
                const float h0 = __uint_as_float(h << 16), h1 = __uint_as_float(h & 0xffff0000u);
                const unsigned int r = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)(p0 - h0), (__bf16)(p1 - h1)});
                lo[qt][j / 4][j % 4] = r;
                const float r0 = (p0 - h0) - __uint_as_float(r << 16), r1 = (p1 - h1) - __uint_as_float(r & 0xffff0000u);
                rest[qt][j / 4][j % 4] = __builtin_bit_cast(unsigned int, bf16x2{(__bf16)r0, (__bf16)r1});
              }
              sum[qt] += p0 + p1;
              asm volatile("" : "+v"(sum[qt]));  // (here, not at the end of the tile)
            }
        };
        constexpr int kReads = 4 * DT / QU;
#pragma unroll
        for (int i = 0; i < QU; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          score(i, sn);
          if (i + kAhead < QU) a[i % kAhead] = lds_read<u32x4>(ka ^ ((i + kAhead) << 5));
#pragma unroll
          for (int j = i * kReads; j < (i + 1) * kReads; ++j) {
            const int dt = j / 2 % DT, half = j % 2, kb = j / (2 * DT);
            vr[dt][kb][half] = lds_read_tr((va ^ (dt << 6)) + (16 * kb + 8 * half) * ROWB);
          }
          exponentials(i * kPairsA / QU, (i + 1) * kPairsA / QU);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (tree) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const short x = vr[dt][kb][e / 4][e % 4];
                const bool bad = (x & 0x7f80) == 0x7f80;
                odd |= bad;
                vr[dt][kb][e / 4][e % 4] = bad ? (short)0 : x;
              }
        }
        auto value = [&](int dt, int kb, const u32x4 (&w)[QT][2]) __attribute__((always_inline)) {
          const s16x4 v0 = vr[dt][kb][0], v1 = vr[dt][kb][1];
          const bf16x8 v = __builtin_bit_cast(bf16x8, s16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) o[qt][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, w[qt][kb]), o[qt][dt], 0, 0, 0);
        };
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          __builtin_amdgcn_sched_barrier(0);
          value(dt, 0, hi);
          exponentials(kPairsA + dt * (8 - kPairsA) / DT, kPairsA + (dt + 1) * (8 - kPairsA) / DT);
        }
        __builtin_amdgcn_sched_barrier(0);
        read_next();
        hide(k1, any1, sn, mw0, mw1);
        if constexpr (SH::FINE) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) value(dt, 0, lo);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) value(dt, 0, rest);
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          __builtin_amdgcn_sched_barrier(0);
          value(dt, 1, hi);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int i = dt * 16 / DT; i < (dt + 1) * 16 / DT; ++i) mx[qt] = i == 0 ? sn[qt][0] : fmaxf(mx[qt], sn[qt][i]);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) asm volatile("" : "+v"(mx[qt]));
        }
        if constexpr (SH::FINE) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) value(dt, 1, lo);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) value(dt, 1, rest);
        }
      }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) l_run[qt] += sum[qt];
      reference(mx);
    };

    // ---- the loop ---------------------------------------------------------------------------------------------------------
    // arrive(i): stage i + 1 is there - this wavefront's requests are counted, those of the others stand behind the barrier -, and
    // all reads of stage i - 1 lie behind it: its place takes stage i - 1 + NS.  (Behind the last stage requests read nothing, but
    // are made, so that the wait can count.)
    const unsigned int mine = kp * KT * 2 * TILE;  // this wavefront's tiles of a stage
    auto place = [&](int i) __attribute__((always_inline)) { return lds0 + i % SH::NS * SH::STAGE + mine; };
    auto arrive = [&](int i) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SH::NS - 3) * NREQ) : "memory");
      lds_barrier();
      request(i - 1 + SH::NS, kc, vc, kt, vt);
    };
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SH::NS - 1 - kEarly) * NREQ) : "memory");
    lds_barrier();
    if (live_wave) {
      read_keys(place(0));
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[qt][i] = 0.f;
#pragma unroll
      for (int i = 0; i < QU; ++i) {
        score(i, s);
        if (i + kAhead < QU) a[i % kAhead] = lds_read<u32x4>((place(0) + kplace) ^ ((i + kAhead) << 5));
      }
      hide(it0 * TPI + kp * KT, true, s, mw0, mw1);
      float mx[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = s[qt][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx[qt] = fmaxf(mx[qt], s[qt][i]);
      }
      reference(mx);
      if constexpr (KT > 1) read_keys(place(0) + 2 * TILE);
    }
    for (int i = 0; i < niter; ++i) {
      if constexpr (KT == 1) {
        arrive(i);
        const int k = (it0 + i) * TPI + kp;
        if (live_wave) {
          read_keys(place(i + 1));
          step(k, place(i), k + TPI, i + 1 < niter, place(i + 1), s, s2, []() {}, mw0, mw1);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[qt] = s2[qt];
        }
      } else {
        static_assert(KT == 2);
        const int k = (it0 + i) * TPI + kp * 2;
        const unsigned int at = place(i), then = place(i + 1);
        if (live_wave)
          step(k, at, k + 1, true, at + 2 * TILE, s, s2, [&]() __attribute__((always_inline)) { arrive(i); read_keys(then); }, mw0, mw1);
        else
          arrive(i);
        if (live_wave)
          step(k + 1, at + 2 * TILE, k + TPI, i + 1 < niter, then, s2, s, [&]() __attribute__((always_inline)) { read_keys(then + 2 * TILE); }, mw0, mw1);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (__builtin_amdgcn_ballot_w64(odd) != 0ull) table[kOdd][0] = 1;
    __syncthreads();  // every request has landed, every tile is consumed: the LDS is free
    if (threadIdx.x == 0) p.odd[slot] = table[kOdd][0];

    // ---- the key parts of a row group joined ------------------------------------------------------------------------------
    if constexpr (SH::KP > 1) {
      float* part = (float*)smem;
      if (kp > 0) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float* its = part + (((kp - 1) * SH::CW + rg) * QT + qt) * (SH::PART / 4);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4*)(its + seg_lane * 4 + (dt * 4 + i) * 256) = f32x4{o[qt][dt][4 * i], o[qt][dt][4 * i + 1], o[qt][dt][4 * i + 2], o[qt][dt][4 * i + 3]};
          its[DT * 1024 + seg_lane] = m_run[qt];
          its[DT * 1024 + 64 + seg_lane] = l_run[qt];
        }
      }
      __syncthreads();
      if (kp == 0) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
          for (int q = 0; q < SH::KP - 1; ++q) {
            const float* its = part + ((q * SH::CW + rg) * QT + qt) * (SH::PART / 4);
            const float mo = its[DT * 1024 + seg_lane], lother = its[DT * 1024 + 64 + seg_lane];
            const float m = fmaxf(m_run[qt], mo), base = m > -INFINITY ? m : 0.f;
            const float a0 = __builtin_amdgcn_exp2f(m_run[qt] - base), a1 = __builtin_amdgcn_exp2f(mo - base);
            l_run[qt] = l_run[qt] * a0 + lother * a1;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 x = *(const f32x4*)(its + seg_lane * 4 + (dt * 4 + i) * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[qt][dt][4 * i + e] = o[qt][dt][4 * i + e] * a0 + x[e] * a1;
              }
            m_run[qt] = m;
          }
      }
      __syncthreads();  // (the next segment's tiles go there)
    }
    // ---- what the segment leaves, in the order of the registers -------------------------------------------------------------
    if (kp == 0 && live_wave) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        l_run[qt] += __shfl_xor(l_run[qt], 32, 64);
        float* po = p.po + ((size_t)slot * (R / 32) + rg * QT + qt) * (DT * 1024) + seg_lane * 4;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *(f32x4*)(po + (dt * 4 + i) * 256) = f32x4{o[qt][dt][4 * i], o[qt][dt][4 * i + 1], o[qt][dt][4 * i + 2], o[qt][dt][4 * i + 3]};
        if (sh == 0) {
          float* ml = p.pml + (size_t)slot * 2 * R + (rg * QT + qt) * 32 + sc;
          ml[0] = m_run[qt];
          ml[R] = l_run[qt];
        }
      }
    }
  }
#endif
}

// ---- the join ------------------------------------------------------------------------------------------------------------
struct PrefixJoinParams {
  PrefixAttnParams a;
  int out_bf16;
  void* out;   // [B][H][max_nodes][dh]
  float* lse;  // [B][H][max_nodes] or null
};

// One workgroup of DHP / 32 wavefronts per (32 rows of a sequence, key head): every wavefront weighs the rows' partial results
// and adds up 32 components of them - the prefix's, then the sequence's own, each in the order of its keys, four at a time
// under way.
template <typename SH>
__global__ __launch_bounds__(2 * SH::DHP) void prefix_join_kernel(PrefixJoinParams p) {
  constexpr int DT = SH::DT, R = SH::R;
  const int lane = threadIdx.x & 63, dt = threadIdx.x >> 6, c = lane & 31, h2 = lane >> 5;
  const int kh = blockIdx.y, b = blockIdx.z, r = blockIdx.x * 32 + c;
  const Work t = read_work<SH>(p.a);
  const int n = __builtin_amdgcn_readlane(t.n, b);
  if ((int)blockIdx.x * 32 >= n * p.a.group) return;
  const bool live = r < n * p.a.group;
  const Deal d = prefix_deal(t.units, SH::GROUPS);
  const int rr = live ? r : 0;  // this row's place in its sequence, and among all rows
  const int rp = __builtin_amdgcn_readlane(t.first, b) * p.a.group + rr;
  float m = -INFINITY, l = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  // partial results w0 + item .. w1 + item of the block of rows that holds `row`
  auto gather = [&](int item, int w0, int w1, int row) __attribute__((always_inline)) {
    const float* ml = p.a.pml + (size_t)item * 2 * R + row % R;
    const float* po = p.a.po + ((size_t)item * (R / 32) + row % R / 32) * (DT * 1024) + dt * 1024 + (h2 * 32 + row % 32) * 4;
    constexpr int kBatch = 4;
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
  };
  if (t.piters > 0) {
    const int item = kh * t.pblocks + rp / R;
    const int first = item * prefix_units<SH>(t.piters) + prefix_block_units(SH::F32);
    gather(item, d.owner(first), d.owner(first + (t.piters - 1) * prefix_shared_weight(R)), rp);
  }
  const int oi = __builtin_amdgcn_readlane(t.iters, b), blk = rr / R;
  const int ou = t.punits + kh * t.head_units + __builtin_amdgcn_readlane(t.unit0, b) +
                 blk * own_units<SH>(oi) + prefix_block_units(SH::F32);
  const int oitem = t.pitems + kh * t.head_blocks + __builtin_amdgcn_readlane(t.block0, b) + blk;
  const int x0 = d.owner(ou), x1 = d.owner(ou + (oi - 1) * kPrefixOwnWeight);
  gather(oitem, x0, x1, rr);
  if (!live) return;
  const int node = r / p.a.group, hg = r - node * p.a.group;
  int odd = 0;
  for (int w = x0; w <= x1; ++w) odd |= p.a.odd[w + oitem];
  if (odd) {  // values of tree nodes that are infinite or not a number, left out so far: into the rows that see them
    const int W = (p.a.max_nodes + 63) >> 6;
    const unsigned long long* mask = p.a.anc_mask + ((size_t)b * p.a.max_nodes + node) * W;
    const unsigned char* vt = p.a.v_tree + ((size_t)b * p.a.H_kv + kh) * p.a.max_nodes * p.a.dh * SH::ES;
    for (int j = 0; j < n; ++j) {
      if (!((mask[j >> 6] >> (j & 63)) & 1ull)) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = 32 * dt + 8 * i + 4 * h2 + e;
          if (at >= p.a.dh) continue;
          float v;
          if constexpr (SH::F32) v = ((const float*)vt)[(size_t)j * p.a.dh + at];
          else v = bf16_bits_to_float(((const unsigned short*)vt)[(size_t)j * p.a.dh + at]);
          if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[i][e] += v;
        }
    }
  }
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
//                                                                                        F32   DHP  QT CW KP KT NS WPE
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 256, FINE> { using type = PrefixShape<false, DHP, 1, 8, 1, 2, 4, 2, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 128, FINE> { using type = PrefixShape<false, DHP, 1, 4, 2, 1, 4, 2, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 64, FINE> { using type = PrefixShape<false, DHP, 1, 2, 2, 1, 4, 1, FINE>; };
template <int DHP, bool FINE> struct ShapeFor<false, DHP, 32, FINE> { using type = PrefixShape<false, DHP, 1, 1, 2, 1, 4, 1, FINE>; };
template <int DHP> struct ShapeFor<true, DHP, 128, true> { using type = PrefixShape<true, DHP, 1, 4, 1, 1, 4, 1, true>; };
template <int DHP> struct ShapeFor<true, DHP, 32, true> { using type = PrefixShape<true, DHP, 1, 1, DHP == 64 ? 2 : 1, 1, 3, 1, true>; };

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
            return hipFuncSetAttribute((const void*)prefix_attn_kernel<SH>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS);
          });
        }
  return e;
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" size_t prefix_verify_attn_workspace_bytes(int B, int H, int H_kv, int dh, int max_nodes) {
  if (B < 1 || H < 1 || H_kv < 1 || H % H_kv || dh < 1 || max_nodes < 1) return 0;
  size_t most = 0;
  for (bool any_prefix : {false, true})
    for (bool f32 : {false, true}) {
      const size_t bytes = prefix_workspace(B, H, H_kv, dh, max_nodes, any_prefix, f32).total;
      most = bytes > most ? bytes : most;
    }
  return most;
}

extern "C" int prefix_verify_attn(ctcspec_ctx* ctx, ctcspec_dtype dt, const void* q, const void* k_prefix, const void* v_prefix,
                                  const int32_t* prefix_len, int prefix_cap, const void* k_cache, const void* v_cache,
                                  const int64_t* kv_off, const int32_t* ctx_len, int kv_cap, const void* k_tree, const void* v_tree,
                                  const int32_t* n_nodes, const uint64_t* anc_mask, int B, int H, int H_kv, int dh, int max_nodes,
                                  float scale, void* workspace, size_t workspace_bytes, ctcspec_dtype out_dt, void* out, float* lse) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, q && prefix_len && kv_off && ctx_len && k_tree && v_tree && n_nodes && anc_mask && workspace && out &&
                           ((k_prefix && v_prefix) || prefix_cap == 0) && ((k_cache && v_cache) || kv_cap == 0),
                  CTCSPEC_EINVAL, "prefix_verify_attn: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && H > 0 && H_kv > 0 && dh > 0 && max_nodes > 0 && prefix_cap >= 0 && kv_cap >= 0, CTCSPEC_EINVAL,
                  "prefix_verify_attn: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, H % H_kv == 0, CTCSPEC_EINVAL, "prefix_verify_attn: H must be a multiple of H_kv");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "prefix_verify_attn: unknown element type");
  CTCSPEC_REQUIRE(ctx, out_dt == CTCSPEC_F32 || (out_dt == CTCSPEC_BF16 && dt == CTCSPEC_BF16), CTCSPEC_EINVAL,
                  "prefix_verify_attn: the output is float, or bf16 with bf16 operands");
  CTCSPEC_REQUIRE(ctx, scale > 0.f && scale <= 2.0e38f, CTCSPEC_EINVAL, "prefix_verify_attn: the scale must be positive and at most 2e38");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && max_nodes <= CTCSPEC_MAX_NODES, CTCSPEC_EUNSUPPORTED,
                  "prefix_verify_attn: dh must be a multiple of 8 and <= %d, max_nodes <= %d", CTCSPEC_MAX_HEAD_DIM, CTCSPEC_MAX_NODES);
  CTCSPEC_REQUIRE(ctx, B <= ctx->lim.max_batch && B <= 64 && max_nodes <= ctx->lim.max_nodes && H <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim && H_kv <= 65535,
                  CTCSPEC_EUNSUPPORTED, "prefix_verify_attn: shape exceeds the context's limits");
  const bool f32 = dt == CTCSPEC_F32, fine = out_dt == CTCSPEC_F32;
  const PrefixWorkspace ws = prefix_workspace(B, H, H_kv, dh, max_nodes, prefix_cap > 0, f32);
  CTCSPEC_REQUIRE(ctx, prefix_units_fit(ws.rows, B, H_kv, (long long)max_nodes * (H / H_kv), prefix_padded_dim(dh), prefix_cap, kv_cap, max_nodes, f32),
                  CTCSPEC_EUNSUPPORTED, "prefix_verify_attn: capacities or rows beyond 2^30, or work of more than 2^31 units");
  for (const void* a : {q, k_prefix, v_prefix, k_cache, v_cache, k_tree, v_tree, (const void*)workspace, (const void*)out})
    CTCSPEC_REQUIRE(ctx, aligned16(a), CTCSPEC_EINVAL, "prefix_verify_attn: pointers must be 16-byte aligned");
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
  p.po = (float*)(base + ws.o); p.pml = (float*)(base + ws.ml); p.odd = (int*)(base + ws.odd);
  j.out_bf16 = out_dt == CTCSPEC_BF16; j.out = out; j.lse = lse;
  hipStream_t st = ctx->stream;
  const hipError_t e = with_shape(f32, prefix_padded_dim(dh), fine, ws.rows, [&](auto shape) {
    using SH = decltype(shape);
    hipLaunchKernelGGL(prefix_attn_kernel<SH>, dim3(SH::GROUPS), dim3(64 * SH::NW), SH::LDS, st, p);
    if (const hipError_t e1 = hipGetLastError(); e1 != hipSuccess) return e1;
    hipLaunchKernelGGL(prefix_join_kernel<SH>, dim3((unsigned)((max_nodes * p.group + 31) / 32), (unsigned)H_kv, (unsigned)B),
                       dim3(2 * SH::DHP), 0, st, j);
    return hipGetLastError();
  });
  CTCSPEC_HIP(ctx, e);
  return CTCSPEC_OK;
}
