// q4_verify_attn: rows of a workgroup, which tiles of keys a window leaves, and the workspace.  The work is dealt to the workgroups as in
// prefix_plan.h, or in pieces of blocks.  Code without HIP, so that a test can ask it.
#pragma once

#include "prefix_plan.h"

namespace ctcspec {

constexpr int kQ4Tiles = 4;  // tiles of 32 keys in an iteration: one for each wavefront of a workgroup

// Query rows of a workgroup (nodes of a sequence x heads that share a key head), and the workgroups that a compute unit holds at once: with
// 32 rows the registers of three wavefronts a SIMD hold a row's result and the next tile, with 64 those of two.  (8 sequences x 64 nodes x 32
// heads behind 256 to 2048 rows, four behind 32768, us: 64 rows and two 57 and 253, 32 and three 42 and 210 - of a kernel that had bank conflicts and spilled
// registers, and with codes fetched in another way: 64 rows have not been measured by themselves.)
constexpr int kQ4Rows = 32;
constexpr int kQ4Waves = 3;
constexpr int kQ4Groups = 256 * kQ4Waves;

// The cached tiles that a window leaves: the first `lead`, then those from lead + gap on; `count` of them.  A row at position p >= len sees
// keys above p - window and below sink, so the tiles between the sink and position len - window stay out.
struct Q4Tiles {
  int lead, gap, count;
};
CTCSPEC_BOTH Q4Tiles q4_tiles(int len, int window, int sink) {
  Q4Tiles t;
  const int all = (len + 31) / 32;
  t.lead = t.count = all;
  t.gap = 0;
  if (window > 0 && window <= len) {
    const int lead = ((sink < len ? sink : len) + 31) / 32, from = (len - window + 1) / 32;
    if (lead < from) {
      t.lead = lead;
      t.gap = from - lead;
      t.count = all - t.gap;
    }
  }
  return t;
}

// A block of rows counts as four iterations over the keys beside its own.  (As two: the same times within 2 %.)
CTCSPEC_BOTH constexpr int q4_units(int iters) { return prefix_block_units(false) + iters * kPrefixOwnWeight; }

// A block's iterations in pieces of `most` at the most, as equal as can be: how many pieces, and where the i-th begins.
CTCSPEC_BOTH constexpr int q4_pieces(int iters, int most) { return iters > 0 ? (iters - 1) / most + 1 : 0; }
CTCSPEC_BOTH constexpr int q4_piece_begin(int iters, int pieces, int i) {
  const int each = iters / pieces, more = iters - each * pieces;
  return i * each + (i < more ? i : more);
}
// Such pieces are the shares where they are no more than the workgroups and not much longer than equal shares would be - half as long again, and
// kQ4PieceSlack iterations: equal shares go across blocks, and a second block in a share costs its way in and out -, and are not made shorter than
// kQ4LeastPiece.  (us with equal shares / pieces.  Eight sequences of one length, 32 heads, single tokens behind 480, 992, 2048 rows: 19.7 / 15.8,
// 20.6 / 21.7, 29.0 / 29.8; 64 nodes: 26.2 / 23.0, 38.0 / 31.0, 54.7 / 46.8, 256 to 2048 rows 39 / 39, windows of 4096 73 / 59.)
constexpr int kQ4LeastPiece = 4, kQ4PieceSlack = 4;

// Iterations over a sequence's keys.
CTCSPEC_BOTH int q4_iterations(int nodes, int len, int window, int sink) {
  return (q4_tiles(len, window, sink).count + (nodes + 31) / 32 + kQ4Tiles - 1) / kQ4Tiles;
}
// Whether every block of rows is one workgroup's, in a single launch: where no length makes more than kQ4AloneIterations of them, and every workgroup
// has its place at once.  (bf16, us with a deal and a join / alone, capacities of 16, 448, 960, 1984 rows, all filled.  One sequence, 32
// heads on 8, a node: 10.8 / 7.4, 13.1 / 10.1, 13.7 / 13.0, 14.0 / 19.3; eight 12.4 / 7.5, 14.1 / 10.1, 14.6 / 13.4, 15.3 / 19.5; with 32 key heads
// 12.0 / 7.7, 14.2 / 10.3, 18.3 / 14.2, 24.2 / 20.9, 64 nodes 15.0 / 11.3, 18.7 / 16.2, 24.0 / 22.0, 43.3 / 32.7.  Beyond, alone loses where blocks are few or
// one length is far from the others: 17 iterations, eight sequences, bf16 and float result.  8 key heads, single tokens behind 256 to 2048 rows 14.8 / 20.7 and
// 16.0 / 25.8; 32 key heads 22.0 / 21.7 and 24.7 / 26.6, one behind 2048 and seven behind 64 16.7 / 20.6 and 18.6 / 25.9; 64 nodes 32.0 / 28.1 and
// 40.3 / 36.5, 22.2 / 23.1 and 24.1 / 28.5.  The limit is one for all of these, and for both results, though 256 blocks of many rows would take a higher one.)
constexpr int kQ4AloneIterations = 8;
inline bool q4_alone(long long B, int H_kv, long long seq_rows, int kv_cap, int max_nodes, int window, int sink) {
  long long tiles = (kv_cap + 31LL) / 32;
  const long long seen = (sink + 31LL) / 32 + window / 32 + 3;  // those of a window, and at its ends
  if (window > 0 && seen < tiles) tiles = seen;
  return tiles + (max_nodes + 31) / 32 <= kQ4AloneIterations * kQ4Tiles && B * H_kv * ((seq_rows + kQ4Rows - 1) / kQ4Rows) <= kQ4Groups;
}

// Rows, keys and units are counted in 32 bits: whether that is enough for the largest lengths.
inline bool q4_units_fit(long long B, int H_kv, long long seq_rows, int kv_cap, int max_nodes) {
  if (seq_rows > 1LL << 30 || kv_cap > 1 << 30) return false;
  const long long tiles = (kv_cap + 31LL) / 32 + (max_nodes + 31) / 32;
  const double block = prefix_block_units(false) + (double)kPrefixOwnWeight * (double)((tiles + kQ4Tiles - 1) / kQ4Tiles);
  return (double)B * (double)((seq_rows + kQ4Rows - 1) / kQ4Rows) * block * H_kv < 2147483647.0;
}

struct Q4Workspace {
  size_t o, ml, odd, span, total;
};
// Numbers of partial results: below workgroups + blocks.
inline Q4Workspace q4_workspace(int B, int H, int H_kv, int dh, int max_nodes) {
  Q4Workspace w;
  size_t off = 0;
  auto carve = [&](size_t bytes) { size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
  const long long seq_rows = (long long)max_nodes * (H / H_kv);
  const size_t slots = kQ4Groups + (size_t)H_kv * B * (size_t)((seq_rows + kQ4Rows - 1) / kQ4Rows);
  const int tiles = (dh + 31) / 32;  // of 32 components
  w.o = carve(slots * kQ4Rows * tiles * 32 * sizeof(float));
  w.ml = carve(slots * kQ4Rows * 2 * sizeof(float));
  w.odd = carve(slots * sizeof(int));
  w.span = carve((slots - kQ4Groups) * 4 * sizeof(int));
  w.total = off;
  return w;
}

}  // namespace ctcspec
