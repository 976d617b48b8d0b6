// prefix_verify_attn: rows of a workgroup, how the work is dealt to the workgroups, and the workspace that
// takes.  Code without HIP, so that a test can ask it which shapes a call takes and where its partial results go.
#pragma once

#include <stddef.h>

#if defined(__HIPCC__)
#define CTCSPEC_BOTH __host__ __device__ inline
#else
#define CTCSPEC_BOTH inline
#endif

namespace ctcspec {

constexpr int kPrefixMaxGroups = 512;  // workgroups: one or two for each compute unit, each with an equal share of the work

// Query rows of a workgroup, by the rows that share the prefix's keys (without one: the rows of a sequence): as many as there
// are, up to what the registers hold, so that every key is fetched once for all of them.  (bf16, 32 heads of 128, us.  8 x 64 nodes
// with 128 / 256: behind 2048 keys 81 / 82, 8192 without history 135 / 98, 32768 445 / 352.  8 x 16 nodes with 128 / 256: behind 16384
// keys 75.6 / 83.2, 2048 32.4 / 30.9; 100 nodes behind 4000 31.9 / 36.4.  8 single tokens with 32 / 64 / 128 / 256: 26.7 / 27.2 /
// 28.7 / 30.5; float, 12 heads of 64, with 32 / 128: 25.5 / 28.2.)
inline int prefix_block_rows(long long rows, bool f32) {
  if (rows <= 32) return 32;
  if (f32) return 128;
  return rows <= 64 ? 64 : (rows <= 128 ? 128 : 256);
}

// Units of work: what an iteration over the prefix and one over a sequence's own keys cost (64 keys against all R rows: products;
// 64 keys against the sequence's rows: the keys' way in), and a block of rows besides its iterations (the rows' way in, the
// first keys' way, what it leaves).  8 sequences x 64 nodes behind 2048 keys with 256 to 2048 of their own, us for 2 : 2 / 3 : 2 /
// 4 : 2 with 256 rows 98 / 82 / 84; 256 short blocks of their own behind 32768 keys take 855 us if a block costs nothing, 312 with 8.
// A float iteration is 32 keys or 64, bound by its products, and costs more: 4 sequences x 100 nodes, 12 heads, behind 1500 keys, us with
// 8 / 4 / 3 units a block: 46.5 / 45.1 / 45.6, twice as wide heads 78.5 / 75.9 / 75.7.
CTCSPEC_BOTH constexpr int prefix_shared_weight(int rows) { return rows == 256 ? 3 : 2; }
constexpr int kPrefixOwnWeight = 2;
CTCSPEC_BOTH constexpr int prefix_block_units(bool f32) { return f32 ? 4 : 8; }

// The work is units in a row - iterations over the keys, for block of rows after block of rows -, and workgroup w has
// those from begin(w) to begin(w + 1).  Where its share crosses into another block, it leaves a partial result for each; that
// of block i is number w + i.  From one partial result to the next in order w or i grows, or both: no two share a number.
struct Deal {
  int units, groups;  // workgroups with work
  int each, more;     // units of a workgroup, and how many workgroups have one more
  CTCSPEC_BOTH int begin(int w) const { return w * each + (w < more ? w : more); }
  CTCSPEC_BOTH int owner(int u) const {
    const int big = more * (each + 1);
    return u < big ? u / (each + 1) : more + (u - big) / each;
  }
};
// As few workgroups as need at most kPrefixMinUnits each, up to those there are: all work is one share, or each has at least
// half as many units (7 units are two shares, 4 and 3).  The join reads a partial result from every workgroup between the owners of
// a block's first and last iteration, so each of these has to begin an iteration there: no share may be shorter than one.
constexpr int kPrefixMinUnits = 6;
static_assert((kPrefixMinUnits + 1) / 2 >= prefix_shared_weight(256) && (kPrefixMinUnits + 1) / 2 >= prefix_shared_weight(32) &&
              (kPrefixMinUnits + 1) / 2 >= kPrefixOwnWeight);
// Iterations that begin in the first `units` units of a block of rows, an iteration being `weight` of them.
CTCSPEC_BOTH int prefix_iterations(int units, int weight, bool f32) {
  const int x = units - prefix_block_units(f32);
  return x > 0 ? (x + weight - 1) / weight : 0;
}
CTCSPEC_BOTH Deal prefix_deal(int units, int groups) {
  Deal d;
  const int most = (int)(((unsigned)units + kPrefixMinUnits - 1) / kPrefixMinUnits);
  d.units = units;
  d.groups = most < groups ? most : groups;
  d.each = d.groups ? units / d.groups : 0;
  d.more = units - d.each * d.groups;
  return d;
}
inline int prefix_padded_dim(int dh) { return dh <= 64 ? 64 : 128; }

// Tiles of 32 keys that an iteration takes: one for each of a shape's key parts, two where a wavefront has all keys of 256 rows.
CTCSPEC_BOTH constexpr int prefix_tiles(int rows, int padded_dim, bool f32) { return f32 && (rows > 32 || padded_dim > 64) ? 1 : 2; }

// The most units that a call can have whose workgroups take `rows` rows.
inline double prefix_most_units(int rows, long long B, int H_kv, long long seq_rows, int padded_dim, int prefix_cap, int kv_cap, int max_nodes, bool f32) {
  const long long tiles = prefix_tiles(rows, padded_dim, f32), block = prefix_block_units(f32);
  auto up = [](long long a, long long b) { return (a + b - 1) / b; };
  const long long own = block + kPrefixOwnWeight * up(up(kv_cap, 32) + up(max_nodes, 32), tiles);
  const long long prefix = prefix_cap ? block + prefix_shared_weight(rows) * up(up(prefix_cap, 32), tiles) : 0;
  return ((double)B * up(seq_rows, rows) * own + (double)up(B * seq_rows, rows) * prefix) * H_kv;
}
// Rows, keys and units are counted in 32 bits: whether that is enough for the largest lengths.
inline bool prefix_units_fit(int rows, long long B, int H_kv, long long seq_rows, int padded_dim, int prefix_cap, int kv_cap, int max_nodes, bool f32) {
  return B * seq_rows <= 1LL << 30 && prefix_cap <= 1 << 30 && kv_cap <= 1 << 30 &&
         prefix_most_units(rows, B, H_kv, seq_rows, padded_dim, prefix_cap, kv_cap, max_nodes, f32) < 2147483647.0;
}

struct PrefixWorkspace {
  int rows;  // of a workgroup
  size_t o, ml, odd, total;
};
// Numbers of partial results: below workgroups + blocks.
inline PrefixWorkspace prefix_workspace(int B, int H, int H_kv, int dh, int max_nodes, bool any_prefix, bool f32) {
  PrefixWorkspace w;
  size_t off = 0;
  auto carve = [&](size_t bytes) { size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
  const long long seq_rows = (long long)max_nodes * (H / H_kv), all_rows = seq_rows * B;
  w.rows = prefix_block_rows(any_prefix ? all_rows : seq_rows, f32);
  const size_t blocks = (size_t)H_kv * ((all_rows + w.rows - 1) / w.rows + B * ((seq_rows + w.rows - 1) / w.rows));
  const size_t slots = kPrefixMaxGroups + blocks;
  w.o = carve(slots * w.rows * prefix_padded_dim(dh) * sizeof(float));
  w.ml = carve(slots * w.rows * 2 * sizeof(float));
  w.odd = carve(slots * sizeof(int));
  w.total = off;
  return w;
}

}  // namespace ctcspec
