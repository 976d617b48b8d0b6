// prefix_verify_attn: rows of a workgroup in its two passes, how the work is dealt to the workgroups, and the workspace that
// takes.  Code without HIP, so that a test can ask it which shapes a call takes and where its partial results go.
#pragma once

#include <stddef.h>

#if defined(__HIPCC__)
#define CTCSPEC_BOTH __host__ __device__ inline
#else
#define CTCSPEC_BOTH inline
#endif

namespace ctcspec {

constexpr int kPrefixMaxGroups = 512;  // workgroups of a pass: one or two for each compute unit, each with an equal share of the work

// Query rows of a workgroup, by the rows that may share keys (of all sequences for the prefix, of one for its own keys): as many
// as there are, up to what the registers hold - every key is then fetched once for all of them.
inline int prefix_block_rows(long long rows, bool f32) {
  if (rows <= 32) return 32;
  if (f32) return 128;
  return rows <= 64 ? 64 : (rows <= 128 ? 128 : 256);
}

// A pass has units of work in a row - iterations over the keys, for block of rows after block of rows -, and workgroup w has
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
// A share is at least kPrefixMinUnits: what it leaves costs about as much as so many iterations.
constexpr int kPrefixMinUnits = 2;
CTCSPEC_BOTH Deal prefix_deal(int units, int groups) {
  Deal d;
  const int most = (int)(((unsigned)units + kPrefixMinUnits - 1) / kPrefixMinUnits);
  d.units = units;
  d.groups = most < groups ? most : groups;
  d.each = d.groups ? units / d.groups : 0;
  d.more = units - d.each * d.groups;
  return d;
}
// units of a pass are counted in 32 bits: whether that is enough for the largest lengths
inline bool prefix_units_fit(long long sequences, int H_kv, long long rows, int cap, int max_nodes) {
  return sequences * H_kv * ((rows + 31) / 32) * ((cap + 31LL) / 32 + max_nodes / 32 + 1) < (1LL << 31);
}

// (256 rows of a sequence's own do not fit the registers with their masks)
constexpr int kPrefixOwnRows = 128;

inline int prefix_padded_dim(int dh) { return dh <= 64 ? 64 : 128; }

struct PrefixWorkspace {
  int prefix_rows, own_rows;       // rows of a workgroup
  size_t prefix_o, prefix_ml, own_o, own_ml, own_odd, total;
};
// Numbers of partial results: below workgroups + blocks.
inline PrefixWorkspace prefix_workspace(int B, int H, int H_kv, int dh, int max_nodes, bool f32) {
  PrefixWorkspace w;
  size_t off = 0;
  auto carve = [&](size_t bytes) { size_t at = off; off = (off + bytes + 255) / 256 * 256; return at; };
  const long long seq_rows = (long long)max_nodes * (H / H_kv), all_rows = seq_rows * B;
  w.prefix_rows = prefix_block_rows(all_rows, f32);
  w.own_rows = prefix_block_rows(seq_rows < kPrefixOwnRows ? seq_rows : kPrefixOwnRows, f32);
  const size_t prefix_slots = kPrefixMaxGroups + (size_t)H_kv * ((all_rows + w.prefix_rows - 1) / w.prefix_rows);
  const size_t own_slots = kPrefixMaxGroups + (size_t)B * H_kv * ((seq_rows + w.own_rows - 1) / w.own_rows);
  const size_t row = (size_t)prefix_padded_dim(dh) * sizeof(float);
  w.prefix_o = carve(prefix_slots * w.prefix_rows * row);
  w.prefix_ml = carve(prefix_slots * w.prefix_rows * 2 * sizeof(float));
  w.own_o = carve(own_slots * w.own_rows * row);
  w.own_ml = carve(own_slots * w.own_rows * 2 * sizeof(float));
  w.own_odd = carve(own_slots * sizeof(int));
  w.total = off;
  return w;
}

}  // namespace ctcspec
