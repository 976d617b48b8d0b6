"""q4_plan.h, asked on the CPU: which tiles of keys a window leaves, and that partial results lie inside the workspace."""
import functools
import os
import subprocess
import tempfile

import launch_plans

PROGRAM = r"""
#include <stdio.h>
#include "q4_plan.h"
using namespace ctcspec;
int main() {
  char what;
  long long a, b, c, d, e;
  while (scanf(" %c %lld %lld %lld %lld %lld", &what, &a, &b, &c, &d, &e) == 6) {
    if (what == 't') {
      const Q4Tiles t = q4_tiles(a, b, c);
      printf("%d %d %d\n", t.lead, t.gap, t.count);
    } else if (what == 'a') {  // alone, and the most iterations that a length makes
      int most = 0;
      for (int len = 0; len <= b; ++len) {
        const int n = q4_iterations(c, len, d, e);
        most = n > most ? n : most;
      }
      printf("%d %d 0\n", (int)q4_alone(a, 8, c, b, c, d, e), most);
    } else if (what == 'p') {
      const int pieces = q4_pieces(a, b);
      for (int i = 0; i <= pieces; ++i) printf("%d %d %d\n", pieces, i, pieces ? q4_piece_begin(a, pieces, i) : 0);
    } else if (what == 'f') {
      printf("%d 0 0\n", (int)q4_units_fit(a, b, c, d, e));
    } else {
      const Q4Workspace w = q4_workspace(a, b, c, d, e);
      printf("%d %zu %zu\n", kQ4Groups, w.o, w.total);
    }
  }
}
"""


@functools.lru_cache(maxsize=None)
def _program():
    at = tempfile.mkdtemp(prefix="q4_plan")
    with open(os.path.join(at, "plan.cpp"), "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", launch_plans.CSRC, os.path.join(at, "plan.cpp"), "-o", os.path.join(at, "plan")], check=True)
    return os.path.join(at, "plan")


def ask(lines):
    text = "\n".join(" ".join(map(str, line)) for line in lines)
    out = subprocess.run([_program()], input=text, capture_output=True, text=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.split("\n") if line]


def test_a_window_keeps_every_tile_that_a_row_sees():
    cases = [(L, W, S) for L in (0, 1, 31, 32, 33, 64, 100, 999, 1024) for W in (0, 1, 2, 31, 32, 33, 500, 999, 1000, 5000) for S in (0, 1, 32, 33, 700, 9999)]
    for (L, W, S), (lead, gap, count) in zip(cases, ask([("t", *c, 0, 0) for c in cases])):
        tiles = {x if x < lead else x + gap for x in range(count)}
        seen = {j // 32 for j in range(L) if not W or j > L - W or j < S}  # (a row at a later position sees fewer)
        assert seen <= tiles <= set(range((L + 31) // 32)), (L, W, S)
        assert len(tiles) == count <= len(seen) + 1  # (a window of 1 sees no cached row, its tile is kept)


def test_workgroups_alone_have_few_iterations_whatever_the_lengths():
    cases = [(B, cap, n, W, S) for B in (1, 24, 200) for cap in (0, 16, 500, 896, 1024, 3000) for n in (1, 33, 128) for W, S in ((0, 0), (1, 0), (31, 5), (700, 100), (2900, 0))]
    got = ask([("a", *c) for c in cases])
    for (B, cap, n, W, S), (alone, most, _) in zip(cases, got):
        assert not alone or (most <= 8 and B * 8 * -(-n // 32) <= 768), (B, cap, n, W, S)
        if W == 0:
            assert alone == (most <= 8 and B * 8 * -(-n // 32) <= 768)
    assert {a for a, *_ in got} == {0, 1}


def test_pieces_cover_a_block():
    for iters in (0, 1, 2, 3, 7, 64, 257, 2000, 8_388_609):
        for most in (1, 2, 4, 5, 86, 300, 30000):
            if iters / most > 5000:
                continue
            got = ask([("p", iters, most, 0, 0, 0)])
            begins = [x[2] for x in got]
            assert got[0][0] == -(-iters // most) and begins[0] == 0 and begins[-1] == iters
            sizes = [b - a for a, b in zip(begins, begins[1:])]
            assert all(1 <= x <= most for x in sizes) and (not sizes or max(sizes) - min(sizes) <= 1)


def test_units_are_counted_for_the_largest_lengths():
    # 64 x 32 x 4 blocks of 32 rows, 8 units each and 2 for every iteration of 4 tiles: 2^31 > 8192 (8 + 2 x) allows x = 131067, 524268 tiles, of
    # which the tree has 4
    last = (524268 - 4) * 32
    fits = ask([("f", 64, 32, 128, 30_000_000, 128), ("f", 64, 32, 128, 40_000_000, 128), ("f", 1, 1, 1, 1 << 30, 1), ("f", 1, 1, 1, (1 << 30) + 1, 1),
                ("f", 1, 1, (1 << 30) + 1, 8, 128), ("f", 64, 32, 128, last, 128), ("f", 64, 32, 128, last + 1, 128)])
    assert [f[0] for f in fits] == [0, 0, 1, 0, 0, 1, 0]


def test_workspace_has_room_for_every_partial_result():
    for B, H, Hkv, dh, N in ((1, 1, 1, 8, 1), (8, 32, 32, 128, 64), (64, 40, 8, 96, 128), (3, 32, 1, 64, 1)):
        (groups, o, total), = ask([("w", B, H, Hkv, dh, N)])
        blocks = Hkv * B * -(-(N * H // Hkv) // 32)
        slots = groups + blocks  # a part for each workgroup, and one more where a block of rows ends in its share
        assert o == 0 and total >= slots * (32 * (-(-dh // 32) * 32 + 2) + 1) * 4 + blocks * 16
