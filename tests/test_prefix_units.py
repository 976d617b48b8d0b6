"""What prefix_verify_attn counts in 32 bits (csrc/prefix_plan.h: code without HIP), on the CPU: calls whose units fit are accepted, up to
the last one, and no others."""
import os
import random
import subprocess

import pytest

import paper_2412_00061_amd as pkg

CSRC = os.path.join(os.path.dirname(os.path.abspath(pkg.__file__)), "csrc")
PROGRAM = r"""
#include <stdio.h>
#include "prefix_plan.h"
using namespace ctcspec;
int main() {
  int B, H, H_kv, dh, N, P, cap, f32;
  while (scanf("%d %d %d %d %d %d %d %d", &B, &H, &H_kv, &dh, &N, &P, &cap, &f32) == 8) {
    const int rows = prefix_workspace(B, H, H_kv, dh, N, P > 0, f32).rows;
    const long long seq_rows = (long long)N * (H / H_kv);
    printf("%d %.0f %d\n", rows, prefix_most_units(rows, B, H_kv, seq_rows, prefix_padded_dim(dh), P, cap, N, f32),
           (int)prefix_units_fit(rows, B, H_kv, seq_rows, prefix_padded_dim(dh), P, cap, N, f32));
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """[(B, H, H_kv, dh, max_nodes, prefix_cap, kv_cap, float)] -> [(rows of a workgroup, most units, whether they fit)]."""
    at = tmp_path_factory.mktemp("units")
    (at / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++20", "-I", CSRC, str(at / "p.cpp"), "-o", str(at / "p")], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in calls)
        out = subprocess.run([str(at / "p")], input=text, capture_output=True, text=True, check=True).stdout.split()
        return [(int(out[i]), int(out[i + 1]), out[i + 2] == "1") for i in range(0, len(out), 3)]

    return run


def units(rows, B, H, H_kv, dh, N, P, cap, f32):
    """With every sequence, tree and the prefix as long as they may be, as the kernel counts them: an iteration over the keys is
    64 of them, 32 for float blocks of 128 rows and float heads beyond 64; it is 2 units, against the prefix 3 for 256 rows; a block is
    8 more, 4 for float."""
    keys = 32 if f32 and (rows == 128 or dh > 64) else 64
    seq_rows, block = N * (H // H_kv), 4 if f32 else 8
    tiles = lambda n: -(-n // 32)  # noqa: E731
    own = block + 2 * -(-(tiles(cap) + tiles(N)) * 32 // keys)
    prefix = block + (3 if rows == 256 else 2) * -(-P // keys) if P else 0
    return H_kv * (B * -(-seq_rows // rows) * own + -(-B * seq_rows // rows) * prefix)


def test_units_of_the_longest_call(ask):
    rng = random.Random(2)
    calls = []
    for _ in range(500):
        H_kv, group = rng.choice([1, 2, 3, 8, 32]), rng.choice([1, 1, 4, 7])
        calls.append((rng.randint(1, 64), H_kv * group, H_kv, 8 * rng.randint(1, 16), rng.randint(1, 128), rng.choice([0, 1, 33, 5000, 1 << 22, 1 << 27]),
                      rng.choice([0, 1, 64, 2000, 1 << 20, 1 << 26]), rng.randint(0, 1)))
    for c, (rows, most, fit) in zip(calls, ask(calls)):
        assert most == units(rows, *c), c
        assert fit == (most < 2 ** 31 - 1), c
    assert {r for r, _, _ in ask(calls)} == {32, 64, 128, 256}


@pytest.mark.parametrize("call", [(64, 32, 32, 128, 128), (64, 32, 1, 16, 128), (1, 64, 64, 64, 1), (8, 32, 8, 128, 64)], ids=str)
@pytest.mark.parametrize("f32", [0, 1])
def test_both_sides_of_the_limit(ask, call, f32):
    """The longest prefix, and the longest histories, that fit; one row more does not."""
    for at in (5, 6):
        low, high = 1, (1 << 30) + 1  # fits, does not
        while high - low > 1:
            mid = (low + high) // 2
            low, high = (mid, high) if ask([(*call, *((mid, 70) if at == 5 else (70, mid)), f32)])[0][2] else (low, mid)
        below, above = ([*call, *((n, 70) if at == 5 else (70, n)), f32] for n in (low, high))
        (rows, _, fits), (_, _, does_not) = ask([below, above])
        assert fits and not does_not and units(rows, *below) < 2 ** 31 - 1
        assert low == 1 << 30 or units(rows, *above) >= 2 ** 31 - 1
        if call[:3] == (64, 32, 32) and not f32:  # (as the header says)
            assert low >= (4e7 if at == 5 else 3e7)


def test_a_long_prefix_of_many_sequences_fits(ask):
    """(64 sequences x 128 nodes, 32 heads, four million rows: 2e8 units)"""
    (rows, most, fit), = ask([(64, 32, 32, 128, 128, 1 << 22, 4096, 0)])
    assert rows == 256 and fit and most < 3e8
