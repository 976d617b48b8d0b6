"""How prefix_verify_attn deals its work out (csrc/prefix_plan.h: code without HIP), on the CPU: every unit once, every partial
result in a place of its own inside the workspace, workspaces that serve smaller calls."""
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
// blocks of rows with so many units each -> 0 or what is wrong
static int check(const long long* units, int blocks, int groups) {
  static bool taken[1 << 20];
  static long long covered[1 << 16];
  long long total = 0;
  for (int i = 0; i < blocks; ++i) { total += units[i]; covered[i] = 0; }
  const Deal d = prefix_deal((int)total, groups);
  if (d.groups > groups || (total > 0) != (d.groups > 0)) return 1;
  if (d.begin(d.groups) != total) return 2;
  for (int s = 0; s < groups + blocks; ++s) taken[s] = false;
  long long start = 0;
  int block = 0;
  for (int w = 0; w < d.groups; ++w) {
    long long u = d.begin(w);
    const long long u1 = d.begin(w + 1);
    if (u >= u1) return 3;
    if (d.owner(u) != w || d.owner(u1 - 1) != w) return 4;
    while (u < u1) {
      while (u >= start + units[block]) start += units[block++];
      const long long room = start + units[block] - u, n = room < u1 - u ? room : u1 - u;
      const int slot = w + block;
      if (slot >= groups + blocks || taken[slot]) return 5;
      taken[slot] = true;
      covered[block] += n;
      u += n;
    }
  }
  for (int i = 0; i < blocks; ++i) if (covered[i] != units[i]) return 6;
  return 0;
}
int main() {
  int blocks;
  static long long units[1 << 16];
  while (scanf("%d", &blocks) == 1) {
    for (int i = 0; i < blocks; ++i) if (scanf("%lld", units + i) != 1) return 1;
    printf("%d\n", check(units, blocks, kPrefixMaxGroups) + 10 * check(units, blocks, 256));
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++20", "-I", CSRC, str(at / "p.cpp"), "-o", str(at / "p")], check=True)
    return str(at / "p")


def test_every_unit_once_and_every_partial_result_in_its_own_place(program):
    rng = random.Random(1)
    cases = [[1], [0, 0, 1, 0], [2], [255], [256], [257], [511], [513], [1] * 300, [0] * 5, [1 << 30, 3], [7] * 5000]
    for _ in range(400):
        n = rng.choice([1, 2, 8, 32, 65, 700])
        most = rng.choice([1, 3, 40, 5000])
        cases.append([rng.randint(0, most) for _ in range(n)])
    text = "\n".join(f"{len(c)} " + " ".join(map(str, c)) for c in cases)
    got = subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert got == ["0"] * len(cases)


@pytest.mark.parametrize("H,H_kv,dh", [(4, 4, 16), (32, 32, 128), (40, 8, 128), (12, 1, 64)])
def test_workspace_grows(H, H_kv, dh):
    last = None
    for B in (1, 2, 3, 7, 8, 13, 64):
        row = [pkg.prefix_verify_attn_workspace_bytes(B, H, H_kv, dh, N) for N in range(1, 129)]
        assert row == sorted(row) and row[0] > 0
        assert last is None or all(a <= b for a, b in zip(last, row))
        last = row


def test_workspace_of_no_shape():
    for bad in [(0, 4, 4, 64, 8), (1, 4, 3, 64, 8), (1, 0, 1, 64, 8), (1, 4, 0, 64, 8), (1, 4, 4, 0, 8), (1, 4, 4, 64, 0)]:
        assert pkg.prefix_verify_attn_workspace_bytes(*bad) == 0
