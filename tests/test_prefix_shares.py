"""What prefix_verify_attn's join reads is what its workgroups have left (csrc/prefix_plan.h: code without HIP), on the CPU: of the workgroups
between the owners of a block's first and last iteration every one begins an iteration of the block, and no other does."""
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
// blocks of so many iterations with so many units each -> 0 or what is wrong
static int check(const int* iters, const int* weight, int blocks, int groups, bool f32) {
  static int units[1 << 13];
  int total = 0;
  for (int i = 0; i < blocks; ++i) total += units[i] = prefix_block_units(f32) + iters[i] * weight[i];
  const Deal d = prefix_deal(total, groups);
  int at = 0;
  for (int i = 0; i < blocks; ++i) {
    const int first = at + prefix_block_units(f32);
    const int w0 = d.owner(first), w1 = d.owner(first + (iters[i] - 1) * weight[i]);
    int sum = 0;
    for (int w = 0; w < d.groups; ++w) {
      int a = d.begin(w) - at, b = d.begin(w + 1) - at;  // of the block's units
      a = a < 0 ? 0 : a;
      b = b > units[i] ? units[i] : b;
      const int here = a < b ? prefix_iterations(b, weight[i], f32) - prefix_iterations(a, weight[i], f32) : 0;
      if ((here > 0) != (w0 <= w && w <= w1)) return 1;
      sum += here;
    }
    if (sum != iters[i]) return 2;
    at += units[i];
  }
  return 0;
}
int main() {
  int blocks, f32;
  static int iters[1 << 13], weight[1 << 13];
  while (scanf("%d %d", &f32, &blocks) == 2) {
    for (int i = 0; i < blocks; ++i) if (scanf("%d %d", iters + i, weight + i) != 2) return 1;
    printf("%d\n", check(iters, weight, blocks, kPrefixMaxGroups, f32) + 10 * check(iters, weight, blocks, 256, f32));
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("shares")
    (at / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++20", "-I", CSRC, str(at / "p.cpp"), "-o", str(at / "p")], check=True)
    return str(at / "p")


def test_a_partial_result_from_every_workgroup_that_the_join_asks(program):
    rng = random.Random(5)
    cases = [(f32, [(i, w)]) for f32 in (0, 1) for w in (2, 3) for i in range(1, 200)]  # (few units: the shortest shares)
    for _ in range(400):
        n, most = rng.choice([1, 2, 3, 8, 65, 400]), rng.choice([1, 2, 5, 40, 2000])
        shared = rng.randint(0, n)
        cases.append((rng.randint(0, 1), [(rng.randint(1, most), rng.choice([2, 3]) if i < shared else 2) for i in range(n)]))
    text = "\n".join(f"{f} {len(c)} " + " ".join(f"{i} {w}" for i, w in c) for f, c in cases)
    got = subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert got == ["0"] * len(cases)


def test_a_share_is_all_work_or_half_of_six_units(tmp_path):
    (tmp_path / "p.cpp").write_text(r"""
#include <initializer_list>
#include <stdio.h>
#include "prefix_plan.h"
using namespace ctcspec;
int main() {
  int least = 1 << 30;
  for (int groups : {256, 512})
    for (int units = kPrefixMinUnits + 1; units < 20000; ++units) {
      const Deal d = prefix_deal(units, groups);
      for (int w : {0, d.groups - 1}) least = d.begin(w + 1) - d.begin(w) < least ? d.begin(w + 1) - d.begin(w) : least;
    }
  printf("%d %d", least, prefix_deal(kPrefixMinUnits, 512).groups);
}
""")
    subprocess.run(["g++", "-O1", "-std=c++20", "-I", CSRC, str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    assert subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout == "3 1"
