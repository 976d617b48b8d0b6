"""filter_plan.h, asked on the CPU: the bounds of the listing rounds fall, so that no token is listed twice."""
import os
import subprocess

import numpy as np
import pytest

import launch_plans

PROGRAM = r"""
#include <stdio.h>
#include "filter_plan.h"
using namespace ctcspec;
int main() {
  for (unsigned parts = 1; parts <= 4096; ++parts) {
    for (int round = 0; round < kFilterPartRounds; ++round) printf("%u ", filter_parts_above(parts, round));
    printf("\n");
  }
  const float inf = __builtin_inff(), at[] = {-inf, -3.4e38f, -7.5f, -1.f, 0.f, 2.f, 30.f, 3.4e38f};
  for (float upto : at)
    for (float bound : at)
      for (float least : at)
        if (least <= upto) printf("%d ", filter_next_bound(upto, bound, least) <= upto && filter_next_bound(upto, bound, least) >= least &&
                                         (bound > upto || bound < least || filter_next_bound(upto, bound, least) == bound));
}
"""


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    at = tmp_path_factory.mktemp("filter_plan")
    (at / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", launch_plans.CSRC, str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)
    return subprocess.run([os.path.join(at, "plan")], capture_output=True, text=True, check=True).stdout.splitlines()


def test_the_rounds_take_more_and_more_parts(answers):
    counts = np.array([[int(x) for x in line.split()] for line in answers[:4096]])
    parts = np.arange(1, 4097)
    assert np.all(counts[:, 0] >= 1) and np.all(np.diff(counts, axis=1) >= 0) and np.all(counts[:, -1] <= parts)
    assert np.all(counts[:, 0] <= parts / 4 + 1) and np.all(counts[:, -1] >= 0.97 * parts)


def test_bounds_do_not_rise(answers):
    assert set(answers[4096].split()) == {"1"}


def test_every_token_is_listed_once(answers):
    """The rounds replayed: bounds below the counted parts' largest logits, tokens from one bound up to the last."""
    counts = [[int(x) for x in line.split()] for line in answers[:4096]]
    rng = np.random.default_rng(1)
    for V in range(1, 700):
        z = rng.standard_normal(V)
        parts = np.sort([z[i:i + 4].max() for i in range(0, V, 4)])[::-1]
        listed, upto = np.zeros(V, dtype=int), np.inf
        for count in counts[len(parts) - 1] + [None]:
            bound = -np.inf if count is None else parts[count - 1] - 0.01
            listed += (z >= bound) & (z < upto)
            upto = bound
        assert np.all(listed == 1), V
