// verify_sample_filtered: the bounds between which candidates are listed, round after round, where top-p alone decides how many it takes.
// Code without HIP, so that a test can ask it.
#pragma once

#include "prefix_plan.h"

namespace ctcspec {

constexpr int kFilterPartRounds = 3;  // rounds that the parts give a bound for; the one behind them lists what is left

// How many of the parts' largest logits the bound of a round lies below: a quarter of them, three quarters, nearly all.  Of any number of parts from 1 on:
// never fewer than in the round before.
CTCSPEC_BOTH unsigned int filter_parts_above(unsigned int parts, int round) {
  return round == 0 ? parts / 4 + 1 : (round == 1 ? parts - parts / 4 : parts - parts / 40);
}

// The bound of the next round, which lists the tokens from it up to `upto`, the last one's: never above that - tokens between the two would be listed
// a second time -, and not below `least`, where no token is wanted any more (never above `upto` itself).
CTCSPEC_BOTH float filter_next_bound(float upto, float bound, float least) {
  const float lower = bound < upto ? bound : upto;
  return lower > least ? lower : least;
}

}  // namespace ctcspec
