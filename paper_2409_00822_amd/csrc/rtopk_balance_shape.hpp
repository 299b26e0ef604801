// A router's balance loss: limits, and how a call's tokens are laid over lanes and workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

constexpr int kMaxExperts = 1024;
constexpr int kMaxBalanceGroups = 1 << 20;
constexpr int kBalanceWaves = 4;  // of a workgroup

// A token's row of E logits over `lanes` lanes (a power of two), `loads` 128-bit loads each; a wavefront takes 64 / lanes tokens at a time.
struct RouterLanes {
  int lanes, loads;
};
// X(lanes, loads)
#define RTOPK_ROUTER_LIST(X) \
  X(1, 1) X(2, 1) X(4, 1) X(8, 1) X(16, 1) X(32, 1) X(64, 1) X(2, 2) X(4, 2) X(8, 2) X(16, 2) X(32, 2) X(64, 2) X(64, 4)
constexpr bool is_router_of(int dtype, int loads) { return dtype == 0 || loads <= 2; }

// Two loads to a lane where a token's picks still have a lane each: what is done once for all columns of a lane is then done for half as many lanes (us with one
// and with two: loss 262144 x 256 bfloat16 37.1 and 33.7, 500000 x 100 43.8 and 41.0; gradient 16384 x 64 fp32 6.6 and 5.1, 1048576 x 128 bfloat16 111 and 108).
// A gradient takes one where two would not be whole 128-byte lines each, since stores of parts of lines go to memory by themselves (262144 tokens: 252 bfloat16 62 and
// 73, 96 22.8 and 26.3, 60 fp32 26 and 40, 32 13.5 and 16.4; whole lines: 192 bfloat16 with picked values 53.9 and 48.9, 96 fp32 50.5 and 40.8).
inline RouterLanes router_lanes(int E, int dtype, int k, bool grad) {
  const int v = logits_width(dtype), chunks = (E + v - 1) / v;
  int n = 1;
  while (n < 64 && n < chunks) n *= 2;
  if (chunks > 64) return {64, chunks <= 128 ? 2 : 4};
  return n >= 4 && n / 2 >= k && (!grad || (n >= 16 && E % (8 * v) == 0)) ? RouterLanes{n / 2, 2} : RouterLanes{n, 1};
}

// `per_group` workgroups to a group, `rows` tokens each (the last one what is left).
struct BalanceLayout {
  int64_t rows;
  int per_group;
};

// About 1024 workgroups, which is all that fit the GPU at once (us with 512, 1024, 1536, 2048 and 4096: loss 262144 x 256 bfloat16 49.4, 38.7, 42.2, 40.1, 48.9, gradient
// 1048576 x 128 167, 117, 143, 121, 119).
inline BalanceLayout balance_layout(int64_t groups, int64_t per, const RouterLanes& r, bool spread) {
  const int64_t at_once = kBalanceWaves * (64 / r.lanes);  // tokens that a workgroup takes at a time
  if (!spread || per <= at_once) return {per, 1};
  int64_t n = (1024 + groups - 1) / groups, most = (per + at_once - 1) / at_once;
  if (n > most) n = most;
  const int64_t rows = ((per + n - 1) / n + at_once - 1) / at_once * at_once;
  return {rows, (int)((per + rows - 1) / rows)};
}

constexpr int kJoinCols = 32;  // columns that a workgroup joins, all of them where there are
constexpr int kFewParts = 32;  // or fewer parts to join

// A workgroup's sum of squared log-sum-exps, tokens that count, picks.
struct BalancePart {
  double z;
  int32_t counted, picked;
};

// Device memory for the workgroups' partial results: 64-bit sums of probabilities, the above, what blocks of columns have for a loss, picks, counters.
inline int64_t balance_workspace(int64_t groups, int E, const BalanceLayout& l) {
  if (l.per_group <= 1) return 0;
  const int64_t parts = groups * l.per_group, blocks = (E + kJoinCols - 1) / kJoinCols;
  return 8 * parts * E + 16 * parts + 8 * groups * blocks + 4 * parts * E + 4 * groups;
}

}  // namespace rtopk
