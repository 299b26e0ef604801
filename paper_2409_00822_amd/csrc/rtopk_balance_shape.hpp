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

// Two loads to a lane where a token's picks still have a lane each: what is done once for all columns of a lane is then done for half as many lanes.
inline RouterLanes router_lanes(int E, int dtype, int k) {
  const int v = logits_width(dtype), chunks = (E + v - 1) / v;
  int n = 1;
  while (n < 64 && n < chunks) n *= 2;
  if (chunks > 64) return {64, chunks <= 128 ? 2 : 4};
  return n >= 4 && n / 2 >= k ? RouterLanes{n / 2, 2} : RouterLanes{n, 1};
}

// `per_group` workgroups to a group, `rows` tokens each (the last one what is left).
struct BalanceLayout {
  int64_t rows;
  int per_group;
};

inline BalanceLayout balance_layout(int64_t groups, int64_t per, int E, int dtype, int k, bool spread) {
  const RouterLanes r = router_lanes(E, dtype, k);
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
