// A router's balance loss: limits, and how a call's tokens are laid over lanes and workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

namespace rtopk {

constexpr int kMaxExperts = 1024;
constexpr int kMaxBalanceGroups = 1 << 20;
constexpr int kBalanceWaves = 4;  // of a workgroup

// A token's row of E logits over `lanes` lanes (a power of two), `loads` 128-bit loads each; a wavefront takes 64 / lanes tokens at a time.
struct RouterLanes {
  int lanes, loads;
};
// X(lanes, loads)
#define RTOPK_ROUTER_LIST(X) X(1, 1) X(2, 1) X(4, 1) X(8, 1) X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(64, 4)

inline RouterLanes router_lanes(int E, int dtype) {
  const int v = dtype == 0 ? 4 : 8, chunks = (E + v - 1) / v;
#define X(n, l) \
  if (chunks <= n * l) return {n, l};
  RTOPK_ROUTER_LIST(X)
#undef X
  return {0, 0};
}

// `per_group` workgroups to a group, `rows` tokens each (the last one what is left).
struct BalanceLayout {
  int64_t rows;
  int per_group;
};

inline BalanceLayout balance_layout(int64_t groups, int64_t per, int E, int dtype, bool spread) {
  const RouterLanes r = router_lanes(E, dtype);
  const int64_t at_once = kBalanceWaves * (64 / r.lanes);  // tokens that a workgroup takes at a time
  if (!spread || per <= at_once) return {per, 1};
  int64_t n = (1024 + groups - 1) / groups, most = (per + at_once - 1) / at_once;
  if (n > most) n = most;
  const int64_t rows = ((per + n - 1) / n + at_once - 1) / at_once * at_once;
  return {rows, (int)((per + rows - 1) / rows)};
}

// Device memory for the workgroups' partial results: 64-bit sums of probabilities and of squared log-sum-exps, picks, tokens.
inline int64_t balance_workspace(int64_t groups, int E, const BalanceLayout& l) {
  return l.per_group > 1 ? groups * l.per_group * (8 * ((int64_t)E + 1) + 8 * (((int64_t)E + 2) / 2)) : 0;
}

}  // namespace rtopk
