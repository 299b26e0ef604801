// Instantiations: a router's balance loss.
#include "rtopk_balance.hpp"

namespace rtopk {

namespace {

template <int DT>
hipError_t balance_of_type(const BalanceArgs& a, hipStream_t s) {
  const RouterLanes r = router_lanes(a.E, DT, a.k, false);
  const dim3 grid((uint32_t)(a.groups * a.per_group)), block(64 * kBalanceWaves);
#define X(n, l)                                                                                           \
  if constexpr (is_router_of(DT, l))                                                                      \
    if (r.lanes == n && r.loads == l)                                                                     \
      return a.E % logits_width(DT) != 0 ? launch_kernel(balance_kernel<DT, n, l, true>, grid, block, 0, s, a) \
                                         : launch_kernel(balance_kernel<DT, n, l, false>, grid, block, 0, s, a);
  RTOPK_ROUTER_LIST(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_balance(int dtype, const BalanceArgs& a, hipStream_t s) {
  return dtype == kF32 ? balance_of_type<kF32>(a, s) : dtype == kF16 ? balance_of_type<kF16>(a, s) : balance_of_type<kBF16>(a, s);
}

hipError_t launch_balance_join(const BalanceArgs& a, hipStream_t s) {
  if (a.per_group <= kFewParts) return launch_kernel(balance_join_kernel<256, 256>, dim3((uint32_t)(a.groups * ceil_div(a.E, 256))), dim3(256), 0, s, a);
  return launch_kernel(balance_join_kernel<1024, kJoinCols>, dim3((uint32_t)(a.groups * ceil_div(a.E, kJoinCols))), dim3(1024), 0, s, a);
}

}  // namespace rtopk
