// Instantiations: gradient of a router's balance loss.
#include "rtopk_balance.hpp"

namespace rtopk {

namespace {

template <int DT, int N, int LOADS>
hipError_t grad_of(const BalanceArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)(a.groups * a.per_group)), block(64 * kBalanceWaves);
  if (a.E % logits_width(DT) == 0)
    return a.grad_vals ? launch_kernel(balance_grad_kernel<DT, N, LOADS, true, false>, grid, block, 0, s, a)
                       : launch_kernel(balance_grad_kernel<DT, N, LOADS, false, false>, grid, block, 0, s, a);
  if constexpr (LOADS == 1 || N == 64)
    return a.grad_vals ? launch_kernel(balance_grad_kernel<DT, N, LOADS, true, true>, grid, block, 0, s, a)
                       : launch_kernel(balance_grad_kernel<DT, N, LOADS, false, true>, grid, block, 0, s, a);
  return hipErrorInvalidValue;
}

template <int DT>
hipError_t grad_of_type(const BalanceArgs& a, hipStream_t s) {
  const RouterLanes r = router_lanes(a.E, DT, a.k, true);
#define X(n, l)                                            \
  if constexpr (is_router_of(DT, l) && (l == 1 || n >= 8)) \
    if (r.lanes == n && r.loads == l) return grad_of<DT, n, l>(a, s);
  RTOPK_ROUTER_LIST(X)
#undef X
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_balance_grad(int dtype, const BalanceArgs& a, hipStream_t s) {
  return dtype == kF32 ? grad_of_type<kF32>(a, s) : dtype == kF16 ? grad_of_type<kF16>(a, s) : grad_of_type<kBF16>(a, s);
}

}  // namespace rtopk
