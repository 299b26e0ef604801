// Instantiations: gradient kernels of the operators on rows of logits.
#include "rtopk_logits.hpp"

namespace rtopk {

namespace {

template <int DT, int W>
hipError_t grad_of_waves(int op, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  const dim3 grid((uint32_t)(rows * a.segments)), block(64 * W);
  if (op == kOpDistill) return launch_kernel(logits_grad_kernel<DT, kOpDistill, false, false, W>, grid, block, list_bytes(a.k), s, a);
  return a.grad_entropy ? launch_kernel(logits_grad_kernel<DT, kOpTokens, true, false, W>, grid, block, list_bytes(a.k), s, a)
                        : launch_kernel(logits_grad_kernel<DT, kOpTokens, false, false, W>, grid, block, list_bytes(a.k), s, a);
}

template <int DT>
hipError_t grad_of_type(int op, int waves, bool join, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  if (join)
    return launch_kernel(logits_grad_kernel<DT, kOpDistill, false, true, 4>, dim3((uint32_t)(rows * a.segments)), dim3(256), list_bytes(a.k), s, a);
  if constexpr (DT != kF32)
    if (waves == 1) return grad_of_waves<DT, 1>(op, a, rows, s);
  return grad_of_waves<DT, 4>(op, a, rows, s);
}

template <int DT>
hipError_t row_of_type(int waves, int loads, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  const dim3 grid((uint32_t)rows), block((uint32_t)(64 * waves));
#define X(w, r, q)                     \
  if constexpr (is_held_by(DT, w, r)) \
    if (waves == w && loads == r + q) return launch_kernel(distill_held_kernel<DT, w, r, q>, grid, block, list_bytes(a.k), s, a);
  RTOPK_HELD_LIST(X)
#undef X
  return launch_kernel(distill_row_kernel<DT, 8>, grid, dim3(512), list_bytes(a.k), s, a);
}

}  // namespace

hipError_t launch_logits_grad(int dtype, int op, int waves, bool join, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32   ? grad_of_type<kF32>(op, waves, join, a, rows, s)
         : dtype == kF16 ? grad_of_type<kF16>(op, waves, join, a, rows, s)
                         : grad_of_type<kBF16>(op, waves, join, a, rows, s);
}

hipError_t launch_distill_row(int dtype, int waves, int loads, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32 ? row_of_type<kF32>(waves, loads, a, rows, s) : dtype == kF16 ? row_of_type<kF16>(waves, loads, a, rows, s) : row_of_type<kBF16>(waves, loads, a, rows, s);
}

}  // namespace rtopk
