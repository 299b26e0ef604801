// Instantiations: gradient kernels of the operators on rows of logits.
#include "rtopk_logits.hpp"

namespace rtopk {

namespace {

template <int DT>
hipError_t grad_of_type(int op, bool join, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  const dim3 grid((uint32_t)(rows * a.segments)), block(256);
  if (op == kOpDistill)
    return join ? launch_kernel(logits_grad_kernel<DT, kOpDistill, false, true>, grid, block, 0, s, a)
                : launch_kernel(logits_grad_kernel<DT, kOpDistill, false, false>, grid, block, 0, s, a);
  return a.grad_entropy ? launch_kernel(logits_grad_kernel<DT, kOpTokens, true, false>, grid, block, 0, s, a)
                        : launch_kernel(logits_grad_kernel<DT, kOpTokens, false, false>, grid, block, 0, s, a);
}

template <int DT>
hipError_t row_of_type(int waves, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  const dim3 grid((uint32_t)rows);
  switch (waves) {
    case 1: return launch_kernel(distill_row_kernel<DT, 1>, grid, dim3(64), 0, s, a);
    case 4: return launch_kernel(distill_row_kernel<DT, 4>, grid, dim3(256), 0, s, a);
    default: return launch_kernel(distill_row_kernel<DT, 16>, grid, dim3(1024), 0, s, a);
  }
}

}  // namespace

hipError_t launch_logits_grad(int dtype, int op, bool join, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32   ? grad_of_type<kF32>(op, join, a, rows, s)
         : dtype == kF16 ? grad_of_type<kF16>(op, join, a, rows, s)
                         : grad_of_type<kBF16>(op, join, a, rows, s);
}

hipError_t launch_distill_row(int dtype, int waves, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32 ? row_of_type<kF32>(waves, a, rows, s) : dtype == kF16 ? row_of_type<kF16>(waves, a, rows, s) : row_of_type<kBF16>(waves, a, rows, s);
}

}  // namespace rtopk
