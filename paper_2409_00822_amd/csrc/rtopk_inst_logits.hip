// Instantiations: forward kernels of the operators on rows of logits.
#include "rtopk_logits.hpp"

namespace rtopk {

namespace {

template <int DT, int OP, bool TOP>
hipError_t rows_of(int waves, bool split, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  if (split) return launch_kernel(logits_rows_kernel<DT, 4, OP, TOP, true>, dim3((uint32_t)(rows * a.segments)), dim3(256), 0, s, a);
  const dim3 grid((uint32_t)rows);
  const size_t lds = OP == kOpDistill ? list_bytes(a.k) : 0;
  switch (waves) {
    case 1: return launch_kernel(logits_rows_kernel<DT, 1, OP, TOP, false>, grid, dim3(64), lds, s, a);
    case 4: return launch_kernel(logits_rows_kernel<DT, 4, OP, TOP, false>, grid, dim3(256), lds, s, a);
    case 8: return launch_kernel(logits_rows_kernel<DT, 8, OP, TOP, false>, grid, dim3(512), lds, s, a);
    default: return launch_kernel(logits_rows_kernel<DT, 16, OP, TOP, false>, grid, dim3(1024), lds, s, a);
  }
}

template <int DT>
hipError_t rows_of_type(int op, int waves, bool split, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  if (op == kOpDistill) return rows_of<DT, kOpDistill, false>(waves, split, a, rows, s);
  return a.k > 0 ? rows_of<DT, kOpTokens, true>(waves, split, a, rows, s) : rows_of<DT, kOpTokens, false>(waves, split, a, rows, s);
}

template <int DT>
hipError_t join_of_type(int op, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  const dim3 grid((uint32_t)rows), block(256);
  if (op == kOpDistill) return launch_kernel(logits_join_kernel<DT, kOpDistill, false>, grid, block, list_bytes(a.k), s, a);
  return a.k > 0 ? launch_kernel(logits_join_kernel<DT, kOpTokens, true>, grid, block, 0, s, a)
                 : launch_kernel(logits_join_kernel<DT, kOpTokens, false>, grid, block, 0, s, a);
}

}  // namespace

hipError_t launch_logits_rows(int dtype, int op, int waves, bool split, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32   ? rows_of_type<kF32>(op, waves, split, a, rows, s)
         : dtype == kF16 ? rows_of_type<kF16>(op, waves, split, a, rows, s)
                         : rows_of_type<kBF16>(op, waves, split, a, rows, s);
}

hipError_t launch_logits_join(int dtype, int op, const LogitsArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32 ? join_of_type<kF32>(op, a, rows, s) : dtype == kF16 ? join_of_type<kF16>(op, a, rows, s) : join_of_type<kBF16>(op, a, rows, s);
}

}  // namespace rtopk
