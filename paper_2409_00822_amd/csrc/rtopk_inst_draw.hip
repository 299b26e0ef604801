// Instantiations: tokens drawn from rows of logits, verified drafts.
#include "rtopk_draw.hpp"

namespace rtopk {

namespace {

template <int DT>
hipError_t draw_of_type(const DrawArgs& a, int64_t rows, hipStream_t s) {
  return launch_kernel(draw_kernel<DT, 16>, dim3((uint32_t)rows), dim3(1024), 0, s, a);
}

}  // namespace

hipError_t launch_draw(int dtype, const DrawArgs& a, int64_t rows, hipStream_t s) {
  return dtype == kF32 ? draw_of_type<kF32>(a, rows, s) : dtype == kF16 ? draw_of_type<kF16>(a, rows, s) : draw_of_type<kBF16>(a, rows, s);
}

}  // namespace rtopk
