// Instantiations: tokens drawn from rows of logits, verified drafts.
#include "rtopk_draw.hpp"

namespace rtopk {

namespace {

template <int DT>
hipError_t draw_of_type(int waves, const DrawArgs& a, int64_t n, hipStream_t s) {
  const dim3 grid((uint32_t)n), block(64 * waves);
  return waves == 1   ? launch_kernel(draw_kernel<DT, 1>, grid, block, 0, s, a)
         : waves == 4 ? launch_kernel(draw_kernel<DT, 4>, grid, block, 0, s, a)
         : waves == 8 ? launch_kernel(draw_kernel<DT, 8>, grid, block, 0, s, a)
                      : launch_kernel(draw_kernel<DT, 16>, grid, block, 0, s, a);
}

template <int DT>
hipError_t test_of_type(int waves, const DrawArgs& a, int pos0, int positions, int64_t n, hipStream_t s) {
  const dim3 grid((uint32_t)(n * positions)), block(64 * waves);
  return waves == 4   ? launch_kernel(draw_test_kernel<DT, 4>, grid, block, 0, s, a, pos0, positions)
         : waves == 8 ? launch_kernel(draw_test_kernel<DT, 8>, grid, block, 0, s, a, pos0, positions)
                      : launch_kernel(draw_test_kernel<DT, 16>, grid, block, 0, s, a, pos0, positions);
}

template <int DT>
hipError_t mass_of_type(const DrawArgs& a, int64_t n, hipStream_t s) {
  const int64_t rows = draw_rows(a.G, a.draft != nullptr);
  return launch_kernel(draw_mass_kernel<DT>, dim3((uint32_t)ceil_div(a.pieces, kDrawWaves), (uint32_t)(n * rows)), dim3(64 * kDrawWaves), 0, s, a);
}

template <int DT>
hipError_t rest_of_type(const DrawArgs& a, int64_t n, hipStream_t s) {
  return launch_kernel(draw_rest_kernel<DT>, dim3((uint32_t)ceil_div(a.pieces, kDrawWaves), (uint32_t)n), dim3(64 * kDrawWaves), 0, s, a);
}

template <int DT>
hipError_t pick_of_type(const DrawArgs& a, int64_t n, hipStream_t s) {
  return launch_kernel(draw_pick_kernel<DT>, dim3((uint32_t)n), dim3(64 * kDrawWaves), 0, s, a);
}

template <int DT>
hipError_t join_of_type(const DrawArgs& a, int64_t n, hipStream_t s) {
  if (a.G == 0) return launch_kernel(draw_take_kernel<DT, kDrawWaves>, dim3((uint32_t)n), dim3(64 * kDrawWaves), 0, s, a);
  return launch_kernel(draw_join_kernel<DT, kDrawWaves>, dim3((uint32_t)(n * a.groups)), dim3(64 * kDrawWaves), 0, s, a);
}

}  // namespace

hipError_t launch_draw(int dtype, int waves, const DrawArgs& a, int64_t n, hipStream_t s) {
  return dtype == kF32 ? draw_of_type<kF32>(waves, a, n, s) : dtype == kF16 ? draw_of_type<kF16>(waves, a, n, s) : draw_of_type<kBF16>(waves, a, n, s);
}

hipError_t launch_draw_test(int dtype, int waves, const DrawArgs& a, int pos0, int positions, int64_t n, hipStream_t s) {
  return dtype == kF32   ? test_of_type<kF32>(waves, a, pos0, positions, n, s)
         : dtype == kF16 ? test_of_type<kF16>(waves, a, pos0, positions, n, s)
                         : test_of_type<kBF16>(waves, a, pos0, positions, n, s);
}

hipError_t launch_draw_mass(int dtype, const DrawArgs& a, int64_t n, hipStream_t s) {
  return dtype == kF32 ? mass_of_type<kF32>(a, n, s) : dtype == kF16 ? mass_of_type<kF16>(a, n, s) : mass_of_type<kBF16>(a, n, s);
}

hipError_t launch_draw_join(int dtype, const DrawArgs& a, int64_t n, hipStream_t s) {
  return dtype == kF32 ? join_of_type<kF32>(a, n, s) : dtype == kF16 ? join_of_type<kF16>(a, n, s) : join_of_type<kBF16>(a, n, s);
}

hipError_t launch_draw_rest(int dtype, const DrawArgs& a, int64_t n, hipStream_t s) {
  return dtype == kF32 ? rest_of_type<kF32>(a, n, s) : dtype == kF16 ? rest_of_type<kF16>(a, n, s) : rest_of_type<kBF16>(a, n, s);
}

hipError_t launch_draw_pick(int dtype, const DrawArgs& a, int64_t n, hipStream_t s) {
  return dtype == kF32 ? pick_of_type<kF32>(a, n, s) : dtype == kF16 ? pick_of_type<kF16>(a, n, s) : pick_of_type<kBF16>(a, n, s);
}

}  // namespace rtopk
