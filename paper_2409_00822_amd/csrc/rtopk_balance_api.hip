// C ABI of a router's balance loss: argument checks, layout, launches.  Declarations and the full contract are in include/rtopk.h.
#include "rtopk.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_balance_dispatch.hpp"
#include "rtopk_checks.hpp"

namespace {

using namespace rtopk::checks;
using rtopk::BalanceArgs;

// The part of the checks that both calls share, and the arguments they fill.
int tokens_of(BalanceArgs& a, const void* logits, int32_t dtype, int64_t N, int32_t E, int64_t stride, const void* cols, int32_t col_bytes, int32_t k,
              int32_t groups) {
  if (!is_type(dtype) || (col_bytes != 1 && col_bytes != 4)) return RTOPK_ERR_BAD_TYPE;
  if (N < 0 || E < 1 || k < 1 || k > E || groups < 1 || groups > rtopk::kMaxBalanceGroups || N % groups != 0 || (N > 1 && stride < E))
    return RTOPK_ERR_BAD_SHAPE;
  if (E > rtopk::kMaxExperts || (col_bytes == 1 && E > 256)) return RTOPK_ERR_M_TOO_LARGE;
  if (N / groups > INT32_MAX || N > INT64_MAX / 16 / E || (N > 1 && stride > INT64_MAX / 16 / N)) return RTOPK_ERR_BAD_SHAPE;
  a.x = logits;
  a.stride = stride;
  a.per = N / groups;
  a.groups = groups;
  a.E = E;
  a.k = k;
  a.cols = cols;
  a.col_bytes = col_bytes;
  return RTOPK_OK;
}

inline uint64_t rows_bytes(int64_t N, int32_t E, int64_t stride, int dtype) {
  return N > 0 ? ((uint64_t)(N - 1) * (N > 1 ? (uint64_t)stride : 0) + (uint64_t)E) * size_of(dtype) : 0;
}

}  // namespace

extern "C" {

int64_t rtopk_balance_workspace_bytes(int64_t N, int32_t E, int32_t dtype, int32_t k, int32_t groups) {
  if (N < 1 || E < 1 || k < 1 || k > E || E > rtopk::kMaxExperts || !is_type(dtype) || groups < 1 || groups > rtopk::kMaxBalanceGroups || N % groups != 0) return 0;
  return rtopk::balance_workspace(groups, E, rtopk::balance_layout(groups, N / groups, rtopk::router_lanes(E, dtype, k, false), true));
}

int rtopk_balance_loss(const void* logits, int32_t dtype, int64_t N, int32_t E, int64_t stride, const void* cols, int32_t col_bytes, int32_t k,
                       int32_t groups, float* out_loss, float* out_z, float* out_probs, int32_t* out_counts, int32_t* out_rows, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  BalanceArgs a{};
  if (const int status = tokens_of(a, logits, dtype, N, E, stride, cols, col_bytes, k, groups)) return status;
  if (workspace_bytes < 0 || N / groups > INT32_MAX / k) return RTOPK_ERR_BAD_SHAPE;
  if ((N > 0 && (!logits || !cols)) || !out_loss || !out_counts || !out_rows) return RTOPK_ERR_NULL_POINTER;
  const uint64_t n = (uint64_t)N, g = (uint64_t)groups;
  const Buffer buffers[] = {{logits, rows_bytes(N, E, stride, dtype), size_of(dtype), false},
                            {cols, n * k * col_bytes, (uint64_t)col_bytes, false},
                            {out_loss, g * 4, 4, true},
                            {out_z, g * 4, 4, true},
                            {out_probs, g * E * 4, 4, true},
                            {out_counts, g * E * 4, 4, true},
                            {out_rows, g * 4, 4, true},
                            {workspace, (uint64_t)workspace_bytes, 16, true}};
  if (const int status = check_buffers(buffers)) return status;
  a.loss = out_loss;
  a.z = out_z;
  a.probs = out_probs;
  a.counts = out_counts;
  a.counted = out_rows;
  const rtopk::RouterLanes lanes = rtopk::router_lanes(E, dtype, k, false);
  rtopk::BalanceLayout l = rtopk::balance_layout(groups, a.per, lanes, true);
  if (l.per_group > 1 && (!workspace || workspace_bytes < rtopk::balance_workspace(groups, E, l))) l = rtopk::balance_layout(groups, a.per, lanes, false);
  a.rows = l.rows;
  a.per_group = l.per_group;
  const int64_t parts = (int64_t)groups * l.per_group;
  if (l.per_group > 1) {
    const int64_t blocks = (E + rtopk::kJoinCols - 1) / rtopk::kJoinCols;
    a.part_p = static_cast<double*>(workspace);
    a.part_z = reinterpret_cast<rtopk::BalancePart*>(a.part_p + parts * E);
    a.part_dot = reinterpret_cast<double*>(a.part_z + parts);
    a.part_n = reinterpret_cast<int32_t*>(a.part_dot + groups * blocks);
    a.arrived = a.part_n + parts * E;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = rtopk::launch_balance(dtype, a, s);
  if (err == hipSuccess && l.per_group > 1) err = rtopk::launch_balance_join(a, s);
  return err == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

int rtopk_balance_loss_backward(const float* grad_loss, const float* grad_z, const float* grad_vals, const void* logits, int32_t dtype, int64_t N, int32_t E,
                                int64_t stride, const void* cols, int32_t col_bytes, int32_t k, int32_t groups, const int32_t* counts, const int32_t* rows,
                                void* grad_logits, int64_t grad_stride, void* stream) {
  BalanceArgs a{};
  if (const int status = tokens_of(a, logits, dtype, N, E, stride, cols, col_bytes, k, groups)) return status;
  if (N > 1 && (grad_stride < E || grad_stride > INT64_MAX / 16 / N)) return RTOPK_ERR_BAD_SHAPE;
  if (N == 0) return RTOPK_OK;
  if (!grad_loss || !logits || !cols || !counts || !rows || !grad_logits) return RTOPK_ERR_NULL_POINTER;
  const uint64_t n = (uint64_t)N, g = (uint64_t)groups;
  const bool in_place = grad_logits == logits && (N <= 1 || grad_stride == stride);
  const Buffer buffers[] = {{in_place ? nullptr : logits, rows_bytes(N, E, stride, dtype), size_of(dtype), false},
                            {cols, n * k * col_bytes, (uint64_t)col_bytes, false},
                            {grad_loss, g * 4, 4, false},
                            {grad_z, g * 4, 4, false},
                            {grad_vals, n * k * 4, 4, false},
                            {counts, g * E * 4, 4, false},
                            {rows, g * 4, 4, false},
                            {grad_logits, rows_bytes(N, E, grad_stride, dtype), size_of(dtype), true}};
  if (const int status = check_buffers(buffers)) return status;
  a.grad_loss = grad_loss;
  a.grad_z = grad_z;
  a.grad_vals = grad_vals;
  a.counts_in = counts;
  a.counted_in = rows;
  a.grad_x = grad_logits;
  a.grad_stride = grad_stride;
  const rtopk::BalanceLayout l = rtopk::balance_layout(groups, a.per, rtopk::router_lanes(E, dtype, k, true), true);
  a.rows = l.rows;
  a.per_group = l.per_group;
  return rtopk::launch_balance_grad(dtype, a, static_cast<hipStream_t>(stream)) == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

}  // extern "C"
