// Host-side table between the C ABI of a router's balance loss (rtopk_balance_api.hip) and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_balance_shape.hpp"

namespace rtopk {

// A call's arguments; what it does not use is null or 0.
struct BalanceArgs {
  const void* x;  // [groups * per][E] logits, rows `stride` elements apart
  int64_t stride, per;  // per: tokens of a group
  int64_t rows;         // tokens of a workgroup
  int groups, per_group;
  int E, k;
  const void* cols;  // [groups * per][k]
  int col_bytes;
  float *loss, *z, *probs;  // [groups], [groups], [groups][E]
  int32_t *counts, *counted;  // [groups][E], [groups]
  double* part_p;       // [groups][per_group][E]
  BalancePart* part_z;  // [groups][per_group]
  double* part_dot;     // [groups][blocks of columns]
  int32_t* part_n;      // [groups][per_group][E]
  int32_t* arrived;     // [groups]
  // gradient
  const float *grad_loss, *grad_z, *grad_vals;  // [groups], [groups] or null, [groups * per][k] or null
  const int32_t *counts_in, *counted_in;
  void* grad_x;
  int64_t grad_stride;
};

hipError_t launch_balance(int dtype, const BalanceArgs& a, hipStream_t stream);
hipError_t launch_balance_join(const BalanceArgs& a, hipStream_t stream);
hipError_t launch_balance_grad(int dtype, const BalanceArgs& a, hipStream_t stream);

}  // namespace rtopk
