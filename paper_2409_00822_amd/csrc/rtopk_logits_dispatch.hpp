// Host-side table between the C ABI of the operators on rows of logits (rtopk_logits_api.hip) and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

enum LogitsOp : int {
  kOpTokens = 0,  // log probabilities of given tokens, entropy, top alternatives
  kOpDistill = 1  // loss against a teacher's list
};

// A call's arguments, as every kernel gets them; what an operator does not use is null or 0.
struct LogitsArgs {
  const void* x;  // [N][M] logits, rows `stride` elements apart
  int64_t N, stride;
  int64_t row0;   // first row of the launch
  int M, k;       // k: alternatives (forward, tokens), given tokens (backward, tokens) or the teacher's entries
  float inv_t, c; // 1 / temperature, log2(e) / temperature
  const void* tokens;  // [N][tokens_per_row], 32 or 64 bits
  int tokens_per_row, token64;
  const void* teacher_vals;  // [N][k]
  const int32_t* teacher_cols;
  int teacher_dtype, log_probs;
  float *logprobs, *entropy, *lse, *loss, *top_logprobs;
  int32_t* top_cols;
  const float *grad, *grad_entropy, *lse_in, *entropy_in;
  void* grad_x;
  int64_t grad_stride;
  int segments, seg_cols;
  int far_group;  // (backward) segments that share a workgroup where the row's sums are taken again
  float4* part;         // [N][segments] maximum, S, A
  uint64_t* part_keys;  // [N][segments][k]
};

// Each enqueues its kernel for rows [a.row0, a.row0 + rows); dtype: of the logits.
hipError_t launch_logits_rows(int dtype, int op, int waves, bool split, const LogitsArgs& a, int64_t rows, hipStream_t stream);
hipError_t launch_logits_join(int dtype, int op, const LogitsArgs& a, int64_t rows, hipStream_t stream);
hipError_t launch_logits_grad(int dtype, int op, int waves, bool join, const LogitsArgs& a, int64_t rows, hipStream_t stream);
// (waves, loads) of RTOPK_HELD_LIST: the row in registers; loads 0: read twice
hipError_t launch_distill_row(int dtype, int waves, int loads, const LogitsArgs& a, int64_t rows, hipStream_t stream);

}  // namespace rtopk
