// Host-side table between the C ABI of drawn tokens and verified drafts (rtopk_draw_api.hip) and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_draw_shape.hpp"

namespace rtopk {

// A call's arguments; what it does not use is null or 0.
struct DrawArgs {
  const void* target;  // [B][G + 1][M] logits
  int64_t target_seq, target_pos;  // elements between sequences, between a sequence's rows
  const void* draft;  // [B][G][M], null: a draft stands for itself
  int64_t draft_seq, draft_pos;
  const void* drafts;  // [B][G] tokens, 32 or 64 bits
  int token64, G, M;
  const float* uniforms;  // [B][G + 1]
  const float* temperatures;  // [B], or null: `temperature`
  double temperature, c;       // log2(e) / temperature
  int64_t B, row0;  // sequences; first one of the launch
  void* tokens;     // [B][G + 1], as the drafts
  int32_t* accepted;  // [B], optional
  int pieces, piece_cols;  // of a row
  // sequences spread over workgroups
  int groups;        // workgroups that draw_join_kernel has for a sequence
  double2* part;     // [B][rows][pieces] masses; tested: [B][3][pieces] of target and draft, and what is left of their difference
  double* rest;      // [B][pieces] sums of max(p - q, 0); tested: how near a column's ratio comes to that of fp32 sums
  int32_t* arrived;  // [B]
  float2* near;      // [B][G][2] (tested) maxima and sums in fp32
  uint8_t* accepts;  // [B][G] (tested) what has been accepted
};

// Each enqueues its kernel for sequences [a.row0, a.row0 + n).
hipError_t launch_draw(int dtype, int waves, const DrawArgs& a, int64_t n, hipStream_t stream);  // a workgroup to a sequence
hipError_t launch_draw_test(int dtype, int waves, const DrawArgs& a, int pos0, int positions, int64_t n, hipStream_t stream);
hipError_t launch_draw_mass(int dtype, const DrawArgs& a, int64_t n, hipStream_t stream);
hipError_t launch_draw_join(int dtype, const DrawArgs& a, int64_t n, hipStream_t stream);
hipError_t launch_draw_rest(int dtype, const DrawArgs& a, int64_t n, hipStream_t stream);
hipError_t launch_draw_pick(int dtype, const DrawArgs& a, int64_t n, hipStream_t stream);

}  // namespace rtopk
