// Host-side table between the C ABI of drawn tokens and verified drafts (rtopk_draw_api.hip) and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rtopk {

constexpr int kMaxDrafts = 128;  // drafted tokens of a sequence

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
  double temperature;
  int64_t B, row0;  // sequences; first one of the launch
  void* tokens;     // [B][G + 1], as the drafts
  int32_t* accepted;  // [B], optional
};

hipError_t launch_draw(int dtype, const DrawArgs& a, int64_t rows, hipStream_t stream);

}  // namespace rtopk
