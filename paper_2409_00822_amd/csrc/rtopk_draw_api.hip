// C ABI of drawn tokens and verified drafts: argument checks, layout, launches.  Declarations and the full contract are in include/rtopk.h.
#include "rtopk.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rtopk_checks.hpp"
#include "rtopk_dispatch.hpp"
#include "rtopk_draw_dispatch.hpp"

namespace {

using namespace rtopk::checks;
using rtopk::DrawArgs;

// Rows [sequences][positions][M], `seq` and `pos` elements apart: RTOPK_OK and their bytes, or what is wrong with the strides.  Rows may lie in any order
// (positions first, too).
int rows_of_sequences(int64_t B, int64_t positions, int32_t M, int64_t seq, int64_t pos, uint64_t size, uint64_t& bytes) {
  if ((B > 1 && seq < M) || (positions > 1 && pos < M)) return RTOPK_ERR_BAD_SHAPE;
  const int64_t most = INT64_MAX / 16;
  if ((B > 1 && seq > most / B) || (positions > 1 && pos > most / positions)) return RTOPK_ERR_BAD_SHAPE;
  bytes = ((uint64_t)(B > 1 ? (B - 1) * seq : 0) + (uint64_t)(positions > 1 ? (positions - 1) * pos : 0) + (uint64_t)M) * size;
  return RTOPK_OK;
}

}  // namespace

extern "C" {

int64_t rtopk_verify_workspace_bytes(int64_t B, int32_t G, int32_t M, int32_t dtype, int32_t draft_logits) {
  if (B < 1 || G < 0 || G > rtopk::kMaxDrafts || M < 1 || M > rtopk::kMaxLogitsM || !is_type(dtype) || (draft_logits & ~1) != 0) return 0;
  const auto need = [&](bool draft) { return rtopk::draw_workspace(B, G, draft, rtopk::draw_layout(B, G, M, dtype, draft)); };
  const int64_t without = need(false), with = draft_logits != 0 && G > 0 ? need(true) : 0;
  return without > with ? without : with;  // (a call at temperature 0 is laid out without its draft logits)
}

int rtopk_verify_drafts(const void* target_logits, const void* draft_logits, int32_t dtype, int64_t B, int32_t G, int32_t M, int64_t target_seq_stride,
                        int64_t target_pos_stride, int64_t draft_seq_stride, int64_t draft_pos_stride, const void* drafts, int32_t token_bytes,
                        const float* uniforms, const float* temperatures, double temperature, void* out_tokens, int32_t* out_accepted, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || (token_bytes != 4 && token_bytes != 8)) return RTOPK_ERR_BAD_TYPE;
  if (B < 0 || G < 0 || G > rtopk::kMaxDrafts || M < 1 || workspace_bytes < 0) return RTOPK_ERR_BAD_SHAPE;
  if (M > rtopk::kMaxLogitsM) return RTOPK_ERR_M_TOO_LARGE;
  if (!temperatures && (!(temperature >= 0.0) || !isfinite(temperature) || (temperature > 0.0 && !isfinite(1.44269504088896340736 / temperature))))
    return RTOPK_ERR_BAD_TEMPERATURE;
  if (B == 0) return RTOPK_OK;
  if (B > INT64_MAX / 16 / (G + 1)) return RTOPK_ERR_BAD_SHAPE;
  const bool certain = !temperatures && temperature == 0.0;
  uint64_t target_bytes = 0, draft_bytes = 0;
  if (const int status = rows_of_sequences(B, G + 1, M, target_seq_stride, target_pos_stride, size_of(dtype), target_bytes)) return status;
  if (G == 0 || certain) draft_logits = nullptr;
  if (draft_logits)
    if (const int status = rows_of_sequences(B, G, M, draft_seq_stride, draft_pos_stride, size_of(dtype), draft_bytes)) return status;
  if (!target_logits || (G > 0 && !drafts) || (!certain && !uniforms) || !out_tokens) return RTOPK_ERR_NULL_POINTER;
  const uint64_t n = (uint64_t)B, g = (uint64_t)G;
  const Buffer buffers[] = {{target_logits, target_bytes, size_of(dtype), false},
                            {draft_logits, draft_bytes, size_of(dtype), false},
                            {drafts, n * g * token_bytes, (uint64_t)token_bytes, false},
                            {uniforms, n * (g + 1) * 4, 4, false},
                            {temperatures, n * 4, 4, false},
                            {out_tokens, n * (g + 1) * token_bytes, (uint64_t)token_bytes, true},
                            {out_accepted, n * 4, 4, true},
                            {workspace, (uint64_t)workspace_bytes, 16, true}};
  if (const int status = check_buffers(buffers)) return status;
  DrawArgs a{};
  a.target = target_logits;
  a.target_seq = target_seq_stride;
  a.target_pos = target_pos_stride;
  a.draft = draft_logits;
  a.draft_seq = draft_seq_stride;
  a.draft_pos = draft_pos_stride;
  a.drafts = drafts;
  a.token64 = token_bytes == 8;
  a.G = G;
  a.M = M;
  a.uniforms = uniforms;
  a.temperatures = temperatures;
  a.temperature = temperature;
  a.c = 1.44269504088896340736 / temperature;
  a.B = B;
  a.tokens = out_tokens;
  a.accepted = out_accepted;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool draft = draft_logits != nullptr;
  rtopk::DrawLayout l = rtopk::draw_layout(B, G, M, dtype, draft);
  if (l.spread && (!workspace || workspace_bytes < rtopk::draw_workspace(B, G, draft, l))) l = rtopk::draw_layout_whole(B, M, dtype);
  a.pieces = l.pieces;
  a.piece_cols = l.cols;
  hipError_t err = hipSuccess;
  // launch(sequences) for slices whose workgroups fit one launch: 2^31 threads, 65535 rows of a grid with `rows` to a sequence (0: without)
  const auto sliced = [&](int64_t each, int64_t rows, auto launch) {
    int64_t most = (1 << 21) / each;
    if (rows > 0 && most > 65535 / rows) most = 65535 / rows;
    for (a.row0 = 0; a.row0 < B && err == hipSuccess; a.row0 += most) err = launch(B - a.row0 < most ? B - a.row0 : most);
  };
  if (l.spread) {
    a.groups = l.groups;
    const int64_t rows = rtopk::kept_rows(G, draft, l);
    a.part = static_cast<double2*>(workspace);
    a.rest = reinterpret_cast<double*>(a.part + B * rows * l.pieces);
    if (l.tested) {
      const int64_t groups = rtopk::ceil_div(l.pieces, rtopk::kDrawWaves);
      a.near = reinterpret_cast<float2*>(a.rest + B * l.pieces);
      a.accepts = reinterpret_cast<uint8_t*>(a.near + 2 * B * G);
      for (int pos = 0, launch = 0, positions; pos < G; pos += positions, ++launch) {
        positions = l.positions + launch / 2;
        if (positions > G - pos) positions = G - pos;
        sliced(positions, 0, [&](int64_t n) { return rtopk::launch_draw_test(dtype, l.test_waves, a, pos, positions, n, s); });
      }
      sliced(groups, 1, [&](int64_t n) { return rtopk::launch_draw_rest(dtype, a, n, s); });
      sliced(1, 0, [&](int64_t n) { return rtopk::launch_draw_pick(dtype, a, n, s); });
    } else {
      a.arrived = reinterpret_cast<int32_t*>(a.rest + B * l.pieces);
      sliced(rows * rtopk::ceil_div(l.pieces, rtopk::kDrawWaves), rows, [&](int64_t n) { return rtopk::launch_draw_mass(dtype, a, n, s); });
      sliced(l.groups, 0, [&](int64_t n) { return rtopk::launch_draw_join(dtype, a, n, s); });
    }
  } else {
    sliced(1, 0, [&](int64_t n) { return rtopk::launch_draw(dtype, l.waves, a, n, s); });
  }
  return err == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

int rtopk_sample_tokens(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const float* uniforms, const float* temperatures,
                        double temperature, void* out_tokens, int32_t token_bytes, void* workspace, int64_t workspace_bytes, void* stream) {
  return rtopk_verify_drafts(logits, nullptr, dtype, N, 0, M, stride, M, 0, 0, nullptr, token_bytes, uniforms, temperatures, temperature, out_tokens, nullptr,
                             workspace, workspace_bytes, stream);
}

}  // extern "C"
