// Drawn tokens and verified drafts: limits, and how a call's sequences are laid over workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

constexpr int kMaxDrafts = 128;  // drafted tokens of a sequence

// segments 1: a workgroup of `waves` wavefronts to a sequence; else each row over that many workgroups of four, `cols` columns each (the last one what is
// left).
struct DrawLayout {
  int waves, segments, cols;
};

inline int draw_rows(int G, bool draft) { return draft ? 2 * G + 1 : G + 1; }

inline DrawLayout draw_layout_whole(int64_t B, int M) { return {M <= 2048 || B > 512 ? 4 : (B > 256 ? 8 : 16), 1, M}; }

inline DrawLayout draw_layout(int64_t B, int G, int M, int dtype, bool draft) {
  const int step = 256 * logits_width(dtype);  // a 128-bit load of each thread
  if (B >= 256 || M <= step) return draw_layout_whole(B, M);
  int64_t cols = step;
  while (cols < 4 * step && B * draw_rows(G, draft) * ceil_div(M, 2 * cols) >= 1024) cols *= 2;
  while (ceil_div(M, cols) > kMaxLogitsSegments) cols *= 2;
  DrawLayout l = {4, (int)ceil_div(M, cols), (int)cols};
  return l.segments > 1 ? l : draw_layout_whole(B, M);
}

// Device memory: masses of the segments, their sums of max(p - q, 0), a counter for each sequence.
inline int64_t draw_workspace(int64_t B, int G, bool draft, const DrawLayout& l) {
  return l.segments > 1 ? B * l.segments * (16 * (int64_t)draw_rows(G, draft) + 8) + 16 * ((B * 4 + 15) / 16) : 0;
}

}  // namespace rtopk
