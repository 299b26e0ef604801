// Drawn tokens and verified drafts: limits, and how a call's sequences are laid over workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

constexpr int kMaxDrafts = 128;  // drafted tokens of a sequence

constexpr int kDrawWaves = 4;    // of a workgroup that shares a sequence with others
constexpr int kMostPieces = 64;  // of a row that one workgroup takes

// A row in `pieces` pieces of `cols` columns (the last one what is left), a whole number of 128-bit loads of a wavefront.  spread: a wavefront of any workgroup
// to a piece; else a workgroup of `waves` wavefronts to a sequence.
struct DrawLayout {
  bool spread;
  int waves, pieces, cols;
};

inline int draw_rows(int G, bool draft) { return draft ? 2 * G + 1 : G + 1; }

// Pieces of `loads` loads, more where there would be more than `most` pieces.
inline DrawLayout draw_pieces(int M, int dtype, int64_t loads, int most) {
  const int64_t step = 64 * logits_width(dtype);
  if (ceil_div(M, loads * step) > most) loads = ceil_div(M, most * step);
  return {false, 4, (int)ceil_div(M, loads * step), (int)(loads * step)};
}

inline DrawLayout draw_layout_whole(int64_t B, int M, int dtype) {
  DrawLayout l = draw_pieces(M, dtype, 1, kMostPieces);
  l.waves = M <= 2048 || B > 512 ? 4 : (B > 256 ? 8 : 16);
  return l;
}

inline DrawLayout draw_layout(int64_t B, int G, int M, int dtype, bool draft) {
  DrawLayout l = draw_layout_whole(B, M, dtype);
  if (B >= 256 || l.pieces <= 4) return l;
  int64_t loads = 1;
  while (loads < 4 && B * draw_rows(G, draft) * ceil_div(M, 2 * loads * 64 * logits_width(dtype)) >= 4096) loads *= 2;
  l = draw_pieces(M, dtype, loads, 1024);
  l.spread = true;
  return l;
}

// Device memory: masses of the pieces, their sums of max(p - q, 0), a counter for each sequence.
inline int64_t draw_workspace(int64_t B, int G, bool draft, const DrawLayout& l) {
  return l.spread ? B * l.pieces * (16 * (int64_t)draw_rows(G, draft) + 8) + 16 * ((B * 4 + 15) / 16) : 0;
}

}  // namespace rtopk
