// Drawn tokens and verified drafts: limits, and how a call's sequences are laid over workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

constexpr int kMaxDrafts = 128;  // drafted tokens of a sequence

constexpr int kDrawWaves = 4;    // of a workgroup that shares a sequence with others
constexpr int kMostPieces = 64;  // of a row that one workgroup takes
constexpr int64_t kTestedCells = (int64_t)1 << 26;  // logits of a call from which on drafts are tested in fp32 first

// A row in `pieces` pieces of `cols` columns (the last one what is left), a whole number of 128-bit loads of a wavefront.  spread: a wavefront of any workgroup
// to a piece; else a workgroup of `waves` wavefronts to a sequence.  tested: drafts are tested in fp32 beforehand, `positions` of each sequence in a
// launch, by workgroups of `test_waves` wavefronts.
struct DrawLayout {
  bool spread;
  int waves, pieces, cols;
  int groups;  // (spread) workgroups that share a sequence's draw
  bool tested;
  int positions, test_waves;
};

inline int draw_rows(int G, bool draft) { return draft ? 2 * G + 1 : G + 1; }
// Rows of a sequence whose pieces' masses are kept.
inline int kept_rows(int G, bool draft, const DrawLayout& l) { return l.tested ? (draft ? 2 : 1) : draw_rows(G, draft); }

// Pieces of `loads` loads, more where there would be more than `most` pieces.
inline DrawLayout draw_pieces(int M, int dtype, int64_t loads, int most) {
  const int64_t step = 64 * logits_width(dtype);
  if (ceil_div(M, loads * step) > most) loads = ceil_div(M, most * step);
  return {false, 4, (int)ceil_div(M, loads * step), (int)(loads * step), 1, false, 0, 0};
}

inline DrawLayout draw_layout_whole(int64_t B, int M, int dtype) {
  DrawLayout l = draw_pieces(M, dtype, 1, kMostPieces);
  l.waves = M <= 2048 || B > 512 ? 4 : (B > 256 ? 8 : 16);
  return l;
}

inline DrawLayout draw_layout(int64_t B, int G, int M, int dtype, bool draft) {
  DrawLayout l = draw_layout_whole(B, M, dtype);
  if (B > 16384 || l.pieces <= 4) return l;
  const int64_t rows = draw_rows(G, draft), row = 64 * logits_width(dtype);
  const bool tested = rows >= 5 && B * rows * M >= kTestedCells;
  int64_t loads = 1;
  while (loads < 4 && B * (tested ? (draft ? 2 : 1) : rows) * ceil_div(M, 2 * loads * row) >= 4096) loads *= 2;
  l = draw_pieces(M, dtype, loads, 1024);
  l.spread = true;
  if (draft) {
    l.groups = (int)ceil_div(l.pieces, kDrawWaves);
    if (B * l.groups > 1024) l.groups = B < 1024 ? (int)(1024 / B) : 1;
  }
  if (tested) {
    l.tested = true;
    l.positions = (int)(B < 512 ? ceil_div(512, B) : 1);
    if (l.positions > G) l.positions = G;
    const int64_t workgroups = B * l.positions;
    l.test_waves = workgroups <= 256 ? 16 : (workgroups <= 512 ? 8 : 4);
  }
  return l;
}

// Device memory: masses of the pieces, their sums of max(p - q, 0), a counter for each sequence, what the tests have accepted.
inline int64_t draw_workspace(int64_t B, int G, bool draft, const DrawLayout& l) {
  if (!l.spread) return 0;
  return B * l.pieces * (16 * (int64_t)kept_rows(G, draft, l) + 8) + 4 * B + (l.tested ? B * G : 0);
}

}  // namespace rtopk
