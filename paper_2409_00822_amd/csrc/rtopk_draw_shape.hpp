// Drawn tokens and verified drafts: limits, and how a call's sequences are laid over workgroups.  Host code only (no HIP headers), so that a CPU test can
// sweep the rules.
#pragma once

#include <stdint.h>

#include "rtopk_logits_shape.hpp"

namespace rtopk {

constexpr int kMaxDrafts = 128;  // drafted tokens of a sequence

constexpr int kDrawWaves = 4;    // of a workgroup that shares a sequence with others
constexpr int kMostPieces = 64;  // of a row that one workgroup takes
constexpr int kMostTested = 1 << 20;  // columns of rows that are tested in fp32: the sums' errors are bounded for that many

// A row in `pieces` pieces of `cols` columns (the last one what is left), a whole number of 128-bit loads of a wavefront.  spread: a wavefront of any workgroup
// to a piece; else a workgroup of `waves` wavefronts to a sequence.  tested: drafts are tested in fp32 beforehand, `positions` of each sequence in the first
// two launches, one more in the next two, and so on, by workgroups of `test_waves` wavefronts.
struct DrawLayout {
  bool spread;
  int waves, pieces, cols;
  int groups;  // (spread) workgroups that share a sequence's draw
  bool tested;
  int positions, test_waves;
};

inline int draw_rows(int G, bool draft) { return draft ? 2 * G + 1 : G + 1; }
// Rows of pieces' results that are kept of a sequence.
inline int kept_rows(int G, bool draft, const DrawLayout& l) { return l.tested ? 3 : draw_rows(G, draft); }

// Pieces of `loads` loads, more where there would be more than `most` pieces.
inline DrawLayout draw_pieces(int M, int dtype, int64_t loads, int most) {
  const int64_t step = 64 * logits_width(dtype);
  if (ceil_div(M, loads * step) > most) loads = ceil_div(M, most * step);
  return {false, 4, (int)ceil_div(M, loads * step), (int)(loads * step), 1, false, 0, 0};
}

// What lane `lane` of a wavefront reads of a piece of `cols` columns, in loads of V of them: batch(i) for U chunks from i on, 64 apart, while all lanes have U; then
// one(i, is, some) for chunk i, which there `is` for this lane or not; `some`: not for all of them; and rest(c) for a column of what is less than a chunk.
template <int V, int U, typename Batch, typename One, typename Rest>
__attribute__((always_inline)) constexpr void lane_of_piece(int cols, int lane, Batch batch, One one, Rest rest) {
  const int full = cols / V;
  int i = lane;
  if constexpr (U > 1) {
    for (; i - lane + U * 64 <= full; i += U * 64) batch(i);
  }
  for (; i - lane < full; i += 64) one(i, i < full, i - lane + 64 > full);
  if (lane < cols % V) rest(full * V + lane);
}

// One wavefront to a short sequence where there are many, which pays no barriers (tokens of 16384 rows of 1000 bfloat16 logits 41 us, with four 94; 1024 rows
// 7.4 and 8.7, 64 rows 6.7 and 6.5; 4096 x 8000 43 and 49, 1024 x 8000 21 and 16); else four for short rows or many, eight for few of up to 8192
// columns, sixteen for few wide ones.
inline DrawLayout draw_layout_whole(int64_t B, int M, int dtype) {
  DrawLayout l = draw_pieces(M, dtype, 1, kMostPieces);
  if (M <= 8192) l.waves = 2 * B >= M ? 1 : (M <= 2048 || B > 256 ? 4 : 8);
  else l.waves = B > 512 ? 4 : (B > 256 ? 8 : 16);
  return l;
}

// One workgroup to a sequence, us against spread ones: tokens of rows of up to 8192 columns (1 x 8000 bfloat16 7.8 and 8.8, 1024 x 4000 11.7 and 13.2; 64 x 32000 15.1 and
// 10.6, 4096 x 32000 130 and 107); drafts where rows are short and few (256 sequences of one draft, 1000 columns 10.2 and 13.5, 4000 12.1 and 16.5; of four
// drafts 20.1 and 16.5) or sequences many (4096 of four drafts, 1000 columns 56 and 98).  Very many sequences: tokens of 16385 rows of 12000 columns 248 and 233, 32000
// 562 and 520, 131072 1444 and 1543, so that scratch memory is spared; drafts are tested first, which pays (16385 of four drafts, 32000 columns 2686
// and 1775, three of 8000 713 and 555).
inline bool by_workgroups(int64_t B, int G, int M) {
  if (G == 0) return M <= 8192 || B > 16384;
  if (M > kMostTested && B >= 512) return true;
  return G <= 2 ? M <= 4096 : (M <= 2048 && B >= 1024);
}

// Drafts tested beforehand, us against all rows' sums in 64 bits, four drafts: bfloat16, 32000 columns 16 sequences 20.5 and 17.4, 32 21.3 and 21.8, 64 24.5 and 28.0, 256 53.7
// and 70.9; 131072 columns 16 sequences 37.8 and 29.3, 32 39.1 and 44.3, 64 47.7 and 71.8, 256 131 and 260; fp32, 32000 columns 32 sequences 24.7 and 21.0, 128 40.9 and
// 46.1, 131072 columns 16 sequences 47.0 and 32.5, 64 69.5 and 91.0.  A workgroup to a row is slow for few wide rows.  Narrower rows only where they are
// many (8000 columns, eight drafts, 256 sequences 48.4 and 40.3; 4000 columns, four drafts, 4096 sequences 135 and 178).  Those are of drafts with logits; drafts that were
// looked up, on both sides of the same line (tested, with one sequence fewer not): 131072 columns, seven drafts, 32 sequences 24.8 and 32, three drafts, 64 27.1 and 31.5;
// 50001 half 19.5 and 18.8; 32000, three drafts, 66 16.3 and 16.4, seven drafts, 33 15.4 and 15.9.
inline bool test_first(int64_t B, int G, int M, int dtype, bool draft) {
  const int64_t cells = B * draw_rows(G, draft) * M, least = (int64_t)256 * M;
  return G > 0 && M <= kMostTested && (M >= 16384 || B >= 1024) && cells >= (least > (1 << 23) ? least : 1 << 23) + (dtype == 0 ? 1 << 23 : 0);
}

// Loads of a thread of a workgroup that tests drafts made together (eight for sixteen wavefronts, which have no other workgroup beside them).
constexpr int test_loads(int waves) { return waves == 16 ? 8 : 4; }

// Units of 2^-24 of its value that the fp32 sum of a row of M columns about its maximum is off by at most when drafts are tested; far: where maximum / T is beyond
// what sums run along with (far_maximum), so that each term is taken from the maximum itself.  Terms are weighed by what they are of the sum, and by that their
// distances t from the maximum, in powers of two, average to no more than log2 M <= 20 (an entropy less the log of a sum that is 1 or more):
//   each term   the factor log2(e) / T and the exponent rounded, 2 ln 2 t = 28 (far: the difference too, 42); exp2 2 (off by 0.79 units of its last place at
//               most, over all arguments); a factor without all its bits (T > 10^38) 6
//   each batch  near: half its terms to an accumulator, their sum to the thread's 1, scaled before by an exp2, which is off by 1 + its distance, and a product 1
//               (what it is scaled by is 1, exactly, unless the maximum has risen); far: one term behind the other
//   distances that sums are scaled over, 20; two joins of 6 additions, each scaled by 2; from the sums' reference to the maximum 4.  Far: joins of 6 and 16.
constexpr int64_t test_units(int M, int dtype, int waves, bool far) {
  const int64_t width = logits_width(dtype), threads = 64 * waves, loads = test_loads(waves), chunks = M / width + 2;
  return far ? (chunks + threads - 1) / threads * width + 42 + 2 + 6 + 16 : 3 * (chunks / (threads * loads) + loads + 1) + loads * width / 2 + 28 + 2 + 6 + 20 + 2 * (6 + 2) + 4;
}

// A draft is decided on in fp32 where u q and p are farther from each other, relative to p, than both rows' sums may be off; units: of both.  (Roundings behind one another
// and quotients of them add terms of the second order, less than four squares.)  Wider margins cost time, as a draft that is nearer takes its row's workgroup 20 us more.
constexpr double test_margin(int64_t units) {
  const double off = (double)units * 0x1p-24;
  return off + 4.0 * off * off;
}

inline DrawLayout draw_layout(int64_t B, int G, int M, int dtype, bool draft) {
  if (by_workgroups(B, G, M)) return draw_layout_whole(B, M, dtype);
  const int64_t rows = draw_rows(G, draft), row = 64 * logits_width(dtype);
  const bool tested = test_first(B, G, M, dtype, draft);
  int64_t loads = 1;  // of a piece: four where that makes enough wavefronts
  while (loads < 4 && B * (tested ? 1 : rows) * ceil_div(M, 2 * loads * row) >= 4096) loads *= 2;
  DrawLayout l = draw_pieces(M, dtype, loads, 1024);
  l.spread = true;
  if (tested) {
    l.tested = true;
    l.positions = (int)(B < 512 ? ceil_div(512, B) : 1);
    const int64_t workgroups = B * (l.positions < G ? l.positions : G);
    // sixteen for rows of at least their first loads (160 workgroups, rows of 256 KiB 17.6 us and 20.8 with eight; 192, of 98 KiB 8.2 and 7.8)
    l.test_waves = workgroups <= 256 && M >= 16 * 8 * 64 * logits_width(dtype) ? 16 : (workgroups <= 512 ? 8 : 4);
  } else if (draft) {
    l.groups = (int)ceil_div(l.pieces, kDrawWaves);
    if (B * l.groups > 1024) l.groups = B < 1024 ? (int)(1024 / B) : 1;
  }
  return l;
}

// Device memory: the pieces' results; a number for each; untested a counter for each sequence; tested the drafts' fp32 sums and what is accepted.
inline int64_t draw_workspace(int64_t B, int G, bool draft, const DrawLayout& l) {
  if (!l.spread) return 0;
  const int64_t parts = B * l.pieces * 16 * (int64_t)kept_rows(G, draft, l);
  return parts + 8 * B * l.pieces + (l.tested ? 17 * B * G : 4 * B);
}

}  // namespace rtopk
