// Operators on rows of logits: limits, and how a call's rows are laid over workgroups.  Host code only (no HIP headers), so that a CPU
// test can sweep the rules.
#pragma once

#include <stdint.h>

namespace rtopk {

constexpr int kMaxLogitsM = 1 << 24;  // widest row
constexpr int kMaxAlternatives = 128; // top alternatives of a row
constexpr int kMaxList = 1024;        // given tokens of a row, entries of a teacher's list
constexpr int kMaxLogitsSegments = 256;     // workgroups that a row is spread over
constexpr int kMaxMergeKeys = 2048;   // alternatives of all segments of a row that are merged

// Columns of a 128-bit load.
constexpr int logits_width(int dtype) { return dtype == 0 ? 4 : 8; }

// A row over `segments` workgroups of `waves` wavefronts, `cols` columns each (the last one what is left); cols is a multiple of the load's.
struct LogitsLayout {
  int waves, segments, cols;
};

// Rows held on chip by one workgroup, X(wavefronts, 128-bit loads of a thread in registers, in LDS), narrow ones first.  The widest are held by sixteen
// wavefronts in fp32 and by eight in 16 bits (2048 x 65536 fp32 194 us with sixteen, 204 with eight; 8192 x 131072 bfloat16 794 and 776, 4096 x 100000 half
// 324 and 329).
#define RTOPK_HELD_LIST(X) X(1, 4, 0) X(4, 4, 0) X(4, 4, 4) X(8, 4, 4) X(8, 8, 8) X(8, 16, 8) X(8, 24, 8) X(16, 8, 8)
constexpr bool is_held_by(int dtype, int waves, int in_registers) {
  return dtype == 0 ? in_registers != 24 : waves != 16;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Few rows of more than 128 KiB are spread over several workgroups each, in two launches, unless the alternatives' merge costs more than that saves:
// 8 x 131072 bfloat16 without alternatives 8.9 us against 10.0 in one workgroup, with 20 12.7 against 15.6, with 64 30.5 against 22.5; 96 rows 12.8
// against 11.2; 64 x 32000 fp32, k = 20, 13.4 against 10.0.
inline bool spread(int64_t N, int64_t row_bytes, int k) { return N < 96 && row_bytes > 131072 && k <= 32; }

// Rows that one wavefront takes: up to 2048 columns, and up to 16384 where there are rows enough to fill the GPU so, which pays no barriers.
// Four wavefronts and one, us: 16384 x 2500 bfloat16 30.2 and 17.8, with 5 alternatives 62.5 and 32.8, distillation 33.5 and 23.0; 16384 x 4000
// 31.5 and 24.3, 58.6 and 37.9, 32.1 and 27.1; 4096 x 16000 24.2 and 24.3, 33.6 and 29.6, 24.6 and 23.2.  fp32 with alternatives likewise (16384 x 4000, 5
// alternatives 53.6 and 48.2); without them it gains and loses (16384 x 4000 39.1 and 40.9, distillation 43.2 and 46.9; 4096 x 8000 22.9 and 22.1, 23.7 and
// 21.8; 4096 x 16000 41.3 and 41.4, 42.7 and 41.6).  Fewer rows lose: 1000 x 4000 bfloat16, 5 alternatives 8.1 and 9.4.
inline bool short_rows(int64_t N, int M, int k) { return k <= 32 && (M <= 2048 || (M <= 16384 && N >= 4096)); }

// A workgroup for each row: one wavefront for short rows; sixteen where there are no more rows than compute units, eight up to twice as many, four beyond
// (k = 5, bfloat16 rows of 131072 columns with 16, 8 and 4 wavefronts: 200 rows 16.2, 20.6 and 29.6 us, 400 30.2, 26.0 and 32.7, 700 44.8, 41.8 and
// 38.2; without alternatives 200 12.8, 13.7 and 19.9, 400 23.5, 21.9 and 22.7, 700 35.8, 35.1 and 32.3).
inline LogitsLayout logits_layout_whole(int64_t N, int M, int k) {
  return {short_rows(N, M, k) ? 1 : (N <= 256 ? 16 : (N <= 512 ? 8 : 4)), 1, M};
}

inline LogitsLayout logits_layout(int64_t N, int M, int dtype, int k) {
  const int v = logits_width(dtype);
  const int64_t bytes = (int64_t)M * (dtype == 0 ? 4 : 2);
  if (!spread(N, bytes, k)) return logits_layout_whole(N, M, k);
  // segments of 16 KiB, fewer where that makes more workgroups than fill the GPU four times
  int64_t segments = ceil_div(1024, N);
  if (segments > ceil_div(bytes, 16384)) segments = ceil_div(bytes, 16384);
  if (segments > kMaxLogitsSegments) segments = kMaxLogitsSegments;
  if (k > 0 && segments * k > kMaxMergeKeys) segments = kMaxMergeKeys / k;
  LogitsLayout l;
  l.cols = (int)(ceil_div(ceil_div(M, segments), v) * v);
  l.segments = (int)ceil_div(M, l.cols);
  l.waves = 4;
  return l.segments > 1 ? l : logits_layout_whole(N, M, k);
}

struct HeldLayout {
  int waves, loads;  // loads 0: the row is too wide
};

inline HeldLayout held_layout(int M, int dtype) {
  const int64_t chunks = M / logits_width(dtype);  // (a partial one is held apart)
#define X(w, r, q) \
  if (is_held_by(dtype, w, r) && chunks <= 64 * w * (r + q)) return {w, r + q};
  RTOPK_HELD_LIST(X)
#undef X
  return {8, 0};
}

// The segments of a gradient whose row sums are known: 16 KiB (4096 x 131072 bfloat16: 340 us; 8 KiB 395, 32 KiB 350), less, down to 4 KiB, where
// that leaves compute units without work; short rows of 16 bits take one wavefront (16384 x 1000 bfloat16 35 -> 26 us, lists of 32 41 -> 28; the
// same in fp32 33 against 37).  A gradient that takes its logits' place has one segment: a row whose log-sum-exp is large is read whole before any of it
// is written.
inline LogitsLayout logits_grad_layout(int64_t N, int M, int dtype, bool in_place) {
  const int v = logits_width(dtype);
  if (dtype != 0 && M <= 2048) return {1, 1, M};
  if (in_place) return {4, 1, M};
  int64_t cols = 16384 / (dtype == 0 ? 4 : 2);
  while (cols > 1024 * v / 4 && N * ceil_div(M, cols) < 1024) cols /= 2;
  LogitsLayout l;
  l.segments = (int)ceil_div(M, cols);
  l.cols = (int)(ceil_div(ceil_div(M, l.segments), v) * v);
  l.segments = (int)ceil_div(M, l.cols);
  l.waves = 4;
  return l;
}

// Where a saved log-sum-exp is so large that a row's sums are taken again, which the kernel finds out, this many segments of the row share a
// workgroup, so that no more than about 512 workgroups, or one to a row, read a row whole (fp32 at T = 0.01, each segment's workgroup against this: 2048 x 65536 697 -> 316 us,
// 16 x 1048576 728 -> 185, 512 x 32000 88 -> 53, 64 x 32000 14.9 -> 12.7; with 256 workgroups 128 x 32000 16.0 against 16.7, 256 x 32000 32.4
// against 30.1).  Up to four segments read the row each, from the caches (1024 x 32000 bfloat16 54.7 against 61.7, 2048 x 8192 31.2 against 35.8).
constexpr int kFarWorkgroups = 512;
inline int far_group(int64_t N, int segments) {
  if (segments <= 4) return 1;
  const int64_t group = ceil_div(N * segments, kFarWorkgroups);
  return group < segments ? (int)group : segments;
}

// Device memory for the segments' partial results: maximum, sum and weighted sum of each, then its alternatives.
inline int64_t logits_workspace(int64_t N, const LogitsLayout& l, int k) {
  return l.segments > 1 ? N * l.segments * (16 + 8 * (int64_t)k) : 0;
}

}  // namespace rtopk
