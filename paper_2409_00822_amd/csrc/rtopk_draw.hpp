// Tokens drawn from rows of logits, and drafted tokens verified against them, for gfx950 (MI355X).
//
// A row x at temperature T has the probabilities p_v = e_v / S, e_v = 2^((x_v - r) c), c = log2(e) / T, S = sum e, about any reference r.  By a number u in
// [0, 1) it gives the lowest column v with  e_0 + ... + e_v > u S.  A draft d, drawn from q, is accepted where u q_d < p_d; the first one that is not is
// replaced by a draw from  max(p - q, 0), so that all tokens are distributed as the target's.
//
// Which column a sum passes a threshold at is a whole number: a rounding moves it, and with it the text that follows.  Differences, powers and sums are
// therefore 64-bit here: their errors, 10^-13 of a row's mass, move one draw in 10^7 of a vocabulary of 131072 columns, where fp32 sums would move one in
// a hundred.  That also spares the maximum: in 64 bits r = 0 does for all rows whose sum lies within 2^+-500, which is looked at afterwards.
//
// Bound by the vector ALU: a logit is sixteen 64-bit instructions, of 4.3 to 5 cycles each for 64 of them on a SIMD, 80 cycles in all, where HBM brings
// 128 bytes in 48.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_draw_dispatch.hpp"
#include "rtopk_logits.hpp"

namespace rtopk {

constexpr double kLog2e64 = 1.44269504088896340736;
constexpr double kLeastMass = 0x1p-40;  // of max(p - q, 0): below it p and q are the same but for rounding
constexpr double kLeastSum = 0x1p-500, kMostSum = 0x1p500;  // of a row about r = 0: no term overflows, and what underflows is nothing beside them

// ---- powers and sums ------------------------------------------------------------------------------

// 2^t, as exact as a sum of 10^5 of them needs it: 2^f on [-1/2, 1/2] by a polynomial of degree 9 that is 1 at 0 (interpolated at Chebyshev's nodes, off by
// 3.7 10^-14 of the value), times a whole power.  NaN for infinities and NaN; 0 for what is far below.
__device__ __forceinline__ double power2_finite(double t) {
  const double n = __builtin_rint(t), f = t - n;
  double p = 1.02031210633917292e-7;
  p = __builtin_fma(p, f, 1.3255224878668817e-6);
  p = __builtin_fma(p, f, 0.000015252686846267719);
  p = __builtin_fma(p, f, 0.000154034558524538394);
  p = __builtin_fma(p, f, 0.00133335581790431111);
  p = __builtin_fma(p, f, 0.00961812915940255819);
  p = __builtin_fma(p, f, 0.0555041086647604239);
  p = __builtin_fma(p, f, 0.240226506958129882);
  p = __builtin_fma(p, f, 0.693147180559945309);
  p = __builtin_fma(p, f, 1.0);
  int whole;
  asm("v_cvt_i32_f64 %0, %1" : "=v"(whole) : "v"(n));  // (clamps, which a C++ conversion does not promise)
  return __builtin_amdgcn_ldexp(p, whole);
}
// The same with 0 for -inf; NaN stays.
__device__ __forceinline__ double power2(double t) { return power2_finite(t < -1100.0 ? -1100.0 : t); }

// f of the 64 lanes' values, the same in every lane.
template <typename F>
__device__ __forceinline__ double wave_reduce(double v, F f) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = f(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
  return wave_reduce(v, [](double a, double b) { return a + b; });
}

// A row's sum of powers about ref.  Nothing but -inf: s = 0; a NaN or +inf: s = NaN.
struct Mass {
  double ref, s;
  __device__ __forceinline__ double power(float x, double c) const { return power2(((double)x - ref) * c); }
  __device__ __forceinline__ double over() const { return s == 0.0 ? 0.0 : 1.0 / s; }
};

// Columns [0, cols) from `row` on, for one wavefront: 128-bit chunks, chunk i for lane i mod 64, U at a time; then the chunks left and what is less than one.
// Rows of 16-bit values that start at an odd one have their first column apart, as Segment has it.
template <int DT>
struct Piece {
  using L = Logits<DT>;
  Segment<DT> g;
  __device__ __forceinline__ Piece(const typename L::elem* row, int cols) : g(row, cols) {}
  // whole(chunks, U) for full batches, part(chunk) for single ones, which may hold -inf for what lies outside
  template <int U, typename F, typename P>
  __device__ __forceinline__ void each(int lane, F whole, P part) const {
    int i = lane;
    for (; i - lane + (U - 1) * 64 + 63 < g.full; i += U * 64) {
      u4_vec w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = L::load(g.body + (uint32_t)(i + u * 64) * L::V);
      whole(w);
    }
    for (; i < g.chunks(); i += 64) part(i < g.full ? L::load(g.body + (uint32_t)i * L::V) : g.partial());
  }
};

// Sum of the powers about 0 of a piece, over the wavefront.  Masked columns make a first sum NaN; it is then taken again with -inf as the type's lowest
// value, and so are all that follow.
template <int DT>
__device__ __forceinline__ double piece_sum(const typename Logits<DT>::elem* row, int cols, int lane, double c) {
  using L = Logits<DT>;
  constexpr int U = DT == kF32 ? 4 : 2;
  double s = 0.0;
  bool masked = false;
  const auto masked_power = [&](float x) { return power2_finite((double)(x == kNegInf ? -3.402823466e38f : x) * c); };
  Piece<DT>(row, cols).template each<U>(
      lane,
      [&](u4_vec(&w)[U]) {
        double a[2] = {0.0, 0.0};
        if (!masked) {
#pragma unroll
          for (int i = 0; i < U * L::V; ++i) a[i & 1] += power2_finite((double)L::at(w[i / L::V], i % L::V) * c);
        }
        if (masked || __any(!(a[0] + a[1] == a[0] + a[1]))) {
          masked = true;
          a[0] = a[1] = 0.0;
          apart(w);
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < L::V; ++i) a[i & 1] += masked_power(L::at(w[u], i));
        }
        s += a[0] + a[1];
      },
      [&](const u4_vec& w) {
#pragma unroll
        for (int i = 0; i < L::V; ++i) s += masked_power(L::at(w, i));
      });
  return wave_sum(s);
}

// f(column, value) for the thread's share of `cols` columns from `row` on, in 128-bit loads; i: the thread's number of T.
template <int DT, typename F>
__device__ __forceinline__ void each_of(const typename Logits<DT>::elem* row, int cols, int i, int T, F f) {
  using L = Logits<DT>;
  const int full = cols / L::V;
  for (; i < full; i += T) {
    const u4_vec w = L::load(row + (int64_t)i * L::V);
#pragma unroll
    for (int c = 0; c < L::V; ++c) f(i * L::V + c, L::at(w, c));
  }
  if (i == full)
    for (int c = full * L::V; c < cols; ++c) f(c, L::widen(row[c]));
}

template <int W>
struct DrawRoom {
  double s[W];  // sums of the wavefronts' pieces, in order
  float m[W];
  uint64_t key[W];
  int nan[W], past[W], last[W];
};

// Columns of each wavefront's piece of a row.
template <int DT, int W>
__device__ __forceinline__ int piece_cols(int cols) {
  constexpr int V = Logits<DT>::V;
  return ((cols + W - 1) / W + V - 1) / V * V;
}

// A row's (or segment's) mass, in every thread; the pieces' sums in room.s.
template <int DT, int W>
__device__ __forceinline__ Mass block_mass(const typename Logits<DT>::elem* row, int M, double c, DrawRoom<W>& room) {
  constexpr int T = 64 * W;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int piece = piece_cols<DT, W>(M), from = min(wave * piece, M), cols = min(piece, M - from);
  const auto join = [&](double s) {
    if (lane == 0) room.s[wave] = s;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) all += room.s[w];
    return all;
  };
  const double s = piece_sum<DT>(row + from, cols, lane, c);
  __syncthreads();
  Mass t = {0.0, join(s)};
  if (!(t.s >= kLeastSum && t.s <= kMostSum)) {  // about the maximum then
    float m = kNegInf;
    each_of<DT>(row, M, threadIdx.x, T, [&](int, float x) { m = fmaxf(m, x); });
    m = wave_max(m);
    if (lane == 0) room.m[wave] = m;
    __syncthreads();
    for (int w = 0; w < W; ++w) m = fmaxf(m, room.m[w]);
    t.ref = m == kNegInf ? 0.0 : (double)m;
    double u = 0.0;
    each_of<DT>(row + from, cols, lane, 64, [&](int, float x) { u += t.power(x, c); });
    t.s = join(wave_sum(u));
  }
  return t;
}

// Temperature 0: place_key of the largest logit, 0 where there is none, and whether there is a NaN; in every thread.
struct Best {
  uint64_t key;
  bool nan;
  __device__ __forceinline__ int col() const { return nan || key == 0 ? -1 : place_col(key); }
};

template <int DT, int W>
__device__ __forceinline__ Best block_best(const typename Logits<DT>::elem* row, int first, int cols, DrawRoom<W>& room) {
  constexpr int T = 64 * W;
  Best b = {0, false};
  each_of<DT>(row + first, cols, threadIdx.x, T, [&](int col, float x) {
    const uint64_t key = x > kNegInf ? place_key(order_key(x), first + col) : 0;
    b.key = key > b.key ? key : b.key;
    b.nan |= x != x;
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)b.key, d);
    b.key = o > b.key ? o : b.key;
  }
  b.nan = __any(b.nan);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    room.key[threadIdx.x >> 6] = b.key;
    room.nan[threadIdx.x >> 6] = b.nan;
  }
  __syncthreads();
  for (int w = 0; w < W; ++w) {
    b.key = room.key[w] > b.key ? room.key[w] : b.key;
    b.nan |= room.nan[w] != 0;
  }
  return b;
}

// ---- draws ----------------------------------------------------------------------------------------

// What a column weighs in a draw: its probability in p, without a rejected draft's column, or less its probability in q.
struct Weights {
  Mass p, q;
  double c, over_p, over_q;
  int without;  // a column that weighs nothing, -1: none
  bool less;    // p - q
  __device__ __forceinline__ double at(int col, float xp, float xq) const {
    const double v = p.power(xp, c) * over_p;
    if (less) return fmax(v - q.power(xq, c) * over_q, 0.0);
    return col == without ? 0.0 : v;
  }
  __device__ __forceinline__ bool is_number() const { return over_p == over_p && (!less || over_q == over_q); }
};

// f(weights of a chunk's columns, its first column) for chunks i, i + T, ... of `cols` columns from `first` on, and of what is less than one.
template <int DT, typename F>
__device__ __forceinline__ void each_weight(const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int first, int cols, int i, int T, F f) {
  using L = Logits<DT>;
  const int full = cols / L::V, rest = cols % L::V;
  const auto *a = p + first, *b = (w.less ? q : p) + first;
  double v[L::V];
  for (; i < full; i += T) {
    const u4_vec x = L::load(a + (int64_t)i * L::V), y = w.less ? L::load(b + (int64_t)i * L::V) : x;
#pragma unroll
    for (int c = 0; c < L::V; ++c) v[c] = w.at(first + i * L::V + c, L::at(x, c), L::at(y, c));
    f(v, first + i * L::V);
  }
  if (i == full && rest != 0) {
#pragma unroll
    for (int c = 0; c < L::V; ++c) v[c] = c < rest ? w.at(first + full * L::V + c, L::widen(a[full * L::V + c]), L::widen(b[full * L::V + c])) : 0.0;
    f(v, first + full * L::V);
  }
}

// Inclusive sums over the lanes.
__device__ __forceinline__ double wave_scan(double v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// Of n pieces with the given sums, in order: the first that the cumulated sum passes `goal` in, or the last that has any; -1: none has.  before: the sum of
// those in front of it.  Each wavefront for itself.
template <typename F>
__device__ __forceinline__ int passing(int n, double goal, double& before, F sum) {
  const int lane = threadIdx.x & 63;
  double all = before;
  int at = -1;
  for (int j = 0; j < n; j += 64) {
    const double s = j + lane < n ? sum(j + lane) : 0.0, to = all + wave_scan(s, lane);
    const uint64_t have = __ballot(s > 0.0), past = __ballot(s > 0.0 && to > goal);
    if (have != 0) {
      const int l = past != 0 ? __builtin_ctzll(past) : 63 - __builtin_clzll(have);
      at = j + l;
      before = __shfl(to - s, l);
    }
    if (past != 0) break;
    all = __shfl(to, 63);
  }
  return at;
}

// The column of [first, first + cols) that the cumulated weight, `before` at `first`, passes `goal` in, or the last that has any; in every thread.  Cut into a
// piece for each wavefront, and the piece that it passes in again, until a thread has a chunk of it.
template <int DT, int W>
__device__ int block_find(const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int first, int cols, double before, double goal, DrawRoom<W>& room) {
  constexpr int V = Logits<DT>::V, T = 64 * W;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  while (cols > T * V) {
    const int piece = piece_cols<DT, W>(cols), from = min(wave * piece, cols);
    double s = 0.0;
    each_weight<DT>(w, p, q, first + from, min(piece, cols - from), lane, 64, [&](const double(&v)[V], int) {
#pragma unroll
      for (int c = 0; c < V; ++c) s += v[c];
    });
    s = wave_sum(s);
    __syncthreads();
    if (lane == 0) room.s[wave] = s;
    __syncthreads();
    const int j = passing(W, goal, before, [&](int i) { return room.s[i]; });
    if (j < 0) return -1;
    first += j * piece;
    cols = min(piece, cols - j * piece);
  }
  double v[V], s = 0.0;
  int col = 0;
#pragma unroll
  for (int c = 0; c < V; ++c) v[c] = 0.0;
  each_weight<DT>(w, p, q, first, cols, threadIdx.x, T, [&](const double(&x)[V], int at) {
#pragma unroll
    for (int c = 0; c < V; ++c) {
      v[c] = x[c];
      s += x[c];
    }
    col = at;
  });
  double to = wave_scan(s, lane);
  __syncthreads();
  if (lane == 63) room.s[wave] = to;
  __syncthreads();
  for (int j = 0; j < wave; ++j) before += room.s[j];
  to += before;
  const uint64_t have = __ballot(s > 0.0), past = __ballot(s > 0.0 && to > goal);
  const int one = past != 0 ? __builtin_ctzll(past) : 63 - __builtin_clzll(have | 1);
  if (lane == one) {
    double sum = to - s;
    int at = -1;
#pragma unroll
    for (int c = V - 1; c >= 0; --c)
      if (at < 0 && v[c] > 0.0) at = c;  // the last
    bool found = false;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      sum += v[c];
      if (past != 0 && !found && v[c] > 0.0 && sum > goal) {
        found = true;
        at = c;
      }
    }
    room.past[wave] = past != 0 ? col + at : -1;
    room.last[wave] = have != 0 ? col + at : -1;
  }
  __syncthreads();
  int at = -1;
  for (int j = W - 1; j >= 0; --j)
    if (at < 0) at = room.last[j];
  for (int j = W - 1; j >= 0; --j)
    if (room.past[j] >= 0) at = room.past[j];
  return at;
}

// A draw by u from the weights of a row's columns, the pieces' sums known (`summed`: in room.s, of p about w.p.ref) or not.  Draws from p where the weights' whole
// is no more than kLeastMass.
template <int DT, int W>
__device__ int block_draw(Weights w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int M, double u, bool summed, DrawRoom<W>& room) {
  constexpr int V = Logits<DT>::V;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int piece = piece_cols<DT, W>(M), from = min(wave * piece, M), cols = min(piece, M - from);
  for (;;) {
    const bool part = w.less || !summed || (w.without >= from && w.without < from + cols);
    double s = 0.0;
    if (part) {
      each_weight<DT>(w, p, q, from, cols, lane, 64, [&](const double(&v)[V], int) {
#pragma unroll
        for (int c = 0; c < V; ++c) s += v[c];
      });
      s = wave_sum(s);
    } else {
      s = room.s[wave] * w.over_p;
    }
    __syncthreads();
    if (lane == 0) room.s[wave] = s;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int j = 0; j < W; ++j) all += room.s[j];
    if ((w.less || w.without >= 0) && !(all > kLeastMass)) {
      w.less = false;
      w.without = -1;
      summed = false;
      continue;
    }
    if (!(all > 0.0)) return -1;
    const double goal = fmax(u * all, 0.0);  // (NaN: 0)
    double before = 0.0;
    const int j = passing(W, goal, before, [&](int i) { return room.s[i]; });
    if (j < 0) return -1;
    return block_find<DT, W>(w, p, q, j * piece, min(piece, M - j * piece), before, goal, room);
  }
}

__device__ __forceinline__ int draft_at(const DrawArgs& a, int64_t n, int pos) {  // -1: none
  if (pos >= a.G) return -1;
  const int64_t i = n * a.G + pos, t = a.token64 ? static_cast<const int64_t*>(a.drafts)[i] : static_cast<const int32_t*>(a.drafts)[i];
  return t >= 0 && t < a.M ? (int)t : -1;
}

__device__ __forceinline__ void write_token(const DrawArgs& a, int64_t i, int token) {
  if (a.token64) static_cast<int64_t*>(a.tokens)[i] = token;
  else static_cast<int32_t*>(a.tokens)[i] = token;
}

// The accepted drafts, the drawn token, -1 behind it.
__device__ __forceinline__ void write_sequence(const DrawArgs& a, int64_t n, int accepted, int drawn, int T) {
  for (int j = threadIdx.x; j <= a.G; j += T) write_token(a, n * (a.G + 1) + j, j < accepted ? draft_at(a, n, j) : (j == accepted ? drawn : -1));
  if (threadIdx.x == 0 && a.accepted) a.accepted[n] = accepted;
}

// A sequence's temperature, its factor, and what is to be done with it.
struct Heat {
  double T, c;
  __device__ __forceinline__ Heat(const DrawArgs& a, int64_t n) : T(a.temperatures ? (double)a.temperatures[n] : a.temperature), c(kLog2e64 / T) {}
  __device__ __forceinline__ bool certain() const { return T == 0.0; }
  __device__ __forceinline__ bool none() const { return !(T >= 0.0 && T < __builtin_inf()); }
};

// One workgroup takes a sequence: its rows one after the other until a draft is rejected, then the draw.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  __shared__ DrawRoom<W> room;
  const int64_t n = a.row0 + blockIdx.x;
  const Heat heat(a, n);
  const auto* target = static_cast<const elem*>(a.target) + n * a.target_seq;
  const auto* draft = static_cast<const elem*>(a.draft) + (a.draft ? n * a.draft_seq : 0);
  int pos = 0, drawn = -1;
  if (heat.certain()) {
    for (;; ++pos) {
      drawn = block_best<DT, W>(target + pos * a.target_pos, 0, a.M, room).col();
      if (drawn < 0 || draft_at(a, n, pos) != drawn) break;
    }
  } else if (!heat.none()) {
    Weights w;
    w.c = heat.c;
    const elem *p, *q;
    for (;; ++pos) {
      p = target + pos * a.target_pos;
      q = draft + pos * a.draft_pos;
      w.p = block_mass<DT, W>(p, a.M, w.c, room);
      w.over_p = w.p.over();
      w.without = -1;
      w.less = false;
      const int d = draft_at(a, n, pos);
      if (d < 0) break;
      double q_d = 1.0;
      if (a.draft) {
        w.q = block_mass<DT, W>(q, a.M, w.c, room);
        w.over_q = w.q.over();
        q_d = w.q.power(Logits<DT>::widen(q[d]), w.c) * w.over_q;
        w.less = true;
      } else {
        w.without = d;
      }
      if (!((double)a.uniforms[n * (a.G + 1) + pos] * q_d < w.p.power(Logits<DT>::widen(p[d]), w.c) * w.over_p)) break;
    }
    if (w.is_number()) drawn = block_draw<DT, W>(w, p, q, a.M, (double)a.uniforms[n * (a.G + 1) + a.G], !w.less, room);
  }
  write_sequence(a, n, pos, drawn, 64 * W);
}

// ---- few sequences, spread over workgroups ---------------------------------------------------------

// Row `row` of a sequence's 2 G + 1: its target's rows first, then its draft's.
template <int DT>
__device__ __forceinline__ const typename Logits<DT>::elem* row_of(const DrawArgs& a, int64_t n, int row) {
  using elem = typename Logits<DT>::elem;
  return row <= a.G ? static_cast<const elem*>(a.target) + n * a.target_seq + row * a.target_pos
                    : static_cast<const elem*>(a.draft) + n * a.draft_seq + (row - a.G - 1) * a.draft_pos;
}

// How many drafts a sequence has; each wavefront for itself.
__device__ __forceinline__ int drafts_of(const DrawArgs& a, int64_t n) {
  const int lane = threadIdx.x & 63;
  for (int j = 0; j < a.G; j += 64) {
    const uint64_t none = __ballot(j + lane >= a.G || draft_at(a, n, j + lane) < 0);
    if (none != 0) return j + __builtin_ctzll(none);
  }
  return a.G;
}

// The mass of a segment of a row (at temperature 0: its best column) to scratch memory.  All rows that may be looked at, those behind a rejected draft
// among them: their workgroups have the GPU to themselves otherwise.
template <int DT>
__global__ __launch_bounds__(256) void draw_mass_kernel(DrawArgs a) {
  constexpr int W = 4;
  __shared__ DrawRoom<W> room;
  const int seg = (int)(blockIdx.x % (uint32_t)a.segments), rows = a.draft ? 2 * a.G + 1 : a.G + 1;
  const uint32_t of = blockIdx.x / (uint32_t)a.segments;
  const int row = (int)(of % (uint32_t)rows);
  const int64_t n = a.row0 + of / (uint32_t)rows;
  if (seg == 0 && row == 0 && threadIdx.x == 0) a.arrived[n] = 0;
  const Heat heat(a, n);
  if (heat.none() || (heat.certain() && row > a.G)) return;
  if (a.G > 0) {
    const int g = drafts_of(a, n);
    if (row <= a.G ? row > g : row - a.G - 1 >= g) return;
  }
  const auto* x = row_of<DT>(a, n, row);
  const int first = seg * a.seg_cols, cols = min(a.seg_cols, a.M - first);
  double2 out;
  if (heat.certain()) {
    const Best b = block_best<DT, W>(x, first, cols, room);
    out = make_double2(b.nan ? 1.0 : 0.0, __longlong_as_double((long long)b.key));
  } else {
    const Mass t = block_mass<DT, W>(x + first, cols, heat.c, room);
    out = make_double2(t.ref, t.s);
  }
  if (threadIdx.x == 0) a.part[(n * rows + row) * a.segments + seg] = out;
}

// A row's mass from its segments', in every lane.
__device__ __forceinline__ Mass join_mass(const DrawArgs& a, int64_t n, int rows, int row, double c) {
  const int lane = threadIdx.x & 63;
  const double2* part = a.part + (n * rows + row) * a.segments;
  Mass t = {0.0, 0.0};
  for (int j = lane; j < a.segments; j += 64) {
    const double2 p = part[j];
    if (p.y != 0.0) {  // (NaN too)
      const double ref = t.s == 0.0 ? p.x : fmax(t.ref, p.x);
      if (ref != t.ref) t.s *= t.s == 0.0 ? 1.0 : power2((t.ref - ref) * c);
      t.s += ref == p.x ? p.y : p.y * power2((p.x - ref) * c);
      t.ref = ref;
    }
  }
  const double ref = wave_reduce(t.s == 0.0 ? -__builtin_inf() : t.ref, [](double u, double v) { return fmax(u, v); });
  if (ref == -__builtin_inf()) return {0.0, 0.0};
  if (t.s != 0.0 && t.ref != ref) t.s *= power2((t.ref - ref) * c);
  return {ref, wave_sum(t.s)};
}

__device__ __forceinline__ Best join_best(const DrawArgs& a, int64_t n, int rows, int row) {
  const int lane = threadIdx.x & 63;
  const double2* part = a.part + (n * rows + row) * a.segments;
  Best b = {0, false};
  for (int j = lane; j < a.segments; j += 64) {
    const uint64_t key = (uint64_t)__double_as_longlong(part[j].y);
    b.key = key > b.key ? key : b.key;
    b.nan |= part[j].x != 0.0;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)b.key, d);
    b.key = o > b.key ? o : b.key;
  }
  b.nan = __any(b.nan);
  return b;
}

// Joins the masses, finds the first rejected draft and draws.  Where the draw is from max(p - q, 0) each of `segments` workgroups takes a segment's sum of
// it, and the last one of the sequence that is done (counted from 0, which draw_mass_kernel set) goes on; else the first one does it alone.  Which one is
// last changes nothing: sums lie in memory and are taken in order.
template <int DT>
__global__ __launch_bounds__(256) void draw_join_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  constexpr int W = 4, T = 64 * W;
  __shared__ DrawRoom<W> room;
  __shared__ double2 mass[2 * kMaxDrafts + 1];
  __shared__ int best[kMaxDrafts + 1], last;
  const int parts = a.draft ? a.segments : 1, seg = (int)(blockIdx.x % (uint32_t)parts), rows = a.draft ? 2 * a.G + 1 : a.G + 1;
  const int64_t n = a.row0 + blockIdx.x / (uint32_t)parts;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Heat heat(a, n);
  if (heat.none()) {
    if (seg == 0) write_sequence(a, n, 0, -1, T);
    return;
  }
  const int g = a.G > 0 ? drafts_of(a, n) : 0;
  if (heat.certain()) {
    if (seg != 0) return;
    for (int row = wave; row <= g; row += W) {
      const int col = join_best(a, n, rows, row).col();
      if (lane == 0) best[row] = col;
    }
    __syncthreads();
    int pos = 0;
    while (pos < g && best[pos] >= 0 && best[pos] == draft_at(a, n, pos)) ++pos;
    write_sequence(a, n, pos, best[pos], T);
    return;
  }
  for (int i = wave; i < 2 * g + 1; i += W) {
    const int row = i <= g ? i : a.G + i - g;
    if (row > a.G && !a.draft) break;
    const Mass t = join_mass(a, n, rows, row, heat.c);
    if (lane == 0) mass[row] = make_double2(t.ref, t.s);
  }
  __syncthreads();
  const auto mass_of = [&](int row) { return Mass{mass[row].x, mass[row].y}; };
  int pos = g;  // the first rejected draft
  for (int j = 0; j < g; j += 64) {
    bool rejected = false;
    const int i = j + lane;
    if (i < g) {
      const int d = draft_at(a, n, i);
      const Mass p = mass_of(i);
      double q_d = 1.0;
      if (a.draft) {
        const Mass q = mass_of(a.G + 1 + i);
        q_d = q.power(Logits<DT>::widen(row_of<DT>(a, n, a.G + 1 + i)[d]), heat.c) * q.over();
      }
      rejected = !((double)a.uniforms[n * (a.G + 1) + i] * q_d < p.power(Logits<DT>::widen(row_of<DT>(a, n, i)[d]), heat.c) * p.over());
    }
    const uint64_t mask = __ballot(rejected);
    if (mask != 0) {
      pos = j + __builtin_ctzll(mask);
      break;
    }
  }
  Weights w;
  w.c = heat.c;
  w.p = mass_of(pos);
  w.over_p = w.p.over();
  w.without = pos < g && !a.draft ? draft_at(a, n, pos) : -1;
  w.less = pos < g && a.draft;
  const elem *p = row_of<DT>(a, n, pos), *q = p;
  if (w.less) {
    w.q = mass_of(a.G + 1 + pos);
    w.over_q = w.q.over();
    q = row_of<DT>(a, n, a.G + 1 + pos);
  }
  if (!w.is_number() || !w.less) {
    if (seg != 0) return;
    if (!w.is_number()) {
      write_sequence(a, n, pos, -1, T);
      return;
    }
  }
  const auto segment_cols = [&](int j) { return min(a.seg_cols, a.M - j * a.seg_cols); };
  const auto weigh = [&](int j) {  // a segment's weight, over the workgroup
    double s = 0.0;
    each_weight<DT>(w, p, q, j * a.seg_cols, segment_cols(j), threadIdx.x, T, [&](const double(&v)[Logits<DT>::V], int) {
#pragma unroll
      for (int c = 0; c < Logits<DT>::V; ++c) s += v[c];
    });
    s = wave_sum(s);
    __syncthreads();
    if (lane == 0) room.s[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int j = 0; j < W; ++j) s += room.s[j];
    return s;
  };
  double* rest = a.rest + n * a.segments;
  if (w.less) {
    const double s = weigh(seg);
    if (threadIdx.x == 0) {
      __hip_atomic_store(rest + seg, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(a.arrived + n, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    }
    __syncthreads();
    if (!last) return;
  }
  double special = 0.0;  // the segment without the draft that stood for itself
  const int special_seg = w.without >= 0 ? w.without / a.seg_cols : -1;
  if (special_seg >= 0) special = weigh(special_seg);
  for (;;) {
    const double2* part = a.part + (n * rows + pos) * a.segments;
    const auto sum = [&](int j) {
      if (w.less) return __hip_atomic_load(rest + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (j == special_seg && w.without >= 0) return special;
      const double2 t = part[j];
      return t.y * (t.x == w.p.ref || t.y == 0.0 ? 1.0 : power2((t.x - w.p.ref) * w.c)) * w.over_p;
    };
    double all = 0.0;
    for (int j = lane; j < a.segments; j += 64) all += sum(j);
    all = wave_sum(all);
    if ((w.less || w.without >= 0) && !(all > kLeastMass)) {
      w.less = false;
      w.without = -1;
      continue;
    }
    int drawn = -1;
    if (all > 0.0) {
      const double goal = fmax((double)a.uniforms[n * (a.G + 1) + a.G] * all, 0.0);  // (NaN: 0)
      double before = 0.0;
      const int j = passing(a.segments, goal, before, sum);
      if (j >= 0) drawn = block_find<DT, W>(w, p, q, j * a.seg_cols, segment_cols(j), before, goal, room);
    }
    write_sequence(a, n, pos, drawn, T);
    return;
  }
}

}  // namespace rtopk
