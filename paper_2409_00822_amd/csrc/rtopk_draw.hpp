// Tokens drawn from rows of logits, and drafted tokens verified against them, for gfx950 (MI355X).
//
// A row x at temperature T has the probabilities p_v = e_v / S, e_v = 2^((x_v - max x) c), c = log2(e) / T, S = sum e.  By a number u in [0, 1) it
// gives the lowest column v with  e_0 + ... + e_v > u S.  A draft d, drawn from q, is accepted where u q_d < p_d; the first one that is not is
// replaced by a draw from  max(p - q, 0), so that all tokens are distributed as the target's.
//
// Which column a sum passes a threshold at is a whole number: a rounding moves it, and with it the text that follows.  Differences, powers and sums are
// therefore 64-bit here: their errors, 10^-13 of a row's mass, move one draw in 10^7 of a vocabulary of 131072 columns, where fp32 sums would move one in
// a hundred.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_draw_dispatch.hpp"
#include "rtopk_logits.hpp"

namespace rtopk {

constexpr double kLog2e64 = 1.44269504088896340736;
constexpr double kLeastMass = 0x1p-40;  // of max(p - q, 0): below it p and q are the same but for rounding

// 2^t for t <= 0 (or little above), as exact as a sum of 10^5 of them needs it: 2^f on [-1/2, 1/2] by a polynomial of degree 9 that is 1 at 0 (interpolated
// at Chebyshev's nodes, off by 3.7 10^-14 of the value), times a whole power.  -inf gives 0, NaN stays.
__device__ __forceinline__ double power2(double t) {
  t = t < -1100.0 ? -1100.0 : t;
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
  return __builtin_amdgcn_ldexp(p, (int)n);
}

// Sum of the 64 lanes, the same in every lane.
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// A row's maximum, and its sum of powers about it.  An empty row (nothing but -inf) has m = -inf, s = 0; one with a NaN or +inf has s = NaN.
struct Mass {
  float m;
  double s;
  __device__ __forceinline__ double power(float x, double c) const { return power2(((double)x - (m == kNegInf ? 0.0 : (double)m)) * c); }
  __device__ __forceinline__ void rise_to(float top, double c) {
    if (top != m) s *= power2(((double)m - (double)top) * c);  // (m = -inf: s is 0)
    m = top;
  }
};

// The best column of a row at temperature 0: place_key of its largest logit, 0 where there is none (nothing but -inf, a NaN).
struct Best {
  uint64_t key;
  bool nan;
};

template <int W>
struct DrawRoom {
  double s[W];
  float m[W];
  uint64_t key[W];
  int nan[W];
  int found;
};

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

// The row's mass, in every thread.
template <int DT, int W>
__device__ __forceinline__ Mass block_mass(const typename Logits<DT>::elem* row, int M, double c, DrawRoom<W>& room) {
  constexpr int T = 64 * W;
  Mass t = {kNegInf, 0.0};
  each_of<DT>(row, M, threadIdx.x, T, [&](int, float x) {
    if (x > t.m) t.rise_to(x, c);
    t.s += t.power(x, c);
  });
  t.rise_to(wave_max(t.m), c);
  t.s = wave_sum(t.s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    room.m[threadIdx.x >> 6] = t.m;
    room.s[threadIdx.x >> 6] = t.s;
  }
  __syncthreads();
  float top = room.m[0];
  for (int w = 1; w < W; ++w) top = fmaxf(top, room.m[w]);
  Mass all = {top, 0.0};
  for (int w = 0; w < W; ++w) {
    Mass u = {room.m[w], room.s[w]};
    u.rise_to(top, c);
    all.s += u.s;
  }
  return all;
}

template <int DT, int W>
__device__ __forceinline__ int block_best(const typename Logits<DT>::elem* row, int M, DrawRoom<W>& room) {
  constexpr int T = 64 * W;
  Best b = {0, false};
  each_of<DT>(row, M, threadIdx.x, T, [&](int col, float x) {
    const uint64_t key = x > kNegInf ? place_key(order_key(x), col) : 0;
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
  uint64_t key = 0;
  bool nan = false;
  for (int w = 0; w < W; ++w) {
    key = room.key[w] > key ? room.key[w] : key;
    nan |= room.nan[w] != 0;
  }
  return nan || key == 0 ? -1 : place_col(key);
}

// What a column weighs in a draw: its probability in p, without a rejected draft's column, or less its probability in q.
struct Weights {
  Mass p, q;
  double c, over_p, over_q;
  int without;  // a column that weighs nothing, -1: none
  bool less;    // p - q
  __device__ __forceinline__ double at(int col, float xp, float xq) const {
    if (less) return fmax(p.power(xp, c) * over_p - q.power(xq, c) * over_q, 0.0);
    return col == without ? 0.0 : p.power(xp, c) * over_p;
  }
};

// The same for the columns' weights; q null where they need p only.
template <int DT, typename F>
__device__ __forceinline__ void each_weight(const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int first, int cols, int i, int T, F f) {
  using L = Logits<DT>;
  const int full = cols / L::V;
  const auto *a = p + first, *b = (w.less ? q : p) + first;
  for (; i < full; i += T) {
    const u4_vec x = L::load(a + (int64_t)i * L::V), y = w.less ? L::load(b + (int64_t)i * L::V) : x;
#pragma unroll
    for (int c = 0; c < L::V; ++c) f(w.at(first + i * L::V + c, L::at(x, c), L::at(y, c)));
  }
  if (i == full)
    for (int c = full * L::V; c < cols; ++c) f(w.at(first + c, L::widen(a[c]), L::widen(b[c])));
}

// Of pieces with the given sums, in order: the first that the cumulated sum passes `goal` in, or the last that has any; -1: none has.  before: the sum of
// those in front of it.
template <typename F>
__device__ __forceinline__ int passing(int pieces, double goal, double& before, F sum) {
  double all = before;
  int at = -1;
  for (int j = 0; j < pieces; ++j) {
    const double s = sum(j);
    if (s > 0.0) {
      at = j;
      before = all;
    }
    if (all + s > goal && s > 0.0) break;
    all += s;
  }
  return at;
}

// A draw by u from the weights of a row's columns: the row is cut into a piece for each wavefront, and the piece that the cumulated weight passes u of
// the whole in is cut again, until there is a column to a lane.  `fall`: draws from p where the weights' whole is no more than kLeastMass.
template <int DT, int W>
__device__ int block_draw(Weights w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int M, double u, DrawRoom<W>& room) {
  constexpr int V = Logits<DT>::V;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int first = 0, cols = M;
  double before = 0.0, goal = -1.0;
  while (cols > 64 || goal < 0.0) {
    const int piece = ((cols + W - 1) / W + V - 1) / V * V;
    const int from = min(wave * piece, cols), n = min(piece, cols - from);
    double s = 0.0;
    each_weight<DT>(w, p, q, first + from, n, lane, 64, [&](double x) { s += x; });
    s = wave_sum(s);
    __syncthreads();
    if (lane == 0) room.s[wave] = s;
    __syncthreads();
    if (goal < 0.0) {
      double all = 0.0;
      for (int j = 0; j < W; ++j) all += room.s[j];
      if ((w.less || w.without >= 0) && !(all > kLeastMass)) {
        w.less = false;
        w.without = -1;
        continue;
      }
      if (!(all > 0.0)) return -1;
      goal = fmax(u * all, 0.0);  // (NaN: 0)
    }
    const int j = passing(W, goal, before, [&](int i) { return room.s[i]; });
    if (j < 0) return -1;
    first += j * piece;
    cols = min(piece, cols - j * piece);
  }
  if (wave == 0) {
    const int col = first + lane;
    double s = lane < cols ? w.at(col, Logits<DT>::widen(p[col]), w.less ? Logits<DT>::widen(q[col]) : 0.0f) : 0.0;
    const bool any = s > 0.0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double o = __shfl_up(s, d);
      if (lane >= d) s += o;
    }
    const uint64_t have = __ballot(any), past = __ballot(any && before + s > goal);
    if (lane == 0) room.found = have == 0 ? -1 : first + (past != 0 ? __builtin_ctzll(past) : 63 - __builtin_clzll(have));
  }
  __syncthreads();
  return room.found;
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

// One workgroup takes a sequence: its rows one after the other until a draft is rejected, then the draw.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  __shared__ DrawRoom<W> room;
  const int64_t n = a.row0 + blockIdx.x;
  const double T = a.temperatures ? (double)a.temperatures[n] : a.temperature, c = kLog2e64 / T;
  const auto* target = static_cast<const elem*>(a.target) + n * a.target_seq;
  const auto* draft = static_cast<const elem*>(a.draft) + (a.draft ? n * a.draft_seq : 0);
  int pos = 0, drawn = -1;
  if (T == 0.0) {
    for (;; ++pos) {
      drawn = block_best<DT, W>(target + pos * a.target_pos, a.M, room);
      if (drawn < 0 || draft_at(a, n, pos) != drawn) break;
    }
  } else if (T > 0.0 && T < __builtin_inf()) {
    Weights w;
    w.c = c;
    const elem *p, *q;
    for (;; ++pos) {
      p = target + pos * a.target_pos;
      q = draft + pos * a.draft_pos;
      w.p = block_mass<DT, W>(p, a.M, c, room);
      w.over_p = w.p.s == 0.0 ? 0.0 : 1.0 / w.p.s;
      w.without = -1;
      w.less = false;
      const int d = draft_at(a, n, pos);
      if (d < 0) break;
      double q_d = 1.0;
      if (a.draft) {
        w.q = block_mass<DT, W>(q, a.M, c, room);
        w.over_q = w.q.s == 0.0 ? 0.0 : 1.0 / w.q.s;
        q_d = w.q.power(Logits<DT>::widen(q[d]), c) * w.over_q;
        w.less = true;
      } else {
        w.without = d;
      }
      if (!((double)a.uniforms[n * (a.G + 1) + pos] * q_d < w.p.power(Logits<DT>::widen(p[d]), c) * w.over_p)) break;
    }
    if (w.over_p == w.over_p && (!w.less || w.over_q == w.over_q))
      drawn = block_draw<DT, W>(w, p, q, a.M, (double)a.uniforms[n * (a.G + 1) + a.G], room);
  }
  write_sequence(a, n, pos, drawn, 64 * W);
}

}  // namespace rtopk
