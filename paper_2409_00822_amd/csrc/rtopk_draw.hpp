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
// Bound by the vector ALU: 64 logits are 17 instructions, most of them 64-bit, of 5 cycles each on a SIMD, and three more for a piece's start and end: 100 cycles, where HBM
// brings the 128 bytes in 48.  Slower: powers of bfloat16 logits from tables in LDS (43 us against 52 before the sums, but 64-bit reads keep a compute unit's LDS
// busy for 26 cycles each, and with what corrects 32-bit ones 63), pieces of 2 or 8 loads of a wavefront (93 and 101 us against 87 with 4, 2047 x 50001 half).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <utility>

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
// 2^(x c), 0 for a masked x at any c (one that is finite may be the type's lowest value and weigh something at a very high temperature).
__device__ __forceinline__ double masked_power(float x, double c) { return power2_finite(x == kNegInf ? -1100.0 : (double)x * c); }

// A 64-bit value moved by a DPP permutation, 0 where it comes from no lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, ROWS == 0xf), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, ROWS == 0xf);
  return __longlong_as_double((long long)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ double lane_value(double v, int lane) {  // lane: uniform
  const long long b = __double_as_longlong(v);
  return __longlong_as_double((long long)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}
// Inclusive sums over the lanes.
__device__ __forceinline__ double wave_scan(double v) {
  v += moved<0x111, 0xf>(v);  // row_shr:1
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);  // row_bcast:15
  v += moved<0x143, 0xc>(v);  // row_bcast:31
  return v;
}
// Sum of the lanes, the same in every lane.
__device__ __forceinline__ double wave_sum(double v) { return lane_value(wave_scan(v), 63); }

// A row's (or a piece's) sum of powers about ref.  Nothing but -inf: s = 0; a NaN or +inf: s = NaN.
struct Mass {
  double ref, s;
  __device__ __forceinline__ double power(float x, double c) const { return power2(((double)x - ref) * c); }
  __device__ __forceinline__ double over() const { return s == 0.0 ? 0.0 : 1.0 / s; }
};

// Waits until the wavefront's stores are where those of other workgroups are: in memory, if they were made past the caches.
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ---- pieces of rows -------------------------------------------------------------------------------

// A row is cut into pieces of a whole number of 128-bit loads of a wavefront (draw_pieces); a wavefront sums a piece, and what a row's pieces sum to says
// which of them a draw falls in.

// Sum of the powers about 0 of U chunks.  Masked columns make it NaN; it is then taken again with nothing for -inf, and so are all that follow.
template <int DT, int U>
__device__ __forceinline__ double chunk_powers(u4_vec (&w)[U], double c, bool& masked) {
  using L = Logits<DT>;
  double a[2] = {0.0, 0.0};
  if (!masked) {
#pragma unroll
    for (int i = 0; i < U * L::V; ++i) a[i & 1] += power2_finite((double)L::at(w[i / L::V], i % L::V) * c);
  }
  if (masked || __any(!(a[0] + a[1] == a[0] + a[1]))) {
    masked = true;
    a[0] = a[1] = 0.0;
    apart(w);
#pragma unroll 1
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < L::V; ++i) a[i & 1] += masked_power(L::at(w[u], i), c);
  }
  return a[0] + a[1];
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

// The mass of a piece, in every lane of its wavefront.
template <int DT>
__device__ __forceinline__ Mass piece_mass(const typename Logits<DT>::elem* piece, int cols, int lane, double c) {
  using L = Logits<DT>;
  constexpr int U = DT == kF32 ? 4 : 2;
  double s = 0.0;
  bool masked = false;
  lane_of_piece<L::V, U>(
      cols, lane,
      [&](int i) {
        u4_vec w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = L::load(piece + (uint32_t)(i + u * 64) * L::V);
        s += chunk_powers<DT, U>(w, c, masked);
      },
      [&](int i, bool is, bool some) {
        u4_vec w[1] = {u4_vec{L::kLow, L::kLow, L::kLow, L::kLow}};
        if (is) w[0] = L::load(piece + (uint32_t)i * L::V);
        masked |= some;
        s += chunk_powers<DT, 1>(w, c, masked);
      },
      [&](int col) { s += masked_power(L::widen(piece[col]), c); });
  Mass t = {0.0, wave_sum(s)};
  if (!(t.s >= kLeastSum && t.s <= kMostSum)) {  // about the maximum then
    float m = kNegInf;
    each_of<DT>(piece, cols, lane, 64, [&](int, float x) { m = fmaxf(m, x); });
    m = wave_max(m);
    t.ref = m == kNegInf ? 0.0 : (double)m;
    s = 0.0;
    each_of<DT>(piece, cols, lane, 64, [&](int, float x) { s += t.power(x, c); });
    t.s = wave_sum(s);
  }
  return t;
}

// f(0), ..., f(n - 1) of memory, one to a lane, 64 at a time: the first 128 are held in registers, for all loops over them.
template <typename F>
struct Held {
  using T = decltype(std::declval<F>()(0));
  int n;
  F f;
  T v[2];
  __device__ __forceinline__ Held(int n, F f) : n(n), f(f), v{} {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if ((int)(threadIdx.x & 63) + 64 * i < n) v[i] = f((int)(threadIdx.x & 63) + 64 * i);
  }
  __device__ __forceinline__ T at(int j) const { return j < 64 ? v[0] : (j < 128 ? v[1] : f(j)); }  // j: the lane's, below n
};

// A row's mass from its pieces' (ref, s), in every lane; each wavefront for itself.
template <typename H>
__device__ __forceinline__ Mass join_held(const H& part, double c) {
  const int lane = threadIdx.x & 63;
  Mass t = {0.0, 0.0};
  for (int j = lane; j < part.n; j += 64) {
    const double2 p = part.at(j);
    if (p.y != 0.0) {  // (NaN too)
      const double ref = t.s == 0.0 ? p.x : fmax(t.ref, p.x);
      if (ref != t.ref && t.s != 0.0) t.s *= power2((t.ref - ref) * c);
      t.s += ref == p.x ? p.y : p.y * power2((p.x - ref) * c);
      t.ref = ref;
    }
  }
  const uint64_t some = __ballot(t.s != 0.0);
  if (some == 0) return {0.0, 0.0};
  double ref = lane_value(t.ref, __builtin_ctzll(some));
  if (__any(t.s != 0.0 && t.ref != ref)) {  // (seldom: all are about 0)
    ref = t.s != 0.0 ? t.ref : -__builtin_inf();
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) ref = fmax(ref, __shfl_xor(ref, d));
    if (t.s != 0.0 && t.ref != ref) t.s *= power2((t.ref - ref) * c);
  }
  return {ref, wave_sum(t.s)};
}
__device__ __forceinline__ Mass join_mass(const double2* part, int pieces, double c) {
  return join_held(Held(pieces, [=](int j) { return part[j]; }), c);
}

// Temperature 0: place_key of the largest logit, 0 where there is none, and whether there is a NaN.
struct Best {
  uint64_t key;
  bool nan;
  __device__ __forceinline__ void take(const Best& b) {
    key = b.key > key ? b.key : key;
    nan |= b.nan;
  }
  __device__ __forceinline__ int col() const { return nan || key == 0 ? -1 : place_col(key); }
  // (as a piece's mass is stored)
  __device__ __forceinline__ double2 stored() const { return make_double2(nan ? 1.0 : 0.0, __longlong_as_double((long long)key)); }
  static __device__ __forceinline__ Best from(const double2& p) { return {(uint64_t)__double_as_longlong(p.y), p.x != 0.0}; }
};

__device__ __forceinline__ Best wave_best(Best b) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) b.take({(uint64_t)__shfl_xor((unsigned long long)b.key, d), false});
  b.nan = __any(b.nan);
  return b;
}

template <int DT>
__device__ __forceinline__ Best piece_best(const typename Logits<DT>::elem* row, int first, int cols, int lane) {
  Best b = {0, false};
  float top = kNegInf;
  int at = 0;
  each_of<DT>(row + first, cols, lane, 64, [&](int col, float x) {
    if (x > top) {  // (columns ascend)
      top = x;
      at = col;
    }
    b.nan |= x != x;
  });
  if (top > kNegInf) b.key = place_key(order_key(top), first + at);
  return wave_best(b);
}

__device__ __forceinline__ Best join_best(const double2* part, int pieces) {
  Best b = {0, false};
  for (int j = threadIdx.x & 63; j < pieces; j += 64) b.take(Best::from(part[j]));
  return wave_best(b);
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
    if (less) return fmax(__builtin_fma(p.power(xp, c), over_p, -(q.power(xq, c) * over_q)), 0.0);
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
  if (w.less && w.p.ref == 0.0 && w.q.ref == 0.0) {  // (mostly; neither row has a NaN or +inf)
    const auto power = [&](float x) { return power2_finite(fmax((double)x * w.c, -1100.0)); };
    for (; i < full; i += T) {
      const u4_vec x = L::load(a + (int64_t)i * L::V), y = L::load(b + (int64_t)i * L::V);
#pragma unroll
      for (int c = 0; c < L::V; ++c) v[c] = fmax(__builtin_fma(power(L::at(x, c)), w.over_p, -(power(L::at(y, c)) * w.over_q)), 0.0);
      f(v, first + i * L::V);
    }
  } else {
    for (; i < full; i += T) {
      const u4_vec x = L::load(a + (int64_t)i * L::V), y = w.less ? L::load(b + (int64_t)i * L::V) : x;
#pragma unroll
      for (int c = 0; c < L::V; ++c) v[c] = w.at(first + i * L::V + c, L::at(x, c), L::at(y, c));
      f(v, first + i * L::V);
    }
  }
  if (i == full && rest != 0) {
#pragma unroll
    for (int c = 0; c < L::V; ++c) v[c] = c < rest ? w.at(first + full * L::V + c, L::widen(a[full * L::V + c]), L::widen(b[full * L::V + c])) : 0.0;
    f(v, first + full * L::V);
  }
}

// A piece's weight, in every lane of its wavefront.
template <int DT>
__device__ __forceinline__ double piece_weight(const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int first, int cols, int lane) {
  double s = 0.0;
  each_weight<DT>(w, p, q, first, cols, lane, 64, [&](const double(&v)[Logits<DT>::V], int) {
#pragma unroll
    for (int c = 0; c < Logits<DT>::V; ++c) s += v[c];
  });
  return wave_sum(s);
}

// Of n pieces with the given sums, in order: the first that the cumulated sum passes `goal` in, or the last that has any; -1: none has.  before: the sum of
// those in front of it.  Each wavefront for itself.
template <typename F>
__device__ __forceinline__ int passing(int n, double goal, double& before, F sum) {
  const int lane = threadIdx.x & 63;
  double all = before;
  int at = -1;
  for (int j = 0; j < n; j += 64) {
    const double s = j + lane < n ? sum(j + lane) : 0.0, to = all + wave_scan(s);
    const uint64_t have = __ballot(s > 0.0), past = __ballot(s > 0.0 && to > goal);
    if (have != 0) {
      const int l = past != 0 ? __builtin_ctzll(past) : 63 - __builtin_clzll(have);
      at = j + l;
      before = lane_value(to - s, l);
    }
    if (past != 0) break;
    all = lane_value(to, 63);
  }
  return at;
}

template <int W>
struct FindRoom {
  double s[W];
  int past[W], last[W];
};

// The column of [first, first + cols) that the cumulated weight, `before` at `first`, passes `goal` in, or the last that has any; in every thread.  Cut into a
// part for each wavefront, and the part that it passes in again, until a thread has a chunk of it.
template <int DT, int W>
__device__ int block_find(const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int first, int cols, double before, double goal, FindRoom<W>& room) {
  constexpr int V = Logits<DT>::V, T = 64 * W;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if constexpr (W == 1) {  // one wavefront: a part after the other
    if (cols > T * V) {
      int at = -1;
      double all = before;
      for (int from = 0; from < cols; from += T * V) {
        const double s = piece_weight<DT>(w, p, q, first + from, min(T * V, cols - from), lane);
        if (s > 0.0) {
          at = from;
          before = all;
        }
        all += s;
        if (s > 0.0 && all > goal) break;
      }
      if (at < 0) return -1;
      first += at;
      cols = min(T * V, cols - at);
    }
  } else {
    while (cols > T * V) {  // (a part is smaller: W > 1)
      const int part = ((cols + W - 1) / W + V - 1) / V * V, from = min(wave * part, cols);
      const double s = piece_weight<DT>(w, p, q, first + from, min(part, cols - from), lane);
      __syncthreads();
      if (lane == 0) room.s[wave] = s;
      __syncthreads();
      const int j = passing(W, goal, before, [&](int i) { return room.s[i]; });
      if (j < 0) return -1;
      first += j * part;
      cols = min(part, cols - j * part);
    }
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
  double to = wave_scan(s);
  __syncthreads();
  if (lane == 63) room.s[wave] = to;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < W; ++j) before += j < wave ? room.s[j] : 0.0;
  to += before;
  const uint64_t have = __ballot(s > 0.0), past = __ballot(s > 0.0 && to > goal);
  const int one = past != 0 ? __builtin_ctzll(past) : 63 - __builtin_clzll(have | 1);
  if (lane == one) {
    double sum = to - s;
    int at = 0;
#pragma unroll
    for (int c = 0; c < V; ++c) at = v[c] > 0.0 ? c : at;  // the last
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
#pragma unroll
  for (int j = 0; j < W; ++j) at = room.last[j] >= 0 ? room.last[j] : at;
#pragma unroll
  for (int j = W - 1; j >= 0; --j) at = room.past[j] >= 0 ? room.past[j] : at;
  return at;
}

// A draw by u from the weights of a row, sum(j) its pieces' sums of them; -2: their whole is no more than `least`.
template <int DT, int W, typename S>
__device__ __forceinline__ int block_draw_of(const DrawArgs& a, const Weights& w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, S sum, double u, double least,
                                             FindRoom<W>& room) {
  const int lane = threadIdx.x & 63;
  const Held held(a.pieces, sum);
  double all = 0.0;
  for (int j = lane; j < a.pieces; j += 64) all += held.at(j);
  all = wave_sum(all);
  if (!(all > least)) return -2;
  const double goal = fmax(u * all, 0.0);  // (NaN: 0)
  double before = 0.0;
  const int j = passing(a.pieces, goal, before, [&](int i) { return held.at(i); });
  return j < 0 ? -1 : block_find<DT, W>(w, p, q, j * a.piece_cols, min(a.piece_cols, a.M - j * a.piece_cols), before, goal, room);
}

// What a piece with mass t weighs in p.
__device__ __forceinline__ double weight_of(const Weights& w, const double2& t) {
  return t.y * (t.x == w.p.ref || t.y == 0.0 ? 1.0 : power2((t.x - w.p.ref) * w.c)) * w.over_p;
}

// A draw from the weights of a row: rest(j) are its pieces' sums where they are p - q, else part(j) their masses in p.  Draws from p where the weights' whole is
// no more than kLeastMass.
template <int DT, int W, typename P, typename R>
__device__ int block_draw(const DrawArgs& a, Weights w, const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, P part, R rest, double u, FindRoom<W>& room) {
  int at = -2;
  if (w.less) {
    at = block_draw_of<DT, W>(a, w, p, q, rest, u, kLeastMass, room);
  } else if (w.without >= 0) {
    // the piece with the draft that stood for itself, without it
    const int special = w.without / a.piece_cols, first = special * a.piece_cols, wave = threadIdx.x >> 6;
    double s = 0.0;
    each_weight<DT>(w, p, q, first, min(a.piece_cols, a.M - first), threadIdx.x, 64 * W, [&](const double(&v)[Logits<DT>::V], int) {
#pragma unroll
      for (int c = 0; c < Logits<DT>::V; ++c) s += v[c];
    });
    s = wave_sum(s);
    if (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) room.s[wave] = s;
      __syncthreads();
      s = 0.0;
#pragma unroll
      for (int i = 0; i < W; ++i) s += room.s[i];
    }
    at = block_draw_of<DT, W>(a, w, p, q, [&](int j) { return j == special ? s : weight_of(w, part(j)); }, u, kLeastMass, room);
  }
  if (at != -2) return at;
  w.less = false;
  w.without = -1;
  return max(block_draw_of<DT, W>(a, w, p, q, [&](int j) { return weight_of(w, part(j)); }, u, 0.0, room), -1);
}

// ---- sequences ------------------------------------------------------------------------------------

__device__ __forceinline__ int draft_at(const DrawArgs& a, int64_t n, int pos) {  // -1: none
  if (pos >= a.G) return -1;
  const int64_t i = n * a.G + pos, t = a.token64 ? static_cast<const int64_t*>(a.drafts)[i] : static_cast<const int32_t*>(a.drafts)[i];
  return t >= 0 && t < a.M ? (int)t : -1;
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

__device__ __forceinline__ void write_token(const DrawArgs& a, int64_t i, int token) {
  if (a.token64) static_cast<int64_t*>(a.tokens)[i] = token;
  else static_cast<int32_t*>(a.tokens)[i] = token;
}

// The accepted drafts, the drawn token, -1 behind it.
__device__ __forceinline__ void write_sequence(const DrawArgs& a, int64_t n, int accepted, int drawn, int T) {
  for (int j = threadIdx.x; j <= a.G; j += T) write_token(a, n * (a.G + 1) + j, j < accepted ? draft_at(a, n, j) : (j == accepted ? drawn : -1));
  if (threadIdx.x == 0 && a.accepted) a.accepted[n] = accepted;
}

// A sequence's temperature and its factor.
struct Heat {
  double T, c;
  __device__ __forceinline__ Heat(const DrawArgs& a, int64_t n) : T(a.temperatures ? (double)a.temperatures[n] : a.temperature), c(a.temperatures ? kLog2e64 / T : a.c) {}
  __device__ __forceinline__ bool certain() const { return T == 0.0; }
  __device__ __forceinline__ bool none() const { return !(T >= 0.0 && T < __builtin_inf()); }
};

// Row `row` of a sequence's 2 G + 1: its target's rows first, then its draft's.
template <int DT>
__device__ __forceinline__ const typename Logits<DT>::elem* row_of(const DrawArgs& a, int64_t n, int row) {
  using elem = typename Logits<DT>::elem;
  return row <= a.G ? static_cast<const elem*>(a.target) + n * a.target_seq + row * a.target_pos
                    : static_cast<const elem*>(a.draft) + n * a.draft_seq + (row - a.G - 1) * a.draft_pos;
}

// One workgroup takes a sequence: its rows one after the other until a draft is rejected, then the draw.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  __shared__ FindRoom<W> room;
  __shared__ double2 part[kMostPieces], draft_part[kMostPieces];  // masses of pieces; then the sums of p - q in the latter's place
  const int64_t n = a.row0 + blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Heat heat(a, n);
  int pos = 0;
  const auto each_piece = [&](auto f) {
    for (int j = wave; j < a.pieces; j += W) f(j, j * a.piece_cols, min(a.piece_cols, a.M - j * a.piece_cols));
  };
  int drawn = -1;
  if (heat.certain()) {
    for (;; ++pos) {
      const elem* x = row_of<DT>(a, n, pos);
      __syncthreads();
      each_piece([&](int j, int first, int cols) {
        const Best b = piece_best<DT>(x, first, cols, lane);
        if (lane == 0) part[j] = b.stored();
      });
      __syncthreads();
      drawn = join_best(part, a.pieces).col();
      if (drawn < 0 || draft_at(a, n, pos) != drawn) break;
    }
  } else if (!heat.none()) {
    Weights w;
    w.c = heat.c;
    const elem *p, *q;
    const auto row_mass = [&](const elem* x, double2* to) {
      __syncthreads();
      each_piece([&](int j, int first, int cols) {
        const Mass t = piece_mass<DT>(x + first, cols, lane, w.c);
        if (lane == 0) to[j] = make_double2(t.ref, t.s);
      });
      __syncthreads();
      return join_mass(to, a.pieces, w.c);
    };
    for (;; ++pos) {
      p = q = row_of<DT>(a, n, pos);
      w.p = row_mass(p, part);
      w.over_p = w.p.over();
      w.without = -1;
      w.less = false;
      const int d = draft_at(a, n, pos);
      if (d < 0) break;
      double q_d = 1.0;
      if (a.draft) {
        q = row_of<DT>(a, n, a.G + 1 + pos);
        w.q = row_mass(q, draft_part);
        w.over_q = w.q.over();
        q_d = w.q.power(Logits<DT>::widen(q[d]), w.c) * w.over_q;
        w.less = true;
      } else {
        w.without = d;
      }
      if (!((double)a.uniforms[n * (a.G + 1) + pos] * q_d < w.p.power(Logits<DT>::widen(p[d]), w.c) * w.over_p)) break;
    }
    if (w.is_number()) {
      double* rest = reinterpret_cast<double*>(draft_part);
      if (w.less) {
        __syncthreads();
        each_piece([&](int j, int first, int cols) {
          const double s = piece_weight<DT>(w, p, q, first, cols, lane);
          if (lane == 0) rest[j] = s;
        });
        __syncthreads();
      }
      drawn = block_draw<DT, W>(a, w, p, q, [&](int j) { return part[j]; }, [&](int j) { return rest[j]; }, (double)a.uniforms[n * (a.G + 1) + a.G], room);
    }
  }
  write_sequence(a, n, pos, drawn, 64 * W);
}

// ---- drafts tested beforehand ----------------------------------------------------------------------

// The first of `most` positions whose draft the tests have rejected; each wavefront for itself.
__device__ __forceinline__ int tested_up_to(const DrawArgs& a, int64_t n, int most) {
  const int lane = threadIdx.x & 63;
  for (int j = 0; j < most; j += 64) {
    const uint64_t stop = __ballot(j + lane >= most || a.accepts[n * a.G + min(j + lane, most - 1)] == 0);
    if (stop != 0) return j + __builtin_ctzll(stop);
  }
  return most;
}

// 269 MB of bfloat16 logits by 512 workgroups 42 us (6.4 TB/s, vector ALU 67 %); 84 MB by 160 of 16 wavefronts 18 (160 of 256 compute units, whose ALUs are what is
// waited for).  256 sequences of seven drafts in phases of two, two and three positions 117 us; of three and four 111, but where fewer drafts are accepted that
// reads more rows for nothing.
// Tests positions [pos0, pos0 + positions) of the sequences whose drafts before that have been accepted, a workgroup to each: most rows are read once, in fp32, at
// the rate of HBM, and those behind a rejected draft not at all.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_test_kernel(DrawArgs a, int pos0, int positions) {
  using elem = typename Logits<DT>::elem;
  constexpr int T = 64 * W;
  __shared__ float4 sums[W];
  __shared__ double2 part[W];
  const int64_t n = a.row0 + blockIdx.x / (uint32_t)positions;
  const int pos = pos0 + (int)(blockIdx.x % (uint32_t)positions), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Heat heat(a, n);
  if (heat.none() || pos >= drafts_of(a, n) || tested_up_to(a, n, pos0) < pos0) return;
  const int d = draft_at(a, n, pos), cols = (a.M + W - 1) / W, first = min(wave * cols, a.M), mine = min(cols, a.M - first);
  const elem *p = row_of<DT>(a, n, pos), *q = a.draft ? row_of<DT>(a, n, a.G + 1 + pos) : p;
  bool accepted;
  if (heat.certain()) {
    const Best b = piece_best<DT>(p, first, mine, lane);
    if (lane == 0) part[wave] = b.stored();
    __syncthreads();
    accepted = join_best(part, W).col() == d;
  } else {
    const double u = (double)a.uniforms[n * (a.G + 1) + pos];
    const float c = (float)heat.c;
    int64_t units = 0;
    const auto near = [&](const elem* x, int which) {
      const Segment<DT> g(x, a.M);
      const Stats t = segment_stats<DT, W, false>(g, thread_stats<DT, T, test_loads(W), false, false>(g, c), c, sums);
      __syncthreads();
      units += test_units(a.M, DT, W, far_maximum(t.m, c));
      if (threadIdx.x == 0) a.near[2 * (n * a.G + pos) + which] = make_float2(t.m, t.s);
      return power2(((double)Logits<DT>::widen(x[d]) - (double)t.m) * heat.c) / (double)t.s;
    };
    double p_d = near(p, 0), uq = a.draft ? u * near(q, 1) : u;
    const double margin = test_margin(units);
    accepted = uq < p_d * (1.0 - margin);
    if (!accepted && !(uq > p_d * (1.0 + margin))) {  // (nearer than the sums are exact: again, in 64 bits)
      const auto exact = [&](const elem* x) {
        const Mass t = piece_mass<DT>(x + first, mine, lane, heat.c);
        __syncthreads();
        if (lane == 0) part[wave] = make_double2(t.ref, t.s);
        __syncthreads();
        const Mass all = join_mass(part, W, heat.c);
        return all.power(Logits<DT>::widen(x[d]), heat.c) * all.over();
      };
      p_d = exact(p);
      uq = a.draft ? u * exact(q) : u;
      accepted = uq < p_d;
    }
  }
  if (threadIdx.x == 0) a.accepts[n * a.G + pos] = accepted;
}

// ---- sequences spread over workgroups --------------------------------------------------------------

// Rows of a sequence whose masses are kept: of all its positions, the target's first.
__device__ __forceinline__ int rows_of(const DrawArgs& a) { return a.draft ? 2 * a.G + 1 : a.G + 1; }

// The masses of pieces of a row (at temperature 0: their best columns) to scratch memory, a piece to a wavefront.  All rows that may be looked at, those behind a
// rejected draft among them: few sequences leave the GPU room for that.  2047 x 50001 half: 71 us, 2.9 TB/s, vector ALU busy 96 % of the time (640
// instructions to a wavefront of 2048 columns); 64 x 131072 bfloat16 9.
template <int DT>
__global__ __launch_bounds__(64 * kDrawWaves) void draw_mass_kernel(DrawArgs a) {
  const uint32_t rows = (uint32_t)rows_of(a);
  const int piece = (int)blockIdx.x * kDrawWaves + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63, row = rows == 1 ? 0 : (int)(blockIdx.y % rows);
  const int64_t n = a.row0 + (rows == 1 ? blockIdx.y : blockIdx.y / rows);
  if (blockIdx.x == 0 && row == 0 && threadIdx.x == 0) a.arrived[n] = 0;
  if (piece >= a.pieces) return;
  const Heat heat(a, n);
  if (heat.none() || (heat.certain() && row > a.G)) return;
  if (a.G > 0) {
    const int g = drafts_of(a, n);
    if (row <= a.G ? row > g : row - a.G - 1 >= g) return;
  }
  const auto* x = row_of<DT>(a, n, row);
  const int first = piece * a.piece_cols, cols = min(a.piece_cols, a.M - first);
  double2 out;
  if (heat.certain()) {
    out = piece_best<DT>(x, first, cols, lane).stored();
  } else {
    const Mass t = piece_mass<DT>(x + first, cols, lane, heat.c);
    out = make_double2(t.ref, t.s);
  }
  if (lane == 0) a.part[(n * rows + row) * a.pieces + piece] = out;
}

// The draws of sequences without drafts from their masses, a chain of three loads: 3.2 us for one row, 9.8 for 2047.  By the kernel for drafts, with a third more
// registers and loads twice, 5.6 and 15.6; with sixteen wavefronts one in six longer.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_take_kernel(DrawArgs a) {
  __shared__ FindRoom<W> room;
  const int64_t n = a.row0 + blockIdx.x;
  const Heat heat(a, n);
  const double2* part = a.part + n * a.pieces;
  int drawn = -1;
  if (heat.certain()) {
    drawn = join_best(part, a.pieces).col();
  } else if (!heat.none()) {
    const double u = (double)a.uniforms[n];
    const Held held(a.pieces, [=](int j) { return part[j]; });
    Weights w;
    w.c = heat.c;
    w.p = w.q = join_held(held, w.c);
    w.over_p = w.over_q = w.p.over();
    w.without = -1;
    w.less = false;
    if (w.is_number()) {
      const auto* p = row_of<DT>(a, n, 0);
      drawn = max(block_draw_of<DT, W>(a, w, p, p, [&](int j) { return weight_of(w, held.at(j)); }, u, 0.0, room), -1);
    }
  }
  if (threadIdx.x == 0) {
    write_token(a, n, drawn);
    if (a.accepted) a.accepted[n] = 0;
  }
}

// Joins the masses, finds the first rejected draft and draws: a chain of some eight loads, 11 us for one sequence of four drafts, 32000
// columns fp32.  Where the draw is from max(p - q, 0) the sequence's workgroups take its pieces' sums, and the
// last one of them that is done (counted from 0, which draw_mass_kernel set) goes on; else the first one does it alone.  Which one is last changes
// nothing: sums lie in memory and are taken in order.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void draw_join_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  constexpr int T = 64 * W;
  __shared__ FindRoom<W> room;
  __shared__ double2 mass[2 * kMaxDrafts + 1];
  __shared__ int best[kMaxDrafts + 1], last;
  const uint32_t groups = (uint32_t)a.groups;
  const int group = (int)(blockIdx.x % groups), rows = rows_of(a);
  const int64_t n = a.row0 + blockIdx.x / groups;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Heat heat(a, n);
  if (heat.none()) {
    if (group == 0) write_sequence(a, n, 0, -1, T);
    return;
  }
  const int g = drafts_of(a, n);
  const double2* parts = a.part + n * rows * a.pieces;
  if (heat.certain()) {
    if (group != 0) return;
    for (int row = wave; row <= g; row += W) {
      const int col = join_best(parts + (int64_t)row * a.pieces, a.pieces).col();
      if (lane == 0) best[row] = col;
    }
    __syncthreads();
    int pos = 0;
    while (pos < g && best[pos] >= 0 && best[pos] == draft_at(a, n, pos)) ++pos;
    write_sequence(a, n, pos, best[pos], T);
    return;
  }
  // what the tests need, before the masses are there
  float p_at = 0.0f, q_at = 0.0f, u = 0.0f;
  const auto look = [&](int i) {
    if (i < g) {
      const int d = draft_at(a, n, i);
      u = a.uniforms[n * (a.G + 1) + i];
      p_at = Logits<DT>::widen(row_of<DT>(a, n, i)[d]);
      if (a.draft) q_at = Logits<DT>::widen(row_of<DT>(a, n, a.G + 1 + i)[d]);
    }
  };
  look(lane);
  for (int i = wave; i < (a.draft ? 2 * g + 1 : g + 1); i += W) {
    const int row = i <= g ? i : a.G + i - g;
    const Mass t = join_mass(parts + (int64_t)row * a.pieces, a.pieces, heat.c);
    if (lane == 0) mass[row] = make_double2(t.ref, t.s);
  }
  __syncthreads();
  const auto mass_of = [&](int row) { return Mass{mass[row].x, mass[row].y}; };
  int pos = g;  // of the first rejected draft, or behind them all
  for (int j = 0; j < g; j += 64) {
    bool rejected = false;
    const int i = j + lane;
    if (j > 0) look(i);
    if (i < g) {
      const Mass p = mass_of(i);
      double q_d = 1.0;
      if (a.draft) {
        const Mass q = mass_of(a.G + 1 + i);
        q_d = q.power(q_at, heat.c) * q.over();
      }
      rejected = !((double)u * q_d < p.power(p_at, heat.c) * p.over());
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
    if (group != 0) return;
    if (!w.is_number()) {
      write_sequence(a, n, pos, -1, T);
      return;
    }
  }
  double* rest = a.rest + n * a.pieces;
  if (w.less) {
    for (int piece = group * W + wave; piece < a.pieces; piece += a.groups * W) {
      const int first = piece * a.piece_cols;
      const double s = piece_weight<DT>(w, p, q, first, min(a.piece_cols, a.M - first), lane);
      if (lane == 0) __hip_atomic_store(rest + piece, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // the stores, and the loads of the last workgroup, go past the caches, which need not be written back then; a barrier alone does not wait for stores
    stores_done();
    __syncthreads();
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(a.arrived + n, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)groups - 1;
    __syncthreads();
    if (!last) return;
  }
  const double2* part = parts + (int64_t)pos * a.pieces;
  const int drawn = block_draw<DT, W>(
      a, w, p, q, [&](int j) { return part[j]; }, [&](int j) { return __hip_atomic_load(rest + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); },
      (double)a.uniforms[n * (a.G + 1) + a.G], room);
  write_sequence(a, n, pos, drawn, T);
}

// ---- the draws of tested sequences -----------------------------------------------------------------

// With e_p and e_q the powers of two rows about 0, their sums S and l = S_p / S_q, a piece has  sum max(e_p - l e_q, 0) / S_p  of p - q.  That is taken in the pass
// that finds the sums: about the tests' fp32 ratio k of them, A = sum max(e_p - k e_q, 0) and B = sum of e_q where that is not 0, so that
// A - (l - k) B is the piece's sum if no column's ratio lies between l and k.  l and k differ by 10^-7 of them or so, and few pieces have such a column, but
// rows that are alike in most columns have many: the distance of k from the nearest ratio that is nearer than k kNear is kept, and a piece that has one within
// l - k is summed again when l is known.
struct Rest {
  double p, q, a, b, nearest;
};
constexpr double kNear = 0x1p-16;

template <int DT>
__device__ __forceinline__ Rest piece_rest(const typename Logits<DT>::elem* p, const typename Logits<DT>::elem* q, int cols, int lane, double c, double ratio) {
  using L = Logits<DT>;
  Rest r = {0.0, 0.0, 0.0, 0.0, __builtin_inf()};
  const double near = ratio * kNear;
  bool masked = false;
  const auto add = [&](double ep, double eq, Rest& t, bool& close) {
    const double d = __builtin_fma(-ratio, eq, ep);
    t.p += ep;
    t.q += eq;
    t.a += fmax(d, 0.0);
    t.b += d > 0.0 ? eq : 0.0;
    close |= fabs(d) < near * eq;
  };
  const auto approach = [&](float x, float y) {
    const double eq = masked_power(y, c), d = __builtin_fma(-ratio, eq, masked_power(x, c));
    if (fabs(d) < near * eq) r.nearest = fmin(r.nearest, fabs(d) / eq);
  };
  lane_of_piece<L::V, 1>(
      cols, lane, [](int) {},
      [&](int i, bool is, bool) {
        Rest t = {0.0, 0.0, 0.0, 0.0, 0.0};
        bool close = false;
        u4_vec x[1], y[1];
        if (is) {
          x[0] = L::load(p + (int64_t)i * L::V);
          y[0] = L::load(q + (int64_t)i * L::V);
          if (!masked) {
#pragma unroll
            for (int k = 0; k < L::V; ++k) add(power2_finite((double)L::at(x[0], k) * c), power2_finite((double)L::at(y[0], k) * c), t, close);
          }
        }
        if (masked || __any(!(t.p + t.q == t.p + t.q))) {  // (-inf, or what is no number)
          masked = true;
          close = false;
          t = {0.0, 0.0, 0.0, 0.0, 0.0};
          if (is) {
            apart(x);
            apart(y);
#pragma unroll
            for (int k = 0; k < L::V; ++k) add(masked_power(L::at(x[0], k), c), masked_power(L::at(y[0], k), c), t, close);
          }
        }
        r.p += t.p;
        r.q += t.q;
        r.a += t.a;
        r.b += t.b;
        if (__any(close)) {  // (seldom)
          if (close) {
#pragma unroll 1
            for (int k = 0; k < L::V; ++k) approach(L::widen(p[(int64_t)i * L::V + k]), L::widen(q[(int64_t)i * L::V + k]));
          }
        }
      },
      [&](int col) {
        const float x = L::widen(p[col]), y = L::widen(q[col]);
        bool close = false;
        add(masked_power(x, c), masked_power(y, c), r, close);
        approach(x, y);
      });
  if (__any(r.nearest < __builtin_inf())) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) r.nearest = fmin(r.nearest, __shfl_xor(r.nearest, d));
  }
  return {wave_sum(r.p), wave_sum(r.q), wave_sum(r.a), wave_sum(r.b), r.nearest};
}

// S_p / S_q from the tests' fp32 sums.
__device__ __forceinline__ double near_ratio(const DrawArgs& a, int64_t n, int pos, double c) {
  const float2 p = a.near[2 * (n * a.G + pos)], q = a.near[2 * (n * a.G + pos) + 1];
  return (double)p.y / (double)q.y * power2(((double)p.x - (double)q.x) * c);
}

// 256 sequences, rows of 131072 bfloat16 columns: 61 to 62 us, 43 instructions to 64 pairs of columns, vector ALU 92 % busy.  (Sums first and what is left of p - q in a second
// launch: 226 us for the whole call, and 177 so.)
// The pieces of the row that a sequence draws from, one to a wavefront: its mass, and that of the draft's row and what is left of p - q where a draft was rejected.
template <int DT>
__global__ __launch_bounds__(64 * kDrawWaves) void draw_rest_kernel(DrawArgs a) {
  const int piece = (int)blockIdx.x * kDrawWaves + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t n = a.row0 + blockIdx.y;
  const Heat heat(a, n);
  if (piece >= a.pieces || heat.none()) return;
  const int g = drafts_of(a, n), pos = tested_up_to(a, n, g), first = piece * a.piece_cols, cols = min(a.piece_cols, a.M - first);
  const auto* p = row_of<DT>(a, n, pos);
  double2* part = a.part + 3 * n * a.pieces + piece;
  if (heat.certain()) {
    const Best b = piece_best<DT>(p, first, cols, lane);
    if (lane == 0) *part = b.stored();
  } else if (pos == g || !a.draft) {
    const Mass t = piece_mass<DT>(p + first, cols, lane, heat.c);
    if (lane == 0) *part = make_double2(t.ref, t.s);
  } else {
    const Rest r = piece_rest<DT>(p + first, row_of<DT>(a, n, a.G + 1 + pos) + first, cols, lane, heat.c, near_ratio(a, n, pos, heat.c));
    if (lane == 0) {
      *part = make_double2(0.0, r.p);
      part[a.pieces] = make_double2(0.0, r.q);
      part[2 * a.pieces] = make_double2(r.a, r.b);
      a.rest[n * a.pieces + piece] = r.nearest;
    }
  }
}

// The draw of a sequence from those: a chain of loads, 8 us for 32 to 256 sequences.
template <int DT>
__global__ __launch_bounds__(64 * kDrawWaves) void draw_pick_kernel(DrawArgs a) {
  using elem = typename Logits<DT>::elem;
  constexpr int W = kDrawWaves, T = 64 * W;
  __shared__ FindRoom<W> room;
  const int64_t n = a.row0 + blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Heat heat(a, n);
  if (heat.none()) {
    write_sequence(a, n, 0, -1, T);
    return;
  }
  const int g = drafts_of(a, n), pos = tested_up_to(a, n, g);
  double2 *part = a.part + 3 * n * a.pieces, *draft_part = part + a.pieces, *rest = part + 2 * a.pieces;
  if (heat.certain()) {
    write_sequence(a, n, pos, join_best(part, a.pieces).col(), T);
    return;
  }
  Weights w;
  w.c = heat.c;
  w.p = join_mass(part, a.pieces, w.c);
  w.over_p = w.p.over();
  w.without = pos < g && !a.draft ? draft_at(a, n, pos) : -1;
  w.less = pos < g && a.draft;
  const elem *p = row_of<DT>(a, n, pos), *q = p;
  double more = 0.0;  // l - k
  if (w.less) {
    q = row_of<DT>(a, n, a.G + 1 + pos);
    w.q = join_mass(draft_part, a.pieces, w.c);
    const double k = near_ratio(a, n, pos, w.c), l = w.p.s / w.q.s;
    const auto in_range = [](double s) { return s >= kLeastSum && s <= kMostSum; };
    if (in_range(w.p.s) && in_range(w.q.s) && fabs(l - k) < 0.5 * kNear * k) {
      more = l - k;
      w.over_q = w.q.over();
      const double* nearest = a.rest + n * a.pieces;
      for (int j0 = 0; j0 < a.pieces; j0 += 64) {  // (each W-th piece is the wavefront's)
        const int mine = j0 + lane;
        uint64_t again = __ballot(mine < a.pieces && mine % W == wave && nearest[min(mine, a.pieces - 1)] <= 1.001 * fabs(more));
        for (; again != 0; again &= again - 1) {
          const int j = j0 + __builtin_ctzll(again), first = j * a.piece_cols;
          const double s = piece_weight<DT>(w, p, q, first, min(a.piece_cols, a.M - first), lane);
          if (lane == 0) rest[j] = make_double2(w.p.s * s, 0.0);
        }
      }
      __syncthreads();
    } else {  // sums about 0 leave their range, or there are none: about the maxima, here
      __syncthreads();
      for (int j = wave; j < a.pieces; j += W) {
        const int first = j * a.piece_cols, cols = min(a.piece_cols, a.M - first);
        const Mass s = piece_mass<DT>(p + first, cols, lane, w.c), t = piece_mass<DT>(q + first, cols, lane, w.c);
        if (lane == 0) {
          part[j] = make_double2(s.ref, s.s);
          draft_part[j] = make_double2(t.ref, t.s);
        }
      }
      __syncthreads();
      w.p = join_mass(part, a.pieces, w.c);
      w.q = join_mass(draft_part, a.pieces, w.c);
      w.over_p = w.p.over();
      w.over_q = w.q.over();
      if (w.is_number()) {
        for (int j = wave; j < a.pieces; j += W) {
          const int first = j * a.piece_cols;
          const double s = piece_weight<DT>(w, p, q, first, min(a.piece_cols, a.M - first), lane);
          if (lane == 0) rest[j] = make_double2(w.p.s * s, 0.0);
        }
      }
      __syncthreads();
    }
    w.over_q = w.q.over();
  }
  int drawn = -1;
  if (w.is_number())
    drawn = block_draw<DT, W>(
        a, w, p, q, [&](int j) { return part[j]; }, [&](int j) { return fmax(__builtin_fma(-more, rest[j].y, rest[j].x), 0.0) * w.over_p; },
        (double)a.uniforms[n * (a.G + 1) + a.G], room);
  write_sequence(a, n, pos, drawn, T);
}

}  // namespace rtopk
