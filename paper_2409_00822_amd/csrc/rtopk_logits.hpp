// Operators on rows of logits for gfx950 (MI355X): log probabilities of given tokens with entropy and top alternatives, distillation
// from a teacher's top logits, and the gradients of both.
//
// With x a row of M logits, T the temperature, m = max x:
//   S = sum_v exp((x_v - m) / T),  A = sum_v exp((x_v - m) / T) (x_v - m)
//   log-sum-exp = m / T + ln S,  ln q_v = (x_v - m) / T - ln S,  entropy = ln S - A / (S T)
// so a row is read once: a thread keeps the maximum, S and A of the columns it has seen and scales the two sums when its maximum
// rises; threads, wavefronts and workgroups are joined by the same rule.  Sums are fp32 whatever the logits' type.  A row whose logits
// are all -inf has S = 0: log-sum-exp -inf, entropy 0, log probabilities -inf, gradient 0.
//
// Gradients have the form  dx_v = alpha q_v - beta q_v (ln q_v + H) + sum_{j: c_j = v} w_j  with few pairs (c_j, w_j): the given tokens or
// the teacher's entries.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_kernel.hpp"
#include "rtopk_logits_dispatch.hpp"

namespace rtopk {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kFar = -1e30f;  // stands for x - m where x is -inf, so that exp(x - m) (x - m) is 0

// A log-sum-exp beyond this has too few digits behind its point for a gradient: x / T - lse would be off by 6e-5 and more, and by all of ln S
// where a row is nothing but the type's lowest value.  The row's sums are then taken again.
constexpr float kLargeLse = 1024.0f;

// ---- loads and stores -----------------------------------------------------------------------------

typedef uint32_t u4_vec __attribute__((ext_vector_type(4)));
typedef u4_vec u4_half __attribute__((aligned(2)));  // from any element of a row
typedef u4_vec u4_word __attribute__((aligned(4)));

template <int DT>
struct Logits {
  static constexpr int V = DT == kF32 ? 4 : 8;  // values of a 128-bit load
  using elem = typename std::conditional<DT == kF32, float, uint16_t>::type;
  using any4 = typename std::conditional<DT == kF32, u4_word, u4_half>::type;
  static constexpr uint32_t kLow = DT == kF32 ? 0xff800000u : (DT == kF16 ? 0xfc00fc00u : 0xff80ff80u);  // -inf

  static __device__ __forceinline__ float widen(elem v) {
    if constexpr (DT == kF32) return v;
    else if constexpr (DT == kBF16) return __uint_as_float((uint32_t)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
  }
  static __device__ __forceinline__ float at(const u4_vec& w, int c) {
    if constexpr (DT == kF32) return __uint_as_float(w[c]);
    else if constexpr (DT == kBF16) return __uint_as_float((c & 1) ? w[c / 2] & 0xffff0000u : w[c / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[c / 2] >> (16 * (c & 1))));
  }
  // the largest of a load
  static __device__ __forceinline__ float largest(const u4_vec& w) {
    if constexpr (DT == kF16) {
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      const auto two = [&](int i) {
        const uint32_t v = w[i];  // (a bit cast of the element itself takes element 0)
        return __builtin_bit_cast(h2, v);
      };
      const h2 m = __builtin_elementwise_max(__builtin_elementwise_max(two(0), two(1)), __builtin_elementwise_max(two(2), two(3)));
      return vmax((float)m[0], (float)m[1]);
    } else {
      float m = vmax(at(w, 0), at(w, 1));
#pragma unroll
      for (int i = 2; i < V; i += 2) m = vmax3(m, at(w, i), at(w, i + 1));
      return m;
    }
  }
  static __device__ __forceinline__ elem narrow(float v) {  // to nearest even
    if constexpr (DT == kF32) return v;
    else if constexpr (DT == kBF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    else return __builtin_bit_cast(uint16_t, (_Float16)v);
  }
  static __device__ __forceinline__ u4_vec pack(const float (&v)[V]) {
    u4_vec w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == kF32) w[i] = __float_as_uint(v[i]);
      else w[i] = (uint32_t)narrow(v[2 * i]) | (uint32_t)narrow(v[2 * i + 1]) << 16;
    }
    return w;
  }
  static __device__ __forceinline__ u4_vec load(const elem* p) { return *reinterpret_cast<const any4*>(p); }
  static __device__ __forceinline__ u4_vec load_once(const elem* p) { return __builtin_nontemporal_load(reinterpret_cast<const any4*>(p)); }
  static __device__ __forceinline__ void store(elem* p, const u4_vec& w) { __builtin_nontemporal_store(w, reinterpret_cast<any4*>(p)); }
};

// ---- order of the alternatives --------------------------------------------------------------------

// A whole number in the order of the logits; -0 and +0 are equal, NaN counts as -inf; 0 stands for no logit.
constexpr uint32_t kLowKey = 0x007fffffu;  // of -inf
__device__ __forceinline__ uint32_t order_key(float v) {
  if (!(v > kNegInf)) return kLowKey;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}
// The same with the column: larger for the lower one.
__device__ __forceinline__ uint64_t place_key(uint32_t key, int col) { return (uint64_t)key << 32 | (uint32_t)~col; }
__device__ __forceinline__ int place_col(uint64_t key) { return (int)~(uint32_t)key; }

// ---- sums -----------------------------------------------------------------------------------------

// Of the 64 lanes, in every lane, in a fixed order: within 16 lanes by DPP permutations, then across them to lane 63.
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, float none, F f) {
  const auto moved = [&](auto ctrl, auto rows) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using all = std::integral_constant<int, 0xf>;
  v = f(v, moved(std::integral_constant<int, 0xb1>{}, all{}));                                  // quad_perm [1, 0, 3, 2]
  v = f(v, moved(std::integral_constant<int, 0x4e>{}, all{}));                                  // quad_perm [2, 3, 0, 1]
  v = f(v, moved(std::integral_constant<int, 0x141>{}, all{}));                                 // row_half_mirror
  v = f(v, moved(std::integral_constant<int, 0x140>{}, all{}));                                 // row_mirror
  v = f(v, moved(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));    // row_bcast:15
  v = f(v, moved(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));    // row_bcast:31
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, kNegInf, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}

struct Stats {
  float m, s, a;  // maximum, S and A about it
};

// The factor and the sums of `t` about a maximum that is no smaller; c = log2(e) / T.
template <bool ENT>
__device__ __forceinline__ void scale_to(Stats& t, float m, float c) {
  const float about = m == kNegInf ? 0.0f : m;
  const float d = t.m - about, f = __builtin_amdgcn_exp2f(d * c);
  if (ENT) t.a = f * __builtin_fmaf(t.s, fmaxf(d, kFar), t.a);
  t.s *= f;
  t.m = m;
}

// While a row is read the sums are about r = m c, rounded, in powers of two: one fused multiply-add and one exp2 to a logit, and the rounding of r
// is in all terms alike.  s = sum 2^(x c - r), a = sum 2^(x c - r) (x c - r).
struct Running {
  float m, s, a;
};
// Rounding moves r by up to 2^-24 of it, which is small against 1 up to kFarReference; maxima below stay above their reference's place so that no term
// overflows, and a segment whose maximum lies beyond is summed again (segment_stats).
constexpr float kFarReference = 1048576.0f;
__device__ __forceinline__ float reference(float m, float c) { return fmaxf(m * c, -kFarReference); }

template <bool ENT>
__device__ __forceinline__ void rise_to(Running& t, float m, float c) {
  const float d = reference(t.m, c) - reference(m, c), f = __builtin_amdgcn_exp2f(d);
  if (ENT) t.a = f * __builtin_fmaf(t.s, fmaxf(d, kFar), t.a);
  t.s *= f;
  t.m = m;
}

// Whether differences from m c are too coarse: a row of nothing but a mask's large negative value, a very low temperature.
__device__ __forceinline__ bool far_maximum(float m, float c) { return fabsf(m * c) > kFarReference && fabsf(m) < __builtin_inff(); }

// All W wavefronts' sums, in every thread.  `room`: W entries; a barrier lies between its writes and reads.
template <int W, bool ENT>
__device__ __forceinline__ Running block_join(Running t, float c, float4* room) {
  rise_to<ENT>(t, wave_max(t.m), c);
  t.s = wave_sum(t.s);
  if (ENT) t.a = wave_sum(t.a);
  if (W == 1) return t;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = make_float4(t.m, t.s, t.a, 0.0f);
  __syncthreads();
  const int lane = threadIdx.x & 63;  // each wavefront takes them all, one to a lane
  Running u = {kNegInf, 0.0f, 0.0f};
  if (lane < W) u = {room[lane].x, room[lane].y, room[lane].z};
  rise_to<ENT>(u, wave_max(u.m), c);
  u.s = wave_sum(u.s);
  if (ENT) u.a = wave_sum(u.a);
  return u;
}

// Behind the main path: what seldom follows widens the loads again, rather than that every value is kept for it.
template <int U>
__device__ __forceinline__ void apart(u4_vec (&w)[U]) {
#pragma unroll
  for (int u = 0; u < U; ++u) asm volatile("" : "+v"(w[u]));
}

// Takes U loads into a thread's sums; top: their maxima.  MASKED: -inf is to be expected.
template <int DT, int U, bool ENT, bool MASKED>
__device__ __forceinline__ void absorb(u4_vec (&w)[U], float c, Running& t, float (&top)[U]) {
  using L = Logits<DT>;
  float m = t.m;
#pragma unroll
  for (int u = 0; u < U; ++u) top[u] = L::largest(w[u]);
#pragma unroll
  for (int u = 0; u + 1 < U; u += 2) m = vmax3(m, top[u], top[u + 1]);
  if (U % 2 != 0) m = vmax(m, top[U - 1]);
  rise_to<ENT>(t, m, c);
  const float r = reference(t.m, c);
  float s[2] = {0.0f, 0.0f}, a[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < U * L::V; ++i) {
    const float y = __builtin_fmaf(L::at(w[i / L::V], i % L::V), c, -r), e = __builtin_amdgcn_exp2f(y);
    s[i & 1] += e;
    if (ENT) a[i & 1] = __builtin_fmaf(e, MASKED ? fmaxf(y, kFar) : y, a[i & 1]);
  }
  t.s += s[0] + s[1];
  apart(w);
  if (ENT) {
    if (!MASKED && !(a[0] + a[1] == a[0] + a[1])) {  // 0 times -inf, from masked columns
      a[0] = a[1] = 0.0f;
      float again = r;
      asm volatile("" : "+v"(again));
#pragma unroll
      for (int i = 0; i < U * L::V; ++i) {
        const float y = __builtin_fmaf(L::at(w[i / L::V], i % L::V), c, -again);
        a[i & 1] = __builtin_fmaf(__builtin_amdgcn_exp2f(y), fmaxf(y, kFar), a[i & 1]);
      }
    }
    t.a += a[0] + a[1];
  }
}

// ---- a thread's share of a segment ----------------------------------------------------------------

// `cols` columns from `row` on, in chunks of a load's width; chunk i belongs to thread i mod T.  Rows of 16-bit values that start at an odd one
// have their first column (`lead`) apart, so that all loads start at multiples of four bytes: from there they run at the rate of aligned ones
// (8191 x 50001 half: 174 -> 131 us).  What is left at the end (`rest`, less than a chunk) and the lead make up the last chunk.
template <int DT>
struct Segment {
  using L = Logits<DT>;
  const typename L::elem* body;  // of the whole chunks
  int lead, full, rest;
  __device__ __forceinline__ Segment(const typename L::elem* row, int cols) {
    lead = DT == kF32 ? 0 : (int)((reinterpret_cast<uintptr_t>(row) >> 1) & 1);
    body = row + lead;
    full = (cols - lead) / L::V;
    rest = (cols - lead) % L::V;
  }
  __device__ __forceinline__ int chunks() const { return full + (rest + lead != 0); }
  // the last chunk: the rest's columns first, the lead in the last place, -inf between
  __device__ __forceinline__ u4_vec partial() const {
    const int end = full * L::V;
    typename L::elem v[L::V];  // (loaded without a branch, so together)
#pragma unroll
    for (int c = 0; c < L::V; ++c) v[c] = body[c < rest ? end + c : (lead != 0 ? -1 : end)];
    u4_vec w;
#pragma unroll
    for (int c = 0; c < L::V; ++c) {
      const bool is = c < rest || (c == L::V - 1 && lead != 0);
      if constexpr (DT == kF32) w[c] = is ? __float_as_uint(v[c]) : L::kLow;
      else if ((c & 1) == 0) w[c / 2] = is ? v[c] : L::kLow & 0xffffu;
      else w[c / 2] |= (is ? (uint32_t)v[c] : L::kLow & 0xffffu) << 16;
    }
    return w;
  }
  // f(columns from the segment's start, value) for each column of chunk i
  template <typename F>
  __device__ __forceinline__ void each(int i, F f) const {
    const bool whole = i < full;
    const u4_vec w = whole ? L::load(body + (uint32_t)i * L::V) : partial();
#pragma unroll
    for (int c = 0; c < L::V; ++c) {
      if (whole || c < rest) f(lead + i * L::V + c, L::at(w, c));
      else if (DT != kF32 && c == L::V - 1 && lead != 0) f(0, L::at(w, c));
    }
  }
};

// Loads batch b of the thread's whole chunks, U of them.  KEEP: the row is read again by this workgroup.
template <int DT, int T, int U, bool KEEP>
__device__ __forceinline__ void load_batch(const Segment<DT>& g, int b, u4_vec (&w)[U]) {
  using L = Logits<DT>;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const auto* p = g.body + (uint32_t)((int)threadIdx.x + (b * U + u) * T) * L::V;
    w[u] = KEEP ? L::load(p) : L::load_once(p);
  }
}

// What the segment has beyond `batches` of U T whole chunks: fewer than U T, and the partial one.  The last chunk again where a thread has none, so that
// all loads are made together; then the sums of what wavefronts have.  top: the loads' maxima, -inf past the end.
template <int DT, int T, int U, bool ENT>
__device__ __forceinline__ void absorb_rest(const Segment<DT>& g, int batches, float c, Running& t, u4_vec (&w)[U], u4_vec (&end)[1], float (&top)[U],
                                            float (&end_top)[1]) {
  using L = Logits<DT>;
  const int i = threadIdx.x + batches * (U * T);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (g.full > 0) w[u] = L::load(g.body + (uint32_t)min(i + u * T, g.full - 1) * L::V);
  end_top[0] = kNegInf;
  end[0] = u4_vec{L::kLow, L::kLow, L::kLow, L::kLow};
  const bool last = g.rest + g.lead != 0 && (int)threadIdx.x == g.full % T;
  if (last) end[0] = g.partial();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    top[u] = kNegInf;
    if (i - (int)(threadIdx.x & 63) + u * T < g.full) {
      if (i + u * T >= g.full) w[u] = u4_vec{L::kLow, L::kLow, L::kLow, L::kLow};
      float m[1];
      absorb<DT, 1, ENT, true>(reinterpret_cast<u4_vec(&)[1]>(w[u]), c, t, m);
      top[u] = m[0];
    }
  }
  if (last) absorb<DT, 1, ENT, true>(end, c, t, end_top);
}

// S, A and the maximum of the thread's chunks.
template <int DT, int T, int U, bool ENT, bool KEEP>
__device__ __forceinline__ Running thread_stats(const Segment<DT>& g, float c) {
  Running t = {kNegInf, 0.0f, 0.0f};
  u4_vec w[U], end[1];
  float top[U], end_top[1];
  const int batches = g.full / (U * T);
  for (int b = 0; b < batches; ++b) {
    load_batch<DT, T, U, KEEP>(g, b, w);
    absorb<DT, U, ENT, false>(w, c, t, top);
  }
  if (g.chunks() > batches * (U * T)) absorb_rest<DT, T, U, ENT>(g, batches, c, t, w, end, top, end_top);
  return t;
}

// A segment's sums about its maximum, in every thread, from each thread's.  `room` as for block_join.
template <int DT, int W, bool ENT>
__device__ __forceinline__ Stats segment_stats(const Segment<DT>& g, const Running& mine, float c, float4* room) {
  const Running t = block_join<W, ENT>(mine, c, room);
  if (far_maximum(t.m, c)) {
    // x - m is exact or nearly so
    Stats u = {t.m, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < g.chunks(); i += 64 * W)
      g.each(i, [&](int, float x) {
        const float d = x - t.m, e = __builtin_amdgcn_exp2f(d * c);
        u.s += e;
        if (ENT) u.a = __builtin_fmaf(e, fmaxf(d, kFar), u.a);
      });
    u.s = wave_sum(u.s);
    u.a = wave_sum(u.a);
    if (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = make_float4(u.m, u.s, u.a, 0.0f);
      __syncthreads();
      u.s = u.a = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        u.s += room[w].y;
        u.a += room[w].z;
      }
    }
    return u;
  }
  // from about r to about m: r's rounding goes out of the sums
  const float off = t.m == kNegInf ? 0.0f : __builtin_fmaf(t.m, c, -reference(t.m, c)), f = __builtin_amdgcn_exp2f(-off);
  return {t.m, t.s * f, ENT ? __builtin_fmaf(-off, t.s, t.a) * f / c : 0.0f};
}

// ---- top alternatives -----------------------------------------------------------------------------

// The k largest of a row's columns, by value and then by column, from the same pass.  The k-th largest of the threads' maxima is a floor under
// the k-th largest of what they have seen; a column of the first batch, or of a later one, that reaches the floor is listed, and after 1, 2,
// 4, 8 ... batches the floor is raised, so that each doubling lists about k columns.  Each wavefront has a list of its own, so that a place in it
// is a count of lanes and no atomic, and drops what falls below a raised floor.  At the end what has reached the last floor, a little
// over k columns, is ranked by comparing each with each.  The floor is found as the top-k selections find theirs, by
// bisection on a threshold with early stopping: it need not be the k-th exactly.  (Reading the columns of the threads that reach the floor
// again instead takes their lines from memory: 16 bytes used of 128, 8191 x 50000 fp32, k = 20, 397 us against 256.)
template <int W>
struct TopRoom {
  static constexpr int T = 64 * W;
  static constexpr int kList = W == 1 ? 512 : (W == 4 ? 256 : 128);  // of a wavefront
  static constexpr int kAll = W * kList;
  uint64_t found[kAll];  // the wavefronts' lists, one behind the other
  uint64_t best[kMaxAlternatives];
  static constexpr int kKeys = W > 4 ? 256 : T;  // maxima that floors are found among: of two or four threads where there are many
  uint32_t key[kKeys];
  int listed[W];
  uint32_t floor;
  int count, reach;
};

template <bool MAX>
__device__ __forceinline__ uint32_t wave_extreme(uint32_t v) {
  const auto f = [](float a, float b) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    return __uint_as_float(MAX ? max(x, y) : min(x, y));
  };
  return __float_as_uint(wave_reduce(__uint_as_float(v), __uint_as_float(MAX ? 0u : 0xffffffffu), f));
}

// A floor that at least k of the T keys reach, or 0 where fewer than k are not 0; the first wavefront's work.  Few more than k reach it
// unless many are equal.
template <int T>
__device__ __forceinline__ uint32_t find_floor(const uint32_t* keys, int k) {
  constexpr int P = T / 64;
  uint32_t v[P];
  uint32_t lo = 0xffffffffu, hi = 0;
  int have = 0;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    v[p] = keys[threadIdx.x + 64 * p];
    have += __popcll(__ballot(v[p] != 0));
    if (v[p] != 0) lo = min(lo, v[p]);
    hi = max(hi, v[p]);
  }
  if (have < k) return 0;
  uint32_t a = wave_extreme<false>(lo), b = wave_extreme<true>(hi) + 1;  // a is reached by k keys, b by fewer
  const int enough = k + max(8, k / 2);
  while (b - a > 1) {
    const uint32_t mid = a + (b - a) / 2;
    int n = 0;
#pragma unroll
    for (int p = 0; p < P; ++p) n += __popcll(__ballot(v[p] >= mid));
    if (n >= k) {
      a = mid;
      if (n <= enough) break;
    } else {
      b = mid;
    }
  }
  return a;
}

// The lists as one of n keys from the first on.
template <int W>
__device__ __forceinline__ void set_listed(TopRoom<W>& room, int n) {
  if (threadIdx.x < W) room.listed[threadIdx.x] = min(max(n - (int)threadIdx.x * TopRoom<W>::kList, 0), TopRoom<W>::kList);
}

// Ranks the lists' distinct keys: the k largest in order in room.best, 0 where there are fewer.
template <int W>
__device__ __forceinline__ void rank_listed(TopRoom<W>& room, int k) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int all = 0, at = 0;  // at: where the lane's key of the lists' first 64 lies
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int m = room.listed[w];
    if (lane >= all && lane < all + m) at = w * TopRoom<W>::kList + lane - all;
    all += m;
  }
  for (int j = all + threadIdx.x; j < k; j += 64 * W) room.best[j] = 0;
  if (all <= 64) {  // a key to a lane of the first wavefront, each held against all by way of scalar registers
    if (wave == 0) {
      const uint64_t key = lane < all ? room.found[at] : 0;
      int rank = 0;
      for (int i = 0; i < all; ++i) {
        const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, i);
        rank += other > key;
      }
      if (lane < all && rank < k) room.best[rank] = key;
    }
  } else {
    const int n = room.listed[wave];
    for (int j = lane; j < n; j += 64) {
      const uint64_t key = room.found[wave * TopRoom<W>::kList + j];
      int rank = 0;
      for (int w = 0; w < W; ++w) {
        const int m = room.listed[w];
#pragma unroll 8
        for (int i = 0; i < m; ++i) rank += room.found[w * TopRoom<W>::kList + i] > key;
      }
      if (rank < k) room.best[rank] = key;
    }
  }
  __syncthreads();
}

// Columns of the segment whose key reaches `least`, over the workgroup.
template <int DT, int T>
__device__ __forceinline__ int count_reaching(const Segment<DT>& g, uint32_t least, int* slot) {
  if (threadIdx.x == 0) *slot = 0;
  __syncthreads();
  int n = 0;
  for (int i = threadIdx.x; i < g.chunks(); i += T) g.each(i, [&](int, float v) { n += order_key(v) >= least; });
  atomicAdd(slot, n);
  __syncthreads();
  n = *slot;
  __syncthreads();
  return n;
}

// Lists the columns of a load that reach the floor behind the wavefront's `n` (uniform); col(e): of the thread's element e.  n counts on past
// the end.
template <int DT, int W, typename F>
__device__ __forceinline__ void list_chunk(const u4_vec& w, float floor, TopRoom<W>& room, int& n, F col) {
  using L = Logits<DT>;
  uint64_t* list = room.found + (threadIdx.x >> 6) * TopRoom<W>::kList;
  u4_vec here = w;
  asm volatile("" : "+v"(here));  // (else all loads are widened before the branch)
#pragma unroll
  for (int e = 0; e < L::V; ++e) {
    const float v = L::at(here, e);
    const uint64_t mask = __ballot(v >= floor);
    if (mask != 0) {
      const int at = (int)lanes_below(mask, (uint32_t)n);
      if (v >= floor && at < TopRoom<W>::kList) list[at] = place_key(order_key(v), col(e));
      n += __popcll(mask);
    }
  }
}

// Drops what lies below the floor from the wavefront's list.
template <int W>
__device__ __forceinline__ void drop_below(uint32_t least, TopRoom<W>& room, int& n) {
  uint64_t* list = room.found + (threadIdx.x >> 6) * TopRoom<W>::kList;
  const int lane = threadIdx.x & 63;
  int kept = 0;
  for (int i = 0; i < n; i += 64) {
    const uint64_t key = i + lane < n ? list[i + lane] : 0;
    const uint64_t mask = __ballot((uint32_t)(key >> 32) >= least);
    if ((uint32_t)(key >> 32) >= least) list[lanes_below(mask, (uint32_t)kept)] = key;  // (at or before its place, after all lanes' reads)
    kept += __popcll(mask);
  }
  n = kept;
}

// The floor under the k-th largest logit seen so far, in every thread: the smallest finite value where fewer than k threads have seen more
// than -inf.
template <int W>
__device__ __forceinline__ float raise_floor(float seen, int k, TopRoom<W>& room) {
  uint32_t key = order_key(seen);
  constexpr int of = W > 4 ? W / 4 : 1;
  if (of >= 2) key = max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0xb1, 0xf, 0xf, false));
  if (of == 4) key = max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0x4e, 0xf, 0xf, false));
  if (threadIdx.x % of == 0) room.key[threadIdx.x / of] = key == kLowKey ? 0 : key;
  __syncthreads();
  if (threadIdx.x < 64) {
    const uint32_t f = find_floor<TopRoom<W>::kKeys>(room.key, k);
    if (threadIdx.x == 0) room.floor = f == 0 ? kLowKey + 1 : f;
  }
  __syncthreads();
  return order_value(room.floor);
}

// The first columns whose key is `least` follow the n of the first list up to k; the first wavefront's work.  Returns how many there are then.
template <int DT, int W>
__device__ int fill_list(const Segment<DT>& g, int first, int k, uint32_t least, int n, TopRoom<W>& room) {
  uint64_t* list = room.found;
  const int lane = threadIdx.x, chunks = g.chunks();
  if (g.lead != 0 && n < k && order_key(Logits<DT>::widen(g.body[-1])) == least) {
    if (lane == 0) list[n] = place_key(least, first);
    ++n;
  }
  for (int i = lane; n < k && i - lane < chunks; i += 64) {
    int mine = 0;
    if (i < chunks) g.each(i, [&](int col, float v) { mine += col >= g.lead && order_key(v) == least; });
    int before = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(before, d);
      if (lane >= d) before += o;
    }
    const int all = __shfl(before, 63);
    before += n - mine;
    if (mine > 0 && before < k)
      g.each(i, [&](int col, float v) {
        if (col >= g.lead && order_key(v) == least) {
          if (before < k) list[before] = place_key(least, first + col);
          ++before;
        }
      });
    n += all;
  }
  return min(n, k);
}

// More columns reached the floors than there is room for: equal logits in crowds, or logits that ascend.  Bisection over the whole segment, until
// so few columns reach the threshold that they can be listed, or none lies between the bounds; then the columns equal to it fill up.
// `least` is reached by k columns.
template <int DT, int W>
__device__ void list_again(const Segment<DT>& g, int first, int k, uint32_t least, TopRoom<W>& room) {
  constexpr int T = 64 * W, kAll = TopRoom<W>::kAll;
  uint64_t a = least, b = (uint64_t)1 << 32;
  int reach = g.lead + g.full * Logits<DT>::V + g.rest, above = 0;
  bool next = true;  // the first threshold is the one above `least`: all others are equal where a mask has left few columns
  while (b - a > 1 && reach > kAll) {
    const uint32_t mid = next ? (uint32_t)(a + 1) : (uint32_t)(a + (b - a) / 2);
    next = false;
    const int n = count_reaching<DT, T>(g, mid, &room.reach);
    if (n >= k) {
      a = mid;
      reach = n;
    } else {
      b = mid;
      above = n;
    }
  }
  const bool crowd = reach > kAll;  // fewer than k lie above `a`, too many equal it
  const uint32_t listed = (uint32_t)a + (crowd ? 1 : 0);
  if (threadIdx.x == 0) room.count = 0;
  __syncthreads();
  if (!crowd || above > 0)
    for (int i = threadIdx.x; i < g.chunks(); i += T)
      g.each(i, [&](int col, float v) {
        const uint32_t o = order_key(v);
        if (o >= listed) {
          const int at = atomicAdd(&room.count, 1);
          if (at < kAll) room.found[at] = place_key(o, first + col);  // (the lists follow one another)
        }
      });
  __syncthreads();
  int n = room.count;
  __syncthreads();
  if (crowd) {
    if (threadIdx.x < 64) {
      n = fill_list<DT, W>(g, first, k, (uint32_t)a, n, room);
      if (threadIdx.x == 0) room.count = n;
    }
    __syncthreads();
    n = room.count;
  }
  set_listed(room, n);
  __syncthreads();
}

// thread_stats, and the k largest of the segment in room.best, best first (0 where it has fewer columns); first: the segment's first column.
template <int DT, int W, int U, bool ENT>
__device__ Running stats_and_top(const Segment<DT>& g, int first, int k, float c, TopRoom<W>& room) {
  using L = Logits<DT>;
  constexpr int T = 64 * W, kList = TopRoom<W>::kList;
  Running t = {kNegInf, 0.0f, 0.0f};
  float floor = 0.0f;
  int n = 0;  // the wavefront's list
  bool lost = false;
  const auto raise = [&] {
    floor = raise_floor<W>(t.m, k, room);
    lost |= n > kList;
    n = min(n, kList);
    drop_below<W>(order_key(floor), room, n);
  };
  const auto list = [&](const u4_vec(&w)[U], const float(&top)[U], int b) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (__any(top[u] >= floor)) {
        const int col = first + g.lead + ((int)threadIdx.x + (b * U + u) * T) * L::V;
        list_chunk<DT, W>(w[u], floor, room, n, [&](int e) { return col + e; });
      }
  };
  u4_vec w[U];
  float top[U];
  const int batches = g.full / (U * T);
  constexpr bool AHEAD = W == 16 && U == 4;  // few rows: nothing else covers the wait for the next batch (eight loads have no registers left for it)
  if (AHEAD && batches > 0) load_batch<DT, T, U, false>(g, 0, w);
  for (int b = 0; b < batches; ++b) {
    u4_vec next[U];
    if (!AHEAD) load_batch<DT, T, U, false>(g, b, w);
    absorb<DT, U, ENT, false>(w, c, t, top);
    if (AHEAD && b + 1 < batches) load_batch<DT, T, U, false>(g, b + 1, next);
    if ((b & (b + 1)) == 0) raise();
    list(w, top, b);
    if (AHEAD && b + 1 < batches) {
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = next[u];
    }
  }
  if (g.chunks() > batches * (U * T)) {
    u4_vec end[1];
    float end_top[1];
    absorb_rest<DT, T, U, ENT>(g, batches, c, t, w, end, top, end_top);
    raise();
    list(w, top, batches);
    if (__any(end_top[0] >= floor))
      list_chunk<DT, W>(end[0], floor, room, n, [&](int e) { return e < g.rest ? first + g.lead + g.full * L::V + e : first; });
  } else if ((batches & (batches - 1)) != 0) {
    raise();
  }
  lost |= n > kList;
  if ((threadIdx.x & 63) == 0) room.listed[threadIdx.x >> 6] = lost ? kList + 1 : n;
  __syncthreads();
  int all = 0;
  bool again = false;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    all += room.listed[w];
    again |= room.listed[w] > kList;
  }
  if (again) {
    __syncthreads();
    list_again<DT, W>(g, first, k, order_key(floor), room);
  } else if (all < k) {  // all finite ones are listed: those that are not follow in the first list
    __syncthreads();
    if (threadIdx.x < 64) {
      const int filled = fill_list<DT, W>(g, first, k - all + n, kLowKey, n, room), most = min(k, g.lead + g.full * L::V + g.rest);
      if (threadIdx.x == 0) room.listed[0] = filled;
      // Fewer still: a signalling NaN, for which a maximum is NaN, hid columns beside it.  Nothing of such a row is a number: its first columns.
      if (all - n + filled < most) {
        for (int j = threadIdx.x; j < most; j += 64) room.found[j] = place_key(kLowKey, first + j);
        set_listed(room, most);
      }
    }
    __syncthreads();
  }
  rank_listed<W>(room, k);
  return t;
}

// ---- given tokens and the teacher's entries -------------------------------------------------------

__device__ __forceinline__ int token_at(const LogitsArgs& a, int64_t i) {  // -1: left out
  const int64_t t = a.token64 ? static_cast<const int64_t*>(a.tokens)[i] : static_cast<const int32_t*>(a.tokens)[i];
  return t >= 0 && t < a.M ? (int)t : -1;
}

__device__ __forceinline__ float teacher_at(const LogitsArgs& a, int64_t i) {
  if (a.teacher_dtype == kF32) return static_cast<const float*>(a.teacher_vals)[i];
  const uint16_t h = static_cast<const uint16_t*>(a.teacher_vals)[i];
  return a.teacher_dtype == kBF16 ? Logits<kBF16>::widen(h) : Logits<kF16>::widen(h);
}

// Whether the row has an entry that counts, looked up by each wavefront for itself.
__device__ __forceinline__ bool any_entry(const LogitsArgs& a, int64_t n) {
  for (int j = threadIdx.x & 63; j - (int)(threadIdx.x & 63) < a.k; j += 64) {
    const int col = j < a.k ? a.teacher_cols[n * a.k + j] : -1;
    if (__any(col >= 0 && col < a.M && !(teacher_at(a, n * a.k + j) == kNegInf))) return true;  // (NaN counts)
  }
  return false;
}

// A row's list in LDS: three values to an entry in the launch's dynamic memory (list_bytes), so that short lists leave room for more workgroups.
struct ListHead {
  float mass;     // sum of w
  int ascending;  // columns in strictly ascending order, so none twice
};
struct ListRoom {
  int* col;
  float* w;   // the teacher's probability, or the gradient that belongs to a token
  float* lp;  // logarithm of the former
  ListHead& head;
  __device__ __forceinline__ ListRoom(float* memory, int k, ListHead& h)
      : col(reinterpret_cast<int*>(memory)), w(memory + k), lp(memory + 2 * k), head(h) {}
};
inline size_t list_bytes(int k) { return 12 * (size_t)k; }

// The first wavefront writes the row's list to LDS; entries that do not count have column -1 and weight 0.
__device__ __forceinline__ void teacher_list(const LogitsArgs& a, int64_t n, ListRoom& r) {
  const int lane = threadIdx.x;
  const float c = a.c;
  float top = kNegInf;
  bool ascending = true;
  for (int j = lane; j < a.k; j += 64) {
    const int col = a.teacher_cols[n * a.k + j];
    const bool ok = col >= 0 && col < a.M;
    const float t = ok ? teacher_at(a, n * a.k + j) : kNegInf;
    if (j > 0 && a.teacher_cols[n * a.k + j - 1] >= col) ascending = false;
    r.col[j] = ok ? col : -1;
    r.lp[j] = t;
    top = fmaxf(top, t);
  }
  float less = 0.0f, scale = 1.0f;  // ln p = (t - top) / T - less
  if (!a.log_probs) {
    top = wave_max(top);
    if (top == kNegInf) top = 0.0f;
    float z = 0.0f;
    for (int j = lane; j < a.k; j += 64) z += __builtin_amdgcn_exp2f((r.lp[j] - top) * c);
    less = logf(wave_sum(z));
    scale = a.inv_t;
  } else {
    top = 0.0f;
  }
  float mass = 0.0f;
  for (int j = lane; j < a.k; j += 64) {
    const float lp = (r.lp[j] - top) * scale - less;
    const float p = r.lp[j] == kNegInf ? 0.0f : expf(lp);
    if (p == 0.0f) r.col[j] = -1;
    r.lp[j] = lp;
    r.w[j] = p;
    mass += p;
  }
  mass = wave_sum(mass);
  const bool all = __all(ascending);
  if (lane == 0) {
    r.head.mass = mass;
    r.head.ascending = all;
  }
}

__device__ __forceinline__ void token_list(const LogitsArgs& a, int64_t n, ListRoom& r) {
  const int lane = threadIdx.x;
  float mass = 0.0f;
  for (int j = lane; j < a.k; j += 64) {
    const int col = token_at(a, n * a.k + j);
    const float w = col >= 0 ? a.grad[n * a.k + j] : 0.0f;
    r.col[j] = col;
    r.w[j] = w;
    mass += w;
  }
  mass = wave_sum(mass);
  if (lane == 0) {
    r.head.mass = mass;
    r.head.ascending = a.k == 1;
  }
}

// -inf for a row of nothing but -inf, and for no other: what lies beyond fp32 is its last finite number.
__device__ __forceinline__ float log_sum_exp(const LogitsArgs& a, const Stats& t, float ln_s) {
  if (t.s == 0.0f) return kNegInf;
  const float v = __builtin_fmaf(t.m, a.inv_t, ln_s);
  return fabsf(v) == __builtin_inff() && fabsf(t.m) < __builtin_inff() ? copysignf(3.402823466e38f, v) : v;
}

// Loss of the row from its list; the first wavefront's work, in its every lane.
template <int DT>
__device__ __forceinline__ float list_loss(const LogitsArgs& a, const typename Logits<DT>::elem* row, const Stats& t, float ln_s, const ListRoom& r) {
  float loss = 0.0f;
  for (int j = threadIdx.x; j < a.k; j += 64)
    if (r.col[j] >= 0) {
      const float lq = t.s == 0.0f ? kNegInf : (Logits<DT>::widen(row[r.col[j]]) - t.m) * a.inv_t - ln_s;
      loss = __builtin_fmaf(r.w[j], r.lp[j] - lq, loss);
    }
  return wave_sum(loss);
}

// ---- forward --------------------------------------------------------------------------------------

// What a row's sums give: log probabilities of the tokens, entropy, log-sum-exp.
template <int DT>
__device__ __forceinline__ void write_tokens(const LogitsArgs& a, int64_t n, const typename Logits<DT>::elem* row, const Stats& t, float ln_s, int T) {
  const bool empty = t.s == 0.0f;
  for (int g = threadIdx.x; g < a.tokens_per_row; g += T) {
    const int col = token_at(a, n * a.tokens_per_row + g);
    float lp = 0.0f;
    if (col >= 0) lp = empty ? kNegInf : (Logits<DT>::widen(row[col]) - t.m) * a.inv_t - ln_s;
    a.logprobs[n * a.tokens_per_row + g] = lp;
  }
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[n] = log_sum_exp(a, t, ln_s);
    if (a.entropy) a.entropy[n] = empty ? 0.0f : ln_s - t.a / t.s * a.inv_t;
  }
}

template <int W>
__device__ __forceinline__ void write_top(const LogitsArgs& a, int64_t n, const Stats& t, float ln_s, const TopRoom<W>& room) {
  for (int j = threadIdx.x; j < a.k; j += 64 * W) {
    const uint64_t key = room.best[j];
    a.top_logprobs[n * a.k + j] = t.s == 0.0f ? kNegInf : (order_value((uint32_t)(key >> 32)) - t.m) * a.inv_t - ln_s;
    a.top_cols[n * a.k + j] = place_col(key);
  }
}

// One workgroup reads a segment of a row.  SPLIT: its sums and alternatives go to scratch memory for logits_join_kernel; else the segment is the
// row and the results are written.
// Many rows: four wavefronts to a row (eight rows to a compute unit, so that some load while others search), bound by HBM for fp32 (8191 x 50000 250 us,
// 6.55 TB/s; 255 with 20 alternatives), by HBM and the vector ALU in 16 bits, which have twice the terms to a byte (bfloat16 127 us, 6.46 TB/s, its
// ALU 84 % busy; 154 with 20 alternatives; half, odd columns, one alternative 146).  The bfloat16 form with alternatives is held to 80
// registers, six wavefronts to a SIMD: 8191 x 50000, k = 20, 164 -> 154 us.  Few rows: bound by the chain load, sums, floor, ranks, each a
// microsecond or two (1 x 32768 fp32, k = 5, 6.9 us).
template <int DT, int W, int OP, bool TOP, bool SPLIT>
__global__ __launch_bounds__(64 * W, TOP && W == 4 && DT == kBF16 ? 6 : 1) void logits_rows_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  constexpr bool ENT = OP == kOpTokens;
  // fp32 rows of sixteen wavefronts, eight loads and four, us, k = 20: 1 x 32768 7.1 and 8.4, 1 x 20000 7.7 and 8.1, 64 x 24000 9.2 and 9.6, 200 x 32000 10.1 and
  // 10.9, 100 x 65536 (k = 5) 9.9 and 10.8; below one batch and over several of them it loses: 256 x 8000 8.2 and 7.8, 200 x 16000 8.7 and 8.4, 200 x 131072 (k = 5)
  // 24.4 and 20.6.  Twice the values of 16 bits have no registers for it.
  constexpr int U = DT == kF32 && W == 16 ? 8 : 4;
  __shared__ float4 sums[W];
  const int seg = SPLIT ? (int)(blockIdx.x % (uint32_t)a.segments) : 0;
  const int64_t n = a.row0 + (SPLIT ? blockIdx.x / (uint32_t)a.segments : blockIdx.x);
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  const int first = seg * a.seg_cols;
  const Segment<DT> g(row + first, min(a.seg_cols, a.M - first));
  const float c = a.c;
  extern __shared__ float list_memory[];
  __shared__ ListHead head;
  ListRoom list(list_memory, a.k, head);  // (distillation only)
  if constexpr (OP == kOpDistill && !SPLIT) {
    if (threadIdx.x < 64) teacher_list(a, n, list);
  }
  Stats t;
  if constexpr (!TOP) {
    t = segment_stats<DT, W, ENT>(g, thread_stats<DT, T, 4, ENT, false>(g, c), c, sums);
  } else {
    __shared__ TopRoom<W> room;
    t = segment_stats<DT, W, ENT>(g, stats_and_top<DT, W, U, ENT>(g, first, a.k, c, room), c, sums);
    if constexpr (SPLIT) {
      uint64_t* keys = a.part_keys + (n * a.segments + seg) * a.k;
      for (int j = threadIdx.x; j < a.k; j += T) keys[j] = room.best[j];
    } else {
      write_top<W>(a, n, t, logf(t.s), room);
    }
  }
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) a.part[n * a.segments + seg] = make_float4(t.m, t.s, t.a, 0.0f);
  } else if constexpr (OP == kOpTokens) {
    write_tokens<DT>(a, n, row, t, logf(t.s), T);
  } else if (threadIdx.x < 64) {
    const float ln_s = logf(t.s), loss = list_loss<DT>(a, row, t, ln_s, list);
    if (threadIdx.x == 0) {
      a.loss[n] = loss;
      if (a.lse) a.lse[n] = log_sum_exp(a, t, ln_s);
    }
  }
}

// Sums of a row's segments, in every lane: each wavefront takes them all.
template <bool ENT>
__device__ __forceinline__ Stats join_segments(const LogitsArgs& a, int64_t n, float c) {
  Stats t = {kNegInf, 0.0f, 0.0f};
  for (int s = threadIdx.x & 63; s < a.segments; s += 64) {
    const float4 p = a.part[n * a.segments + s];
    Stats u = {p.x, p.y, p.z};
    const float m = fmaxf(t.m, u.m);
    scale_to<ENT>(t, m, c);
    scale_to<ENT>(u, m, c);
    t.s += u.s;
    t.a += u.a;
  }
  scale_to<ENT>(t, wave_max(t.m), c);
  t.s = wave_sum(t.s);
  if (ENT) t.a = wave_sum(t.a);
  return t;
}

// Joins a row's segments.  Its time is that of a launch and a few trips to memory, 3.5 to 6 us (64 x 131072 bfloat16, 20 alternatives: 5.7); a row's last workgroup cannot do the work instead, for
// the counter that would tell it is the last has to be zero beforehand, which is a launch too.
template <int DT, int OP, bool TOP>
__global__ __launch_bounds__(256) void logits_join_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 256;
  const int64_t n = a.row0 + blockIdx.x;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  extern __shared__ float list_memory[];
  __shared__ ListHead head;
  ListRoom list(list_memory, a.k, head);  // (distillation only)
  if constexpr (OP == kOpDistill) {
    if (threadIdx.x < 64) teacher_list(a, n, list);
  }
  const Stats t = join_segments<OP == kOpTokens>(a, n, a.c);
  const float ln_s = logf(t.s);
  if constexpr (TOP) {
    // the segments' alternatives, merged as a segment's columns are: each thread's largest, a floor, what reaches it
    __shared__ TopRoom<4> room;
    const uint64_t* keys = a.part_keys + n * a.segments * a.k;
    const int all = a.segments * a.k;  // at most kMaxMergeKeys
    constexpr int P = kMaxMergeKeys / T;
    uint64_t v[P];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = threadIdx.x + p * T;
      v[p] = i < all ? keys[i] : 0;
      top = max(top, (uint32_t)(v[p] >> 32));
    }
    if (threadIdx.x == 0) room.count = 0;
    uint64_t least = 1;  // any key
    if (all > 128) {  // (so few are ranked as they are)
      room.key[threadIdx.x] = top;
      __syncthreads();
      if (threadIdx.x < 64) {
        const uint32_t f = find_floor<T>(room.key, a.k);
        if (threadIdx.x == 0) room.floor = f;
      }
      __syncthreads();
      least = (uint64_t)max(room.floor, 1u) << 32;  // (0: all that are keys)
    }
    if (all > TopRoom<4>::kAll) {
      // bisection on the whole keys, which are distinct, where more reach the floor than there is room for
      int reach = all;
      const auto count = [&](uint64_t mid) {
        if (threadIdx.x == 0) room.count = 0;
        __syncthreads();
        int n = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) n += v[p] >= mid;
        if (n > 0) atomicAdd(&room.count, n);
        __syncthreads();
        n = room.count;
        __syncthreads();
        return n;
      };
      reach = count(least);
      uint64_t b = ~(uint64_t)0;
      while (reach > TopRoom<4>::kAll) {
        const uint64_t mid = least + (b - least) / 2;
        const int n = count(mid);
        if (n >= a.k) {
          least = mid;
          reach = n;
        } else {
          b = mid;
        }
      }
      if (threadIdx.x == 0) room.count = 0;
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (v[p] >= least) room.found[atomicAdd(&room.count, 1)] = v[p];
    __syncthreads();
    set_listed(room, room.count);
    __syncthreads();
    rank_listed<4>(room, a.k);
    write_top<4>(a, n, t, ln_s, room);
  }
  if constexpr (OP == kOpTokens) {
    write_tokens<DT>(a, n, row, t, ln_s, T);
  } else if (threadIdx.x < 64) {
    const float loss = list_loss<DT>(a, row, t, ln_s, list);
    if (threadIdx.x == 0) {
      a.loss[n] = loss;
      if (a.lse) a.lse[n] = log_sum_exp(a, t, ln_s);
    }
  }
}

// ---- gradients ------------------------------------------------------------------------------------

// dx_v but for the list: alpha q - beta q (ln q + H).  q from the maximum and sum of a row (x - m is exact or nearly so), or from its
// log-sum-exp.
struct Base {
  float alpha, beta, h;  // h: entropy
  float m, inv_t, less;  // ln q = (x - m) inv_t - less
  template <bool ENT>
  __device__ __forceinline__ float at(float x) const {
    float lq = __builtin_fmaf(x - m, inv_t, -less);
    if (ENT) lq = lq < kFar ? kFar : lq;  // (NaN stays)
    const float q = __builtin_amdgcn_exp2f(lq * kLog2e);
    // (q first: beta is 1 / T times a gradient and may be so large that beta ln q leaves fp32, where q is 0 above all)
    return ENT ? __builtin_fmaf(-beta, q * (lq + h), alpha * q) : alpha * q;
  }
};

// A segment of the gradient; ZERO: the base is 0 whatever the logits are, which are not read.
template <int DT, int U, bool ENT, bool ZERO>
__device__ __forceinline__ void write_base(const Segment<DT>& g, typename Logits<DT>::elem* out, int T, const Base& base) {
  using L = Logits<DT>;
  int i = threadIdx.x;
  const u4_vec none = {0, 0, 0, 0};
  const auto turn = [&](const u4_vec& w) {
    float y[L::V];
#pragma unroll
    for (int c = 0; c < L::V; ++c) y[c] = base.template at<ENT>(L::at(w, c));
    return L::pack(y);
  };
  typename L::elem* to = out + g.lead;
  for (; i + (U - 1) * T < g.full; i += U * T) {
    u4_vec w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = ZERO ? none : L::load_once(g.body + (uint32_t)(i + u * T) * L::V);
#pragma unroll
    for (int u = 0; u < U; ++u) L::store(to + (uint32_t)(i + u * T) * L::V, ZERO ? none : turn(w[u]));
  }
  for (; i < g.full; i += T) L::store(to + (uint32_t)i * L::V, ZERO ? none : turn(L::load_once(g.body + (uint32_t)i * L::V)));
  if ((int)threadIdx.x < g.rest + g.lead) {
    const int64_t at = (int)threadIdx.x < g.rest ? (int64_t)g.full * L::V + threadIdx.x : -1;
    to[at] = ZERO ? L::narrow(0.0f) : L::narrow(base.template at<ENT>(L::widen(g.body[at])));
  }
}

// Entry j of the list, after the base has been written (a barrier lies between): where its column lies in the segment and no earlier entry has
// it, the column's one value, rounded once.  base_y: the base at the column; factor * weight(i): what an entry adds.  Unless columns strictly ascend each
// entry is held against all: 2048 x 65536 fp32 with lists of 64 in the order of their values 181 us against 173 in the order of their columns, of 256 1443
// against 189, of 1024 22 ms against 0.39; loss and gradient in one call at 2048 x 50000 182 against 156, 410 against 189, 2.1 ms against 0.37.
template <int DT, typename F>
__device__ __forceinline__ void write_entry(const LogitsArgs& a, const ListRoom& r, int j, int first, int cols, typename Logits<DT>::elem* out,
                                            float factor, float base_y, F weight) {
  const int col = r.col[j];
  if (col < first || col >= first + cols) return;
  float w = weight(j);
  if (!r.head.ascending)
    for (int i = 0; i < a.k; ++i)
      if (i != j && r.col[i] == col) {
        if (i < j) return;
        w += weight(i);
      }
  out[col - first] = Logits<DT>::narrow(__builtin_fmaf(factor, w, base_y));
}

// All entries.  `x`: the logits at the thread's entries, read before the base was written (the gradient may lie in the logits' place).
template <int DT, int T, bool ENT, bool ZERO>
__device__ __forceinline__ void write_list(const LogitsArgs& a, const ListRoom& r, int first, int cols, typename Logits<DT>::elem* out,
                                           const Base& base, float factor, const float (&x)[(kMaxList + T - 1) / T]) {
#pragma unroll
  for (int e = 0; e < (kMaxList + T - 1) / T; ++e) {
    const int j = threadIdx.x + e * T;
    if (j >= a.k) break;
    write_entry<DT>(a, r, j, first, cols, out, factor, ZERO ? 0.0f : base.template at<ENT>(x[e]), [&](int i) { return r.w[i]; });
  }
}

template <int DT, int T>
__device__ __forceinline__ void read_list(const LogitsArgs& a, const ListRoom& r, int first, int cols, const typename Logits<DT>::elem* seg,
                                          float (&x)[(kMaxList + T - 1) / T]) {
#pragma unroll
  for (int e = 0; e < (kMaxList + T - 1) / T; ++e) {
    const int j = threadIdx.x + e * T;
    x[e] = 0.0f;
    if (j < a.k) {
      const int col = r.col[j];
      if (col >= first && col < first + cols) x[e] = Logits<DT>::widen(seg[col - first]);
    }
  }
}

template <int DT, int T, bool ENT>
__device__ __forceinline__ void write_gradient(const LogitsArgs& a, const ListRoom& r, const Segment<DT>& g, int first, int cols,
                                               typename Logits<DT>::elem* out, const Base& base, float factor, bool zero) {
  if (zero) {  // (uniform over the workgroup)
    float x[(kMaxList + T - 1) / T];
    write_base<DT, 4, ENT, true>(g, out, T, base);
    __syncthreads();
    if (factor != 0.0f) write_list<DT, T, ENT, true>(a, r, first, cols, out, base, factor, x);
    return;
  }
  float x[(kMaxList + T - 1) / T];
  read_list<DT, T>(a, r, first, cols, g.body - g.lead, x);
  __syncthreads();
  write_base<DT, 4, ENT, false>(g, out, T, base);
  __syncthreads();
  write_list<DT, T, ENT, false>(a, r, first, cols, out, base, factor, x);
}

// Bound by HBM: logits read once, gradient written once (4096 x 131072 bfloat16, an eighth of the rows not read, 339 us, 5.95 TB/s; 2048 x 65536 fp32,
// lists of 100, 172 us, 6.24 TB/s; this repository's copy kernels reach 6.2 to 6.5).
// A segment of a row's gradient by one workgroup (several, where the row's sums are taken again).  The row's sums are known: its log-sum-exp was saved
// (JOIN false), or the segments' sums lie in scratch memory (JOIN, distillation only), and then the loss is written too.
template <int DT, int OP, bool ENT, bool JOIN, int W>
__global__ __launch_bounds__(64 * W) void logits_grad_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  extern __shared__ float list_memory[];
  __shared__ ListHead head;
  ListRoom list(list_memory, a.k, head);
  __shared__ float4 sums[W];
  const int seg = (int)(blockIdx.x % (uint32_t)a.segments);
  const int64_t n = a.row0 + blockIdx.x / (uint32_t)a.segments;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + n * a.grad_stride;
  int first = seg * a.seg_cols, cols = min(a.seg_cols, a.M - first);
  if (threadIdx.x < 64) {
    if (OP == kOpTokens) token_list(a, n, list);
    else teacher_list(a, n, list);
  }
  Base base;
  base.inv_t = a.inv_t;
  base.m = 0.0f;
  base.less = JOIN ? 0.0f : a.lse_in[n];
  const float up = OP == kOpTokens ? a.inv_t : a.inv_t * a.grad[n];
  bool empty;
  __syncthreads();
  if constexpr (JOIN) {
    const Stats t = join_segments<false>(a, n, a.c);
    base.m = t.m;
    base.less = logf(t.s);
    empty = t.s == 0.0f;
    if (a.loss && seg == 0 && threadIdx.x < 64) {
      const float loss = list_loss<DT>(a, row, t, base.less, list);
      if (threadIdx.x == 0) a.loss[n] = loss;
    }
  } else {
    empty = base.less == kNegInf;
    // (a row without a gradient is not read)
    if (fabsf(base.less) > kLargeLse && fabsf(base.less) < __builtin_inff() && __any(up * head.mass != 0.0f || (ENT && a.inv_t * a.grad_entropy[n] != 0.0f))) {
      // One of `far_group` workgroups takes the row's sums and writes the segments of all: another one in each row, for neighbours lie in different XCDs.
      const int group = seg - seg % a.far_group, of = min(a.far_group, a.segments - group);
      if (seg - group != (int)(n % of)) return;
      first = group * a.seg_cols;
      cols = min(of * a.seg_cols, a.M - first);
      const Segment<DT> all(row, a.M);
      const Stats t = segment_stats<DT, W, false>(all, thread_stats<DT, T, 4, false, true>(all, a.c), a.c, sums);
      base.m = t.m;
      base.less = logf(t.s);
    }
  }
  base.alpha = OP == kOpTokens ? -up * head.mass : up * head.mass;
  base.beta = ENT ? a.inv_t * a.grad_entropy[n] : 0.0f;
  base.h = ENT ? a.entropy_in[n] : 0.0f;
  const bool zero = empty || (base.alpha == 0.0f && base.beta == 0.0f);
  const Segment<DT> g(row + first, cols);
  write_gradient<DT, T, ENT>(a, list, g, first, cols, out + first, base, empty ? 0.0f : (OP == kOpTokens ? up : -up), zero);
}

// Loss and gradient of a row by one workgroup that holds it on chip, so that it is read once and its gradient written once: R loads of each thread in
// registers and, for the widest rows, Q more in LDS.  The first Q loads go on to LDS once they are in the sums, and their registers take
// the last Q.  With eight wavefronts and 128 registers each, two such workgroups share a compute unit, and one's loads and stores overlap
// the other's arithmetic.
// Bound by HBM where rows are wide: 8192 x 131072 bfloat16, lists of 64, an eighth of the rows without entries, 750 us (5.38 TB/s; the streaming gradient
// kernel above takes 762 for all rows' bytes), 4096 x 65536 fp32 380 us (5.65 TB/s), against 930 and 471 us with the row read twice; 2048 x 50000
// fp32, lists of 100, 167 us (147).  Few rows in flight are better than many: 64 KiB rows on 8 wavefronts of 4 + 4 loads 103 us, on 4 of 16 107; 128 KiB
// ones on 8 of 8 + 8 381, on 4 of 24 + 8 405.  Workgroups that stay and load their next row while they store one lose 20 to 30 %.
template <int DT, int W, int R, int Q>
__global__ __launch_bounds__(64 * W, R + Q > 16 && W == 8 ? 4 : 1) void distill_held_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  constexpr int G = R > 16 ? 2 : 4;  // loads that are summed together: more take registers that the row needs
  static_assert(R % G == 0 && Q % G == 0 && Q <= R, "whole groups");
  extern __shared__ float list_memory[];
  __shared__ ListHead head;
  ListRoom list(list_memory, a.k, head);  // (w: the logits at the list's columns)
  __shared__ float4 sums[W];
  __shared__ u4_vec room[Q > 0 ? Q : 1][Q > 0 ? T : 1];
  const int64_t n = a.row0 + blockIdx.x;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + n * a.grad_stride;
  const Segment<DT> g(row, a.M);
  Base base = {0.0f, 0.0f, 0.0f, 0.0f, a.inv_t, 0.0f};
  if (!any_entry(a, n)) {  // no loss, and a gradient of zero whatever the logits are
    if (threadIdx.x == 0) a.loss[n] = 0.0f;
    write_base<DT, 4, false, true>(g, out, T, base);
    return;
  }
  const int wave0 = (int)threadIdx.x - (int)(threadIdx.x & 63);  // what a wavefront has of a load is decided for all its lanes
  const auto load = [&](int chunk, u4_vec& w) {  // chunk: without the thread's own number
    if (wave0 + chunk < g.full) w = L::load_once(g.body + (uint32_t)min((int)threadIdx.x + chunk, g.full - 1) * L::V);
  };
  u4_vec w[R], end[1];
#pragma unroll
  for (int u = 0; u < R; ++u) load(u * T, w[u]);
  const bool last = g.rest + g.lead != 0 && (int)threadIdx.x == g.full % T;
  if (last) end[0] = g.partial();
  if (threadIdx.x < 64) {
    teacher_list(a, n, list);
    for (int j = threadIdx.x; j < a.k; j += 64) list.w[j] = list.col[j] >= 0 ? L::widen(row[list.col[j]]) : 0.0f;
  }
  Running mine = {kNegInf, 0.0f, 0.0f};
  const auto sum = [&](u4_vec(&four)[G], int u) {  // loads u ... u + G - 1
    float top[G], one[1];
    if (wave0 + 63 + (u + G - 1) * T < g.full) {
      absorb<DT, G, false, false>(four, a.c, mine, top);
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (wave0 + (u + i) * T < g.full) {
          u4_vec x[1] = {four[i]};
          if ((int)threadIdx.x + (u + i) * T >= g.full) x[0] = u4_vec{L::kLow, L::kLow, L::kLow, L::kLow};
          absorb<DT, 1, false, true>(x, a.c, mine, one);
        }
    }
  };
  const auto group = [&](int u) -> u4_vec(&)[G] { return reinterpret_cast<u4_vec(&)[G]>(w[u]); };
#pragma unroll
  for (int u = 0; u < Q; u += G) {
    sum(group(u), u);
#pragma unroll
    for (int i = u; i < u + G; ++i) {
      room[i][threadIdx.x] = w[i];
      load((R + i) * T, w[i]);
    }
  }
#pragma unroll
  for (int u = Q; u < R; u += G) sum(group(u), u);
#pragma unroll
  for (int u = 0; u < Q; u += G) sum(group(u), R + u);
  float top[1];
  if (last) absorb<DT, 1, false, true>(end, a.c, mine, top);
  const Stats t = segment_stats<DT, W, false>(g, mine, a.c, sums);
  if (W == 1) __syncthreads();
  base.m = t.m;
  base.less = logf(t.s);
  const float up = a.inv_t * a.grad[n];
  const bool empty = t.s == 0.0f, zero = empty || up * head.mass == 0.0f;
  base.alpha = zero ? 0.0f : up * head.mass;
  if (threadIdx.x < 64) {
    float loss = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += 64)
      if (list.col[j] >= 0) loss = __builtin_fmaf(expf(list.lp[j]), list.lp[j] - (empty ? kNegInf : (list.w[j] - t.m) * a.inv_t - base.less), loss);
    loss = wave_sum(loss);
    if (threadIdx.x == 0) a.loss[n] = loss;
  }
  if (zero) {
    write_base<DT, 4, false, true>(g, out, T, base);
  } else if (far_maximum(t.m, a.c)) {
    write_base<DT, 4, false, false>(g, out, T, base);
  } else {
    // alpha q = 2^(x c - r) (alpha / S about r): a fused multiply-add, an exp2 and a product to a logit
    const float r = reference(t.m, a.c), share = base.alpha / t.s * __builtin_amdgcn_exp2f(-__builtin_fmaf(t.m, a.c, -r));
    const auto turn = [&](const u4_vec& x) {
      float y[L::V];
#pragma unroll
      for (int c = 0; c < L::V; ++c) y[c] = __builtin_amdgcn_exp2f(__builtin_fmaf(L::at(x, c), a.c, -r)) * share;
      return L::pack(y);
    };
    auto* to = out + g.lead;
    const auto store = [&](int u, const u4_vec& x) {
      const int i = threadIdx.x + u * T;
      if (i < g.full) L::store(to + (uint32_t)i * L::V, turn(x));
    };
#pragma unroll
    for (int u = 0; u < R; ++u) store(u < Q ? R + u : u, w[u]);
#pragma unroll
    for (int u = 0; u < Q; ++u) store(u, room[u][threadIdx.x]);
    if (last) {
      const u4_vec y = turn(end[0]);
#pragma unroll
      for (int c = 0; c < L::V; ++c) {
        typename L::elem v;
        if constexpr (DT == kF32) v = __uint_as_float(y[c]);
        else v = (typename L::elem)(y[c / 2] >> (16 * (c & 1)));
        if (c < g.rest) to[(int64_t)g.full * L::V + c] = v;
        else if (DT != kF32 && c == L::V - 1 && g.lead != 0) to[-1] = v;
      }
    }
  }
  __syncthreads();
  if (empty) return;
  for (int j = threadIdx.x; j < a.k; j += T)
    write_entry<DT>(a, list, j, 0, a.M, out, -up, zero ? 0.0f : base.template at<false>(list.w[j]), [&](int i) { return expf(list.lp[i]); });
}

// The same for rows too wide to hold: the row is read twice, the second time from the caches if it is still there.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void distill_row_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  extern __shared__ float list_memory[];
  __shared__ ListHead head;
  ListRoom list(list_memory, a.k, head);
  __shared__ float4 sums[W];
  const int64_t n = a.row0 + blockIdx.x;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + n * a.grad_stride;
  const Segment<DT> g(row, a.M);
  if (threadIdx.x < 64) teacher_list(a, n, list);
  __syncthreads();
  Base base = {0.0f, 0.0f, 0.0f, 0.0f, a.inv_t, 0.0f};
  if (head.mass == 0.0f) {  // no entry counts: no loss, and a gradient of zero whatever the logits are
    if (threadIdx.x == 0) a.loss[n] = 0.0f;
    write_base<DT, 4, false, true>(g, out, T, base);
    return;
  }
  const Stats t = segment_stats<DT, W, false>(g, thread_stats<DT, T, 4, false, true>(g, a.c), a.c, sums);
  base.m = t.m;
  base.less = logf(t.s);
  if (threadIdx.x < 64) {
    const float loss = list_loss<DT>(a, row, t, base.less, list);
    if (threadIdx.x == 0) a.loss[n] = loss;
  }
  __syncthreads();  // the first wavefront has read the logits that the loss needs: a gradient of zero may take their place at once
  const float up = a.inv_t * a.grad[n];
  base.alpha = up * head.mass;
  const bool empty = t.s == 0.0f;
  write_gradient<DT, T, false>(a, list, g, 0, a.M, out, base, empty ? 0.0f : -up, empty || base.alpha == 0.0f);
}

}  // namespace rtopk
