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
  static constexpr int B = DT == kF32 ? 4 : 2;  // bytes of one
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

// A whole number in the order of the logits; -0 and +0 are equal, NaN is above all; 0 stands for no logit.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}
// The same with the column: larger for the lower one.
__device__ __forceinline__ uint64_t place_key(uint32_t key, int col) { return (uint64_t)key << 32 | (uint32_t)~col; }
__device__ __forceinline__ int place_col(uint64_t key) { return (int)~(uint32_t)key; }

// ---- sums -----------------------------------------------------------------------------------------

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

struct Stats {
  float m, s, a;  // maximum, S and A about it (0 where the maximum is -inf)
  __device__ __forceinline__ float about() const { return m == kNegInf ? 0.0f : m; }
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

template <bool ENT>
__device__ __forceinline__ Stats wave_join(Stats t, float c) {
  scale_to<ENT>(t, wave_max(t.m), c);
  t.s = wave_sum(t.s);
  if (ENT) t.a = wave_sum(t.a);
  return t;
}

// All W wavefronts' sums, in every thread.  `room`: W entries; a barrier lies between its writes and reads.
template <int W, bool ENT>
__device__ __forceinline__ Stats block_join(Stats t, float c, float4* room) {
  t = wave_join<ENT>(t, c);
  if (W == 1) return t;
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = make_float4(t.m, t.s, t.a, 0.0f);
  __syncthreads();
  float m = room[0].x;
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, room[w].x);
  Stats all = {m, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < W; ++w) {
    Stats u = {room[w].x, room[w].y, room[w].z};
    scale_to<ENT>(u, m, c);
    all.s += u.s;
    all.a += u.a;
  }
  return all;
}

// Takes U loads into a thread's sums.
template <int DT, int U, bool ENT>
__device__ __forceinline__ void absorb(const u4_vec (&w)[U], float c, Stats& t) {
  using L = Logits<DT>;
  float x[U * L::V];
#pragma unroll
  for (int i = 0; i < U * L::V; ++i) x[i] = L::at(w[i / L::V], i % L::V);
  float m = t.m;
#pragma unroll
  for (int i = 0; i < U * L::V; i += 2) m = vmax3(m, x[i], x[i + 1]);
  scale_to<ENT>(t, m, c);
  const float about = t.about();
  float s[2] = {t.s, 0.0f}, a[2] = {t.a, 0.0f};
#pragma unroll
  for (int i = 0; i < U * L::V; ++i) {
    const float d = x[i] - about, e = __builtin_amdgcn_exp2f(d * c);
    s[i & 1] += e;
    if (ENT) a[i & 1] = __builtin_fmaf(e, fmaxf(d, kFar), a[i & 1]);
  }
  t.s = s[0] + s[1];
  t.a = a[0] + a[1];
}

// ---- a thread's share of a segment ----------------------------------------------------------------

// `cols` columns from `row` on, in chunks of a load's width; chunk i belongs to thread i mod T, the last one may be partial.
template <int DT>
struct Segment {
  using L = Logits<DT>;
  const typename L::elem* row;
  int full, rest;  // whole chunks, columns beyond them
  __device__ __forceinline__ Segment(const typename L::elem* r, int cols) : row(r), full(cols / L::V), rest(cols % L::V) {}
  __device__ __forceinline__ int chunks() const { return full + (rest != 0); }
  // chunk `i` (i < chunks()), -inf past the end
  __device__ __forceinline__ u4_vec partial() const {
    u4_vec w = {L::kLow, L::kLow, L::kLow, L::kLow};
    const typename L::elem* p = row + (int64_t)full * L::V;
#pragma unroll
    for (int c = 0; c < L::V - 1; ++c)
      if (c < rest) {
        if constexpr (DT == kF32) w[c] = __float_as_uint(p[c]);
        else w[c / 2] = (c & 1) ? (w[c / 2] & 0xffffu) | (uint32_t)p[c] << 16 : (w[c / 2] & 0xffff0000u) | p[c];
      }
    return w;
  }
  // f(columns from the segment's start, value) for each column of chunk i
  template <typename F>
  __device__ __forceinline__ void each(int i, F f) const {
    const int width = i < full ? L::V : rest;
    const u4_vec w = i < full ? L::load(row + (uint32_t)i * L::V) : partial();
#pragma unroll
    for (int c = 0; c < L::V; ++c)
      if (c < width) f(i * L::V + c, L::at(w, c));
  }
};

// S, A and the maximum of the thread's chunks.  KEEP: the row is read again by this workgroup.
template <int DT, int U, bool ENT, bool KEEP>
__device__ __forceinline__ Stats thread_stats(const Segment<DT>& g, int T, float c) {
  using L = Logits<DT>;
  Stats t = {kNegInf, 0.0f, 0.0f};
  int i = threadIdx.x;
  for (; i + (U - 1) * T < g.full; i += U * T) {
    u4_vec w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const auto* p = g.row + (uint32_t)(i + u * T) * L::V;
      w[u] = KEEP ? L::load(p) : L::load_once(p);
    }
    absorb<DT, U, ENT>(w, c, t);
  }
  if (i < g.full) {  // chunks past the last are -inf: they add nothing
    u4_vec w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = L::load(g.row + (uint32_t)min(i + u * T, g.full - 1) * L::V);
#pragma unroll
    for (int u = 1; u < U; ++u)
      if (i + u * T >= g.full) w[u] = u4_vec{L::kLow, L::kLow, L::kLow, L::kLow};
    absorb<DT, U, ENT>(w, c, t);
  }
  if (g.rest != 0 && (int)threadIdx.x == g.full % T) {
    const u4_vec w[1] = {g.partial()};
    absorb<DT, 1, ENT>(w, c, t);
  }
  return t;
}

// ---- top alternatives -----------------------------------------------------------------------------

// The k largest of a row's columns, by value and then by column.  Every thread knows the largest logit it has seen; the k-th largest of
// these is a floor under the k-th largest of the row, and only threads whose maximum reaches the floor can hold columns that do: about k
// threads' columns are read again, and what reaches the floor, a little over k columns, is ranked by comparing each with each.
// The floor is found as the top-k selections find theirs, by bisection on a threshold with early stopping: it need not be the k-th exactly.
constexpr int kMaxCandidates = 1024;

template <int T>
struct TopRoom {
  uint64_t found[kMaxCandidates];
  uint64_t best[kMaxAlternatives];
  uint32_t key[T];
  uint16_t holder[T];
  uint32_t floor;
  int holders, count;
};

// A floor that at least k of the T keys reach, or 1 where fewer than k are not 0; the first wavefront's work.  Few more than k reach it
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
  if (have <= k) return 1;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
  }
  uint64_t a = __builtin_amdgcn_readfirstlane(lo), b = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(hi) + 1;
  const int enough = k + max(8, k / 2);
  while (b - a > 1) {  // a is reached by k keys, b by fewer
    const uint32_t mid = (uint32_t)(a + (b - a) / 2);
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
  return (uint32_t)a;
}

// Ranks room.count (at most kMaxCandidates) distinct keys: the k largest in order in room.best, 0 where there are fewer.
template <int T>
__device__ __forceinline__ void rank_found(TopRoom<T>& room, int k) {
  const int n = room.count;
  for (int j = n + threadIdx.x; j < k; j += T) room.best[j] = 0;
  for (int j = threadIdx.x; j < n; j += T) {
    const uint64_t key = room.found[j];
    int rank = 0;
    for (int i = 0; i < n; ++i) rank += room.found[i] > key;
    if (rank < k) room.best[rank] = key;
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

// The k largest of the segment in room.best, best first (0 where it has fewer columns); first: the segment's first column.
// `mine`: the thread's maximum, or whatever (`any` false) where it has no column.
template <int DT, int T>
__device__ void segment_top(const Segment<DT>& g, int first, int k, float mine, bool any, TopRoom<T>& room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t key = any ? order_key(mine) : 0;
  room.key[threadIdx.x] = key;
  if (threadIdx.x == 0) {
    room.holders = 0;
    room.count = 0;
  }
  __syncthreads();
  if (wave == 0) {
    const uint32_t f = find_floor<T>(room.key, k);
    if (lane == 0) room.floor = f;
  }
  __syncthreads();
  uint32_t least = room.floor;
  if (any && key >= least) room.holder[atomicAdd(&room.holders, 1)] = (uint16_t)threadIdx.x;
  __syncthreads();
  const int holders = room.holders, chunks = g.chunks();
  for (int h = wave; h < holders; h += T / 64)
    for (int64_t i = room.holder[h] + (int64_t)lane * T; i < chunks; i += 64 * T)
      g.each((int)i, [&](int col, float v) {
        const uint32_t o = order_key(v);
        if (o >= least) {
          const int at = atomicAdd(&room.count, 1);
          if (at < kMaxCandidates) room.found[at] = place_key(o, first + col);
        }
      });
  __syncthreads();
  if (room.count > kMaxCandidates) {
    // Equal logits in crowds, or the largest ones in few threads' columns: bisection over the whole segment, until so few columns reach the
    // threshold that they can be listed, or none lies between the bounds.  least is reached by k columns.
    __syncthreads();  // (all have read the count)
    uint64_t a = least, b = (uint64_t)1 << 32;
    int reach = g.full * Logits<DT>::V + g.rest, above = 0;
    bool next = true;  // the first threshold is the one above `least`: all others are equal where a mask has left few columns
    while (b - a > 1 && reach > kMaxCandidates) {
      const uint32_t mid = next ? (uint32_t)(a + 1) : (uint32_t)(a + (b - a) / 2);
      next = false;
      const int n = count_reaching<DT, T>(g, mid, &room.holders);
      if (n >= k) {
        a = mid;
        reach = n;
      } else {
        b = mid;
        above = n;
      }
    }
    least = (uint32_t)a;
    const uint32_t listed = reach > kMaxCandidates ? least + 1 : least;  // (least is then below the largest key of all)
    if (threadIdx.x == 0) room.count = 0;
    __syncthreads();
    if (reach <= kMaxCandidates || above > 0)
      for (int i = threadIdx.x; i < chunks; i += T)
        g.each(i, [&](int col, float v) {
          const uint32_t o = order_key(v);
          if (o >= listed) {
            const int at = atomicAdd(&room.count, 1);
            if (at < kMaxCandidates) room.found[at] = place_key(o, first + col);
          }
        });
    __syncthreads();
    if (reach > kMaxCandidates && wave == 0) {  // fewer than k lie above `least`: the first columns that equal it fill up
      int n = room.count;
      for (int i = lane; n < k && i - lane < chunks; i += 64) {
        int mine_n = 0;
        if (i < chunks) g.each(i, [&](int, float v) { mine_n += order_key(v) == least; });
        int before = mine_n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int o = __shfl_up(before, d);
          if (lane >= d) before += o;
        }
        const int all = __shfl(before, 63);
        before += n - mine_n;
        if (mine_n > 0 && before < k)
          g.each(i, [&](int col, float v) {
            if (order_key(v) == least) {
              if (before < k) room.found[before] = place_key(least, first + col);
              ++before;
            }
          });
        n += all;
      }
      if (lane == 0) room.count = min(n, k);
    }
    __syncthreads();
  }
  rank_found<T>(room, k);
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

struct ListRoom {
  int col[kMaxList];
  float w[kMaxList];   // the teacher's probability, or the gradient that belongs to a token
  float lp[kMaxList];  // logarithm of the former
  float mass;          // sum of w
  int ascending;       // columns in strictly ascending order, so none twice
};

// The first wavefront writes the row's list to LDS; entries that do not count have column -1 and weight 0.
__device__ __forceinline__ void teacher_list(const LogitsArgs& a, int64_t n, ListRoom& r) {
  const int lane = threadIdx.x;
  const float c = a.inv_t * kLog2e;
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
    r.mass = mass;
    r.ascending = all;
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
    r.mass = mass;
    r.ascending = a.k == 1;
  }
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
    if (a.lse) a.lse[n] = empty ? kNegInf : __builtin_fmaf(t.m, a.inv_t, ln_s);
    if (a.entropy) a.entropy[n] = empty ? 0.0f : ln_s - t.a / t.s * a.inv_t;
  }
}

template <int T>
__device__ __forceinline__ void write_top(const LogitsArgs& a, int64_t n, const Stats& t, float ln_s, const TopRoom<T>& room) {
  for (int j = threadIdx.x; j < a.k; j += T) {
    const uint64_t key = room.best[j];
    a.top_logprobs[n * a.k + j] = t.s == 0.0f ? kNegInf : (order_value((uint32_t)(key >> 32)) - t.m) * a.inv_t - ln_s;
    a.top_cols[n * a.k + j] = place_col(key);
  }
}

// One workgroup reads a segment of a row.  SPLIT: its sums and alternatives go to scratch memory for logits_join_kernel; else the segment is the
// row and the results are written.
template <int DT, int W, int OP, bool TOP, bool SPLIT>
__global__ __launch_bounds__(64 * W) void logits_rows_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  constexpr bool ENT = OP == kOpTokens;
  __shared__ float4 sums[W];
  const int seg = SPLIT ? (int)(blockIdx.x % (uint32_t)a.segments) : 0;
  const int64_t n = a.row0 + (SPLIT ? blockIdx.x / (uint32_t)a.segments : blockIdx.x);
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  const int first = seg * a.seg_cols;
  const Segment<DT> g(row + first, min(a.seg_cols, a.M - first));
  const float c = a.inv_t * kLog2e;
  __shared__ typename std::conditional<OP == kOpDistill && !SPLIT, ListRoom, int>::type list;
  if constexpr (OP == kOpDistill && !SPLIT) {
    if (threadIdx.x < 64) teacher_list(a, n, list);
  }
  const Stats mine = thread_stats<DT, 4, ENT, TOP>(g, T, c);
  const Stats t = block_join<W, ENT>(mine, c, sums);
  if constexpr (TOP) {
    __shared__ TopRoom<T> room;
    segment_top<DT, T>(g, first, a.k, mine.m, (int)threadIdx.x < g.chunks(), room);
    if constexpr (SPLIT) {
      uint64_t* keys = a.part_keys + (n * a.segments + seg) * a.k;
      for (int j = threadIdx.x; j < a.k; j += T) keys[j] = room.best[j];
    } else {
      write_top<T>(a, n, t, logf(t.s), room);
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
      if (a.lse) a.lse[n] = t.s == 0.0f ? kNegInf : __builtin_fmaf(t.m, a.inv_t, ln_s);
    }
  }
}

// Sums of a row's segments, in every thread of a workgroup of W wavefronts.
template <int W, bool ENT>
__device__ __forceinline__ Stats join_segments(const LogitsArgs& a, int64_t n, float c, float4* room) {
  Stats t = {kNegInf, 0.0f, 0.0f};
  for (int s = threadIdx.x; s < a.segments; s += 64 * W) {
    const float4 p = a.part[n * a.segments + s];
    Stats u = {p.x, p.y, p.z};
    const float m = fmaxf(t.m, u.m);
    scale_to<ENT>(t, m, c);
    scale_to<ENT>(u, m, c);
    t.s += u.s;
    t.a += u.a;
  }
  return block_join<W, ENT>(t, c, room);
}

template <int DT, int OP, bool TOP>
__global__ __launch_bounds__(256) void logits_join_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 256;
  __shared__ float4 sums[4];
  const int64_t n = a.row0 + blockIdx.x;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  __shared__ typename std::conditional<OP == kOpDistill, ListRoom, int>::type list;
  if constexpr (OP == kOpDistill) {
    if (threadIdx.x < 64) teacher_list(a, n, list);
  }
  const Stats t = join_segments<4, OP == kOpTokens>(a, n, a.inv_t * kLog2e, sums);
  const float ln_s = logf(t.s);
  if constexpr (TOP) {
    // the segments' alternatives, merged as a segment's columns are: each thread's largest, a floor, what reaches it
    __shared__ TopRoom<T> room;
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
    room.key[threadIdx.x] = top;
    if (threadIdx.x == 0) room.count = 0;
    __syncthreads();
    if (threadIdx.x < 64) {
      const uint32_t f = find_floor<T>(room.key, a.k);
      if (threadIdx.x == 0) room.floor = f;
    }
    __syncthreads();
    uint64_t least = (uint64_t)room.floor << 32;
    int n_reach = 0;
#pragma unroll
    for (int p = 0; p < P; ++p) n_reach += v[p] >= least;
    if (n_reach > 0) atomicAdd(&room.count, n_reach);
    __syncthreads();
    int reach = room.count;
    __syncthreads();
    // more than there is room for: bisection on the whole keys, which are distinct
    uint64_t b = ~(uint64_t)0;
    while (reach > kMaxCandidates) {
      const uint64_t mid = least + (b - least) / 2;
      if (threadIdx.x == 0) room.count = 0;
      __syncthreads();
      n_reach = 0;
#pragma unroll
      for (int p = 0; p < P; ++p) n_reach += v[p] >= mid;
      if (n_reach > 0) atomicAdd(&room.count, n_reach);
      __syncthreads();
      const int got = room.count;
      __syncthreads();
      if (got >= a.k) {
        least = mid;
        reach = got;
      } else {
        b = mid;
      }
    }
    if (threadIdx.x == 0) room.count = 0;
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (v[p] >= least) room.found[atomicAdd(&room.count, 1)] = v[p];
    __syncthreads();
    rank_found<T>(room, a.k);
    write_top<T>(a, n, t, ln_s, room);
  }
  if constexpr (OP == kOpTokens) {
    write_tokens<DT>(a, n, row, t, ln_s, T);
  } else if (threadIdx.x < 64) {
    const float loss = list_loss<DT>(a, row, t, ln_s, list);
    if (threadIdx.x == 0) {
      a.loss[n] = loss;
      if (a.lse) a.lse[n] = t.s == 0.0f ? kNegInf : __builtin_fmaf(t.m, a.inv_t, ln_s);
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
    return ENT ? q * (alpha - beta * (lq + h)) : alpha * q;
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
  for (; i + (U - 1) * T < g.full; i += U * T) {
    u4_vec w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = ZERO ? none : L::load_once(g.row + (uint32_t)(i + u * T) * L::V);
#pragma unroll
    for (int u = 0; u < U; ++u) L::store(out + (uint32_t)(i + u * T) * L::V, ZERO ? none : turn(w[u]));
  }
  for (; i < g.full; i += T) L::store(out + (uint32_t)i * L::V, ZERO ? none : turn(L::load_once(g.row + (uint32_t)i * L::V)));
  if ((int)threadIdx.x < g.rest) {
    const uint32_t at = (uint32_t)g.full * L::V + threadIdx.x;
    out[at] = ZERO ? L::narrow(0.0f) : L::narrow(base.template at<ENT>(L::widen(g.row[at])));
  }
}

// The columns of the list that lie in the segment, after the base has been written (a barrier lies between): one value, rounded once, from
// the thread of the column's first entry.  `x`: the logits at the thread's entries, read before the base was written (the gradient may lie
// in the logits' place).  sign * r.w: what an entry adds.
template <int DT, int T, bool ENT, bool ZERO>
__device__ __forceinline__ void write_list(const LogitsArgs& a, const ListRoom& r, int first, int cols, typename Logits<DT>::elem* out,
                                           const Base& base, float factor, const float (&x)[(kMaxList + T - 1) / T]) {
#pragma unroll
  for (int e = 0; e < (kMaxList + T - 1) / T; ++e) {
    const int j = threadIdx.x + e * T;
    if (j >= a.k) break;
    const int col = r.col[j];
    if (col < first || col >= first + cols) continue;
    float w = r.w[j];
    bool again = false;
    if (!r.ascending)
      for (int i = 0; i < a.k; ++i)
        if (i != j && r.col[i] == col) {
          if (i < j) again = true;
          w += r.w[i];
        }
    if (again) continue;
    const float y = ZERO ? 0.0f : base.template at<ENT>(x[e]);
    out[col - first] = Logits<DT>::narrow(__builtin_fmaf(factor, w, y));
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
  read_list<DT, T>(a, r, first, cols, g.row, x);
  __syncthreads();
  write_base<DT, 4, ENT, false>(g, out, T, base);
  __syncthreads();
  write_list<DT, T, ENT, false>(a, r, first, cols, out, base, factor, x);
}

// A segment of a row's gradient by one workgroup.  The row's sums are known: its log-sum-exp was saved (JOIN false), or the segments' sums
// lie in scratch memory (JOIN, distillation only), and then the loss is written too.
template <int DT, int OP, bool ENT, bool JOIN>
__global__ __launch_bounds__(256) void logits_grad_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 256;
  __shared__ ListRoom list;
  __shared__ float4 sums[4];
  const int seg = (int)(blockIdx.x % (uint32_t)a.segments);
  const int64_t n = a.row0 + blockIdx.x / (uint32_t)a.segments;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + n * a.grad_stride;
  const int first = seg * a.seg_cols, cols = min(a.seg_cols, a.M - first);
  const Segment<DT> g(row + first, cols);
  if (threadIdx.x < 64) {
    if (OP == kOpTokens) token_list(a, n, list);
    else teacher_list(a, n, list);
  }
  Base base;
  base.inv_t = a.inv_t;
  bool empty;
  if constexpr (JOIN) {
    const Stats t = join_segments<4, false>(a, n, a.inv_t * kLog2e, sums);
    base.m = t.m;
    base.less = logf(t.s);
    empty = t.s == 0.0f;
    if (a.loss && seg == 0 && threadIdx.x < 64) {
      const float loss = list_loss<DT>(a, row, t, base.less, list);
      if (threadIdx.x == 0) a.loss[n] = loss;
    }
  } else {
    base.m = 0.0f;
    base.less = a.lse_in[n];
    empty = base.less == kNegInf;
    __syncthreads();
    if (fabsf(base.less) > kLargeLse && fabsf(base.less) < __builtin_inff()) {
      const Stats t = block_join<4, false>(thread_stats<DT, 4, false, true>(Segment<DT>(row, a.M), T, a.inv_t * kLog2e), a.inv_t * kLog2e, sums);
      base.m = t.m;
      base.less = logf(t.s);
    }
  }
  const float up = OP == kOpTokens ? a.inv_t : a.inv_t * a.grad[n];
  base.alpha = OP == kOpTokens ? -up * list.mass : up * list.mass;
  base.beta = ENT ? a.inv_t * a.grad_entropy[n] : 0.0f;
  base.h = ENT ? a.entropy_in[n] : 0.0f;
  const bool zero = empty || (base.alpha == 0.0f && base.beta == 0.0f);
  write_gradient<DT, T, ENT>(a, list, g, first, cols, out + first, base, empty ? 0.0f : (OP == kOpTokens ? up : -up), zero);
}

// Loss and gradient of a row by one workgroup: the row is read twice, the second time from the caches.
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void distill_row_kernel(LogitsArgs a) {
  using L = Logits<DT>;
  constexpr int T = 64 * W;
  __shared__ ListRoom list;
  __shared__ float4 sums[W];
  const int64_t n = a.row0 + blockIdx.x;
  const auto* row = static_cast<const typename L::elem*>(a.x) + n * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + n * a.grad_stride;
  const Segment<DT> g(row, a.M);
  if (threadIdx.x < 64) teacher_list(a, n, list);
  __syncthreads();
  Base base = {0.0f, 0.0f, 0.0f, 0.0f, a.inv_t, 0.0f};
  if (list.mass == 0.0f) {  // no entry counts: no loss, and a gradient of zero whatever the logits are
    if (threadIdx.x == 0) a.loss[n] = 0.0f;
    write_base<DT, 4, false, true>(g, out, T, base);
    return;
  }
  const Stats t = block_join<W, false>(thread_stats<DT, 4, false, true>(g, T, a.inv_t * kLog2e), a.inv_t * kLog2e, sums);
  base.m = t.m;
  base.less = logf(t.s);
  if (threadIdx.x < 64) {
    const float loss = list_loss<DT>(a, row, t, base.less, list);
    if (threadIdx.x == 0) a.loss[n] = loss;
  }
  const float up = a.inv_t * a.grad[n];
  base.alpha = up * list.mass;
  const bool empty = t.s == 0.0f;
  write_gradient<DT, T, false>(a, list, g, 0, a.M, out, base, empty ? 0.0f : -up, empty || base.alpha == 0.0f);
}

}  // namespace rtopk
