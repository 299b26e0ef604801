// A router's balance loss and its gradient for gfx950 (MI355X).
//
// Tokens come in groups; token t of a group has E logits x_t and the columns that a selection picked for it, and counts if any of them lies in [0, E).
// With p_t = softmax(x_t), n the group's tokens that count, f_e the share of all picks that expert e got, P_e = (1 / n) sum_t p_te:
//   loss = E sum_e f_e P_e  (1 where either is even),   z = (1 / n) sum_t lse_t^2
// and, f held constant (it is piecewise so), with w_e = E f_e g_loss / n:
//   dx_te = p_te (w_e - sum_j p_tj w_j + 2 g_z lse_t / n) + the gradients of the token's picked values at their columns
//
// A token's row lies in a few lanes, 64 / lanes tokens to a wavefront, and is read once; maxima and sums go over those lanes.  Forward, a lane keeps the sums of
// its columns' probabilities over the tokens it sees, in fp32 for kFlush turns and in 64 bits over lanes and (LDS) over these; picks are counted by integer atomics
// in LDS, whose order changes nothing.  Workgroups leave their sums in scratch memory and a second kernel joins them in order.
//
// Bound by HBM and the vector ALU alike: 262144 x 256 bfloat16 28 to 29 us (5.0 TB/s, ALU 84 % busy) and 4.6 for the join; gradient 1048576 x 128 bfloat16 with picked
// values 109 us (603 MB, 5.5 TB/s, ALU 62 %).  Four tokens' loads in flight and moved columns out of the loads' way took the gradient from 315 us to
// 136, sums of lanes by one instruction a step to 117, two loads to a lane to 108.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_balance_dispatch.hpp"
#include "rtopk_logits.hpp"

namespace rtopk {

constexpr int kFlush = 64;  // tokens of a lane that fp32 sums run over
constexpr float kFarMaximum = 1024.0f;  // log2(e) times a maximum beyond this is too coarse a reference: differences from the maximum are taken first

// Over each N lanes (a power of two), the same in all of them: within 16 lanes by DPP permutations that are part of the maximum or sum, then by swaps of rows.
// (The maximum in assembly: a C++ one first quiets what might be a signalling NaN.)
template <int N>
__device__ __forceinline__ float lanes_max(float v) {
  if constexpr (N >= 2) asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf" : "+v"(v));
  if constexpr (N >= 4) asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf" : "+v"(v));
  if constexpr (N >= 8) asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf" : "+v"(v));
  if constexpr (N >= 16) asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_mirror row_mask:0xf bank_mask:0xf" : "+v"(v));
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (N >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  const auto dpp = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
  if constexpr (N >= 2) v += dpp(std::integral_constant<int, 0xb1>{});   // quad_perm [1, 0, 3, 2]
  if constexpr (N >= 4) v += dpp(std::integral_constant<int, 0x4e>{});   // quad_perm [2, 3, 0, 1]
  if constexpr (N >= 8) v += dpp(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (N >= 16) v += dpp(std::integral_constant<int, 0x140>{}); // row_mirror
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (N >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Sums in 64 bits of each lane's C values, over the lanes that have the same place among their N.  Each swap of rows leaves a lane half of the sums: it has those of
// kHeld values from number `first` on, and of the lanes with the same ones the first N of 16 write them.  (All sums in all lanes instead: 500000 x 100 bfloat16
// 39.9 us against 37.8, 1048576 x 4 20.4 against 19.4.)
template <int N, int C>
struct PlacesSums {
  static constexpr int kHeld = N >= 64 ? C : (N == 32 ? C / 2 : C / 4);
  double s[C];
  int first;
  bool writes;
  template <int LOADS, int V>
  __device__ __forceinline__ explicit PlacesSums(const float (&p)[LOADS][V]) {
    const int lane = threadIdx.x & 63;
    first = (N <= 32 ? lane / 32 * (C / 2) : 0) + (N <= 16 ? lane / 16 % 2 * (C / 4) : 0);
    writes = N >= 16 || lane % 16 < N;
    if constexpr (N >= 64) {
#pragma unroll
      for (int k = 0; k < C; ++k) s[k] = p[k / V][k % V];
    } else {
#pragma unroll
      for (int k = 0; k < C / 2; ++k) {
        const int j = k + C / 2;
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(p[k / V][k % V]), __float_as_uint(p[j / V][j % V]), false, false);
        s[k] = (double)__uint_as_float(r[0]) + (double)__uint_as_float(r[1]);
      }
    }
    if constexpr (N <= 16) {
#pragma unroll
      for (int k = 0; k < C / 4; ++k) {
        const uint64_t u = (uint64_t)__double_as_longlong(s[k]), v = (uint64_t)__double_as_longlong(s[k + C / 4]);
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)v, false, false), hi = __builtin_amdgcn_permlane16_swap(u >> 32, v >> 32, false, false);
        s[k] = __longlong_as_double((long long)((uint64_t)hi[0] << 32 | lo[0])) + __longlong_as_double((long long)((uint64_t)hi[1] << 32 | lo[1]));
      }
    }
    const auto add_turned = [&](auto by) {  // row_ror
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        const uint64_t b = (uint64_t)__double_as_longlong(s[k]);
        const uint32_t lo = __builtin_amdgcn_mov_dpp((int)b, 0x120 + decltype(by)::value, 0xf, 0xf, true);
        const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(b >> 32), 0x120 + decltype(by)::value, 0xf, 0xf, true);
        s[k] += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
      }
    };
    if constexpr (N <= 8) add_turned(std::integral_constant<int, 8>{});
    if constexpr (N <= 4) add_turned(std::integral_constant<int, 4>{});
    if constexpr (N <= 2) add_turned(std::integral_constant<int, 2>{});
    if constexpr (N <= 1) add_turned(std::integral_constant<int, 1>{});
  }
};

// The columns of a token's row that a lane has: chunk i of the lane is chunk `sub + i N` of the row.  RAGGED: the row is no whole number of chunks; its last chunk is
// moved back to end with it, and what that shares with the chunk before is held twice and counts once (`keep`).  Rows narrower than a chunk are loaded
// by the element.
template <int DT, int N, int LOADS, bool RAGGED>
struct RouterLane {
  using L = Logits<DT>;
  using elem = typename L::elem;
  static constexpr int V = L::V;
  int at[LOADS];  // first column of the chunk
  bool has[LOADS];
  float keep[LOADS][V];
  static __device__ __forceinline__ int first_of(int E, int c0) { return RAGGED ? (E < V ? 0 : min(c0, E - V)) : c0; }
  __device__ __forceinline__ RouterLane(int E, int sub) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c0 = (sub + i * N) * V;
      has[i] = c0 < E;
      at[i] = first_of(E, c0);
#pragma unroll
      for (int c = 0; c < V; ++c) keep[i][c] = !RAGGED || (has[i] && at[i] + c >= c0 && at[i] + c < E) ? 1.0f : 0.0f;
    }
  }
  // -inf where the lane has nothing, or there is no such token
  __device__ __forceinline__ void load(const elem* row, int E, bool is, u4_vec (&w)[LOADS]) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) w[i] = u4_vec{L::kLow, L::kLow, L::kLow, L::kLow};
    if (!RAGGED || E >= V) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        if (is && has[i]) w[i] = L::load_once(row + at[i]);
    } else {
      typename L::elem v[V];
      if (is && has[0]) {
#pragma unroll
        for (int c = 0; c < V; ++c) v[c] = row[c < E ? c : 0];
#pragma unroll
        for (int c = 0; c < V; ++c) {
          if constexpr (DT == kF32) w[0][c] = c < E ? __float_as_uint(v[c]) : L::kLow;
          else if ((c & 1) == 0) w[0][c / 2] = c < E ? v[c] : L::kLow & 0xffffu;
          else w[0][c / 2] |= (c < E ? (uint32_t)v[c] : L::kLow & 0xffffu) << 16;
        }
      }
    }
  }
  static __device__ __forceinline__ void leave_out(bool is, u4_vec (&w)[LOADS]) {  // (padding may hold NaN)
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int h = 0; h < 4; ++h) w[i][h] = is ? L::kLow : w[i][h];
  }
  __device__ __forceinline__ float kept(float v, int i, int c) const { return RAGGED ? v * keep[i][c] : v; }
};

// A row's powers about its maximum in the lane's columns, and their sum.  One fused multiply-add and one exp2 to a logit: the rounding of the reference
// m log2(e) is in all powers alike, and in the log-sum-exp that is formed about it.
template <int DT, int N, int LOADS, bool RAGGED>
struct RouterRow {
  using R = RouterLane<DT, N, LOADS, RAGGED>;
  using L = Logits<DT>;
  static constexpr int V = L::V;
  float e[LOADS][V], m, s;
  __device__ __forceinline__ RouterRow(const R& r, u4_vec (&w)[LOADS]) {
    m = L::largest(w[0]);
#pragma unroll
    for (int i = 1; i < LOADS; ++i) m = vmax(m, L::largest(w[i]));
    m = lanes_max<N>(m);
    if (m == kNegInf) m = 0.0f;
    const float about = m * kLog2e;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) e[i][c] = __builtin_amdgcn_exp2f(__builtin_fmaf(L::at(w[i], c), kLog2e, -about));
    if (__any(fabsf(m) > kFarMaximum)) {
      apart(w);
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int c = 0; c < V; ++c)
          if (fabsf(m) > kFarMaximum) e[i][c] = __builtin_amdgcn_exp2f((L::at(w[i], c) - m) * kLog2e);
    }
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if (RAGGED) s = __builtin_fmaf(e[i][c], r.keep[i][c], s);
        else s += e[i][c];
      }
    s = lanes_sum<N>(s);
  }
};

// 1 / s of a sum of powers about the maximum (1 <= s <= kMaxExperts, or 0, or NaN), and the log-sum-exp, 0 for a row of nothing but -inf.
__device__ __forceinline__ float over_of(float s) { return s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(s); }
__device__ __forceinline__ float lse_of(float m, float s) {
  constexpr float kLn2 = 0.69314718055994530942f;
  const float log2_s = __builtin_amdgcn_logf(s), v = fabsf(m) > kFarMaximum ? __builtin_fmaf(log2_s, kLn2, m) : (m * kLog2e + log2_s) * kLn2;
  return s == 0.0f ? 0.0f : v;
}

// A column as it is stored, and whether it is a pick: looked at apart, so that a load is not waited for before the next one.
__device__ __forceinline__ int stored_col(const BalanceArgs& a, const char* p) {
  return a.col_bytes == 1 ? (int)*reinterpret_cast<const uint8_t*>(p) : *reinterpret_cast<const int32_t*>(p);
}
__device__ __forceinline__ int pick_of(const BalanceArgs& a, int col) { return (uint32_t)col < (uint32_t)a.E ? col : -1; }  // -1: none
__device__ __forceinline__ int pick_from(const BalanceArgs& a, const char* p) { return pick_of(a, stored_col(a, p)); }

// Whether a token of the lane's row has any pick: `any` of its N lanes, given their ballot.
template <int N>
__device__ __forceinline__ bool any_lane(uint64_t ballot, int of) {
  const uint64_t mask = N == 64 ? ~(uint64_t)0 : ((uint64_t)1 << (N % 64)) - 1;
  return ((ballot >> (of * N)) & mask) != 0;
}
// The ballot of a wavefront whose tokens all have k picks in their first k lanes.
template <int N>
__device__ __forceinline__ uint64_t full_ballot(int k) {
  const uint64_t row = k >= N ? (N == 64 ? ~(uint64_t)0 : ((uint64_t)1 << (N % 64)) - 1) : ((uint64_t)1 << k) - 1;
  uint64_t all = 0;
#pragma unroll
  for (int i = 0; i < 64; i += N) all |= row << i;
  return all;
}

// A batch's loads are waited for once, here: a wait further on would also be one for the stores that have been made since.
template <int U, int LOADS>
__device__ __forceinline__ void arrived(u4_vec (&w)[U][LOADS], int (&col)[U]) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    apart(w[u]);
    asm volatile("" : "+v"(col[u]));
  }
}

// To nearest even, two values by one instruction where there is one.
template <int DT>
__device__ __forceinline__ u4_vec pack_rounded(const float (&v)[Logits<DT>::V]) {
  if constexpr (DT == kBF16) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    u4_vec w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{v[2 * i], v[2 * i + 1]}), b2));
    return w;
  } else {
    return Logits<DT>::pack(v);
  }
}

// Loads of a lane that are made together.
constexpr int balance_batch(int loads) { return loads == 1 ? 4 : (loads == 2 ? 2 : 1); }

__device__ __forceinline__ double lanes_total(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

// ---- loss -----------------------------------------------------------------------------------------

// A column's results; returns what it adds to the group's loss before the factors.
__device__ __forceinline__ double write_column(const BalanceArgs& a, int g, int e, double sum, int picks, int counted) {
  const double mean = counted > 0 ? sum / counted : 0.0;
  if (a.probs) a.probs[(int64_t)g * a.E + e] = (float)mean;
  a.counts[(int64_t)g * a.E + e] = picks;
  return picks > 0 ? mean * picks : 0.0;  // (what was never picked adds nothing, whatever it is)
}

__device__ __forceinline__ void write_group(const BalanceArgs& a, int g, double dot, double z, int counted, int picked) {
  a.loss[g] = picked > 0 ? (float)(a.E * dot / picked) : 0.0f;
  if (a.z) a.z[g] = counted > 0 ? (float)(z / counted) : 0.0f;
  a.counted[g] = counted;
}

template <int DT, int N, int LOADS, bool RAGGED>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_kernel(BalanceArgs a) {
  using R = RouterLane<DT, N, LOADS, RAGGED>;
  constexpr int W = kBalanceWaves, T = 64 * W, PER = 64 / N, V = R::V, COLS = N * LOADS * V, U = balance_batch(LOADS);
  __shared__ double sums[W][COLS];
  __shared__ double z_sums[W];
  __shared__ int picks[COLS], tokens[W], all_picks[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % N, of = lane / N;
  const int g = blockIdx.x / a.per_group, part = blockIdx.x % a.per_group;
  const int64_t first = part * a.rows, end = first + a.rows < a.per ? first + a.rows : a.per, base = (int64_t)g * a.per;
  const auto* x = static_cast<const typename R::elem*>(a.x) + base * a.stride;
  const R r(a.E, sub);
  const uint64_t full = full_ballot<N>(a.k);
  float p[LOADS][V] = {};
  double z = 0.0;
  int counted = 0, picked = 0, turns = 0;  // (counts of the wavefront)
  const auto flush = [&] {
    const PlacesSums<N, LOADS * V> sum(p);
#pragma unroll
    for (int h = 0; h < sum.kHeld; ++h) {
      const int i = (sum.first + h) / V, c0 = (sub + i * N) * V, at = R::first_of(a.E, c0) + (sum.first + h) % V;
      if (sum.writes && c0 < a.E && (!RAGGED || (at >= c0 && at < a.E))) sums[wave][at] += sum.s[h];
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) p[i][c] = 0.0f;
  };
  const int64_t t1 = first + wave * (PER * U) + of;  // the lane's first token
  const auto* px = x + t1 * a.stride;
  const char* pc = static_cast<const char*>(a.cols) + ((base + t1) * a.k + sub) * a.col_bytes;
  u4_vec w[U][LOADS];
  int col[U];
  const auto load = [&](int64_t left) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool is = u * PER + of < left;
      r.load(px + u * PER * a.stride, a.E, is, w[u]);
      col[u] = -1;
      if (is && sub < a.k) col[u] = stored_col(a, pc + u * PER * a.k * a.col_bytes);
    }
  };
  int64_t left = end - first - wave * (PER * U);
  load(left);  // (before all else: the first batch comes meanwhile)
  for (int e = threadIdx.x; e < COLS; e += T) {
    picks[e] = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) sums[w][e] = 0.0;
  }
  if (part == 0 && threadIdx.x == 0 && a.arrived) a.arrived[g] = 0;
  __syncthreads();
  for (; left > 0; left -= W * PER * U, px += W * PER * U * a.stride, pc += W * PER * U * a.k * a.col_bytes, load(left)) {
    arrived(w, col);
    float own_m = 0.0f, own_s = 0.0f;  // of the token whose number is the lane's
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * PER >= left) break;  // (uniform)
      const bool any = (uint32_t)col[u] < (uint32_t)a.E;
      uint64_t ballot = __ballot(any);
      if (any) atomicAdd(&picks[col[u]], 1);
      picked += __popcll(ballot);
      if (ballot == full && a.k <= N) {
        counted += PER;
      } else {
        for (int j = N; j < a.k; j += N) {
          const int more = sub + j < a.k && u * PER + of < left ? pick_from(a, pc + (u * PER * a.k + j) * a.col_bytes) : -1;
          if (more >= 0) atomicAdd(&picks[more], 1);
          const uint64_t b = __ballot(more >= 0);
          picked += __popcll(b);
          ballot |= b;
        }
        const bool counts = any_lane<N>(ballot, of);
        counted += __popcll(__ballot(counts && sub == 0));
        R::leave_out(!counts, w[u]);
      }
      const RouterRow<DT, N, LOADS, RAGGED> row(r, w[u]);
      const float over = over_of(row.s);
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int c = 0; c < V; ++c) p[i][c] = __builtin_fmaf(row.e[i][c], over, p[i][c]);
      if constexpr (N >= U) {
        own_m = sub == u ? row.m : own_m;
        own_s = sub == u ? row.s : own_s;
      } else {
        const double lse = sub == 0 ? (double)lse_of(row.m, row.s) : 0.0;
        z = __builtin_fma(lse, lse, z);
      }
    }
    if constexpr (N >= U) {
      const double lse = lse_of(own_m, own_s);
      z = __builtin_fma(lse, lse, z);
    }
    turns += U;
    if (turns >= kFlush) {
      flush();
      turns = 0;
    }
  }
  flush();
  z = lanes_total(z);
  if (lane == 0) {
    z_sums[wave] = z;
    tokens[wave] = counted;
    all_picks[wave] = picked;
  }
  __syncthreads();
  z = 0.0;
  counted = picked = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    z += z_sums[w];
    counted += tokens[w];
    picked += all_picks[w];
  }
  double dot = 0.0;
  for (int e = threadIdx.x; e < a.E; e += T) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) v += sums[w][e];
    if (a.per_group == 1) {
      dot += write_column(a, g, e, v, picks[e], counted);
    } else {
      a.part_p[(int64_t)blockIdx.x * a.E + e] = v;
      a.part_n[(int64_t)blockIdx.x * a.E + e] = picks[e];
    }
  }
  if (a.per_group == 1) {
    dot = lanes_total(dot);
    __syncthreads();
    if (lane == 0) z_sums[wave] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      dot = 0.0;
#pragma unroll
      for (int w = 0; w < W; ++w) dot += z_sums[w];
      write_group(a, g, dot, z, counted, picked);
    }
  } else if (threadIdx.x == 0) {
    a.part_z[blockIdx.x] = BalancePart{z, counted, picked};
  }
}

// Joins a group's workgroups, in order: C columns by a workgroup, its threads in slices of the parts.  The last of a group's that is done (counted from 0, which
// balance_kernel set) adds up what each has for the loss, in order.  What it reads of the others is stored and loaded past the caches, so that no cache
// has to be written back, which takes 5 us.
template <int T, int C>
__global__ __launch_bounds__(T) void balance_join_kernel(BalanceArgs a) {
  constexpr int S = T / C, W = T / 64;
  __shared__ double p[S][C], of_wave[2][W];
  __shared__ int n[S][C], counts[2][W];
  const int blocks = (a.E + C - 1) / C, g = blockIdx.x / blocks, block = blockIdx.x % blocks;
  const int slice = threadIdx.x / C, c = threadIdx.x % C, e = block * C + c, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at = (int64_t)g * a.per_group;
  double s = 0.0, z = 0.0;
  int k = 0, counted = 0, picked = 0;
  if (e < a.E) {
#pragma unroll 4
    for (int j = slice; j < a.per_group; j += S) {
      s += a.part_p[(at + j) * a.E + e];
      k += a.part_n[(at + j) * a.E + e];
    }
  }
  for (int j = threadIdx.x; j < a.per_group; j += T) {
    const BalancePart q = a.part_z[at + j];
    z += q.z;
    counted += q.counted;
    picked += q.picked;
  }
  z = lanes_total(z);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    counted += __shfl_xor(counted, d);
    picked += __shfl_xor(picked, d);
  }
  if (lane == 0) {
    of_wave[0][wave] = z;
    counts[0][wave] = counted;
    counts[1][wave] = picked;
  }
  if (S > 1) {
    p[slice][c] = s;
    n[slice][c] = k;
  }
  __syncthreads();
  z = 0.0;
  counted = picked = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    z += of_wave[0][w];
    counted += counts[0][w];
    picked += counts[1][w];
  }
  double dot = 0.0;
  if (slice == 0 && e < a.E) {
#pragma unroll
    for (int i = 1; i < S; ++i) {
      s += p[i][c];
      k += n[i][c];
    }
    dot = write_column(a, g, e, s, k, counted);
  }
  dot = lanes_total(dot);
  if (lane == 0) of_wave[1][wave] = dot;
  __syncthreads();
  if (threadIdx.x != 0) return;
  dot = 0.0;
  for (int w = 0; w < W; ++w) dot += of_wave[1][w];
  if (blocks > 1) {
    double* dots = a.part_dot + (int64_t)g * blocks;
    __hip_atomic_store(dots + block, dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the store is done (a fence of the workgroup would not wait for it)
    if (__hip_atomic_fetch_add(a.arrived + g, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != blocks - 1) return;
    dot = 0.0;
    for (int i = 0; i < blocks; ++i) dot += __hip_atomic_load(dots + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  write_group(a, g, dot, z, counted, picked);
}

// ---- gradient -------------------------------------------------------------------------------------

// LDS of one wavefront: what it writes there it reads again itself, in the order of the program.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The picked values' gradients at their columns of the wavefront's tokens, 0 elsewhere: as the lanes hold the columns, in planes of four so that the
// lanes' 128-bit reads meet no bank twice.  A column that two lanes hold is written for both.
template <int DT, int N, int LOADS, bool RAGGED>
struct PickedTile {
  static constexpr int V = Logits<DT>::V, PER = 64 / N, PLANE = N * LOADS * 4;
  float (&at)[PER][V / 4][PLANE];
  int E, of;
  __device__ __forceinline__ float* place(int chunk, int c) const { return &at[of][c / 4][chunk * 4 + c % 4]; }
  // where a column is held: for the lane that has it, and for the one whose chunk ends with the row
  struct Places {
    float *own, *end;
    __device__ __forceinline__ void put(float v) const {
      if (!RAGGED || own) *own = v;
      if (RAGGED && end) *end = v;
    }
  };
  __device__ __forceinline__ Places places(int col) const {
    if (!RAGGED || E < V) return {place(col / V, col % V), nullptr};
    const int last = (E - 1) / V;
    return {col / V != last ? place(col / V, col % V) : nullptr, col >= E - V ? place(last, col - (E - V)) : nullptr};
  }
  __device__ __forceinline__ void put(int col, float v) const { places(col).put(v); }
  __device__ __forceinline__ void get(int chunk, float (&v)[V]) const {
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
      const float4 f = *reinterpret_cast<const float4*>(&at[of][h][chunk * 4]);
      v[4 * h] = f.x;
      v[4 * h + 1] = f.y;
      v[4 * h + 2] = f.z;
      v[4 * h + 3] = f.w;
    }
  }
};

template <int DT, int N, int LOADS, bool VALS, bool RAGGED>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_grad_kernel(BalanceArgs a) {
  using R = RouterLane<DT, N, LOADS, RAGGED>;
  using L = Logits<DT>;
  using Tile = PickedTile<DT, N, LOADS, RAGGED>;
  constexpr int W = kBalanceWaves, PER = 64 / N, V = R::V, U = balance_batch(LOADS);
  __shared__ __align__(16) float tiles[VALS ? W : 1][PER][V / 4][Tile::PLANE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % N, of = lane / N;
  const int g = blockIdx.x / a.per_group, part = blockIdx.x % a.per_group;
  const int64_t first = part * a.rows, end = first + a.rows < a.per ? first + a.rows : a.per, base = (int64_t)g * a.per;
  const auto* x = static_cast<const typename L::elem*>(a.x) + base * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + base * a.grad_stride;
  const R r(a.E, sub);
  const uint64_t full = full_ballot<N>(a.k);
  const int64_t t1 = first + wave * (PER * U) + of;  // the lane's first token
  const auto* px = x + t1 * a.stride;
  auto* to = out + t1 * a.grad_stride;
  const char* pc = static_cast<const char*>(a.cols) + ((base + t1) * a.k + sub) * a.col_bytes;
  const float* pv = a.grad_vals + (VALS ? (base + t1) * a.k + sub : 0);
  u4_vec raw[U][LOADS];
  int col[U];
  float val[U];
  const auto load = [&](int64_t left) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool is = u * PER + of < left;
      r.load(px + u * PER * a.stride, a.E, is, raw[u]);
      col[u] = -1;
      val[u] = 0.0f;
      if (is && sub < a.k) {
        col[u] = stored_col(a, pc + u * PER * a.k * a.col_bytes);
        if (VALS) val[u] = pv[u * PER * a.k];
      }
    }
  };
  int64_t left = end - first - wave * (PER * U);
  load(left);  // (before all else: the first batch comes meanwhile)
  // w_e of the lane's columns
  float w[LOADS][V];
  double all = 0.0;
  for (int e = lane; e < a.E; e += 64) all += a.counts_in[(int64_t)g * a.E + e];
  all = lanes_total(all);
  const int tokens = a.counted_in[g];
  const double over_n = tokens > 0 ? 1.0 / tokens : 0.0, each = all > 0.0 ? a.E * (double)a.grad_loss[g] * over_n / all : 0.0;
  const float z2 = a.grad_z ? (float)(2.0 * a.grad_z[g] * over_n) : 0.0f;
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int e = r.at[i] + c;
      w[i][c] = (float)a.counts_in[(int64_t)g * a.E + min(e, a.E - 1)];  // (no branch: together)
    }
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
#pragma unroll
    for (int c = 0; c < V; ++c) w[i][c] *= (float)each;
  const Tile tile{tiles[VALS ? wave : 0], a.E, of};
  if constexpr (VALS) {
    for (int c = lane; c < PER * V / 4 * Tile::PLANE; c += 64) (&tiles[wave][0][0][0])[c] = 0.0f;
    wave_fence();
  }
  for (; left > 0; left -= W * PER * U, px += W * PER * U * a.stride, to += W * PER * U * a.grad_stride, pc += W * PER * U * a.k * a.col_bytes,
                  pv += VALS ? W * PER * U * a.k : 0, load(left)) {
    arrived(raw, col);
    if (VALS) {
#pragma unroll
      for (int u = 0; u < U; ++u) asm volatile("" : "+v"(val[u]));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * PER >= left) break;  // (uniform)
      const bool is = u * PER + of < left;
      const char* entry = pc + u * PER * a.k * a.col_bytes;
      const float* value = pv + (VALS ? u * PER * a.k : 0);
      col[u] = pick_of(a, col[u]);
      uint64_t ballot = __ballot(col[u] >= 0);
      bool left_out = false, once = true;  // picks that ascend, so that none is there twice
      if (VALS) {
        const int before = __builtin_amdgcn_update_dpp(0, col[u], 0x138, 0xf, 0xf, false);  // wave_shr:1
        once = !__any(col[u] >= 0 && sub > 0 && !(before >= 0 && before < col[u]));
      }
      if (!(ballot == full && a.k <= N)) {
        for (int j = N; j < a.k; j += N) {
          const int mine = sub + j < a.k && is ? pick_from(a, entry + j * a.col_bytes) : -1;
          ballot |= __ballot(mine >= 0);
          if (VALS) {
            const int before = mine >= 0 ? pick_from(a, entry + (j - 1) * a.col_bytes) : -1;
            once = once && !__any(mine >= 0 && !(before >= 0 && before < mine));
          }
        }
        left_out = !any_lane<N>(ballot, of);
        R::leave_out(left_out, raw[u]);
      }
      const RouterRow<DT, N, LOADS, RAGGED> row(r, raw[u]);
      // f(column, the gradients that it gets) for the picks of the lane, but for the first where there is one to a column
      const auto picked = [&](auto f) {
        if (once) {
          for (int j = N; j < a.k; j += N) {
            const int mine = sub + j < a.k && is ? pick_from(a, entry + j * a.col_bytes) : -1;
            if (mine >= 0) f(mine, value[j]);
          }
        } else if (is) {
          for (int j = sub; j < a.k; j += N) {
            const int mine = pick_from(a, entry + (j - sub) * a.col_bytes);
            if (mine < 0) continue;
            float v = value[j - sub];  // the first entry of a column adds up all that have it
            bool earlier = false;
            for (int i = 0; i < a.k; ++i)
              if (i != j && pick_from(a, entry + (i - sub) * a.col_bytes) == mine) {
                earlier |= i < j;
                v += value[i - sub];
              }
            if (!earlier) f(mine, v);
          }
        }
      };
      typename Tile::Places own = {};
      const bool first_pick = VALS && once && col[u] >= 0;
      if constexpr (VALS) {
        if (first_pick) {
          own = tile.places(col[u]);
          own.put(val[u]);
        }
        picked([&](int c, float v) { tile.put(c, v); });
        wave_fence();
      }
      const float over = over_of(row.s);
      float dot = 0.0f;
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int c = 0; c < V; ++c) dot = __builtin_fmaf(r.kept(row.e[i][c], i, c), w[i][c], dot);
      dot = lanes_sum<N>(dot) * over;
      const float both = ((z2 == 0.0f ? 0.0f : z2 * lse_of(row.m, row.s)) - dot) * over;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        float d[V], v[V];
        if (VALS) tile.get(sub + i * N, v);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float t = __builtin_fmaf(w[i][c], over, both);
          d[c] = VALS ? __builtin_fmaf(row.e[i][c], t, v[c]) : row.e[i][c] * t;
        }
        if (__any(left_out)) {  // (0, whatever the group's gradients are)
#pragma unroll
          for (int c = 0; c < V; ++c) d[c] = left_out ? 0.0f : d[c];
        }
        if (is && r.has[i]) {
          auto* at = to + u * PER * a.grad_stride + r.at[i];
          if (!RAGGED || a.E >= V) {
            L::store(at, pack_rounded<DT>(d));
          } else {
#pragma unroll
            for (int c = 0; c < V; ++c)
              if (c < a.E) at[c] = L::narrow(d[c]);
          }
        }
      }
      if constexpr (VALS) {
        wave_fence();
        if (first_pick) own.put(0.0f);
        picked([&](int c, float) { tile.put(c, 0.0f); });
        wave_fence();
      }
    }
  }
}

}  // namespace rtopk
