// A router's balance loss and its gradient for gfx950 (MI355X).
//
// Tokens come in groups; token t of a group has E logits x_t and the columns that a selection picked for it, and counts if any of them lies in [0, E).
// With p_t = softmax(x_t), n the group's tokens that count, f_e the share of all picks that expert e got, P_e = (1 / n) sum_t p_te:
//   loss = E sum_e f_e P_e  (1 where either is even),   z = (1 / n) sum_t lse_t^2
// and, f held constant (it is piecewise so), with w_e = E f_e g_loss / n:
//   dx_te = p_te (w_e - sum_j p_tj w_j + 2 g_z lse_t / n) + the gradients of the token's picked values at their columns
//
// A token's row lies in a few lanes, 64 / lanes tokens to a wavefront, and is read once; maxima and sums go over those lanes.  Forward, a lane keeps the sums of
// its columns' probabilities over the tokens it sees, in fp32 for kFlush turns and in 64 bits (LDS) over these; picks are counted by integer atomics
// in LDS, whose order changes nothing.  Workgroups leave their sums in scratch memory and a second kernel joins them in order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk_balance_dispatch.hpp"
#include "rtopk_logits.hpp"

namespace rtopk {

constexpr int kFlush = 64;  // turns that fp32 sums run over

// f over each N lanes (a power of two), the same in all of them.
template <int N, typename F>
__device__ __forceinline__ float lanes_reduce(float v, F f) {
  const auto dpp = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
  if constexpr (N >= 2) v = f(v, dpp(std::integral_constant<int, 0xb1>{}));   // quad_perm [1, 0, 3, 2]
  if constexpr (N >= 4) v = f(v, dpp(std::integral_constant<int, 0x4e>{}));   // quad_perm [2, 3, 0, 1]
  if constexpr (N >= 8) v = f(v, dpp(std::integral_constant<int, 0x141>{}));  // row_half_mirror
  if constexpr (N >= 16) v = f(v, dpp(std::integral_constant<int, 0x140>{})); // row_mirror
  if constexpr (N >= 32) v = f(v, __shfl_xor(v, 16));
  if constexpr (N >= 64) v = f(v, __shfl_xor(v, 32));
  return v;
}
template <int N>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_reduce<N>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_reduce<N>(v, [](float a, float b) { return a + b; });
}

// The lane's columns of a token's row: chunk i of the lane is chunk `lane + i N` of the row.
template <int DT, int N, int LOADS>
struct RouterRow {
  using L = Logits<DT>;
  static constexpr int V = L::V;
  float x[LOADS][V];
  static __device__ __forceinline__ int column(int sub, int i) { return (sub + i * N) * V; }
  __device__ __forceinline__ void load(const typename L::elem* row, int E, int sub, bool is) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c0 = column(sub, i);
      if (is && c0 + V <= E) {
        const u4_vec w = L::load_once(row + c0);
#pragma unroll
        for (int c = 0; c < V; ++c) x[i][c] = L::at(w, c);
      } else {
#pragma unroll
        for (int c = 0; c < V; ++c) x[i][c] = is && c0 + c < E ? L::widen(row[c0 + c]) : kNegInf;
      }
    }
  }
  // x becomes the probabilities; the log-sum-exp (-inf for a row of nothing but -inf, whose probabilities are 0)
  __device__ __forceinline__ float softmax() {
    float m = x[0][0], s = 0.0f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) m = vmax(m, x[i][c]);
    m = lanes_max<N>(m);
    const float about = m == kNegInf ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        x[i][c] = __builtin_amdgcn_exp2f((x[i][c] - about) * kLog2e);
        s += x[i][c];
      }
    s = lanes_sum<N>(s);
    const float over = s == 0.0f ? 0.0f : 1.0f / s;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) x[i][c] *= over;
    return s == 0.0f ? kNegInf : about + logf(s);
  }
};

__device__ __forceinline__ int pick_at(const BalanceArgs& a, int64_t i) {  // -1: none
  const int c = a.col_bytes == 1 ? static_cast<const uint8_t*>(a.cols)[i] : static_cast<const int32_t*>(a.cols)[i];
  return c >= 0 && c < a.E ? c : -1;
}

// The results of a group from its sums; all threads of a workgroup.  sum_p(e), picks(e): of column e.
template <int T, typename P, typename C>
__device__ __forceinline__ void write_balance(const BalanceArgs& a, int g, double z, int counted, double* room, P sum_p, C picks) {
  double dot = 0.0, all = 0.0;
  const double over = counted > 0 ? 1.0 / counted : 0.0;
  for (int e = threadIdx.x; e < a.E; e += T) {
    const double mean = sum_p(e) * over;
    const int n = picks(e);
    if (a.probs) a.probs[(int64_t)g * a.E + e] = (float)mean;
    a.counts[(int64_t)g * a.E + e] = n;
    if (n > 0) dot += mean * n;  // (what was never picked adds nothing, whatever it is)
    all += n;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    dot += __shfl_xor(dot, d);
    all += __shfl_xor(all, d);
  }
  if ((threadIdx.x & 63) == 0) {
    room[2 * (threadIdx.x >> 6)] = dot;
    room[2 * (threadIdx.x >> 6) + 1] = all;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    dot = all = 0.0;
    for (int w = 0; w < T / 64; ++w) {
      dot += room[2 * w];
      all += room[2 * w + 1];
    }
    a.loss[g] = all > 0.0 ? (float)(a.E * dot / all) : 0.0f;
    if (a.z) a.z[g] = (float)(z * over);
    a.counted[g] = counted;
  }
}

template <int DT, int N, int LOADS>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_kernel(BalanceArgs a) {
  using R = RouterRow<DT, N, LOADS>;
  constexpr int W = kBalanceWaves, T = 64 * W, PER = 64 / N, V = R::V, COLS = N * LOADS * V;
  __shared__ double sums[W][COLS];
  __shared__ double z_sums[W];
  __shared__ double room[2 * W];
  __shared__ int picks[COLS], tokens[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % N, of = lane / N;
  const int g = blockIdx.x / a.per_group, part = blockIdx.x % a.per_group;
  const int64_t first = part * a.rows, end = first + a.rows < a.per ? first + a.rows : a.per, base = (int64_t)g * a.per;
  for (int e = threadIdx.x; e < COLS; e += T) {
    picks[e] = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) sums[w][e] = 0.0;
  }
  __syncthreads();
  const auto* x = static_cast<const typename Logits<DT>::elem*>(a.x) + base * a.stride;
  float p[LOADS][V] = {};
  double z_all = 0.0;
  int counted = 0, turns = 0;
  const auto flush = [&] {
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        float v = p[i][c];
#pragma unroll
        for (int d = N; d < 64; d <<= 1) v += __shfl_xor(v, d);
        if (of == 0) sums[wave][R::column(sub, i) + c] += v;
        p[i][c] = 0.0f;
      }
  };
  for (int64_t t0 = first + wave * PER; t0 < end; t0 += W * PER) {
    const int64_t t = t0 + of;
    R r;
    r.load(x + t * a.stride, a.E, sub, t < end);
    bool any = false;
    if (t < end)
      for (int j = sub; j < a.k; j += N) {
        const int col = pick_at(a, (base + t) * a.k + j);
        any |= col >= 0;
        if (col >= 0) atomicAdd(&picks[col], 1);
      }
    const uint64_t mask = N == 64 ? ~(uint64_t)0 : ((uint64_t)1 << (N % 64)) - 1;
    const bool counts = ((__ballot(any) >> (of * N)) & mask) != 0;
    const float lse = r.softmax();
    if (counts) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int c = 0; c < V; ++c) p[i][c] += r.x[i][c];
      if (sub == 0) {
        if (lse != kNegInf) z_all = __builtin_fma((double)lse, (double)lse, z_all);
        ++counted;
      }
    }
    if (++turns % kFlush == 0) flush();
  }
  flush();
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    z_all += __shfl_xor(z_all, d);
    counted += __shfl_xor(counted, d);
  }
  if (lane == 0) {
    z_sums[wave] = z_all;
    tokens[wave] = counted;
  }
  __syncthreads();
  z_all = 0.0;
  counted = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    z_all += z_sums[w];
    counted += tokens[w];
  }
  const auto sum_p = [&](int e) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) v += sums[w][e];
    return v;
  };
  if (a.per_group == 1) {
    write_balance<T>(a, g, z_all, counted, room, sum_p, [&](int e) { return picks[e]; });
  } else {
    for (int e = threadIdx.x; e < a.E; e += T) {
      a.part_p[(int64_t)blockIdx.x * a.E + e] = sum_p(e);
      a.part_n[(int64_t)blockIdx.x * a.E + e] = picks[e];
    }
    if (threadIdx.x == 0) {
      a.part_z[blockIdx.x] = z_all;
      a.part_rows[blockIdx.x] = counted;
    }
  }
}

// Joins a group's workgroups, in order.
template <int T>
__global__ __launch_bounds__(T) void balance_join_kernel(BalanceArgs a) {
  __shared__ double p[kMaxExperts], room[T / 32];
  __shared__ int n[kMaxExperts];
  __shared__ double z;
  __shared__ int counted;
  const int g = blockIdx.x;
  const int64_t at = (int64_t)g * a.per_group;
  for (int e = threadIdx.x; e < a.E; e += T) {
    double s = 0.0;
    int c = 0;
    for (int j = 0; j < a.per_group; ++j) {
      s += a.part_p[(at + j) * a.E + e];
      c += a.part_n[(at + j) * a.E + e];
    }
    p[e] = s;
    n[e] = c;
  }
  if (threadIdx.x == 0) {
    double s = 0.0;
    int c = 0;
    for (int j = 0; j < a.per_group; ++j) {
      s += a.part_z[at + j];
      c += a.part_rows[at + j];
    }
    z = s;
    counted = c;
  }
  __syncthreads();
  write_balance<T>(a, g, z, counted, room, [&](int e) { return p[e]; }, [&](int e) { return n[e]; });
}

// LDS of one wavefront: what it writes there it reads again itself, in the order of the program.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int DT, int N, int LOADS, bool VALS>
__global__ __launch_bounds__(64 * kBalanceWaves) void balance_grad_kernel(BalanceArgs a) {
  using R = RouterRow<DT, N, LOADS>;
  using L = Logits<DT>;
  constexpr int W = kBalanceWaves, PER = 64 / N, V = R::V, COLS = N * LOADS * V;
  __shared__ float tile[VALS ? W : 1][VALS ? PER : 1][VALS ? COLS : 1];  // the picked values' gradients at their columns, 0 elsewhere
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % N, of = lane / N;
  const int g = blockIdx.x / a.per_group, part = blockIdx.x % a.per_group;
  const int64_t first = part * a.rows, end = first + a.rows < a.per ? first + a.rows : a.per, base = (int64_t)g * a.per;
  const auto* x = static_cast<const typename L::elem*>(a.x) + base * a.stride;
  auto* out = static_cast<typename L::elem*>(a.grad_x) + base * a.grad_stride;
  // w_e of the lane's columns
  float w[LOADS][V];
  double all = 0.0;
  for (int e = lane; e < a.E; e += 64) all += a.counts_in[(int64_t)g * a.E + e];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
  const int tokens = a.counted_in[g];
  const double over = tokens > 0 ? 1.0 / tokens : 0.0, each = all > 0.0 ? a.E * (double)a.grad_loss[g] * over / all : 0.0;
  const float z2 = a.grad_z ? (float)(2.0 * a.grad_z[g] * over) : 0.0f;
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int e = R::column(sub, i) + c;
      w[i][c] = e < a.E ? (float)(each * a.counts_in[(int64_t)g * a.E + e]) : 0.0f;
    }
  if constexpr (VALS) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) tile[wave][of][R::column(sub, i) + c] = 0.0f;
    wave_fence();
  }
  for (int64_t t0 = first + wave * PER; t0 < end; t0 += W * PER) {
    const int64_t t = t0 + of;
    R r;
    r.load(x + t * a.stride, a.E, sub, t < end);
    bool any = false;
    if (t < end)
      for (int j = sub; j < a.k; j += N) {
        const int col = pick_at(a, (base + t) * a.k + j);
        any |= col >= 0;
        if (VALS && col >= 0) {
          // the first entry of a column adds up all that have it
          float v = a.grad_vals[(base + t) * a.k + j];
          bool earlier = false;
          for (int i = 0; i < a.k; ++i)
            if (i != j && pick_at(a, (base + t) * a.k + i) == col) {
              earlier |= i < j;
              v += a.grad_vals[(base + t) * a.k + i];
            }
          if (!earlier) tile[wave][of][col] = v;
        }
      }
    const uint64_t mask = N == 64 ? ~(uint64_t)0 : ((uint64_t)1 << (N % 64)) - 1;
    const bool counts = ((__ballot(any) >> (of * N)) & mask) != 0;
    if constexpr (VALS) wave_fence();
    const float lse = r.softmax();
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int c = 0; c < V; ++c) dot = __builtin_fmaf(r.x[i][c], w[i][c], dot);
    dot = lanes_sum<N>(dot);
    const float both = (lse == kNegInf ? 0.0f : z2 * lse) - dot;
    if (t < end) {
      auto* to = out + t * a.grad_stride;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int c0 = R::column(sub, i);
        float d[V];
#pragma unroll
        for (int c = 0; c < V; ++c) {
          d[c] = counts ? r.x[i][c] * (w[i][c] + both) : 0.0f;
          if (VALS) d[c] += tile[wave][of][c0 + c];
        }
        if (c0 + V <= a.E) L::store(to + c0, L::pack(d));
        else
          for (int c = 0; c < V; ++c)
            if (c0 + c < a.E) to[c0 + c] = L::narrow(d[c]);
      }
    }
    if constexpr (VALS) {
      wave_fence();
      if (t < end)
        for (int j = sub; j < a.k; j += N) {
          const int col = pick_at(a, (base + t) * a.k + j);
          if (col >= 0) tile[wave][of][col] = 0.0f;
        }
      wave_fence();
    }
  }
}

}  // namespace rtopk
