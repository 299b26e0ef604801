// C ABI of the operators on rows of logits: argument checks, layout, launches.  Declarations and the full contract are in include/rtopk.h.
#include "rtopk.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "rtopk_dispatch.hpp"
#include "rtopk_logits_dispatch.hpp"

namespace {

using rtopk::LogitsArgs;

inline uintptr_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

struct Buffer {
  const void* p;
  uint64_t bytes, align;
  bool written;
};

// RTOPK_OK, or what is wrong with the buffers: alignment, or bytes that a written one shares with another.
template <int C>
int check_buffers(const Buffer (&b)[C]) {
  for (const Buffer& x : b)
    if (!rtopk::is_aligned(addr(x.p), x.align)) return RTOPK_ERR_MISALIGNED;
  for (int i = 0; i < C; ++i)
    for (int j = i + 1; j < C; ++j)
      if ((b[i].written || b[j].written) && b[i].p && b[j].p && rtopk::ranges_overlap(addr(b[i].p), b[i].bytes, addr(b[j].p), b[j].bytes))
        return RTOPK_ERR_OVERLAP;
  return RTOPK_OK;
}

inline uint64_t size_of(int dtype) { return dtype == RTOPK_F32 ? 4 : 2; }
inline bool is_type(int dtype) { return dtype == RTOPK_F32 || dtype == RTOPK_F16 || dtype == RTOPK_BF16; }

// The part of the checks that all share, and the arguments they fill.
int rows_of_logits(LogitsArgs& a, const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, float temperature) {
  if (!is_type(dtype)) return RTOPK_ERR_BAD_TYPE;
  if (N < 0 || M < 1 || (N > 1 && stride < M)) return RTOPK_ERR_BAD_SHAPE;
  if (M > rtopk::kMaxLogitsM) return RTOPK_ERR_M_TOO_LARGE;
  const float inv_t = 1.0f / temperature;
  const float c = (float)(1.44269504088896340736 / (double)temperature);
  if (!(temperature > 0.0f) || !isfinite(temperature) || !isfinite(c)) return RTOPK_ERR_BAD_TEMPERATURE;
  if (N > 0 && stride > (INT64_MAX / 8) / N) return RTOPK_ERR_BAD_SHAPE;
  a.x = logits;
  a.N = N;
  a.M = M;
  a.stride = stride;
  a.inv_t = inv_t;
  a.c = c;
  return RTOPK_OK;
}

inline uint64_t rows_bytes(int64_t N, int32_t M, int64_t stride, int dtype) {
  return ((uint64_t)(N - 1) * (N > 1 ? (uint64_t)stride : 0) + (uint64_t)M) * size_of(dtype);
}

// The layout of the rows' pass, spread over workgroups only where there is memory for the parts.
rtopk::LogitsLayout lay_out(LogitsArgs& a, int dtype, int k, void* workspace, int64_t workspace_bytes) {
  rtopk::LogitsLayout l = rtopk::logits_layout(a.N, a.M, dtype, k);
  if (l.segments > 1 && (!workspace || workspace_bytes < rtopk::logits_workspace(a.N, l, k))) l = rtopk::logits_layout_whole(a.N, a.M, k);
  a.segments = l.segments;
  a.seg_cols = l.cols;
  a.part = static_cast<float4*>(workspace);
  a.part_keys = l.segments > 1 ? reinterpret_cast<uint64_t*>(a.part + a.N * l.segments) : nullptr;
  return l;
}

// launch(rows) for slices of the rows whose workgroups fit one launch (2^31 threads).
template <typename F>
hipError_t sliced(LogitsArgs& a, F launch) {
  const int64_t most = (1 << 21) / a.segments;
  for (a.row0 = 0; a.row0 < a.N; a.row0 += most) {
    const int64_t rows = a.N - a.row0 < most ? a.N - a.row0 : most;
    const hipError_t err = launch(rows);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

int forward(LogitsArgs& a, int dtype, int op, int k, void* workspace, int64_t workspace_bytes, void* stream) {
  const rtopk::LogitsLayout l = lay_out(a, dtype, k, workspace, workspace_bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_rows(dtype, op, l.waves, l.segments > 1, a, rows, s); });
  if (err == hipSuccess && l.segments > 1) err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_join(dtype, op, a, rows, s); });
  return err == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

inline bool in_place(const LogitsArgs& a) { return a.grad_x == a.x && (a.N <= 1 || a.grad_stride == a.stride); }

int backward(LogitsArgs& a, int dtype, int op, void* stream) {
  const rtopk::LogitsLayout l = rtopk::logits_grad_layout(a.N, a.M, dtype, in_place(a));
  a.segments = l.segments;
  a.seg_cols = l.cols;
  a.far_group = rtopk::far_group(a.N, l.segments);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_grad(dtype, op, l.waves, false, a, rows, s); });
  return err == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

// The teacher's list: shared checks and arguments.
int teacher_of(LogitsArgs& a, const void* vals, int32_t dtype, const int32_t* cols, int32_t k, int32_t log_probs) {
  if (!is_type(dtype)) return RTOPK_ERR_BAD_TYPE;
  if (k < 1 || k > rtopk::kMaxList || (log_probs & ~1) != 0) return RTOPK_ERR_BAD_SHAPE;
  a.teacher_vals = vals;
  a.teacher_dtype = dtype;
  a.teacher_cols = cols;
  a.k = k;
  a.log_probs = log_probs;
  return RTOPK_OK;
}

// The gradient's rows: RTOPK_OK with the bytes to hold against the other buffers (0 where it lies in the logits' place).
int gradient_of(LogitsArgs& a, int dtype, void* grad_logits, int64_t grad_stride, Buffer& out) {
  if (a.N > 1 && grad_stride < a.M) return RTOPK_ERR_BAD_SHAPE;
  if (grad_stride > (INT64_MAX / 8) / a.N) return RTOPK_ERR_BAD_SHAPE;
  a.grad_x = grad_logits;
  a.grad_stride = grad_stride;
  out = {grad_logits, rows_bytes(a.N, a.M, grad_stride, dtype), size_of(dtype), true};
  return RTOPK_OK;
}

}  // namespace

extern "C" {

int64_t rtopk_logits_workspace_bytes(int64_t N, int32_t M, int32_t dtype, int32_t k) {
  if (N < 1 || M < 1 || M > rtopk::kMaxLogitsM || !is_type(dtype) || k < 0 || k > rtopk::kMaxAlternatives || k > M) return 0;
  return rtopk::logits_workspace(N, rtopk::logits_layout(N, M, dtype, k), k);
}

int rtopk_token_logprobs(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const void* tokens, int32_t token_bytes,
                         int32_t G, int32_t k, float temperature, float* out_logprobs, float* out_entropy, float* out_lse,
                         float* out_top_logprobs, int32_t* out_top_cols, void* workspace, int64_t workspace_bytes, void* stream) {
  LogitsArgs a{};
  if (const int status = rows_of_logits(a, logits, dtype, N, M, stride, temperature)) return status;
  if (token_bytes != 4 && token_bytes != 8) return RTOPK_ERR_BAD_TYPE;
  if (G < 0 || G > rtopk::kMaxList || k < 0 || k > rtopk::kMaxAlternatives || k > M || workspace_bytes < 0) return RTOPK_ERR_BAD_SHAPE;
  if (N == 0) return RTOPK_OK;
  if (!logits || (G > 0 && (!tokens || !out_logprobs)) || (k > 0 && (!out_top_logprobs || !out_top_cols))) return RTOPK_ERR_NULL_POINTER;
  const uint64_t n = (uint64_t)N;
  const Buffer buffers[] = {{logits, rows_bytes(N, M, stride, dtype), size_of(dtype), false},
                            {tokens, n * G * token_bytes, (uint64_t)token_bytes, false},
                            {out_logprobs, n * G * 4, 4, true},
                            {out_entropy, n * 4, 4, true},
                            {out_lse, n * 4, 4, true},
                            {out_top_logprobs, n * k * 4, 4, true},
                            {out_top_cols, n * k * 4, 4, true},
                            {workspace, (uint64_t)workspace_bytes, 16, true}};
  if (const int status = check_buffers(buffers)) return status;
  a.tokens = tokens;
  a.token64 = token_bytes == 8;
  a.tokens_per_row = G;
  a.k = k;
  a.logprobs = out_logprobs;
  a.entropy = out_entropy;
  a.lse = out_lse;
  a.top_logprobs = out_top_logprobs;
  a.top_cols = out_top_cols;
  return forward(a, dtype, rtopk::kOpTokens, k, workspace, workspace_bytes, stream);
}

int rtopk_token_logprobs_backward(const float* grad_logprobs, const float* grad_entropy, const void* logits, int32_t dtype, int64_t N, int32_t M,
                                  int64_t stride, const void* tokens, int32_t token_bytes, int32_t G, const float* lse, const float* entropy,
                                  float temperature, void* grad_logits, int64_t grad_stride, void* stream) {
  LogitsArgs a{};
  if (const int status = rows_of_logits(a, logits, dtype, N, M, stride, temperature)) return status;
  if (token_bytes != 4 && token_bytes != 8) return RTOPK_ERR_BAD_TYPE;
  if (G < 0 || G > rtopk::kMaxList) return RTOPK_ERR_BAD_SHAPE;
  if (N == 0) return RTOPK_OK;
  if (!logits || !lse || !grad_logits || (G > 0 && (!tokens || !grad_logprobs)) || (grad_entropy && !entropy)) return RTOPK_ERR_NULL_POINTER;
  Buffer out;
  if (const int status = gradient_of(a, dtype, grad_logits, grad_stride, out)) return status;
  const uint64_t n = (uint64_t)N;
  const Buffer buffers[] = {{in_place(a) ? nullptr : logits, rows_bytes(N, M, stride, dtype), size_of(dtype), false},
                            {tokens, n * G * token_bytes, (uint64_t)token_bytes, false},
                            {grad_logprobs, n * G * 4, 4, false},
                            {grad_entropy, n * 4, 4, false},
                            {lse, n * 4, 4, false},
                            {grad_entropy ? entropy : nullptr, n * 4, 4, false},
                            out};
  if (const int status = check_buffers(buffers)) return status;
  a.tokens = tokens;
  a.token64 = token_bytes == 8;
  a.tokens_per_row = a.k = G;
  a.grad = grad_logprobs;
  a.grad_entropy = grad_entropy;
  a.lse_in = lse;
  a.entropy_in = entropy;
  return backward(a, dtype, rtopk::kOpTokens, stream);
}

int rtopk_distill(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const void* teacher_vals, int32_t teacher_dtype,
                  const int32_t* teacher_cols, int32_t k, int32_t log_probs, float temperature, float* out_loss, float* out_lse,
                  void* workspace, int64_t workspace_bytes, void* stream) {
  LogitsArgs a{};
  if (const int status = rows_of_logits(a, logits, dtype, N, M, stride, temperature)) return status;
  if (const int status = teacher_of(a, teacher_vals, teacher_dtype, teacher_cols, k, log_probs)) return status;
  if (workspace_bytes < 0) return RTOPK_ERR_BAD_SHAPE;
  if (N == 0) return RTOPK_OK;
  if (!logits || !teacher_vals || !teacher_cols || !out_loss) return RTOPK_ERR_NULL_POINTER;
  const uint64_t n = (uint64_t)N;
  const Buffer buffers[] = {{logits, rows_bytes(N, M, stride, dtype), size_of(dtype), false},
                            {teacher_vals, n * k * size_of(teacher_dtype), size_of(teacher_dtype), false},
                            {teacher_cols, n * k * 4, 4, false},
                            {out_loss, n * 4, 4, true},
                            {out_lse, n * 4, 4, true},
                            {workspace, (uint64_t)workspace_bytes, 16, true}};
  if (const int status = check_buffers(buffers)) return status;
  a.loss = out_loss;
  a.lse = out_lse;
  return forward(a, dtype, rtopk::kOpDistill, 0, workspace, workspace_bytes, stream);
}

int rtopk_distill_backward(const float* grad_loss, const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride,
                           const void* teacher_vals, int32_t teacher_dtype, const int32_t* teacher_cols, int32_t k, int32_t log_probs,
                           const float* lse, float temperature, void* grad_logits, int64_t grad_stride, void* stream) {
  LogitsArgs a{};
  if (const int status = rows_of_logits(a, logits, dtype, N, M, stride, temperature)) return status;
  if (const int status = teacher_of(a, teacher_vals, teacher_dtype, teacher_cols, k, log_probs)) return status;
  if (N == 0) return RTOPK_OK;
  if (!logits || !teacher_vals || !teacher_cols || !grad_loss || !lse || !grad_logits) return RTOPK_ERR_NULL_POINTER;
  Buffer out;
  if (const int status = gradient_of(a, dtype, grad_logits, grad_stride, out)) return status;
  const uint64_t n = (uint64_t)N;
  const Buffer buffers[] = {{in_place(a) ? nullptr : logits, rows_bytes(N, M, stride, dtype), size_of(dtype), false},
                            {teacher_vals, n * k * size_of(teacher_dtype), size_of(teacher_dtype), false},
                            {teacher_cols, n * k * 4, 4, false},
                            {grad_loss, n * 4, 4, false},
                            {lse, n * 4, 4, false},
                            out};
  if (const int status = check_buffers(buffers)) return status;
  a.grad = grad_loss;
  a.lse_in = lse;
  return backward(a, dtype, rtopk::kOpDistill, stream);
}

int rtopk_distill_with_grad(const float* weights, const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride,
                            const void* teacher_vals, int32_t teacher_dtype, const int32_t* teacher_cols, int32_t k, int32_t log_probs,
                            float temperature, float* out_loss, void* grad_logits, int64_t grad_stride, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  LogitsArgs a{};
  if (const int status = rows_of_logits(a, logits, dtype, N, M, stride, temperature)) return status;
  if (const int status = teacher_of(a, teacher_vals, teacher_dtype, teacher_cols, k, log_probs)) return status;
  if (workspace_bytes < 0) return RTOPK_ERR_BAD_SHAPE;
  if (N == 0) return RTOPK_OK;
  if (!logits || !teacher_vals || !teacher_cols || !weights || !out_loss || !grad_logits) return RTOPK_ERR_NULL_POINTER;
  Buffer out;
  if (const int status = gradient_of(a, dtype, grad_logits, grad_stride, out)) return status;
  const uint64_t n = (uint64_t)N;
  const Buffer buffers[] = {{in_place(a) ? nullptr : logits, rows_bytes(N, M, stride, dtype), size_of(dtype), false},
                            {teacher_vals, n * k * size_of(teacher_dtype), size_of(teacher_dtype), false},
                            {teacher_cols, n * k * 4, 4, false},
                            {weights, n * 4, 4, false},
                            {out_loss, n * 4, 4, true},
                            out,
                            {workspace, (uint64_t)workspace_bytes, 16, true}};
  if (const int status = check_buffers(buffers)) return status;
  a.grad = weights;
  a.loss = out_loss;
  const rtopk::LogitsLayout l = lay_out(a, dtype, 0, workspace, workspace_bytes);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t err;
  if (l.segments == 1) {
    const rtopk::HeldLayout h = rtopk::held_layout(M, dtype);
    err = sliced(a, [&](int64_t rows) { return rtopk::launch_distill_row(dtype, h.waves, h.loads, a, rows, s); });
  } else {
    err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_rows(dtype, rtopk::kOpDistill, l.waves, true, a, rows, s); });
    if (in_place(a) && err == hipSuccess) {
      // the loss needs the logits at the list's columns, which another workgroup may have replaced: in a launch before
      err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_join(dtype, rtopk::kOpDistill, a, rows, s); });
      a.loss = nullptr;
    }
    if (err == hipSuccess) err = sliced(a, [&](int64_t rows) { return rtopk::launch_logits_grad(dtype, rtopk::kOpDistill, l.waves, true, a, rows, s); });
  }
  return err == hipSuccess ? RTOPK_OK : RTOPK_ERR_LAUNCH;
}

}  // extern "C"
