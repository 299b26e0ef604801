/*
 * rtopk.h -- C ABI of the MI355X (gfx950) row-wise top-k library.
 *
 * Operation (RTop-K paper, arXiv 2409.00822, Section 3: problem statement and Algorithms 1 and 2):
 * for each of N rows of M fp32 values, select k (value, column) pairs by a binary search over a
 * threshold between the row's minimum and maximum, counting the elements at or above each midpoint.
 *
 * Common conventions for every entry point below
 * ----------------------------------------------
 *  - All data pointers are DEVICE pointers owned by the caller.  The library never allocates,
 *    frees, copies to the host or synchronises.  Work is enqueued on `stream` (a hipStream_t passed
 *    as void*; NULL means the default stream) and the call returns at once.
 *  - `in`       : [N][M] fp32, dense, row-major, row stride M, read-only, 4-byte aligned.
 *                 Any M and any such alignment take vector loads.  Where the outputs are 16-byte aligned (8-byte for
 *                 16-bit values, 4-byte for byte-wide columns) rows of up to 8192 columns leave in whole groups of four
 *                 pairs, whatever k is; otherwise, and beyond 8192 columns, every pair is stored by itself.
 *  - `out_vals` : [N][k] fp32, row-major.  out_vals[r][j] is the bit pattern of in[r][out_idx[r][j]].
 *  - `out_idx`  : [N][k] column indices, 0-based, strictly ascending within a row
 *                 (int32_t, or uint8_t in the *_u8 variants, which require M <= 256: this is the
 *                 compressed row -- k values plus k byte-wide columns -- that MaxK-GNN's sparse
 *                 aggregation consumes, Section 1 / Fig. 1).
 *  - Input and output buffers must not overlap (checked on the host: RTOPK_ERR_OVERLAP).
 *  - Ties are broken towards the lower column index.
 *  - Preconditions that are NOT checked: every input is finite and |v| < FLT_MAX / 2 (so that
 *    min + max cannot overflow).  With NaN or infinities the selection is unspecified, but the call
 *    still terminates and writes only inside the output buffers.
 *  - Return value: RTOPK_OK (0) when the work was enqueued (or N == 0: nothing to do), otherwise a
 *    negative RTOPK_ERR_* code; every argument check happens on the host before any launch, and on
 *    error nothing was enqueued (but for RTOPK_ERR_LAUNCH from rtopk_select_ws, which makes several launches: the
 *    earlier ones may then run, and the outputs are to be taken as unwritten).  A pending error of the caller's own earlier HIP calls is neither
 *    reported nor cleared.  Faults of the asynchronous work surface at the caller's next
 *    synchronisation, as with any HIP launch.
 *  - Limits: 1 <= k <= M <= rtopk_max_m() = 2^24 for fp32 rows with int32 columns (65536 for rows stored
 *    in 16 bits, the dense form and the backward edge; 256 in the *_u8 variants); 0 <= N; N * M and
 *    N * k must fit in int64_t.  Rows wider than 8192 columns are handled by one workgroup per row, and
 *    then N < 2^31.  Rows wider than 65536 columns are not held on chip but streamed from memory: once
 *    when k is up to about a thousand and the winners are not crowded into one sixteenth of the row,
 *    otherwise once for the minimum and maximum, once per eight search steps and, for k in the
 *    thousands, once more to write the result; a launch of fewer such rows than twice the number of
 *    compute units leaves some of them idle, unless rtopk_select_ws (below) spreads each over several.
 */
#ifndef RTOPK_H_
#define RTOPK_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  RTOPK_OK = 0,
  RTOPK_ERR_NULL_POINTER = -1,  /* a data pointer is NULL while N > 0 */
  RTOPK_ERR_BAD_SHAPE = -2,     /* N < 0, M < 1, k < 1 or k > M */
  RTOPK_ERR_BAD_MAX_ITER = -3,  /* max_iter < 0 */
  RTOPK_ERR_M_TOO_LARGE = -4,   /* M > rtopk_max_m(); M > 65536 for 16-bit rows, dense form, backward edge; M > 256 for *_u8; more than 1024 experts */
  RTOPK_ERR_MISALIGNED = -5,    /* a pointer is not aligned to its element size */
  RTOPK_ERR_LAUNCH = -6,        /* the HIP runtime refused the launch */
  RTOPK_ERR_BAD_EPSILON = -7,   /* eps_rel is negative or NaN */
  RTOPK_ERR_OVERLAP = -8,       /* the input shares bytes with an output, or two outputs with each other */
  RTOPK_ERR_BAD_TEMPERATURE = -9, /* a temperature that is not positive and finite, or whose reciprocal is not (0 is one where tokens are drawn) */
  RTOPK_ERR_BAD_TYPE = -10      /* an element type that is none of RTOPK_F32, RTOPK_F16, RTOPK_BF16, token_bytes neither 4 nor 8, or col_bytes neither 1 nor 4 */
};

/*
 * Early-stopping selection: Algorithm 2 (Section 3.1), taken literally.
 *   lo = min(row), hi = max(row); repeat max_iter times: thres = (lo + hi) * 0.5f in fp32,
 *   cnt = #{v >= thres}, cnt < k ? hi = thres : lo = thres; emit the first k columns with v >= lo.
 * max_iter == 0 is legal and returns the first k columns.  The result is bit-identical to a scalar
 * fp32 evaluation of those steps.  Each step halves hi - lo, so after at most ~300 steps on finite fp32
 * input the rounded midpoint equals lo or hi and further steps change nothing: a max_iter above 512 is
 * run as 512, with bit-identical output (a caller may pass INT32_MAX for "no early stop").
 */
int rtopk_rowwise(const float* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, float* out_vals,
                  int32_t* out_idx, void* stream);

/*
 * Exact selection: Algorithm 1 with epsilon = 0, which Section 3.1 identifies with exact top-k.
 * The search runs until an iteration counts exactly k elements, or until no fp32 value lies strictly
 * between lo and hi; then everything >= hi is taken and the lowest columns of [lo, hi) fill up to k.
 * The result equals the plain definition of top-k with the lower column winning ties.
 */
int rtopk_rowwise_exact(const float* in, int64_t N, int32_t M, int32_t k, float* out_vals, int32_t* out_idx,
                        void* stream);

/* The same two operations writing uint8_t columns (MaxK compressed row layout); require M <= 256. */
int rtopk_rowwise_u8(const float* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, float* out_vals,
                     uint8_t* out_idx, void* stream);
int rtopk_rowwise_exact_u8(const float* in, int64_t N, int32_t M, int32_t k, float* out_vals, uint8_t* out_idx,
                           void* stream);

/*
 * Precision-bounded selection: Algorithm 1 with epsilon = eps_rel * |max(row)| (Section 3.1: epsilon
 * bounds how wide the band of undecided elements around the k-th value may stay, and with it the
 * number of steps; Appendix B, Fig. 7 sweeps it).
 * The search ends when a step counts exactly k, when hi - lo <= epsilon, or when no fp32 value lies
 * strictly between lo and hi.  Everything >= hi is then taken, and the lowest columns of [lo, hi) fill
 * up to k, so every selected value is >= (k-th largest) - epsilon and every rejected one is
 * < (k-th largest) + epsilon.  eps_rel == 0 gives exactly rtopk_rowwise_exact's output.
 *   eps_rel   : >= 0 (negative or NaN: RTOPK_ERR_BAD_EPSILON).
 *   out_iters : optional (may be NULL) device int32_t[N]; receives the exit iteration of each row's
 *               loop as Tables 1 and 5 count it: the number of midpoints evaluated when one of them
 *               counted exactly k, one more than that when the loop ended through its guard.
 */
int rtopk_rowwise_eps(const float* in, int64_t N, int32_t M, int32_t k, float eps_rel, float* out_vals,
                      int32_t* out_idx, int32_t* out_iters, void* stream);

/*
 * The k SMALLEST values per row (Section 3 states the row-wise problem for either end of the order and
 * develops the largest case only).  Defined as the two
 * operations above applied to the negated row, with the original values written out: Algorithm 2's
 * thresholds are midpoints of the negated minimum and maximum, counts are of v <= -thres.  Ties go
 * to the lower column; columns ascend; int32 columns.
 */
int rtopk_rowwise_smallest(const float* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, float* out_vals,
                           int32_t* out_idx, void* stream);
int rtopk_rowwise_exact_smallest(const float* in, int64_t N, int32_t M, int32_t k, float* out_vals, int32_t* out_idx,
                                 void* stream);

/*
 * The fp32 selections above with scratch memory from the caller.  With at least rtopk_workspace_bytes(...) bytes
 * of device memory (16-byte aligned, sharing no byte with the other buffers) rows of more than 32768 columns are
 * spread over several workgroups each, which few or very wide rows need to fill the GPU; the work is then a few launches
 * on `stream` instead of one, and the memory may be used again by later work on that stream.  Without it (NULL, too few
 * bytes, or a shape for which rtopk_workspace_bytes returns 0) the call is the plain entry point's.  Same results.
 * Memory that is enough for N rows is enough to spread any smaller number of the same rows (rtopk_workspace_bytes may
 * return more for these: with as much, they are spread over more workgroups each).
 *   variant   : RTOPK_EARLY (max_iter), RTOPK_EXACT or RTOPK_EPS (eps_rel, optional out_iters; NULL otherwise), with
 *               RTOPK_SMALLEST added for the k smallest (not with RTOPK_EPS); anything else: RTOPK_ERR_BAD_SHAPE.
 */
enum { RTOPK_EARLY = 0, RTOPK_EXACT = 1, RTOPK_EPS = 2, RTOPK_SMALLEST = 4 };
int64_t rtopk_workspace_bytes(int64_t N, int32_t M, int32_t k, int32_t variant, int32_t max_iter);
int rtopk_select_ws(const float* in, int64_t N, int32_t M, int32_t k, int32_t variant, int32_t max_iter, float eps_rel,
                    float* out_vals, int32_t* out_idx, int32_t* out_iters, void* workspace, int64_t workspace_bytes,
                    void* stream);

/*
 * Rows stored in 16 bits: IEEE half (_f16) or bfloat16 (_bf16), passed as raw uint16_t bit patterns.
 * The paper's method is defined in fp32 (Section 3.1); here each row is widened exactly to fp32 as
 * it is loaded and Algorithm 2 / Algorithm 1 (epsilon = 0) run on the widened row, with fp32
 * midpoints.  `in` is [N][M] and `out_vals` is [N][k], both 16-bit and 2-byte aligned (fastest when
 * `in` is 16-byte aligned and M is a multiple of 8); out_vals[r][j] is the bit pattern of
 * in[r][out_idx[r][j]].  Everything else is as for rtopk_rowwise / rtopk_rowwise_exact.
 */
int rtopk_rowwise_f16(const uint16_t* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, uint16_t* out_vals,
                      int32_t* out_idx, void* stream);
int rtopk_rowwise_exact_f16(const uint16_t* in, int64_t N, int32_t M, int32_t k, uint16_t* out_vals, int32_t* out_idx,
                            void* stream);
int rtopk_rowwise_bf16(const uint16_t* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, uint16_t* out_vals,
                       int32_t* out_idx, void* stream);
int rtopk_rowwise_exact_bf16(const uint16_t* in, int64_t N, int32_t M, int32_t k, uint16_t* out_vals,
                             int32_t* out_idx, void* stream);

/*
 * The MaxK non-linearity in dense form (Section 1 and Fig. 1: MaxK-GNN applies row-wise top-k to the
 * feature matrix before aggregation; Section 4.3 measures it inside MaxK-GNN training):
 *   out[r][c] = in[r][c] if column c is one of the k columns selected for row r, +0.0f otherwise.
 * The selected columns are exactly those of rtopk_rowwise_exact (max_iter < 0) or of
 * rtopk_rowwise with that max_iter (max_iter >= 0).  `in` and `out` are [N][M] fp32, dense,
 * row-major, 4-byte aligned (fastest when both are 16-byte aligned and M is a multiple of 4), and must
 * not overlap (RTOPK_ERR_OVERLAP).  One launch; the row is read once and written once, nothing else
 * touches memory.
 */
int rtopk_maxk_dense(const float* in, int64_t N, int32_t M, int32_t k, int32_t max_iter, float* out, void* stream);

/*
 * Backward edge of the MaxK non-linearity (Section 1 and Fig. 1: the row-wise top-k is the non-linearity
 * of a MaxK-GNN layer; Section 4.3 measures it inside MaxK-GNN training).  Forward, a row keeps its k
 * selected entries and every other entry becomes zero, so the derivative with respect to the row is
 * that 0/1 mask, and with the columns the forward pass saved the backward step is data movement:
 *
 *   rtopk_maxk_backward        : grad_in[r][c] = grad_vals[r][j] where c == idx[r][j], 0.0f elsewhere
 *                                (the gradient of the k kept values, scattered into the dense row);
 *   rtopk_maxk_backward_gather : grad_vals[r][j] = grad_out[r][idx[r][j]]
 *                                (the entries of a dense gradient row that flow back through the k kept values).
 *
 *   idx       : [N][k] columns as written by rtopk_rowwise* (int32_t, or uint8_t in the *_u8 variants,
 *               which require M <= 256), read-only.  Columns of a row must be distinct (any order); a
 *               column outside [0, M) is ignored by the scatter and yields 0.0f in the gather, so no
 *               index value can make the kernels touch memory outside the buffers.
 *   grad_vals : [N][k] fp32, row-major (input of the scatter, output of the gather).
 *   grad_in / grad_out : [N][M] fp32, dense, row-major (fastest when 16-byte aligned and M % 4 == 0).
 * All pointers are device pointers, 4-byte aligned (uint8 columns: any alignment); the dense array must
 * not overlap the others, and the gather's output must not overlap idx (RTOPK_ERR_OVERLAP).  One
 * launch per call; every byte of the inputs is read once and every byte of the output written once.
 */
int rtopk_maxk_backward(const float* grad_vals, const int32_t* idx, int64_t N, int32_t M, int32_t k, float* grad_in,
                        void* stream);
int rtopk_maxk_backward_u8(const float* grad_vals, const uint8_t* idx, int64_t N, int32_t M, int32_t k, float* grad_in,
                           void* stream);
int rtopk_maxk_backward_gather(const float* grad_out, const int32_t* idx, int64_t N, int32_t M, int32_t k,
                               float* grad_vals, void* stream);
int rtopk_maxk_backward_gather_u8(const float* grad_out, const uint8_t* idx, int64_t N, int32_t M, int32_t k,
                                  float* grad_vals, void* stream);

/*
 * Operators on rows of logits
 * ---------------------------
 * A row x of M logits (fp32, half or bfloat16) at temperature T stands for the distribution q_v = exp(x_v / T - lse) with
 * lse = ln sum_v exp(x_v / T).  All arithmetic is fp32 on the widened logits; a gradient is rounded once, to nearest even.  Logits may be
 * -inf (masked columns); a row of nothing but -inf has lse -inf, entropy 0, log probabilities -inf and a gradient of zero.  A row with a NaN
 * or +inf gives NaN results for itself (its alternatives' columns are then some columns of the row), and only for itself.
 *
 *   logits        : [N][M] of `dtype`, rows `stride` elements apart (stride >= M where N > 1; what lies between rows is not read),
 *                   aligned to the element.  1 <= M <= rtopk_max_m().
 *   dtype         : RTOPK_F32, RTOPK_F16 or RTOPK_BF16.
 *   temperature   : > 0, finite, as is its reciprocal (RTOPK_ERR_BAD_TEMPERATURE otherwise).
 *   workspace     : with at least rtopk_logits_workspace_bytes(...) bytes of device memory (16-byte aligned, sharing no byte with the other
 *                   buffers) few wide rows are spread over several workgroups each, in two launches (three where a gradient takes its
 *                   logits' place) instead of one; the memory may be used again by later work on that stream.  Without it (NULL, too few
 *                   bytes, or a shape for which that function returns 0) a row is one workgroup's work.  The results of both differ by rounding only.
 *   Outputs may be NULL where marked (optional).  Results do not depend on what else runs: no sum is taken in an order of chance.
 */
enum { RTOPK_F32 = 0, RTOPK_F16 = 1, RTOPK_BF16 = 2 };

/* Device memory for the calls below that take some; k: alternatives of rtopk_token_logprobs, 0 for the others. */
int64_t rtopk_logits_workspace_bytes(int64_t N, int32_t M, int32_t dtype, int32_t k);

/*
 * Log probabilities of given tokens, entropy and top alternatives; every logit is read once.
 *   tokens           : [N][G] columns, int32_t or int64_t (token_bytes 4 or 8), 0 <= G <= 1024 (NULL where G is 0).  A token outside [0, M)
 *                      is left out: its log probability is written as 0.
 *   k                : alternatives of each row, 0 <= k <= min(128, M).
 *   out_logprobs     : [N][G] fp32, ln q at the tokens (NULL where G is 0).
 *   out_entropy      : [N] fp32, -sum_v q_v ln q_v (optional).
 *   out_lse          : [N] fp32 (optional); the backward call takes it.  Finite unless the row has nothing but -inf, a NaN or +inf (beyond fp32: its last
 *                      finite number).
 *   out_top_logprobs : [N][k] fp32, ln q of the k largest logits, largest first; equal logits by ascending column (NULL where k is 0).
 *   out_top_cols     : [N][k] int32_t, their columns (NULL where k is 0).
 */
int rtopk_token_logprobs(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const void* tokens, int32_t token_bytes,
                         int32_t G, int32_t k, float temperature, float* out_logprobs, float* out_entropy, float* out_lse,
                         float* out_top_logprobs, int32_t* out_top_cols, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Gradient of the above with respect to the logits,
 *   (1 / T) (sum_g grad_logprobs_g (1[v == token_g] - q_v) - grad_entropy q_v (ln q_v + entropy)),
 * one launch; logits read once, gradient written once.  Where |lse| is above 1024 it has too few digits, and the row's sums are taken again: its logits are
 * read twice where rows are many (up to five times where they are short), by several workgroups at once where they are few.  Rows whose tokens' gradients sum
 * to zero (tokens left out have none) and whose entropy has no gradient are not read.
 *   grad_logprobs : [N][G] fp32 (NULL where G is 0).      grad_entropy : [N] fp32, or NULL: the entropy has no gradient.
 *   lse           : [N] fp32 as the forward call wrote it at the same temperature.   entropy : [N] fp32 likewise (with grad_entropy only).
 *   grad_logits   : [N][M] of `dtype`, rows grad_stride >= M apart.  It may be the logits themselves (same address and stride), which it then
 *                   replaces; any other overlap is RTOPK_ERR_OVERLAP.
 */
int rtopk_token_logprobs_backward(const float* grad_logprobs, const float* grad_entropy, const void* logits, int32_t dtype, int64_t N, int32_t M,
                                  int64_t stride, const void* tokens, int32_t token_bytes, int32_t G, const float* lse, const float* entropy,
                                  float temperature, void* grad_logits, int64_t grad_stride, void* stream);

/*
 * Distillation from a teacher's top logits: loss_n = sum_j p_j (ln p_j - ln q_{c_j}) over the row's k entries (t_j, c_j), with
 * p = softmax(t / T) over the entries that count, or p_j = exp(t_j) where log_probs is 1 (t are then log probabilities at the temperature, as
 * rtopk_token_logprobs writes them; what mass the list lacks adds nothing).  The pairs may be those of rtopk_rowwise* or of
 * rtopk_token_logprobs, in any order.  An entry whose column is outside [0, M), or whose value is -inf, does not count; a row without
 * any has loss 0 and gradient 0.  Entries with the same column add up.
 *   teacher_vals : [N][k] of teacher_dtype; teacher_cols : [N][k] int32_t; 1 <= k <= 1024.
 *   out_loss     : [N] fp32.      out_lse : [N] fp32 (optional); the backward call takes it.
 */
int rtopk_distill(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const void* teacher_vals, int32_t teacher_dtype,
                  const int32_t* teacher_cols, int32_t k, int32_t log_probs, float temperature, float* out_loss, float* out_lse,
                  void* workspace, int64_t workspace_bytes, void* stream);

/*
 * grad_loss_n dloss_n / dx_v = (grad_loss_n / T) (q_v sum_j p_j - sum_{j: c_j == v} p_j), one launch.  lse, grad_logits: as for
 * rtopk_token_logprobs_backward.  Rows without a gradient (grad_loss 0, or no entry that counts) are not read.
 */
int rtopk_distill_backward(const float* grad_loss, const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride,
                           const void* teacher_vals, int32_t teacher_dtype, const int32_t* teacher_cols, int32_t k, int32_t log_probs,
                           const float* lse, float temperature, void* grad_logits, int64_t grad_stride, void* stream);

/*
 * Both at once, for weights [N] that are known before the loss is (1 / N for a mean): out_loss as rtopk_distill's, not weighted, grad_logits as
 * rtopk_distill_backward's for grad_loss = weights.  Rows of up to 256 KiB are read once (few of more than 128 KiB, which are spread, twice), wider ones
 * twice.  A row without an entry that counts has loss 0 and gradient 0 whatever its logits are.
 */
int rtopk_distill_with_grad(const float* weights, const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride,
                            const void* teacher_vals, int32_t teacher_dtype, const int32_t* teacher_cols, int32_t k, int32_t log_probs,
                            float temperature, float* out_loss, void* grad_logits, int64_t grad_stride, void* workspace,
                            int64_t workspace_bytes, void* stream);

/*
 * Tokens drawn from rows of logits, and drafted tokens verified
 * --------------------------------------------------------------
 * Random numbers are inputs, and a result is a pure function of its inputs: what decides on a token is computed in 64 bits, in an order that
 * depends on the call's sizes only.  A row x at temperature T has probabilities p_v = exp((x_v - max x) / T) / sum; at T = 0 all of it is on the largest logit, the
 * lowest column of equal ones.  By a number u in [0, 1) it gives the lowest column v with  p_0 + ... + p_v > u  (u below 0 or NaN counts as 0; where rounding or
 * u >= 1 leaves none, the last column with p_v > 0).  A row without a distribution -- nothing but -inf, or with a NaN, or with +inf at T > 0 -- gives -1.
 *
 *   logits       : as above; rows may lie apart by any stride >= M.
 *   uniforms     : fp32 (NULL where `temperature` is 0 and temperatures is NULL).
 *   temperatures : [N] or [B] fp32 on the device, one for each sequence, or NULL: `temperature` for all.  0 is the limit above; a sequence whose
 *                  temperature is negative, infinite or NaN gets no token (-1) and no draft accepted.
 *   temperature  : 0, or finite and positive with a finite reciprocal (RTOPK_ERR_BAD_TEMPERATURE); not looked at where temperatures is given.
 *   token_bytes  : of drafts and out_tokens, 4 (int32_t) or 8 (int64_t).
 *   workspace    : as above, rtopk_verify_workspace_bytes(...) bytes, which do for any temperature (for rtopk_sample_tokens with G and draft_logits 0): few
 *                  sequences are then spread over many workgroups, in a few launches.  Drawn tokens of both ways can differ only where u lies within rounding, about 1e-13, of a border.
 */
int64_t rtopk_verify_workspace_bytes(int64_t B, int32_t G, int32_t M, int32_t dtype, int32_t draft_logits);

/* One token of each row: out_tokens [N], by uniforms [N]. */
int rtopk_sample_tokens(const void* logits, int32_t dtype, int64_t N, int32_t M, int64_t stride, const float* uniforms, const float* temperatures,
                        double temperature, void* out_tokens, int32_t token_bytes, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Verification of drafted tokens: a sequence's drafts d_0, d_1, ... are accepted from the first on while  u_i q_i(d_i) < p_i(d_i),  p_i and q_i the
 * distributions of row i of the target and of the draft model.  The first rejected one, at n, is replaced by a draw by u_G from max(p_n - q_n, 0) (from p_n where
 * that sums to no more than 2^-40); where all are accepted one more token is drawn by u_G from the row behind them.  The tokens are then distributed
 * as if drawn from the target one by one, if the drafts were drawn from q.
 *   target_logits : [B][G + 1][M], sequences target_seq_stride and their rows target_pos_stride elements apart, each >= M, in any order.
 *   draft_logits  : [B][G][M] of the same type, likewise; NULL: a draft stands for itself, q_i(d_i) = 1 (as where T is 0).  A row of nothing but -inf has q = 0.
 *   drafts        : [B][G], 0 <= G <= 128.  The first token outside [0, M) ends a sequence's drafts; nothing depends on rows behind the one that the last token is
 *                   drawn from.
 *   uniforms      : [B][G + 1].
 *   out_tokens    : [B][G + 1]: the accepted drafts, the drawn token, -1 behind it.     out_accepted : [B] int32_t, how many were accepted (optional).
 */
int rtopk_verify_drafts(const void* target_logits, const void* draft_logits, int32_t dtype, int64_t B, int32_t G, int32_t M, int64_t target_seq_stride,
                        int64_t target_pos_stride, int64_t draft_seq_stride, int64_t draft_pos_stride, const void* drafts, int32_t token_bytes,
                        const float* uniforms, const float* temperatures, double temperature, void* out_tokens, int32_t* out_accepted, void* workspace,
                        int64_t workspace_bytes, void* stream);

/*
 * A router's balance loss
 * -----------------------
 * N tokens in `groups` groups of N / groups consecutive ones (sequences, or 1: the whole batch); a token has E logits x and the k columns that a selection
 * (rtopk_rowwise*) picked for it.  A column outside [0, E) is no pick, and a token without any (padding) is left out of everything.  With p = softmax(x), n the
 * group's tokens that count, counts_e its picks of expert e, f_e = counts_e / sum counts, P_e = (1 / n) sum_t p_te:
 *   loss = E sum_e f_e P_e  (1 where picks or probabilities are even; 0 for a group without picks),      z = (1 / n) sum_t lse_t^2.
 * Sums over tokens are 64-bit, over at most 64 terms fp32.  A row of nothing but -inf has probabilities 0 and adds nothing to z; a NaN or +inf spoils
 * its group's results, and no other's.
 *   logits     : [N][E] of `dtype`, rows `stride` >= E elements apart, 1 <= E <= 1024 (RTOPK_ERR_M_TOO_LARGE beyond).
 *   cols       : [N][k], int32_t or uint8_t (col_bytes 4 or 1; bytes: E <= 256), 1 <= k <= E, in any order; the same column twice counts twice.
 *   out_loss, out_z (optional) : [groups] fp32.     out_probs (optional) : [groups][E] fp32, P.     out_counts : [groups][E] int32_t.
 *   out_rows   : [groups] int32_t, n.
 *   workspace  : as above, rtopk_balance_workspace_bytes(...) bytes.
 */
int64_t rtopk_balance_workspace_bytes(int64_t N, int32_t E, int32_t dtype, int32_t k, int32_t groups);
int rtopk_balance_loss(const void* logits, int32_t dtype, int64_t N, int32_t E, int64_t stride, const void* cols, int32_t col_bytes, int32_t k,
                       int32_t groups, float* out_loss, float* out_z, float* out_probs, int32_t* out_counts, int32_t* out_rows, void* workspace,
                       int64_t workspace_bytes, void* stream);

/*
 * Gradient of sum_g (grad_loss_g loss_g + grad_z_g z_g) + sum grad_vals . (the picked logits) with respect to the logits; the counts are constants.
 *   grad_loss  : [groups] fp32.     grad_z : [groups] fp32, or NULL.     grad_vals : [N][k] fp32, gradients of the picked values (as rtopk_maxk_backward
 *                takes them), or NULL; those of the same column add up.
 *   counts, rows : as rtopk_balance_loss wrote them (counts may be sums over several processes, whose shares then are the whole's).
 *   grad_logits  : [N][E] of `dtype`, rows grad_stride >= E apart, rounded once; zero for tokens left out.  It may be the logits themselves (same address and
 *                  stride); any other overlap is RTOPK_ERR_OVERLAP.
 */
int rtopk_balance_loss_backward(const float* grad_loss, const float* grad_z, const float* grad_vals, const void* logits, int32_t dtype, int64_t N, int32_t E,
                                int64_t stride, const void* cols, int32_t col_bytes, int32_t k, int32_t groups, const int32_t* counts, const int32_t* rows,
                                void* grad_logits, int64_t grad_stride, void* stream);

/* Human-readable text for a status code (static storage, never NULL). */
const char* rtopk_status_string(int status);

/* Library version, major * 10000 + minor * 100 + patch. */
int rtopk_version(void);

/* Largest supported row width M (fp32 rows, int32 columns). */
int rtopk_max_m(void);

#ifdef __cplusplus
}
#endif

#endif /* RTOPK_H_ */
