/* Operators at the output end of a language model over the encoder's tokens: from hidden states to logits that a token is chosen
 * from.
 *
 *   bpe_add_norm, bpe_add_norm_grad        root-mean-square norm of a sum with the residual, and its gradient
 *   bpe_add_norm_8bit, bpe_quantize_rows   rows of 8-bit integers with a scale each, of such a norm or of a matrix
 *   bpe_project_8bit                       logits from 8-bit rows and 8-bit weights
 *   bpe_adjust_logits, .._grad             penalties for tokens that a string already holds, biases, a grammar's masks
 *
 * Codes, streams, types, sizes, strides, alignment, workspaces and overlapping calls are as for bpe_ops.h.  Matrices of 8-bit
 * integers may have any alignment.  Equal calls give equal bits.
 */
#ifndef BPE_HEAD_H_
#define BPE_HEAD_H_

#include "bpe_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* summed[t] = x[t] + residual[t], rounded to the type; the norm is of that, or of x itself without a residual:
 *   s = summed[t],  rstd[t] = 1 / sqrt(mean over j of s_j^2 + eps),  out[t][j] = s_j * rstd[t] * weight[j].
 *   x, residual, summed, out   [n][dim] of `dtype`; residual and summed may both be NULL.  summed may be x or the residual, and out
 *                              x or the residual, but not summed (same pointer and stride); else nothing that is written overlaps
 *                              anything.
 *   weight  [dim] of weight_dtype: BPE_F32 or `dtype`;  rstd float[n], or NULL.
 *   eps     >= 0.  A row of zeros with eps = 0 gives NaN, as does a row with a NaN; one with infinities gives NaN where they are, else 0.
 *           Of rows whose root mean square is below 2^-128 (with eps = 0) rstd is infinite; out is the formula's all the same. */
int bpe_add_norm(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride,
                 const void* weight, int weight_dtype, float eps, void* summed, int64_t summed_stride, float* rstd, void* out,
                 int64_t out_stride, void* stream);

/* The same norm in 8 bits: with p_j = s_j weight[j], a = max over j of |p_j|,
 *   q[t][j] = 127 p_j / a to the nearest integer, ties to even;  scales[t] = a rstd[t] / 127:  scales[t] q[t][j] stands for out[t][j].
 * Quotients are rounded as if they were exact to 64-bit arithmetic.  Where a = 0 the row and its scale are 0; where a row or the
 * weights hold an infinity or NaN, the row is 0 and its scale NaN.
 *   q  int8 [n][dim], overlapping nothing. */
int bpe_add_norm_8bit(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, const void* residual, int64_t residual_stride,
                      const void* weight, int weight_dtype, float eps, void* summed, int64_t summed_stride, int8_t* q,
                      int64_t q_stride, float* scales, void* stream);

/* The gradients of a norm.  With u_j = grad[t][j] weight[j], h_j = s_j rstd[t] and m = mean over j of u_j h_j,
 *   grad_x[t][j] = rstd[t] (u_j - h_j m) + grad_summed[t][j],   which is the residual's gradient as well;
 *   grad_weight[j] = sum over t of grad[t][j] h_j, with `accumulate` != 0 added to what it holds.
 *   grad, summed (x where there was no residual), grad_x  [n][dim] of `dtype`;  rstd as bpe_add_norm wrote it (of a row whose rstd is
 *   infinite the gradients are no numbers).
 *   grad_summed  of the same, or NULL: zeros.  grad_x may be grad or grad_summed (same pointer and stride), else overlaps nothing.
 *   grad_weight  [dim] of grad_weight_dtype: BPE_F32 or weight_dtype; or NULL: not wanted, and no workspace needed. */
int bpe_add_norm_grad(const void* grad, int dtype, int64_t n, int64_t dim, int64_t grad_stride, const void* summed,
                      int64_t summed_stride, const void* weight, int weight_dtype, const float* rstd, const void* grad_summed,
                      int64_t grad_summed_stride, void* grad_x, int64_t grad_x_stride, void* grad_weight, int grad_weight_dtype,
                      int accumulate, void* workspace, size_t workspace_bytes, void* stream);
/* Bytes of its workspace; 0 for sizes that are out of range. */
size_t bpe_add_norm_grad_workspace_bytes(int64_t n, int64_t dim);

/* Rows in 8 bits: a = max over j of |x[t][j]|, q[t][j] = 127 x[t][j] / a, scales[t] = a / 127; everything as for bpe_add_norm_8bit. */
int bpe_quantize_rows(const void* x, int dtype, int64_t n, int64_t dim, int64_t stride, int8_t* q, int64_t q_stride, float* scales,
                      void* stream);

/* out[t][v] = (sum over k of q[t][k] weight[v][k]) * scales[t] * weight_scales[v]; the sum is exact, then it and both products are rounded
 * to 32 bits, in this order.
 *   q       int8 [n][dim], dim <= BPE_MAX_DIM_8BIT (the sum fits 32 bits);  scales float[n]
 *   weight  int8 [vocab][dim];  weight_scales float[vocab]
 *           both with a stride of at most BPE_MAX_STRIDE_8BIT
 *   out     [n][vocab] of `dtype`, overlapping nothing; n * vocab <= 10^13.
 * Rows that begin at multiples of 4 bytes and have a multiple of 4 columns are read fastest, at multiples of 128 bytes more so. */
#define BPE_MAX_DIM_8BIT 131071
#define BPE_MAX_STRIDE_8BIT 0xfffffe
int bpe_project_8bit(const int8_t* q, int64_t n, int64_t dim, int64_t q_stride, const float* scales, const int8_t* weight,
                     int64_t vocab, int64_t weight_stride, const float* weight_scales, void* out, int dtype, int64_t out_stride,
                     void* stream);

/* Logits as a token is chosen from.  The history of row t is ids[begin[t]] .. ids[end[t] - 1] (bounds outside [0, n_ids] are taken
 * to be 0 and n_ids; ids outside [0, vocab) are padding and count nowhere): a packed batch's string with offsets and offsets + 1,
 * what is before a position with its string's offset and the position, a row of a buffer with its beginning and its length so far.
 * For x = logits[t][v], c the number of times that v is in the history, in this order:
 *   c > 0:  x = x > 0 ? x / repetition : x * repetition;  x = x - (presence + frequency * c)      (divided by the rounded reciprocal)
 *   v is bias_ids[i] for an i in bias_begin[t] .. bias_end[t] - 1:  x = x + bias_values[i]; of several such i the last one counts
 *   bit v % 32 of mask[state[t]][v / 32] is 0:  x = -infinity, whatever it was.
 *   penalties   float[n][3]: repetition (2^-126 to 2^126), presence and frequency of each row; or NULL: those given for all rows.
 *   ids         int32[n_ids]; begin, end int64[n].  begin and end may be NULL: no history.  (Of a history or a list of biases the first
 *               0xfffffff0 are looked at.)
 *   bias_ids, bias_values   int32 and float [n_biases]; bias_begin, bias_end int64[n], bounds as above; both may be NULL: no biases.
 *   mask        int32 [states][mask_stride], mask_stride >= (vocab + 31) / 32 words; or NULL: none.
 *   state       int32[n], each row's mask; a row whose state is outside [0, states) has none.  NULL: row t has mask t (states = n), or
 *               all have the only one (states = 1).
 *   out         [n][vocab] of `dtype`; may be the logits (same pointer and stride), else overlaps nothing.  In place only stretches of
 *               16 bytes in which something changes are written, and read.
 * A mask may leave nothing of a row: it is -infinity throughout. */
int bpe_adjust_logits(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* ids, int64_t n_ids,
                      const int64_t* begin, const int64_t* end, const float* penalties, float repetition, float presence,
                      float frequency, const int32_t* bias_ids, const float* bias_values, int64_t n_biases,
                      const int64_t* bias_begin, const int64_t* bias_end, const int32_t* mask, int64_t states, int64_t mask_stride,
                      const int32_t* state, void* out, int64_t out_stride, void* stream);

/* The gradient with respect to the logits, from that of what bpe_adjust_logits wrote: 0 where the mask's bit is 0, else grad[t][v],
 * and where v is in the history, grad[t][v] / repetition for logits[t][v] > 0 and grad[t][v] * repetition for others.
 *   logits  as they were before; only those of tokens in histories matter, and with them up to 16 bytes of their row about each are read.
 *   out     [n][vocab] of `dtype`; may be grad (same pointer and stride), else overlaps nothing. */
int bpe_adjust_logits_grad(const void* grad, int dtype, int64_t n, int64_t vocab, int64_t grad_stride, const void* logits,
                           int64_t stride, const int32_t* ids, int64_t n_ids, const int64_t* begin, const int64_t* end,
                           const float* penalties, float repetition, const int32_t* mask, int64_t states, int64_t mask_stride,
                           const int32_t* state, void* out, int64_t out_stride, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BPE_HEAD_H_ */
