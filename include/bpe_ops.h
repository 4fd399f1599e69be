/* Operators on token batches: the two ends of a language model that is trained on or scored over what
 * bpe_encode_batch writes.  A batch is packed as the encoder packs it: int32 ids back to back, int64 offsets[batch+1].
 *
 *   bpe_embed_tokens, bpe_embed_tokens_grad            rows of an embedding, and their gradient by sorted tokens
 *   bpe_next_tokens                                    what each position is to predict
 *   bpe_token_logprobs, .._grad, .._and_grad           log-probabilities of tokens from logits, and the logits' gradient
 *   bpe_preference_loss, bpe_policy_loss               two losses over strings, with the logits' gradient
 *
 * Every function returns one of the BPE_* codes of bpe.h and none throws.  All only enqueue kernels on `stream` (a hipStream_t
 * as void*, NULL = the default stream): no synchronisation, no allocation, no host reads of device data, so that they can be
 * captured in a HIP graph.  Arguments are checked before anything is enqueued (BPE_EINVAL: null pointers with non-zero sizes,
 * negative sizes, unknown types, strides below a row's length, pointers not aligned to their type, a short or misaligned
 * workspace); BPE_EHIP if the runtime refuses a launch, with outputs then unspecified.  Pointers are DEVICE pointers of the
 * current device unless marked HOST.  Workspaces are caller-owned, 256-byte aligned, need not be initialised and are garbage
 * afterwards; calls that overlap in time need one each.
 *
 * Matrices are row-major with a stride between rows, in elements, of at least the row's length; pointers need be aligned to
 * their elements only.  Sums, maxima and losses are held in 32 bits or more and rounded once, to the type of the output.
 * Results do not depend on the order in which workgroups run: equal calls give equal bits.
 */
#ifndef BPE_OPS_H_
#define BPE_OPS_H_

#include "bpe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of matrices. */
enum { BPE_F32 = 0, BPE_BF16 = 1, BPE_F16 = 2 };

/* Ids and rows, 0 <= n <= BPE_MAX_TOKENS; columns, 1 <= vocab, dim <= BPE_MAX_COLUMNS.  (Their products may pass 2^32.) */
#define BPE_MAX_TOKENS 0x3fffffff
#define BPE_MAX_COLUMNS 0x1fffffff
/* Strings of the losses: 0 <= batch <= BPE_MAX_STRINGS. */
#define BPE_MAX_STRINGS 0xffffff

/* out[t] = scale * weight[ids[t]], t < n.  An id outside [0, vocab) -- padding -- gives a row of zeros.
 *   weight  [vocab][dim] of `dtype`;  out [n][dim] of the same type, not overlapping weight.
 *   count   one int64, or NULL: if given, rows from min(n, *count) on are left as they are (the encoder's
 *           out_offsets + batch says how many of its ids there are, and need not be fetched for it). */
int bpe_embed_tokens(const void* weight, int dtype, int64_t vocab, int64_t dim, int64_t weight_stride, const int32_t* ids,
                     int64_t n, const int64_t* count, float scale, void* out, int64_t out_stride, void* stream);

/* grad_weight[v] = scale * (sum of grad[t] over all t with ids[t] = v), for every row v, those that no id names (zeros)
 * among them; with `accumulate` != 0 it is added to what grad_weight holds, and rows that no id names are not touched.
 *   grad         [n][dim] of `dtype`; rows whose id is outside [0, vocab), and those from *count on, are not read.
 *   grad_weight  [vocab][dim] of `out_dtype`: BPE_F32 or `dtype`; not overlapping grad.
 * Each row's terms are added in an order that the ids alone determine. */
int bpe_embed_tokens_grad(const void* grad, int dtype, int64_t grad_stride, const int32_t* ids, int64_t n,
                          const int64_t* count, int64_t vocab, int64_t dim, float scale, int accumulate, void* grad_weight,
                          int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream);
/* Bytes of its workspace; 0 for sizes that are out of range. */
size_t bpe_embed_tokens_grad_workspace_bytes(int64_t n, int64_t vocab, int64_t dim);

/* targets[t] = ids[t+1] where t and t+1 belong to one string i (offsets[i] <= t, t+1 < offsets[i+1]) and t+1 is not among
 * the string's first first[i] tokens (a prompt, which is given and not predicted); else -1: "not scored".
 *   offsets  int64[batch+1], non-decreasing; positions outside every string are not scored.
 *   first    int32[batch], or NULL: none.
 *   n        number of ids and targets; ids from offsets[batch] on are not read. */
int bpe_next_tokens(const int32_t* ids, int64_t n, const int64_t* offsets, int32_t batch, const int32_t* first,
                    int32_t* targets, void* stream);

/* logprobs[t] = logits[t][targets[t]] - lse[t], lse[t] = log(sum over j of exp(logits[t][j])).
 * A row whose target is outside [0, vocab) is not scored: it is not read, whatever it holds, and both outputs are 0.
 * Logits of -inf (masked entries) have probability 0; a row without any finite one has no distribution, and gives NaN.
 *   logits  [n][vocab] of `dtype`;  logprobs, lse float[n], either may be NULL.
 *   workspace  may be NULL where none is needed. */
int bpe_token_logprobs(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                       float* logprobs, float* lse, void* workspace, size_t workspace_bytes, void* stream);
/* Bytes of its workspace: 0 where it needs none (only few rows that are long are split among workgroups). */
size_t bpe_token_logprobs_workspace_bytes(int64_t n, int64_t vocab);

/* The gradient with respect to the logits of sum over t of upstream[t] * logprobs[t]:
 *   grad[t][j] = upstream[t] * ((j == targets[t]) - exp(logits[t][j] - lse[t])).
 * Rows that are not scored, and rows whose upstream is 0, get zeros and are not read.
 *   lse   as bpe_token_logprobs wrote it: 32 bits, which is 1e-6 of the gradient for logits of some tens and nothing left of
 *         it for logits of 10^7 (the one-pass form and the losses below keep the maximum and the sum apart, and have no such limit).
 *   grad  [n][vocab] of the logits' type; may be the logits themselves (same pointer and stride), else not overlapping. */
int bpe_token_logprobs_grad(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                            const float* lse, const float* upstream, void* grad, int64_t grad_stride, void* stream);

/* Both in one pass over the logits, for weights that are known before (cross entropy: upstream = -1 / scored tokens).
 * A scored row whose upstream is 0 is read for its log-probability, and its gradient is zeros. */
int bpe_token_logprobs_and_grad(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride,
                                const int32_t* targets, const float* upstream, float* logprobs, float* lse, void* grad,
                                int64_t grad_stride, void* stream);

/* Bytes of workspace that the two losses need; 0 for sizes that are out of range. */
size_t bpe_loss_workspace_bytes(int64_t n, int64_t vocab, int32_t batch);

/* Preference loss on pairs: string 2k is preferred to string 2k+1.  With S_i the sum of logprobs[t] - reference[t] over the
 * scored positions t of string i,
 *   margins[k] = beta * (S_2k - S_2k+1),
 *   loss = mean over k of -(1 - smoothing) log sigmoid(margins[k]) - smoothing log sigmoid(-margins[k]).
 *   offsets    int64[batch+1], batch even; string i is rows offsets[i] .. offsets[i+1) of the logits.
 *   reference  float[n], or NULL (zeros): the reference model's logprobs; not read where a row is not scored.
 *   scale      factor of the gradient (loss scaling, weight of the loss); the loss itself is not scaled.
 *   loss       one float; 0 for no pairs.  margins float[batch/2], logprobs float[n]: either may be NULL.
 *   grad       as above; rows outside every string get zeros (and have logprobs all the same).  A string without scored
 *              positions has S = 0.  A masked target makes S -inf: its pair adds 0 or infinity to the loss (a term whose
 *              weight is 0 is left out), and where it adds 0 its gradient is 0. */
int bpe_preference_loss(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                        const int64_t* offsets, int32_t batch, const float* reference, float beta, float smoothing,
                        float scale, float* loss, float* margins, float* logprobs, void* grad, int64_t grad_stride,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Clipped policy loss with a KL term.  For a scored position t, with r = exp(logprobs[t] - old[t]) and its advantage A,
 *   l_t = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_weight (exp(d) - d - 1),  d = reference[t] - logprobs[t],
 * and loss = sum of w_t l_t, where w_t = 1 / (scored positions of the batch) or, with `by_string`, 1 / (batch * scored
 * positions of its string).  Where the clipped term is the smaller one the gradient has no part of it.
 *   advantages  float[n], or float[batch] with advantage_by_string != 0: one for all of a string.
 *   reference   float[n], or NULL: no KL term, and none where kl_weight is 0.
 *   old, reference and advantages are not read where a row is not scored; positions outside every string are not scored.
 *               A NaN in those of a scored row, or for its log-probability, makes the loss NaN and the row's gradient; an
 *               advantage of 0 has no part in the loss, whatever the ratio, unless that is NaN.
 *   scale, loss, logprobs, grad  as for bpe_preference_loss (but logprobs are 0 outside every string); loss = 0 where nothing
 *                                is scored. */
int bpe_policy_loss(const void* logits, int dtype, int64_t n, int64_t vocab, int64_t stride, const int32_t* targets,
                    const int64_t* offsets, int32_t batch, const float* old, const float* advantages,
                    int advantage_by_string, const float* reference, float clip_low, float clip_high, float kl_weight,
                    int by_string, float scale, float* loss, float* logprobs, void* grad, int64_t grad_stride,
                    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BPE_OPS_H_ */
