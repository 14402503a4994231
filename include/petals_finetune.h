/*
 * petals_finetune.h - C ABI of the client's scoring and of its ends of a fine-tuning step on one GPU.
 *
 * In distributed fine-tuning (Petals paper, Section 2.2) the servers backpropagate through frozen
 * blocks and the client owns what is trained, the loss and both ends of the chain:
 *
 *   petals_client_embed -> petals_span_prefill / _backward -> petals_client_lm_head -> loss
 *   petals_client_embed_backward <- petals_span_backward <- petals_client_lm_head_backward <- its gradient
 *
 * These calls are the second line and the loss.  They work on the client handle of petals_client.h
 * and keep its conventions (device pointers, contiguous row-major tensors, caller-owned memory,
 * a stream, error codes, petals_last_error); all but petals_client_lm_head_backward's store take
 * their scratch memory from the handle's workspace, so one handle serves one stream at a time.
 * Every call can be captured into a graph.  The same inputs give the same bits in every call.
 *
 * Logits may be -infinity (a token that is ruled out: probability 0).  A row of which no logit is
 * above -infinity has no distribution; each call says what it returns for one.  A row of logits with
 * a NaN or +infinity gives NaN for that row's real-valued results (and in-range token ids); other rows
 * are not affected.  Outputs may overlap neither inputs nor each other, but for what is said below.
 */
#ifndef PETALS_FINETUNE_H
#define PETALS_FINETUNE_H

#include "petals_client.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PETALS_LOGPROBS_TOP_MAX 64
#define PETALS_DISTILL_TOP_MAX 1024
#define PETALS_BACKWARD_ROWS_MAX (1 << 20)  /* rows of one of the two backward calls (and 2^30 tokens of any vocabulary here): above it PETALS_ERR_UNSUPPORTED */

/*
 * Log probabilities of given tokens (scoring a text, or showing what a generation was sure of).
 * With q = softmax(logits[t] / temperature):
 *   logprob_out[t]      dev fp32 [M]: log q[tokens[t]]; 0 where tokens[t] is outside [0, V) (no token given)
 *   entropy_out[t]      dev fp32 [M]: -sum_v q_v log q_v
 *   top_out[t][i]       dev int32 [M, top_k]: the token with the i-th largest logit (equal logits: lower index first)
 *   top_logprob_out     dev fp32 [M, top_k]: its log probability
 * logits: dev fp32 [M, V]; tokens: dev int32 [M], may be NULL together with logprob_out; entropy_out may be NULL; with
 * top_k = 0 the last two are NULL.  temperature at least 1e-38 and not infinite; top_k <= min(V, PETALS_LOGPROBS_TOP_MAX), above
 * PETALS_LOGPROBS_TOP_MAX -> PETALS_ERR_UNSUPPORTED.  M <= max_rows_per_call, else PETALS_ERR_CAPACITY.  Sums are held
 * in fp64.  A row without a distribution: all log probabilities -infinity, entropy 0, tokens 0, 1, 2, ...
 */
int petals_client_logprobs(petals_client *client, const float *logits, const int32_t *tokens, int32_t M,
                           float temperature, int32_t top_k, float *logprob_out, float *entropy_out,
                           int32_t *top_out, float *top_logprob_out, void *stream);

/*
 * Loss against a teacher's top logits, and its gradient.  For a row t whose list teacher_tokens[t][0..K) holds the
 * teacher's most likely tokens and teacher_logits[t][0..K) their logits:
 *   p = softmax over the list of teacher_logits[t] / temperature,  q = softmax over the vocabulary of logits[t] / temperature
 *   loss_out[t]       = temperature^2 * sum_k p_k (log p_k - log q[teacher_tokens[t][k]])
 *   grad_logits_out[t][v] = loss_grad[t] * temperature * (q_v - sum of p_k over the entries with token v)
 * (the gradient of sum_t loss_grad[t] * loss_out[t]).  With K = 1 and temperature 1 this is cross-entropy with hard labels.
 *   logits            dev fp32 [M, V]
 *   teacher_tokens    dev int32 [M, K]; an entry outside [0, V) is not part of the list (lists of different lengths,
 *                     positions that are not trained on); a token may stand in a list more than once
 *   teacher_logits    dev fp32 [M, K]
 *   loss_grad         dev fp32 [M], NULL: 1
 *   loss_out          dev fp32 [M], may be NULL if grad_logits_out is given
 *   grad_logits_out   dev fp32 [M, V], may be NULL if loss_out is given; may be the same memory as logits
 * A NaN or +infinity among a row's teacher_logits makes its loss and the gradients of the listed tokens NaN.
 * A row without a list (no entry, or all teacher logits -infinity) has loss 0 and gradient 0.  A row without a distribution
 * of its own (and with a list) has loss +infinity and gradient 0.  1 <= K <= PETALS_DISTILL_TOP_MAX, above it
 * PETALS_ERR_UNSUPPORTED; temperature at least 1e-38 and not infinite; M <= max_rows_per_call, else PETALS_ERR_CAPACITY.
 */
int petals_client_distill(petals_client *client, const float *logits, int32_t M, const int32_t *teacher_tokens,
                          const float *teacher_logits, int32_t K, float temperature, const float *loss_grad,
                          float *loss_out, float *grad_logits_out, void *stream);

/*
 * Backward of petals_client_lm_head: the gradient with respect to its hidden states.
 *   grad_hidden_out[t] = J_t (sum_v grad_logits[t][v] * embeddings[v]),  J_t the derivative of the final LayerNorm at hidden_in[t]
 *   hidden_in         dev fp16 [M, H]: what petals_client_lm_head was given
 *   grad_logits       dev fp32 [M, V], finite
 *   grad_hidden_out   dev fp16 [M, H]: grad_out of petals_span_backward
 * (The roundings of the forward pass count as the identity; matrix and LayerNorm parameters are frozen.)  The product runs on
 * fp16 matrix instructions with fp32 sums; grad_logits is taken as two fp16 values for calls of up to
 * PETALS_HEAD_BACKWARD_PAIR_ROWS rows and as one beyond, scaled per row and section of the vocabulary (1024 columns, beyond
 * those rows 2048) so that the section's largest value is exact and one value rounds by at most 2^-11 of itself down to 2^-29 of
 * the largest, two by 2^-22 down to 2^-18.  grad_hidden_out is rounded to
 * fp16 once, without loss scaling (loss_grad of petals_client_distill can carry a scale).
 * dev_store: 256-byte aligned device memory of petals_client_lm_head_backward_bytes(cfg, M) bytes, contents unspecified
 * before and after.  (That many for a call of M rows: one of fewer rows may need more, being cut up in another way, so a store that
 * serves calls of several sizes has the most that any of them asks for.)  M <= max_rows_per_call, else PETALS_ERR_CAPACITY.
 */
#define PETALS_HEAD_BACKWARD_PAIR_ROWS 64
int petals_client_lm_head_backward_bytes(const petals_client_config *cfg, int32_t M, size_t *bytes);
int petals_client_lm_head_backward(petals_client *client, void *dev_store, const void *hidden_in,
                                   const float *grad_logits, int32_t M, void *grad_hidden_out, void *stream);

/*
 * Backward of petals_client_embed: the gradient with respect to the looked-up rows of the embedding matrix (for prompt
 * tuning: of a client whose matrix is the table of prompt vectors), one row for each DIFFERENT token of the call.
 *   token_ids         dev int32 [M], as given to petals_client_embed (an id outside [0, V) counts as the clamped one)
 *   grad_hidden       dev fp16 [M, H]: grad_in of petals_span_backward
 *   tokens_out        dev int32 [M]: the different tokens in ascending order
 *   grads_out         dev fp32 [M, H]: row i = the gradient of embeddings[tokens_out[i]], through the LayerNorm behind the lookup
 *   count_out         dev int32 [1]: how many there are; entries of the two outputs from there on are left as they were
 * The rows of a token are summed in fp32 in an order that depends on H and on their number alone, then go through the
 * derivative of the LayerNorm once.  M <= max_rows_per_call, else PETALS_ERR_CAPACITY.
 */
int petals_client_embed_backward(petals_client *client, const int32_t *token_ids, const void *grad_hidden, int32_t M,
                                 int32_t *tokens_out, float *grads_out, int32_t *count_out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PETALS_FINETUNE_H */
