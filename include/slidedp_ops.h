/*
 * slidedp_ops.h -- operators of the fine-tuning pass that produces the gradients of slidedp.h:
 * the token embedding, the norms around a block with its gate and residual, the query / key norms
 * with the position rotation, attention over packed documents, distillation from a teacher's top
 * logits and the clipped policy loss, each with its gradient, and clipping by the norm over many
 * gradient tensors. (Not part of the paper, whose Sec. 3.1 takes the layers' forward and backward
 * pass as given; its workloads, Sec. 4.1, are the decoder layers these operators belong to.)
 *
 * Conventions are those of slidedp.h: every call returns SLIDEDP_OK or a negative status and only
 * enqueues work on cuda_stream; the caller owns every buffer, workspaces included; nothing is kept
 * between calls. Results are bit-reproducible: no call adds floating-point numbers with atomics.
 * Calls of this header on one context may go to different streams and come from different threads, also at once (but not
 * beside other calls on that context); workspaces must not be shared by calls that can overlap.
 *
 * The attention, distillation, block-norm and policy-step kernels wait on copies and on blocks of their own launch; every
 * such wait is bounded (about a minute). If one runs out, the results of that call are not complete, and the first of these calls on the
 * context to start after that returns SLIDEDP_ERR_TIMEOUT, once, and does nothing else: any operator of this header; a
 * slidedp_grad_norm_finish or slidedp_grad_norm_finish_from that fetches its results (they are fetched all the same); or
 * slidedp_destroy (which still destroys). A call's own kernels have only been queued when it returns: to know that a step's
 * gradients are complete before they are used, fetch the norm, which waits for the kernels queued before it.
 *
 * BF16 and FP32 tensors need the alignment of their element only; 16-byte aligned bases and
 * strides are faster. All sums, norms and softmax statistics are FP32 and each output is rounded
 * once (attention multiplies some intermediates as BF16: see there). Sizes of zero are no-ops. Factors given as doubles
 * (scale, softcap, temperature, weights, eps) are used as FP32: ones that FP32 makes infinite, or makes zero where they must
 * be positive, are refused.
 */
#ifndef SLIDEDP_OPS_H
#define SLIDEDP_OPS_H

#include "slidedp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SLIDEDP_BF16 = 0, SLIDEDP_F32 = 1 } slidedp_dtype;

/* A device tensor [tokens, heads, head_dim] whose last axis is contiguous: element (t, h, d) is
 * data[t * stride_token + h * stride_head + d], strides in elements, none negative. Views of a
 * fused projection's output are of this form. Outputs must not overlap themselves. */
typedef struct {
  void* data;
  int64_t stride_token, stride_head;
} slidedp_heads;

/* ---- query / key norms with the position rotation -------------------------------------------
 *
 * For each token t and head h of q and of k, with x = the head's head_dim values:
 *   n = x * rsqrt(mean(x^2) + eps) * w            (w = w_q or w_k; NULL: ones)
 *   y = n with the pairs (a, b) of its first rope_dim values turned by the token's angles:
 *       (a cos - b sin, b cos + a sin)
 * interleaved = 0 pairs value p with p + rope_dim / 2, 1 pairs 2p with 2p + 1. cos_sin: device,
 * table_rows rows of rope_dim floats, the rope_dim / 2 cosines before the sines. positions: device,
 * one row index per token (NULL: token t uses row t, so tokens <= table_rows). A token whose
 * position lies outside the table gets NaN in its rotated values (and, backward, in its gradients,
 * hence in dw). head_dim 1..256, rope_dim even, 0..head_dim; heads_q or heads_k may be 0; at most 2^31 - 1 rows
 * (tokens * heads) of each.
 * q, k, w_q, w_k and the outputs have the type `dtype`.
 *
 * Backward: dq, dk are the gradients of q and k, dw_q and dw_k (device, head_dim floats each,
 * nullable) those of the weights, from the gradients dq_out, dk_out of the outputs. The forward's
 * inputs are needed, its outputs are not. y may be x and dq may be dq_out (same address and
 * strides; the same address with other strides is refused), but outputs may not overlap otherwise.
 * workspace: device, slidedp_qk_norm_rope_workspace bytes, 16-byte aligned.
 */
typedef struct {
  int64_t tokens;
  int32_t heads_q, heads_k, head_dim, rope_dim;
  int32_t interleaved;
  int32_t dtype; /* slidedp_dtype */
  int64_t table_rows;
  double eps;
} slidedp_qk_args;

SLIDEDP_API int slidedp_qk_norm_rope(slidedp_ctx* ctx, const slidedp_qk_args* args, const slidedp_heads* q,
                         const slidedp_heads* k, const void* w_q, const void* w_k, const float* cos_sin,
                         const int32_t* positions /* nullable */, const slidedp_heads* q_out,
                         const slidedp_heads* k_out, void* cuda_stream);
SLIDEDP_API int slidedp_qk_norm_rope_backward(slidedp_ctx* ctx, const slidedp_qk_args* args,
                                  const slidedp_heads* q, const slidedp_heads* k, const void* w_q,
                                  const void* w_k, const float* cos_sin, const int32_t* positions,
                                  const slidedp_heads* dq_out, const slidedp_heads* dk_out,
                                  const slidedp_heads* dq, const slidedp_heads* dk, float* dw_q,
                                  float* dw_k, void* workspace, void* cuda_stream);
/* 0 for arguments that the call would refuse. */
SLIDEDP_API size_t slidedp_qk_norm_rope_workspace(const slidedp_qk_args* args);

/* ---- attention over packed documents ---------------------------------------------------------
 *
 * q: [tokens, heads_q, head_dim], k and v: [tokens, heads_kv, head_dim], BF16; heads_q is a
 * multiple of heads_kv and query head h reads key head h / (heads_q / heads_kv).
 *   s_ij = scale * q_i . k_j;  with softcap > 0: s = softcap * tanh(s / softcap);
 *   with slopes (device, heads_q floats): s -= slopes[h] * |i - j|
 *   out_i = sum_j softmax_j(s_ij) v_j,   lse[h * tokens + i] = log sum_j exp(s_ij)
 * over the keys j that query i sees: those of its own document, and if causal those with j <= i or
 * among the first prefix[d] tokens of the document (device, docs values, nullable; only read if
 * causal). cu_docs: device, docs + 1 ascending token offsets, document d being
 * [cu_docs[d], cu_docs[d + 1]); NULL: one document of all tokens (docs is then 1). A token outside
 * every document sees nothing: out = 0, lse = -inf, and its gradients are 0. Offsets are
 * clamped to [0, tokens]; results for descending ones are undefined but nothing is accessed
 * outside the tensors. head_dim 1..256.
 *
 * What a query does not see does not touch its results, whatever it holds: NaN and infinities in other documents, in later
 * keys, in padding. What it sees and is NaN makes its out and lse NaN.
 *
 * With head_dim a multiple of 8 up to 128 and 16-byte aligned views the products run on the tensor cores, with BF16 operands:
 * the probabilities exp(s - max) for out and those of the backward pass for dv, and the gradients of the scores for dq and dk, are
 * rounded to BF16 (each by at most 2^-8 of itself); their sums, the scores, lse, maxima and accumulators are FP32. The backward
 * pass takes the rows' sums of out * d_out from the BF16 `out`. Against arithmetic in 64 bits, with the output's own rounding
 * (0.0017 in the 2-norm), out is off by 0.0020 and the gradients by 0.0024 to 0.0027. A quarter of the forward pass's exponentials
 * are a polynomial (relative error 3e-6). With softcap, tanh is a polynomial where all scores of 32 neighbouring rows and a tile of
 * keys, masked ones included, are below 0.7 of the cap, and made of an exponential elsewhere: both are accurate to FP32's 2^-23,
 * but the last bits of a row may depend on which it was. Other views and head sizes compute in FP32 throughout, one warp per
 * row (2048 tokens, 8 heads of 256: 4.2 ms forward, 12.4 ms backward; of 128 on the tensor cores 33 and 41 us).
 *
 * Backward: the gradients of q, k and v from d_out (the gradient of out), with the forward's out
 * and lse. The slopes are constants and have none. workspace: device,
 * slidedp_attention_workspace bytes, 16-byte aligned.
 *
 * In both directions no output may overlap an input or another output: the kernels read inputs, also of other rows and heads,
 * while they write (in the backward pass two of them at a time). Views that start at the same address are refused.
 */
typedef struct {
  int64_t tokens;
  int32_t heads_q, heads_kv, head_dim;
  int32_t causal;
  int32_t docs;
  int32_t reserved;
  const int32_t* cu_docs;
  const int32_t* prefix;
  const float* slopes;
  double scale, softcap;
} slidedp_attn_args;

SLIDEDP_API int slidedp_attention(slidedp_ctx* ctx, const slidedp_attn_args* args, const slidedp_heads* q,
                      const slidedp_heads* k, const slidedp_heads* v, const slidedp_heads* out,
                      float* lse, void* cuda_stream);
SLIDEDP_API int slidedp_attention_backward(slidedp_ctx* ctx, const slidedp_attn_args* args,
                               const slidedp_heads* q, const slidedp_heads* k, const slidedp_heads* v,
                               const slidedp_heads* out, const float* lse, const slidedp_heads* d_out,
                               const slidedp_heads* dq, const slidedp_heads* dk,
                               const slidedp_heads* dv, void* workspace, void* cuda_stream);
/* 0 for arguments that the call would refuse. */
SLIDEDP_API size_t slidedp_attention_workspace(const slidedp_attn_args* args);

/* ---- distillation from a teacher's top logits ------------------------------------------------
 *
 * For each row (token) r with the student's logits z[0..vocab), the teacher's stored entries
 * (ids[k], t[k]), k < entries, and its hard label:
 *   q = softmax(t / temperature) over the stored entries;  p = softmax(z / temperature)
 *   loss = w_teacher * temperature^2 * sum_k q_k (log q_k - log p[ids[k]])
 *        + w_label * (logsumexp(z) - z[label])
 * An entry whose id, or a label, lies outside [0, vocab) is absent (padding, prompt tokens): a row
 * with no entries has no teacher term, one without label no label term. Repeated ids of a row add
 * up. An entry with q_k = 0 contributes nothing, whatever its p. logits: [rows, vocab] of `dtype`,
 * logits_stride elements from row to row; teacher_ids: [rows, entries] int32, teacher_logits:
 * [rows, entries] floats, both contiguous (entries 0..512); labels: rows int32, nullable.
 * loss: rows floats. lse: 2 * rows floats: logsumexp(z / temperature) of every row, then
 * logsumexp(z) of every row (zeros there if w_label is 0 or labels NULL: the term is off).
 *
 * Gradient: d_logits[r] = row_grad[r] * d loss[r] / d z, with row_grad: rows floats (nullable: ones).
 * slidedp_distill_loss_backward takes the forward's lse (probabilities from it have the relative error of its rounding, up to
 * 8e-6; rows with an lse beyond 128, where that would be more, are summed again); slidedp_distill_step computes loss, lse and
 * gradient in one call that reads the logits once. d_logits may be the logits themselves (same
 * address and stride; the same address with another stride is refused).
 */
typedef struct {
  int64_t rows, vocab;
  int32_t entries;
  int32_t dtype; /* slidedp_dtype of logits and d_logits */
  int64_t logits_stride, d_logits_stride;
  double temperature, w_teacher, w_label;
} slidedp_distill_args;

SLIDEDP_API int slidedp_distill_loss(slidedp_ctx* ctx, const slidedp_distill_args* args, const void* logits,
                         const int32_t* teacher_ids, const float* teacher_logits, const int32_t* labels,
                         float* loss, float* lse, void* cuda_stream);
SLIDEDP_API int slidedp_distill_loss_backward(slidedp_ctx* ctx, const slidedp_distill_args* args,
                                  const void* logits, const int32_t* teacher_ids,
                                  const float* teacher_logits, const int32_t* labels, const float* lse,
                                  const float* row_grad, void* d_logits, void* cuda_stream);
SLIDEDP_API int slidedp_distill_step(slidedp_ctx* ctx, const slidedp_distill_args* args, const void* logits,
                         const int32_t* teacher_ids, const float* teacher_logits, const int32_t* labels,
                         const float* row_grad, float* loss, float* lse, void* d_logits,
                         void* cuda_stream);

/* ---- token embedding -------------------------------------------------------------------------
 *
 * A device matrix whose last axis is contiguous: element (r, c) is data[r * stride + c], the stride in
 * elements and not negative. Rows of an output do not overlap. */
typedef struct {
  void* data;
  int64_t stride;
} slidedp_rows;

/*   out[t] = scale * table[ids[t]]                          table: [vocab, hidden], out: [tokens, hidden] of `dtype`
 *   d_table[v] = scale * sum of d_out[t] over the t with ids[t] = v     d_out of `dtype`, d_table of `grad_dtype`
 * ids: device, one int32 per token. A token whose id lies outside [0, vocab) is absent (padding): its row of out is zeros,
 * its row of d_out is not read. accumulate = 0 writes all of d_table, zeros for ids that no token has; 1 adds to what
 * d_table holds, and touches only the rows of ids that occur. The sum over a row's tokens is FP32 in an order that follows
 * from the ids and the sizes, scaled and (with what was there) rounded once. d_table may not overlap d_out, nor out the table.
 * tokens and vocab up to 2^30, hidden up to 2^20.
 * workspace: device, slidedp_embedding_workspace bytes, 16-byte aligned.
 */
typedef struct {
  int64_t tokens, vocab, hidden;
  int32_t dtype, grad_dtype; /* slidedp_dtype */
  int32_t accumulate;
  int32_t reserved;
  double scale;
} slidedp_embedding_args;

SLIDEDP_API int slidedp_embedding(slidedp_ctx* ctx, const slidedp_embedding_args* args, const slidedp_rows* table, const int32_t* ids,
                      const slidedp_rows* out, void* cuda_stream);
SLIDEDP_API int slidedp_embedding_backward(slidedp_ctx* ctx, const slidedp_embedding_args* args, const int32_t* ids,
                               const slidedp_rows* d_out, const slidedp_rows* d_table, void* workspace, void* cuda_stream);
/* 0 for arguments that the call would refuse. */
SLIDEDP_API size_t slidedp_embedding_workspace(const slidedp_embedding_args* args);

/* ---- the norms around a block, its gate and its residual ---------------------------------------
 *
 * For each token, with x the residual stream, y the block's output (attention or feed-forward), rms(v) =
 * v * rsqrt(mean(v^2) + eps):
 *   n = post_norm ? rms(y) * w_post : y
 *   x' = x + residual_scale * g * n             g = gate, sigmoid(gate) with gate_sigmoid = 1, or 1 without a gate
 *   h = rms(x') * w_pre                          the next block's input, if pre_norm
 * All are [tokens, hidden] of `dtype` (BF16 or FP32), w_post and w_pre (nullable: ones) hidden values of it. gate: none
 * (gate_kind 0), hidden values for all tokens (1), or [tokens, hidden] (2). h is taken from the FP32 x', not from the rounded
 * one. has_y = 0: there is no block before (x' = x is not written, h alone is; post_norm and gate_kind are then 0 and
 * pre_norm is 1). hidden 1..16384; tokens up to 2^30.
 *
 * Backward: from the gradients dx_out of x' (NULL: zeros) and dh of h, the gradients dx, dy, dgate (2: [tokens, hidden] of
 * `dtype`; 1: hidden floats), dw_post and dw_pre (hidden floats each); dgate, dw_post and dw_pre may be NULL, and are not written where
 * the forward call has no such gate or norm. The forward's inputs are needed, its outputs are not.
 *
 * An output may be an input of the same form (same address and stride: x' = x, dx = dx_out, dy = y, ..): each row is read
 * before it is written. The same address with another stride is refused, as are two outputs at one address; outputs may not
 * overlap otherwise. workspace: device, slidedp_block_norm_workspace bytes, 16-byte aligned; needed where dw_post, dw_pre or
 * the dgate of a gate for all tokens is wanted. A sigmoid's slope is g (1 - g) in FP32: off by 2^-24 of one where g is close to it.
 * The squares are added up in FP32: a row whose sum passes its range is
 * normalised to zeros, and eps = 0 makes a row of zeros NaN. Fastest up to 8192 columns (a gradient of FP32 rows with a gate
 * [tokens, hidden]: 7680).
 */
typedef struct {
  int64_t tokens, hidden;
  int32_t dtype; /* slidedp_dtype */
  int32_t has_y, post_norm, pre_norm;
  int32_t gate_kind, gate_sigmoid;
  double residual_scale, eps;
} slidedp_block_norm_args;

SLIDEDP_API int slidedp_block_norm(slidedp_ctx* ctx, const slidedp_block_norm_args* args, const slidedp_rows* x, const slidedp_rows* y,
                       const void* w_post, const slidedp_rows* gate, const void* w_pre, const slidedp_rows* x_out,
                       const slidedp_rows* h_out, void* cuda_stream);
SLIDEDP_API int slidedp_block_norm_backward(slidedp_ctx* ctx, const slidedp_block_norm_args* args, const slidedp_rows* x,
                                const slidedp_rows* y, const void* w_post, const slidedp_rows* gate, const void* w_pre,
                                const slidedp_rows* dx_out, const slidedp_rows* dh_out, const slidedp_rows* dx,
                                const slidedp_rows* dy, const slidedp_rows* dgate, float* dw_post, float* dw_pre,
                                void* workspace, void* cuda_stream);
/* 0 for arguments that the call would refuse. */
SLIDEDP_API size_t slidedp_block_norm_workspace(const slidedp_block_norm_args* args);

/* ---- clipped policy loss ------------------------------------------------------------------------
 *
 * For each row (a sampled token) with the policy's logits z[0..vocab), the token y = labels[row], the log-probability
 * that it was sampled with (old_logp), a reference model's (ref_logp) and its advantage A:
 *   logp = log softmax(z / temperature)[y],  ratio = exp(logp - old_logp),  k = ref_logp - logp
 *   loss = -min(ratio A, clamp(ratio, 1 - clip_low, 1 + clip_high) A) + kl_weight (exp(k) - k - 1)
 * A row whose label lies outside [0, vocab) is absent (prompt, padding): its loss, logp and gradient are 0 and its logits are
 * not read. old_logp NULL: logp itself (the first step on fresh samples: ratio 1, with its gradient). ref_logp NULL: no
 * second term. advantage NULL: no first term; a row with A = 0 has none either, whatever its ratio. So with all three NULL the
 * call computes log-probabilities (loss may then be NULL too). logits: [rows, vocab] of `dtype`, logits_stride elements from row
 * to row; labels: rows int32; old_logp, ref_logp, advantage, loss, logp: rows floats. clip_low and clip_high are not negative
 * (clip_low may exceed 1).
 *
 * Gradient: d_logits[r] = row_grad[r] * d loss[r] / d z, with row_grad: rows floats (nullable: ones). A ratio on the edge of the
 * clipped range counts as inside. slidedp_policy_loss_backward takes the forward's logp, and reads rows twice where that is below -64;
 * slidedp_policy_step computes loss, logp and gradient in one call. d_logits may be the logits themselves (same address and
 * stride; the same address with another stride is refused) and may not overlap them otherwise. A kl_weight of 0 is no second
 * term, whatever ref_logp holds. Rows whose gradient is zero throughout (absent, clipped without a second term, row_grad 0)
 * are zeros whatever their logits hold; in others NaN and +inf among the logits make the row NaN. A row's exponentials are added in
 * FP32, the label's own apart from the others', so that log-probability and gradient keep their digits where the label has all but little
 * of the probability: off by a few FP32 roundings of the sum, and of the exponents, that is of the logits' distances.
 */
typedef struct {
  int64_t rows, vocab;
  int32_t dtype; /* slidedp_dtype of logits and d_logits */
  int32_t reserved;
  int64_t logits_stride, d_logits_stride;
  double temperature, clip_low, clip_high, kl_weight;
} slidedp_policy_args;

SLIDEDP_API int slidedp_policy_loss(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits, const int32_t* labels,
                        const float* old_logp, const float* ref_logp, const float* advantage, float* loss, float* logp,
                        void* cuda_stream);
SLIDEDP_API int slidedp_policy_loss_backward(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits,
                                 const int32_t* labels, const float* old_logp, const float* ref_logp, const float* advantage,
                                 const float* logp, const float* row_grad, void* d_logits, void* cuda_stream);
SLIDEDP_API int slidedp_policy_step(slidedp_ctx* ctx, const slidedp_policy_args* args, const void* logits, const int32_t* labels,
                        const float* old_logp, const float* ref_logp, const float* advantage, const float* row_grad,
                        float* loss, float* logp, void* d_logits, void* cuda_stream);

/* ---- clipping by the norm over many tensors -------------------------------------------------------
 *
 * S = sum over all tensors of (scale * x)^2, norm = sqrt(S), coef = min(1, max_norm / (norm + 1e-6)) or 1 where max_norm <= 0,
 *   out = x * (scale * coef)          (the factor is formed in double and used as FP32)
 * result: device, four doubles: S, norm, coef, and 1.0 if the norm is inf or NaN, 0.0 otherwise, as slidedp_grad_norm_finish has
 * them. So accumulated FP32 gradients of any number of tensors become the clipped BF16 gradients that
 * slidedp_reduce_adamw_chunk takes (with max_norm 0 there). grads, outs: host arrays of `count` tensors each, read before the
 * call returns; outs[i] has grads[i].count elements of either type and may be grads[i] itself (same address and type); outs NULL:
 * only result is written. Tensors need the alignment of their element; they may be empty. A factor of 1 in place writes nothing.
 * With max_norm > 0 a NaN norm makes coef and with it every output NaN, an infinite one makes coef 0. The sums are FP64 in an
 * order that the tensors' sizes and alignment decide. No tensor of outs may overlap another one, or a tensor of grads other than
 * its own.
 * workspace: device, slidedp_clip_grad_norm_workspace bytes, 16-byte aligned.
 */
typedef struct {
  void* data;
  int64_t count;
  int32_t dtype; /* slidedp_dtype */
  int32_t reserved;
} slidedp_tensor;

SLIDEDP_API int slidedp_clip_grad_norm(slidedp_ctx* ctx, const slidedp_tensor* grads, const slidedp_tensor* outs, int32_t count,
                           double scale, double max_norm, double* result, void* workspace, void* cuda_stream);
/* 0 for tensors that the call would refuse. */
SLIDEDP_API size_t slidedp_clip_grad_norm_workspace(const slidedp_tensor* grads, int32_t count);

#ifdef __cplusplus
}
#endif

#endif
