/*
 * slidedp_ops.h -- operators of the fine-tuning pass that produces the gradients of slidedp.h:
 * the query / key norms with the position rotation, attention over packed documents, and
 * distillation from a teacher's top logits, each with its gradient. (Not part of the paper, whose
 * Sec. 3.1 takes the layers' forward and backward pass as given; its workloads, Sec. 4.1, are the
 * decoder layers these operators belong to.)
 *
 * Conventions are those of slidedp.h: every call returns SLIDEDP_OK or a negative status and only
 * enqueues work on cuda_stream; the caller owns every buffer, workspaces included; nothing is kept
 * between calls. Results are bit-reproducible: no call adds floating-point numbers with atomics.
 * Calls of this header on one context may go to different streams and come from different threads, also at once (but not
 * beside other calls on that context); workspaces must not be shared by calls that can overlap.
 *
 * The attention and distillation kernels wait on copies and on blocks of their own launch; every such wait is bounded (about
 * a minute). If one runs out, the results of that call are not complete, and the first of these calls on the
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

#ifdef __cplusplus
}
#endif

#endif
