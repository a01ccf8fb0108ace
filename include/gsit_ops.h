/*
 * gsit_ops.h -- operators around the Interlaced-Mask attention of libgsit.so that a program needs to train the layers of gsit.h or to
 * run them over a stream: rotary positions with several axes, LayerNorm with its gradients, and attention whose scores follow a rule
 * (cap, bias by distance in time, documents, causality), forward, backward, and for the newest positions only.
 *
 * The conventions of gsit.h hold: device pointers, row-major, the caller owns every buffer, asynchronous on `stream`, nothing is
 * allocated or kept, return codes only, the same call gives the same bits every time; padded rows of every output are +0.0 (lse: -inf)
 * and the contents of padded input rows never matter.  gsit_shape describes the problem: batch, seg_len, valid_len, d_model = heads *
 * head_dim and dtype (GSIT_F32 or GSIT_BF16) are read by all calls, phase, custom_mask and scale by the attention.  The packed row
 * layout is not taken (row_start != NULL answers GSIT_ERR_UNSUPPORTED).  Statistics, sums, accumulators, log-sum-exps and the gradients
 * of LayerNorm's parameters are float whatever the type.
 */
#ifndef GSIT_OPS_H_
#define GSIT_OPS_H_

#include "gsit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotary positions.  A head's first 2 n features (n = sections[0] + sections[1] + sections[2], 2 n <= head_dim) are n pairs; pair p
 * belongs to axis a -- the first sections[0] pairs to axis 0 (time), the next sections[1] to axis 1 (height), the rest to axis 2
 * (width) -- and is rotated by the angle position[a] * base^(-p / n).  Pair p is features (p, n + p), or (2 p, 2 p + 1) when
 * `interleaved` is set; features from 2 n on are copied.  Angles are reduced in double, so they are right for every position an
 * int32 holds.
 *   q, k         [B, L, heads, head_dim] and [B, L, kv_heads, head_dim], row strides in elements (k may be NULL: only q)
 *   positions    int32 [axes][B][L], axes = index of the last non-zero section + 1; axis_stride elements between axes, batch_stride
 *                between samples (0: all samples share one row)
 *   q_out, k_out like q and k, row strides of their own; may be q and k themselves (in place)
 * gsit_rotary_bwd takes the gradients of the results and returns those of the inputs (the rotation by the opposite angle). */
typedef struct gsit_rotary {
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  int32_t sections[3];
  int32_t interleaved;
  int32_t kv_heads;         /* heads of k; 0 = heads */
  double base;              /* > 0, e.g. 10000 */
} gsit_rotary;
gsit_status gsit_rotary_fwd(const gsit_shape* shape, const gsit_rotary* rotary, const void* q, int64_t q_row_stride, const void* k,
                            int64_t k_row_stride, void* q_out, int64_t q_out_row_stride, void* k_out, int64_t k_out_row_stride,
                            gsit_stream stream);
gsit_status gsit_rotary_bwd(const gsit_shape* shape, const gsit_rotary* rotary, const void* dq, int64_t dq_row_stride, const void* dk,
                            int64_t dk_row_stride, void* dq_out, int64_t dq_out_row_stride, void* dk_out, int64_t dk_out_row_stride,
                            gsit_stream stream);

/* LayerNorm over rows of d_model <= 8192 features:  y = (x - mean) * rstd * gamma + beta,  rstd = 1 / sqrt(var + eps).
 *   shape        batch, seg_len, valid_len, d_model are read (heads, dtype and the rest are not)
 *   x            [B, L, d] of x_dtype, row stride in elements;  y [B, L, d] of y_dtype
 *   gamma, beta  float [d] or NULL (1, 0);  eps <= 0 selects 1e-5
 *   mean, rstd   float [B, L] or NULL, for the backward pass
 * Backward, with g = dy * gamma and h = (x - mean) * rstd:  dx = rstd * (g - mean_d(g) - h * mean_d(g h)) [+ residual],
 * dgamma = sum over real rows of dy * h,  dbeta = sum of dy.
 *   dy           [B, L, d] of y_dtype;  dx [B, L, d] of x_dtype
 *   residual     [B, L, d] of x_dtype or NULL: the gradient that reaches x past the norm (x also feeds a residual connection); it
 *                is added to dx in float before the one rounding, and may be dx itself
 *   dgamma, dbeta  float [d] or NULL (both or none)
 *   workspace    gsit_layer_norm_bwd_workspace(shape) bytes, 16-byte aligned; may be NULL when dgamma is */
gsit_status gsit_layer_norm_fwd(const gsit_shape* shape, int32_t x_dtype, const void* x, int64_t x_row_stride, const float* gamma,
                                const float* beta, float eps, int32_t y_dtype, void* y, int64_t y_row_stride, float* mean, float* rstd,
                                gsit_stream stream);
size_t gsit_layer_norm_bwd_workspace(const gsit_shape* shape);   /* (size_t)-1 for an invalid shape */
gsit_status gsit_layer_norm_bwd(const gsit_shape* shape, int32_t y_dtype, const void* dy, int64_t dy_row_stride, int32_t x_dtype,
                                const void* x, int64_t x_row_stride, const float* mean, const float* rstd, const float* gamma,
                                const void* residual, int64_t residual_row_stride, void* dx, int64_t dx_row_stride, float* dgamma,
                                float* dbeta, void* workspace, size_t workspace_bytes, gsit_stream stream);

/* Attention over the blocks that the Interlaced Mask opens, with a rule on the scores.  For query i and key j of sample b, head h:
 *   x = scale * q_i . k_j;   softcap > 0:  x <- softcap * tanh(x / softcap);   slopes:  x <- x - slopes[h] * |time_i - time_j|
 * and j is open to i if its block is open, both are real, documents[b][i] == documents[b][j] (when given) and, when `causal` is set,
 * time_j <= time_i or time_j < prefix[b] (when given).  The softmax runs over the open keys; a query without any yields +0 / -inf
 * and takes and gives no gradient.  Query head h reads key head h / (heads / kv_heads).
 * A pair that is closed contributes nothing, whatever the rows hold: NaN or Inf in a row reaches those rows only that a path of open
 * pairs connects to it. */
typedef struct gsit_score_rule {
  float softcap;              /* <= 0: none; finite, and so is scale / softcap */
  int32_t causal;
  int32_t kv_heads;           /* heads of k and v, a divisor of heads; 0 = heads */
  const float* slopes;        /* DEVICE float [heads] or NULL */
  const float* times;         /* DEVICE float [B][L], finite, or NULL: the index inside the own segment */
  const int32_t* documents;   /* DEVICE int32 [B][L] or NULL */
  const float* prefix;        /* DEVICE float [B] or NULL (read when causal is set) */
  int32_t tail;               /* 1: only the newest positions are queries, see q_len */
  int32_t q_len[3];           /* tail: queries per segment, each <= seg_len.  q holds q_len[0] + q_len[1] + q_len[2] rows a sample; row i of
                                 segment s is position valid_len[b][s] - q_len[s] + i of it (padding where that is negative) */
} gsit_score_rule;

/*   q              [B, Lq, heads, hd], k, v [B, L, kv_heads, hd], each with a row stride of its own (elements); Lq = L without tail
 *   out            [B, Lq, d] contiguous;  lse float [B, heads, Lq] or NULL
 *   bf16: head_dim 8, 16, 32 or 64, pointers 16-byte aligned, row strides multiples of 8;  f32: head_dim <= 128
 *   workspace      gsit_scored_attention_fwd_workspace() bytes: none, so NULL and 0 will do */
gsit_status gsit_im_scored_attention_fwd(const gsit_shape* shape, const gsit_score_rule* rule, const void* q, int64_t q_row_stride,
                                         const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, void* out, float* lse,
                                         void* workspace, size_t workspace_bytes, gsit_stream stream);
size_t gsit_scored_attention_fwd_workspace(const gsit_shape* shape, const gsit_score_rule* rule);   /* (size_t)-1: invalid */

/* Gradients of q, k and v (slopes, times and softcap are constants).  rule->tail is not taken (GSIT_ERR_UNSUPPORTED).
 *   dout, out      [B, L, d], row strides of their own;  lse as the forward call wrote it
 *   dq, dk, dv     like q, k, v, row strides of their own: with 3 d and one buffer [B, L, 3, H, hd] they are the gradient of a fused
 *                  projection.  They may not overlap any input.
 *   workspace      gsit_scored_attention_bwd_workspace() bytes, 16-byte aligned */
gsit_status gsit_im_scored_attention_bwd(const gsit_shape* shape, const gsit_score_rule* rule, const void* q, int64_t q_row_stride,
                                         const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, const void* out,
                                         int64_t out_row_stride, const float* lse, const void* dout, int64_t dout_row_stride, void* dq,
                                         int64_t dq_row_stride, void* dk, int64_t dk_row_stride, void* dv, int64_t dv_row_stride,
                                         void* workspace, size_t workspace_bytes, gsit_stream stream);
size_t gsit_scored_attention_bwd_workspace(const gsit_shape* shape, const gsit_score_rule* rule);   /* (size_t)-1: invalid */

#ifdef __cplusplus
}
#endif
#endif /* GSIT_OPS_H_ */
