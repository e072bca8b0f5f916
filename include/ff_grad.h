/*
 * ff_grad.h -- a training step's operators: attention that keeps its statistics, the affine norm, and
 * the gradients of both and of the modulated norm (libff.so).
 *
 * The objectives of ff_loss.h are functions of the velocity; their gradient passes back through the
 * blocks of ff.h.  Of what a block computes besides the projections, attention and the norms are covered
 * here; the gradients of the per-head norm with its rotation, of GELU and of the gated residual are not.
 * Conventions (ownership, asynchrony on `stream`, host-side validation, status codes, ff_last_error)
 * are those of ff.h.  Sums, softmax statistics and gradients are held in float32 and rounded once when
 * stored, except the probabilities and score gradients of bfloat16 attention of head dimension 64 and
 * 128, which are rounded to bfloat16 as operands of the matrix products (0.0020 to 0.0025 of the results'
 * norm off 64 bits, where rounding the results alone is 0.0017).  Every sum runs in a fixed order: results are bitwise
 * reproducible.  The operations that ff_profile_read reports are those of the pairs of a query and a key that it
 * sees, with every sample counted as n_kv keys long (kv_len lies on the device).
 */
#ifndef FF_GRAD_H
#define FF_GRAD_H

#include "ff.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A tensor [B, heads, tokens, head_dim] in any layout with unit stride along head_dim: element
 * (b, h, n, j) at data + b * batch + h * head + n * token + j, strides in elements.  Head-major
 * [B, heads, n, d], token-major [B, n, heads, d] and the slices of a packed projection
 * [B, n, 3, heads, d] are all of this form.  Inputs may repeat elements (strides of 0). */
typedef struct ff_heads {
  void* data;
  int64_t batch, head, token;
} ff_heads;

/* Attention with heads / kv_heads query heads to each key head: query head h reads key head
 * h / (heads / kv_heads).
 *   kv_len  device int32 [B] or NULL: sample b has keys 0 .. kv_len[b] - 1 (values outside
 *           [0, n_kv] are clamped); NULL: n_kv keys.  K and V at or past kv_len are never read.
 *   causal  0, or 1: query i sees key j only if j <= i + kv_len[b] - n_q (the last query sees the last
 *           key).  A key within kv_len enters the products of other queries of its tile with weight 0,
 *           so it has to be finite.
 *   scale   factor of the scores, of a magnitude between 2^-64 and 2^64; 0 stands for 1 / sqrt(head_dim). */
typedef struct ff_attn_shape {
  int64_t B, heads, kv_heads, n_q, n_kv, head_dim;
  int32_t dtype, causal;
  float scale;
  const int32_t* kv_len;
} ff_attn_shape;

/* Workspace bytes of ff_attention_forward (0 where it needs none) and ff_attention_backward. */
int ff_attention_forward_workspace_size(const ff_attn_shape* shape, size_t* bytes /* host, out */);
int ff_attention_backward_workspace_size(const ff_attn_shape* shape, size_t* bytes /* host, out */);

/* out_i = sum_j exp(s_ij - lse_i) v_j, s_ij = scale q_i . k_j, lse_i = log sum_j exp(s_ij) over the keys
 * j that query i sees; a query that sees none has out_i = 0 and lse_i = -inf.
 * Q, out [B, heads, n_q, d], K, V [B, kv_heads, n_kv, d] of dtype; lse float32 [B, heads, n_q], dense.
 * head_dim <= 128, a multiple of 8 (bf16) or 4 (f32), and so are the strides; data 16-byte aligned; heads a
 * multiple of kv_heads.  out and lse overlap no input and not one another, out none of its own elements
 * (FF_EINVAL where it can be told from strides and addresses).  B = 0 or n_q = 0 is a no-op;
 * n_kv = 0 is allowed.  Limits (FF_EUNSUPPORTED): n_q, n_kv <= 2^27, heads <= 2^16, token strides
 * <= 2^24, other strides < 2^40, B heads ((n_q + n_kv) / 32 + 2) < 2^24. */
int ff_attention_forward(const ff_attn_shape* shape, const ff_heads* Q, const ff_heads* K, const ff_heads* V,
                         const ff_heads* out, float* lse, void* workspace, size_t ws_bytes, void* stream);

/* The gradients of ff_attention_forward's out, given that call's out and lse and the gradient dO of out:
 * with P_ij = exp(s_ij - lse_i) (recomputed), D_i = sum_j dO_ij out_ij and dS_ij = P_ij (dO_i . v_j - D_i),
 *   dV_j = sum_i P_ij dO_i,  dK_j = scale sum_i dS_ij q_i,  dQ_i = scale sum_j dS_ij k_j,
 * dK and dV summed over the query heads that share a key head.  Queries that see no key have dQ = 0, keys
 * that no query sees (those past kv_len among them) dK = dV = 0; every element of dQ, dK and dV is written.
 * P is taken from lse, a float32: it is off by 2^-24 |lse| relative, which tells where scores reach 10^5.
 * Operands, layouts and limits as ff_attention_forward; dO, out, dQ like Q; dK, dV like K.  The outputs
 * overlap no input, no other output and none of their own elements (they may be slices of one packed
 * gradient); one at the address of another operand is refused (FF_EINVAL). */
int ff_attention_backward(const ff_attn_shape* shape, const ff_heads* dO, const ff_heads* Q, const ff_heads* K,
                          const ff_heads* V, const ff_heads* out, const float* lse, const ff_heads* dQ,
                          const ff_heads* dK, const ff_heads* dV, void* workspace, size_t ws_bytes, void* stream);

/* y = Norm(x) w + bias per row: x, y [rows, H] (row strides ldx, ldy), w, bias [H] or NULL (1 and 0), all
 * of dtype; norm_kind FF_NORM_LN or FF_NORM_RMS.  y may be x and overlaps nothing else.  rows <= 2^27, H and strides <= 2^22
 * (FF_EUNSUPPORTED); any H, any strides >= H; pointers aligned to an element. */
int ff_norm_affine(const void* x, int64_t ldx, const void* w, const void* bias, void* y, int64_t ldy, int64_t rows,
                   int64_t H, int32_t norm_kind, float eps, int32_t dtype, void* stream);

/* The gradients of y = Norm(x) m + a (m = w, a = bias for the affine norm; m = 1 + scale[b], a = shift[b]
 * for the modulated one, b = row / rows_per_sample), with xh = Norm(x), g = dy m and means over a row:
 *   dx = (g - mean(g) [layer norm only] - xh mean(g xh)) / sqrt(var + eps)  (+ add)
 *   dm = sum over rows of dy xh,  da = sum over rows of dy
 * dy, x, add (or NULL), dx [rows, H] of dtype with row strides lddy, ldx, ldadd, lddx; add is the gradient
 * that reaches x by another way (the residual's).  dx may be dy, x or add (same row stride); nothing else that is
 * written overlaps another operand (FF_EINVAL where an output has its address).  Outputs dw and dbias
 * float32 [H]; dshift and dscale float32 [samples, H] of row stride dmod_ld, samples = ceil(rows /
 * rows_per_sample).  Each output may be NULL.  scale is float32 of row stride mod_ld (mod_ld, dmod_ld >= H).
 * rows = 0 writes dw and dbias zeros.  Limits as ff_norm_affine, and 65535 samples.  FF_EWORKSPACE if the workspace is smaller than
 * ff_norm_backward_workspace_size(rows, H, rows_per_sample) says (the affine norm has rows_per_sample = rows). */
int ff_norm_backward_workspace_size(int64_t rows, int64_t H, int64_t rows_per_sample, size_t* bytes /* host, out */);
int ff_norm_affine_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w, const void* add,
                            int64_t ldadd, void* dx, int64_t lddx, float* dw, float* dbias, int64_t rows, int64_t H,
                            int32_t norm_kind, float eps, int32_t dtype, void* workspace, size_t ws_bytes, void* stream);
int ff_norm_modulate_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* scale,
                              int64_t mod_ld, int64_t rows_per_sample, const void* add, int64_t ldadd, void* dx,
                              int64_t lddx, float* dshift, float* dscale, int64_t dmod_ld, int64_t rows, int64_t H,
                              int32_t norm_kind, float eps, int32_t dtype, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FF_GRAD_H */
