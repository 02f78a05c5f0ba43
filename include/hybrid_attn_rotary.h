/*
 * hybrid_attn_rotary.h -- rotary positions of queries and keys, alone and behind a norm of every head's row; forward and gradients.
 * Part of the C ABI of libhybridattn.so: the conventions of hybrid_attn.h (device pointers on the current device, the caller's stream and
 * buffers, host checks ahead of the first HIP call, ha_status) hold here too.
 */
#ifndef HYBRID_ATTN_ROTARY_H
#define HYBRID_ATTN_ROTARY_H

#include "hybrid_attn_sparse.h"   /* ha_view */

#ifdef __cplusplus
extern "C" {
#endif

/* Rotation by positions.  Of the first rot_dim channels of a row two and two are a pair (x, x'), pair i = 0 .. rot_dim / 2 - 1:
 *
 *   angle = freq[i] * positions[n][axis[i]]
 *   y  = magnitude (x cos angle - x' sin angle)
 *   y' = magnitude (x sin angle + x' cos angle)
 *
 * and the other channels pass through.  A position is n_axes whole numbers (a token of a video: frame, row and column), of any sign; an angle is formed in
 * 64 bits and reduced to one turn before its sine and cosine are taken in fp32, so that far positions are as exact as near ones.  Frequencies are the caller's,
 * scaled for long contexts or not, and magnitude is what such a scaling multiplies the rotated channels with (1 otherwise). */
typedef struct ha_rotary {
  const double *freq;       /* device [rot_dim / 2], radians per position, 8-byte aligned */
  const int32_t *axis;      /* device [rot_dim / 2], or NULL: all 0.  Values outside 0 .. n_axes - 1 count as the nearer end */
  const int32_t *positions; /* device [N, n_axes] of every batch entry, entry b's at positions + b positions_stride_b */
  int64_t positions_stride_b;   /* in elements, 0 or at least N n_axes: 0 is one list for all entries */
  int32_t rot_dim;          /* 0 .. d_head; even, and a multiple of 8 unless interleaved.  0: nothing is rotated, the pointers are not looked at */
  int32_t interleaved;      /* 1: pair i is channels 2 i and 2 i + 1; 0: i and i + rot_dim / 2 */
  int32_t n_axes;           /* 1 .. 4 */
  float magnitude;          /* finite */
} ha_rotary;

/* Rows of queries [B, H, N, d_head] and keys [B, H_kv, N, d_head] at the same positions.  Views as ha_view says, but inputs may have a zero stride along any
 * dimension; outputs overlap no input and no other output unless it is said. */
typedef struct ha_rows_problem {
  int32_t B, H, H_kv, N;    /* H_kv = 0: no keys (their views and weights are not looked at).  N = 0 is allowed */
  int32_t d_head;           /* 64 or 128 */
  int32_t dtype;            /* ha_dtype of all rows.  Everything is computed in fp32 and rounded once */
  float eps;                /* of the norm; finite, not negative */
} ha_rows_problem;

/* Host-only check of both, as every entry point below makes it first.  HA_ERR_UNSUPPORTED beyond 65535 heads (B H or B H_kv) or 2^27 tokens (B N). */
ha_status hybrid_attn_rotary_validate(const ha_rows_problem *p, const ha_rotary *r);

/* Enqueues out = rotation of x, both [B, H, N, d_head] (H_kv is 0).  transposed = 1: the transposed rotation by the same angles with the same magnitude, which is
 * the gradient of x from that of out.  out may be x itself (the same view), and otherwise overlaps no input. */
ha_status hybrid_attn_rotate(const ha_rows_problem *p, const ha_rotary *r, const ha_view *x, const ha_view *out, int32_t transposed, void *hip_stream);

/* Enqueues the rotation of every row's norm, queries and keys in one launch:
 *
 *   n = x / sqrt(mean of x^2 over the row's d_head channels + eps),   out = rotation of (w n)
 *
 * (A row of zeros with eps = 0, or one whose mean square leaves fp32's range, magnitudes beyond some 2^63, has no norm: it gives zeros, infinities or NaN.)
 * w_q, w_k: device fp32 [d_head] for all heads, 16-byte aligned, or NULL: ones.  q_out may be q itself and k_out k. */
ha_status hybrid_attn_norm_rotate(const ha_rows_problem *p, const ha_rotary *r, const ha_view *q, const ha_view *k, const float *w_q, const float *w_k,
                                  const ha_view *q_out, const ha_view *k_out, void *hip_stream);

/* Enqueues the gradients of q, k, w_q and w_k from those of q_out and k_out (grad_q, grad_k) and the inputs of the forward; the norm is formed anew.  grad_in_q may be
 * grad_q or q itself, grad_in_k grad_k or k.  grad_w_q, grad_w_k: device fp32 [d_head], written in full, or NULL.  They are sums in a fixed order (bitwise
 * reproducible), over all rows: 0 where there are none.  workspace: device, 256-byte aligned, hybrid_attn_norm_rotate_grad_workspace_bytes() bytes, only looked at
 * where a weight's gradient is wanted. */
size_t hybrid_attn_norm_rotate_grad_workspace_bytes(const ha_rows_problem *p);
ha_status hybrid_attn_norm_rotate_grad(const ha_rows_problem *p, const ha_rotary *r, const ha_view *grad_q, const ha_view *grad_k, const ha_view *q, const ha_view *k,
                                       const float *w_q, const float *w_k, const ha_view *grad_in_q, const ha_view *grad_in_k, float *grad_w_q, float *grad_w_k,
                                       void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HYBRID_ATTN_ROTARY_H */
