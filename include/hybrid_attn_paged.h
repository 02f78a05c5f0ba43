/*
 * hybrid_attn_paged.h -- caches of keys and values in pages: storing new tokens, attention of new tokens over all that is stored, the weight that every stored
 * token gets in it, and eviction by that weight.
 * Part of the C ABI of libhybridattn.so: the conventions of hybrid_attn.h (device pointers on the current device, the caller's stream and
 * buffers, host checks ahead of the first HIP call, ha_status) hold here too.
 */
#ifndef HYBRID_ATTN_PAGED_H
#define HYBRID_ATTN_PAGED_H

#include "hybrid_attn_rotary.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A batch of B sequences, each with tokens in slots 0 .. key_len[b] - 1.  Slot j of sequence b is row j % page of page page_table[b][j / page] in the pools of keys and
 * values, [n_pages, H_kv, page, d_head] views.  The last n_b of a sequence's tokens are new: their queries are n_b consecutive ones of T rows [T, H, d_head], those from
 * q_offset[b] to q_offset[b + 1] - 1, in the order of their slots.  Query head h reads key head h / (H / H_kv).
 *
 * No value on the device makes a call read or write outside of the tensors: key_len outside 0 .. max_pages * page and offsets outside 0 .. T count as the nearer
 * end, and the tokens on a page whose number is outside 0 .. n_pages - 1 are not there (no query sees them, nothing is stored).  Offsets must not fall; where they do,
 * which rows are computed is not defined.  Rows that belong to no sequence, and those of a sequence behind its first max_new, are left as they were.  Sequences may share pages (a common beginning), but not those that new tokens go to. */
typedef struct ha_paged_problem {
  int32_t B, H, H_kv;     /* H a multiple of H_kv */
  int32_t T;              /* rows of new tokens; 0 is allowed */
  int32_t d_head;         /* 64 or 128 */
  int32_t dtype;          /* ha_dtype of all rows and pages.  HA_F32: as ha_sparse_problem.dtype says, and an infinity counts as NaN */
  int32_t n_pages;        /* pages of the pools */
  int32_t page;           /* slots of a page: 16, 32, 64, 128 or 256 */
  int32_t max_pages;      /* columns of page_table: max_pages * page <= 2^30 */
  int32_t max_new;        /* no sequence has more new tokens than this, 0 .. T.  (It decides how the work is split: the smallest number that holds is best) */
  int32_t causal;         /* 1: a new token sees the slots up to its own; 0: all slots of its sequence */
  float softmax_scale;    /* 1e-30 .. 1e30 */
  const int32_t *page_table;  /* device [B, max_pages] */
  const int32_t *key_len;     /* device [B], with the new tokens */
  const int32_t *q_offset;    /* device [B + 1], or NULL: every sequence has max_new new tokens (T = B max_new) */
} ha_paged_problem;

/* Rows are [T, heads, d_head] views: of an ha_view, stride_n is a token's, stride_h a head's, stride_b is not looked at.  Pools: stride_b is a page's, stride_h a
 * head's, stride_n a slot's.  Strides in elements, multiples of 16 bytes (zero for inputs only), data 16-byte aligned; a page's rows span less than 2^31 bytes.  Outputs overlap no input
 * and no other output unless it is said.
 *
 * Host-only check, as every entry point below makes it first.  HA_ERR_UNSUPPORTED beyond 65535 sequences or heads (B H_kv), 2^20 rows times heads of a group
 * (T H / H_kv) or 2^24 (T H). */
ha_status hybrid_attn_paged_validate(const ha_paged_problem *p);

/* Enqueues the storing of new tokens in one launch: every row of k [T, H_kv, d_head] and v goes to its slot (key_len counts them already), and with q [T, H, d_head] (or NULL) q_out
 * is written, which may be q itself.  norm = 1: queries and keys are normed for each head (eps, w_q and w_k as hybrid_attn_norm_rotate takes them); after
 * that they are rotated by r, whose positions are those of the T rows [T, n_axes] (r NULL: not). */
ha_status hybrid_attn_paged_append(const ha_paged_problem *p, const ha_rotary *r, int32_t norm, float eps, const ha_view *q, const ha_view *k, const ha_view *v,
                                   const float *w_q, const float *w_k, const ha_view *k_pages, const ha_view *v_pages, const ha_view *q_out, void *hip_stream);

/* Enqueues softmax attention of the new tokens over their sequences: out = sum_j p_j v_j, p_j = exp(scale q . k_j - lse), j over the slots that the token sees.  A token
 * that sees none has out = 0 and lse = -infinity.  lse: device fp32 [T, H], or NULL.  What the pools hold in slots that no token of a sequence sees is never used; a NaN or
 * infinity in a slot that some token of a tile of neighbouring ones sees may reach all of that tile.  Logits beyond 2^28 in magnitude may give infinities or NaN, and so may
 * values whose sum, with weights of 2^8 at most, leaves fp32's range before it is divided.
 * Sums are fp32.  That of the weights keeps what its roundings leave out, so that lse does not lose with the number of slots; those of the values are the matrix cores', like any fp32 product's:
 * with values of one sign under nearly equal weights a result is off by some 1e-9 of itself for every slot.  workspace: device, 256-byte aligned,
 * hybrid_attn_paged_workspace_bytes() bytes (0 is possible).  Results are the same bit for bit every time. */
size_t hybrid_attn_paged_workspace_bytes(const ha_paged_problem *p);
ha_status hybrid_attn_paged_forward(const ha_paged_problem *p, const ha_view *q, const ha_view *k_pages, const ha_view *v_pages, const ha_view *out, float *lse,
                                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* Enqueues weights_out[b][h][j] = weights[b][h][j] + sum of exp(scale q . k_j - lse) over the new tokens of sequence b that see slot j and the query heads of key head h: what the
 * slot got in the attention that wrote lse (fp32 [T, H]).  Tokens whose lse is -infinity count as seeing nothing, whatever their queries hold.  weights, weights_out: device fp32 [B, H_kv, max_pages page], contiguous;
 * weights NULL: zeros; weights_out may be weights itself.  Slots that nothing sees (behind key_len, on pages that are not there) get what weights holds.
 * workspace as above, hybrid_attn_paged_weights_workspace_bytes() bytes.  Sums in fp32 in a fixed order, with what roundings leave out of long ones. */
size_t hybrid_attn_paged_weights_workspace_bytes(const ha_paged_problem *p);
ha_status hybrid_attn_paged_weights(const ha_paged_problem *p, const ha_view *q, const ha_view *k_pages, const float *lse, const float *weights, float *weights_out,
                                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* Enqueues the eviction of what has had the least weight.  Of every sequence and key head at most `keep` slots stay: the first keep_first, the last
 * keep_last, and of the others those with the largest weights, of equal ones the lower slot (a NaN is above all numbers); a sequence of no more than
 * `keep` slots keeps all.  What stays is copied, in its order, to slots 0, 1, .. of the pages out_table[b] (device int32 [B, out_pages],
 * out_pages * page >= keep) of the same pools; rows there behind the last one are left as they were.  No page of out_table is one that a sequence of
 * page_table reads, and none stands in it twice; numbers outside 0 .. n_pages - 1 there store nothing, and a slot that is not there is copied as zeros.
 *   len_out      device int32 [B]: slots that stay; not key_len itself
 *   weights_out  device fp32 [B, H_kv, max_pages page]: the weights of what stays, zeros behind them; not weights itself
 *   kept         device int32 [B, H_kv, keep]: the slots that stay, rising, -1 behind the last
 * T, max_new, causal, softmax_scale, q_offset and H of the problem are checked but not used.  keep >= 1, keep_first, keep_last >= 0, keep_first + keep_last <= keep.
 * workspace as above, hybrid_attn_paged_evict_workspace_bytes() bytes. */
size_t hybrid_attn_paged_evict_workspace_bytes(const ha_paged_problem *p, int32_t keep);
ha_status hybrid_attn_paged_evict(const ha_paged_problem *p, int32_t keep, int32_t keep_first, int32_t keep_last, const float *weights, const int32_t *out_table,
                                  int32_t out_pages, const ha_view *k_pages, const ha_view *v_pages, int32_t *len_out, float *weights_out, int32_t *kept, void *workspace,
                                  size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HYBRID_ATTN_PAGED_H */
