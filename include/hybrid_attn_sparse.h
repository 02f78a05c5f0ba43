/*
 * hybrid_attn_sparse.h -- block-sparse attention: choice of key blocks, forward, gradients.
 * Part of the C ABI of libhybridattn.so: the conventions of hybrid_attn.h (device pointers on the current device, the caller's stream and
 * buffers, host checks ahead of the first HIP call, ha_status) hold here too.
 */
#ifndef HYBRID_ATTN_SPARSE_H
#define HYBRID_ATTN_SPARSE_H

#include "hybrid_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Block-sparse attention: softmax attention of every query over blocks of keys that a cheap score selects.  It stands next to the variants
 * of the token split (ha_problem.split_granularity, local_window), which choose softmax tokens by their position; here they are chosen by what
 * the queries and keys hold, and the other tokens do not take part.  (An operator of its own, not the paper's method.)
 *
 * Keys come in blocks of k_block, queries in tiles of q_block consecutive tokens; the last of either may be short.  Query head h reads key head
 * h / (H / H_kv).  One tile of all query heads of one key head shares one list of n_select key blocks:
 *
 *   mean_j  = mean of the keys of block j (those below key_len)                                        hybrid_attn_key_means
 *   score   = sum over the tile's queries and heads of q . mean_j                                      hybrid_attn_select_blocks
 *   list    = the n_select blocks of highest score among those any query of the tile may see
 *   out_i   = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - lse_i),  j over the list's keys that query i sees    hybrid_attn_sparse_forward
 *
 * Query i stands at position q_start[b] + i.  It sees key j of a listed block if j < key_len[b] and, with causal, j <= its position.  A query that
 * sees no key has out = 0 and lse = -infinity, and its gradients are zero.  What the memory of keys and values holds at and behind key_len is
 * never used, and with causal neither is what stands behind the last position of a tile; a NaN or infinity at a key that some query of a tile sees may
 * reach all queries of that tile.  The gradients form the weights anew from lse, an fp32 number, which puts them off by some |lse| 2^-22 of their value; logits
 * (scale q . k) beyond 2^28 in magnitude may give infinities or NaN, in the forward too. */
typedef struct ha_sparse_problem {
  int32_t B, H, H_kv;     /* H a multiple of H_kv */
  int32_t N_q, N_k;       /* 0 is allowed: no queries, or no keys */
  int32_t d_head;         /* 64 or 128 */
  int32_t dtype;          /* ha_dtype of q, k, v, out and their gradients.  HA_F32 tensors are not rounded to bf16: every value is
                             split into three bf16 ones and multiplied in six products with fp32 accumulation, about fp32's own precision
                             (values below some 2^-110 keep fewer bits: a piece is a multiple of 2^-133). */
  int32_t q_block, k_block;   /* 64 or 128 each */
  int32_t n_select;       /* length of a list, 1 .. 2^20 */
  int32_t causal;         /* 0 or 1 */
  int32_t keep_first;     /* hybrid_attn_select_blocks: the first keep_first blocks are in every list that may see them */
  int32_t near_tokens;    /* hybrid_attn_select_blocks: -1 off; w >= 0: so are the blocks with a key within w tokens of the tile's own positions (before
                             them and, without causal, behind them).  With causal it must not be off: the means of blocks that reach past a tile's first
                             position hold later keys, which must not decide anything. */
  float softmax_scale;    /* 1e-30 .. 1e30 */
  const int32_t *q_start; /* device [B], or NULL: N_k - N_q for every batch entry.  |q_start| < 2^30 */
  const int32_t *key_len; /* device [B], or NULL: N_k for every batch entry.  Values outside 0 .. N_k count as the nearer end */
} ha_sparse_problem;

/* A [B, heads, N, d_head] tensor: element (b, h, n, c) at data + b stride_b + h stride_h + n stride_n + c, strides in elements, multiples of 16
 * bytes, data 16-byte aligned.  Strides of dimensions of one entry are not looked at; a zero stride along b or h reads one tensor for all entries
 * (inputs only; refused for outputs: HA_ERR_SHAPE).  stride_n >= d_head, and k_block rows (of keys; q_block rows of queries) span less than 2^31 bytes. */
typedef struct ha_view {
  void *data;
  int64_t stride_b, stride_h, stride_n;
} ha_view;

/* Host-only check of the problem, as every entry point below makes it first.  HA_ERR_UNSUPPORTED beyond 2^20 tiles of queries (B H ceil(N_q / q_block)),
 * 2^23 blocks of keys (B H_kv ceil(N_k / k_block)) or lists of 2^30 entries a head.  Outputs overlap no input and no other output. */
ha_status hybrid_attn_sparse_validate(const ha_sparse_problem *p);

/* Enqueues the block means: means, device fp32 [B, H_kv, ceil(N_k / k_block), d_head].  A block without a key below key_len has mean 0.
 * Sums are formed in double, in a fixed order.  only_last = 0: all blocks.  only_last = m > 0: of every batch entry the last m blocks that hold a
 * key below key_len, the others are left as they are (a cache that grew by a few tokens). */
ha_status hybrid_attn_key_means(const ha_sparse_problem *p, const ha_view *k, int32_t only_last, float *means, void *hip_stream);

/* Enqueues the choice: blocks, device int32 [B, H_kv, ceil(N_q / q_block), n_select], every list in rising order with -1 behind its last block.
 * Blocks without a key below key_len are in no list, and with causal neither are those behind the last position of the tile.  Blocks that are
 * always kept (keep_first, near_tokens) come first, then those of highest score, of equal ones the lower index.  Scores are sums rounded in double, the same bit
 * for bit every time; ones that differ by no more than such roundings may stand in either order.
 * HA_ERR_SHAPE where n_select does not hold the blocks that are always kept, and not all blocks (with q_start, which the host does not read: where there
 * are places at which it would not, blocks that are kept for both reasons counted twice).  (A score that is NaN ranks above all others.)
 * workspace: device, 256-byte aligned, hybrid_attn_select_workspace_bytes() bytes. */
size_t hybrid_attn_select_workspace_bytes(const ha_sparse_problem *p);
ha_status hybrid_attn_select_blocks(const ha_sparse_problem *p, const ha_view *q, const float *means, int32_t *blocks, void *workspace,
                                    size_t workspace_bytes, void *hip_stream);

/* Enqueues one forward.  blocks: device, as hybrid_attn_select_blocks writes it or any other lists: an index outside 0 .. ceil(N_k / k_block) - 1 is
 * skipped, and one that stands twice counts its keys twice.  out: written in full.  lse: device fp32 [B, H, N_q], or NULL: log of the sum of
 * exp(scale q . k) of every query.  Products run in bf16 with fp32 accumulation (HA_F32: see dtype), softmax statistics in fp32.  workspace: device,
 * 256-byte aligned, hybrid_attn_sparse_workspace_bytes() bytes (0 is possible).  Results are the same bit for bit every time. */
size_t hybrid_attn_sparse_workspace_bytes(const ha_sparse_problem *p);
ha_status hybrid_attn_sparse_forward(const ha_sparse_problem *p, const ha_view *q, const ha_view *k, const ha_view *v, const int32_t *blocks,
                                     const ha_view *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Enqueues the gradients of a loss with respect to q, k and v from the gradient with respect to out.  blocks, out and lse as the forward took and
 * left them (the choice of the blocks has no gradient).  dq, dk, dv: written in full, fp32 sums in a fixed order (bitwise reproducible) rounded to
 * dtype; keys in no list, and at and behind key_len, have gradient 0.  workspace: as above, hybrid_attn_sparse_grad_workspace_bytes() bytes.
 * HA_ERR_UNSUPPORTED (and 0 bytes) where all heads' key blocks, and one more for every 64 tiles that list one (8192 queries in HA_F32), are over 2^22. */
size_t hybrid_attn_sparse_grad_workspace_bytes(const ha_sparse_problem *p);
ha_status hybrid_attn_sparse_grad(const ha_sparse_problem *p, const ha_view *q, const ha_view *k, const ha_view *v, const int32_t *blocks,
                                  const ha_view *out, const float *lse, const ha_view *grad_out, const ha_view *grad_q, const ha_view *grad_k,
                                  const ha_view *grad_v, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HYBRID_ATTN_SPARSE_H */
