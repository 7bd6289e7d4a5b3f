/*
 * cw_layer.h -- what a layer of a served model does around its attention over the
 * paged pools of cw.h: the tables of a step from lengths on the GPU, the norm and
 * position rotation of queries and keys with the page write (one position per token, or
 * one for each of several axes), the norms around the residual stream, differential
 * attention, and attention with shaped scores.
 *
 * Ownership, ordering, errors and graph capture are those of cw.h: the caller owns
 * every buffer, work is enqueued on `stream`, every argument is checked before
 * anything is enqueued, nothing is thrown.  Tensors lie on the current device.
 */
#ifndef CW_LAYER_H_
#define CW_LAYER_H_

#include <stddef.h>
#include <stdint.h>

#include "cw.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Block-table entries of a step's new pages and the index arrays of its new tokens,
 * from request lengths in *device* memory (CacheWise Sec. 2: KV prefixes persist in
 * fixed-size blocks, which a block table maps).  No length passes through the host, so a
 * captured call serves every step of up to max_tokens tokens.  It keeps no place in the free
 * list: every call, and every replay of a captured one, takes pages from free_pages[0] on, so the
 * program moves the list on by info[0] pages before the next one (which work captured behind the
 * call can do).  For programs that keep their free pages in such a list; cw_bm_* (cw_policy.h)
 * hands out tables of its own.  The calls that plan on the host (attention, cw_kv_write_pages) take
 * their lengths there.  cu_rows and seq_ids are for the program's own kernels.
 *
 * With held_b = ceil(Lp_b / P) and need_b = ceil((Lp_b + Ls_b) / P):
 *   block_table[b][held_b + i] = free_pages[F_b + i],  0 <= i < need_b - held_b,
 *     F the exclusive sum of need - held: sequences take pages in order; entries
 *     below held_b are kept (and read), other entries are not touched;
 *   cu_rows[b] = exclusive sum of Ls (cu_rows[num_seqs] = all new tokens);
 *   for packed token t = cu_b + i, i < Ls_b: seq_ids[t] = b, positions[t] = Lp_b + i,
 *     slots[t] = block_table[b][positions[t] / P] * P + positions[t] % P;
 *   tokens t from cu_rows[num_seqs] up to max_tokens: -1 in all three arrays;
 *   info = {pages taken, new tokens, sequences that need more than bt_stride pages}.
 * cw_qk_norm_rope takes positions and slots as they are (-1: nothing is written).
 *
 * What does not fit is left out, in bounds, and shows in info: when info[0] >
 * num_free the pages past the list are -1 in the table and the slots on them -1; when
 * info[1] > max_tokens the tokens past the arrays are not written; a sequence takes no
 * pages beyond its table row (its tokens there get slot -1).  A negative length counts
 * as 0.  cu_rows and positions are clipped to INT32_MAX.
 *
 * prefix_lens, suffix_lens: device int32 [num_seqs]; free_pages: device int32
 * [num_free], distinct page ids; block_table: device int32 [num_seqs, bt_stride];
 * cu_rows [num_seqs + 1], seq_ids, positions [max_tokens] int32, slots [max_tokens] and
 * info [3] int64, device, each may be NULL.  page_size 16 or 64, num_seqs up to 2^30.
 * Outputs may overlap neither inputs nor each other (CW_ERR_ALIAS).  Workspace:
 * cw_step_tables_workspace_bytes(num_seqs) bytes, 0 up to 4096 sequences (then it may be
 * NULL).  Needs no cw_init, also under capture. */
size_t cw_step_tables_workspace_bytes(int32_t num_seqs);
cw_status_t cw_build_step_tables(const int32_t* prefix_lens, const int32_t* suffix_lens,
                                 int32_t num_seqs, const int32_t* free_pages, int32_t num_free,
                                 int32_t page_size, int32_t* block_table, int32_t bt_stride,
                                 int32_t max_tokens, int32_t* cu_rows, int32_t* seq_ids,
                                 int32_t* positions, int64_t* slots, int64_t* info,
                                 void* workspace, size_t workspace_bytes, hipStream_t stream);

/* RMS norm of every query and key head, the position rotation and, with pools, the page
 * write of the new tokens' K/V, in one pass over q, k and v:
 *   y = x / sqrt(mean(x^2) + eps) * weight   (per head; weight NULL: y = x)
 *   with c, s the cos and sin of the token's position, for 0 <= i < R / 2:
 *     (y[a], y[b]) <- (y[a] c[i] - y[b] s[i], y[b] c[i] + y[a] s[i])
 *     a, b = i, i + R / 2, or with interleaved != 0: 2 i, 2 i + 1
 * in fp32, rounded once to bf16.  v is not changed.  With pools, token t's K (after
 * norm and rotation) and V go to slot slots[t] % P of page slots[t] / P, with exactly
 * the bytes that cw_kv_write_pages of k_out and v would put there.  With a weight, mean(x^2)
 * must be an fp32 number (a head's values below about 2^60).
 *
 * q bf16 [T, Hq, D], k and v bf16 [T, Hkv, D] with the heads of a token contiguous and
 * q_stride, k_stride, v_stride elements (multiples of 8) from one token to the next, so
 * they may be columns of one projection's output; q_out [T, Hq, D], k_out, v_out
 * [T, Hkv, D] contiguous (what the attention calls take).  v may be NULL (then v_out and
 * the pools must be); v_out may be NULL.  q_weight, k_weight: fp32 [D] or NULL.
 * cos_sin: fp32 [num_positions, R], the R / 2 cosines of a position, then its sines.
 * positions: device int32 [T]; of a token whose position lies outside [0,
 * num_positions) nothing is written.  slots: device int64 [T]; a token whose slot lies
 * outside [0, num_pages * P) is not written to the pools.  Slots of one call must be
 * distinct.  k_pool NULL: no page write (slots, scales unused).
 *
 * head_dim 64 or 128, R a multiple of 16 in 16 .. head_dim, eps finite and >= 0,
 * page_size 16 or 64.  16-byte alignment of every tensor but positions (4) and slots
 * (8).  q_out may be q and k_out may be k, v_out may be v, where that is contiguous;
 * outputs overlap nothing else (CW_ERR_ALIAS).  No workspace; needs no cw_init. */
cw_status_t cw_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride, int32_t num_tokens,
                            int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                            const float* q_weight, const float* k_weight, float eps,
                            const float* cos_sin, int32_t num_positions, int32_t rotary_dim,
                            int32_t interleaved, const int32_t* positions, void* q_out,
                            void* k_out, void* v_out, void* k_pool, void* v_pool,
                            const float* k_scale, const float* v_scale, const int64_t* slots,
                            int32_t num_pages, int32_t page_size, cw_kv_dtype_t kv_dtype,
                            hipStream_t stream);

/* cw_qk_norm_rope for positions with several axes (time, height and width of an image or a
 * video): pair i of a head (0 <= i < R / 2) is rotated by the cos and sin of column i at the
 * token's position on axis axis_of_h[i].  All else as cw_qk_norm_rope.
 *
 * positions: device int32 [num_axes, T]; a token one of whose positions lies outside [0,
 * num_positions) is not written, like one without a position there.  num_axes 1..4; axis_of_h:
 * host int32 [R / 2], each in 0 .. num_axes - 1, read before the call returns. */
cw_status_t cw_qk_norm_rope_axes(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, int32_t num_tokens,
                                 int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                 const float* q_weight, const float* k_weight, float eps,
                                 const float* cos_sin, int32_t num_positions, int32_t rotary_dim,
                                 int32_t interleaved, const int32_t* positions, int32_t num_axes,
                                 const int32_t* axis_of_h, void* q_out, void* k_out, void* v_out,
                                 void* k_pool, void* v_pool, const float* k_scale,
                                 const float* v_scale, const int64_t* slots, int32_t num_pages,
                                 int32_t page_size, cw_kv_dtype_t kv_dtype, hipStream_t stream);

/* The norm of a block's output, its gate, the scaled residual stream and the norm before the
 * next block, in one pass over a token's row of `width` elements:
 *   u  = x / sqrt(mean(x^2) + eps) * post_weight           (post_weight NULL: u = x)
 *   r' = residual_scale * residual + gate * u              (gate NULL: 1)
 *   y  = r' / sqrt(mean(r'^2) + eps) * pre_weight          (pre_weight and y_out NULL: no y)
 * in fp32; r' is rounded once to residual_out's type, y once to bf16, from r' before its
 * rounding.  mean(x^2) and mean(r'^2) must be fp32 numbers (values below about 2^56).
 *
 * x bf16 [T, width], x_stride elements from one token to the next; residual and residual_out
 * contiguous [T, width], bf16 or (residual_fp32 != 0) fp32; y_out bf16 contiguous; post_weight,
 * pre_weight fp32 [width]; gate bf16 [width] for all tokens (gate_stride 0) or a row for each,
 * gate_stride elements apart.  width a multiple of 8 in 8 .. 16384, strides multiples of 8, eps
 * finite and >= 0, residual_scale finite, 16-byte alignment of every tensor.  residual_out may
 * be residual; outputs overlap nothing else (CW_ERR_ALIAS).  No workspace; needs no cw_init. */
cw_status_t cw_residual_norm(const void* x, int64_t x_stride, const void* residual,
                             int32_t residual_fp32, int32_t num_tokens, int32_t width,
                             const float* post_weight, const void* gate, int64_t gate_stride,
                             float residual_scale, const float* pre_weight, float eps,
                             void* residual_out, void* y_out, hipStream_t stream);

/* Attention with shaped scores over the paged cache: scores capped by a tanh, biased by
 * distance, and masked by a window, by documents or by a prefix whose tokens all see each
 * other; for chunks of new tokens and single tokens mixed.  For the new token at position p of
 * its sequence, its query head h and key j:
 *   x_j = softmax_scale q.k_j
 *   x_j <- score_cap tanh(x_j / score_cap)                 (score_cap 0: no cap)
 *   x_j <- x_j - slopes[h] |p - j|                         (slopes NULL: no bias)
 *   out = sum_j softmax(x)_j v_j over the visible keys j, lse = ln sum_j exp(x_j)
 * Key j is visible where all of these hold:
 *   j <= p, or j < full_lens_h[b]: the first full_lens_h[b] tokens of sequence b see each other
 *     (NULL: none do; what lies beyond the sequence's last token counts for nothing).  Tokens
 *     of that prefix that earlier calls cached have seen only what was there then;
 *   j > p - window                                         (window 0: no limit);
 *   j >= key_begins[t], the first visible position of new token t, such as the start of its
 *     document (NULL, or negative: 0).
 * A token that sees no key gets out = 0 and lse = -inf.  With neither of them the call is the
 * attention of cw_step_attention without its page write: the pools are only read.
 *
 * Tensors, pools, scales, block table and lengths as for cw_extend_attention; out bf16 [T, Hq,
 * D], lse fp32 [T, Hq] or NULL; slopes device fp32 [Hq] of either sign, scores and |slope (p - j)|
 * below 2^64; key_begins device int32 [T], any values; full_lens_h host int32 [num_seqs].  score_cap 0 or
 * 2^-10 .. 4096; a capped score is held to score_cap * 2^-20, a biased one to 2^-21 of the largest
 * score and bias of its row.  Block-table entries of pages that lie wholly before the windows of
 * all new tokens of their sequence are not read, nor is what those pages hold: a program may
 * have given them away.
 *
 * Supported: head_dim 64 or 128, page_size 16 or 64, gqa_group 1..16, num_kv_heads 1..1024.
 * Sequences with one new token run on an HBM-streaming kernel, the others on a matrix-core
 * kernel, which over fp8 pools takes q, k_new, v_new and the cached values (code * scale) in
 * fp16: of such a call their magnitudes must lie below 65504 (and are held to 2^-25 where they
 * lie below 2^-14, beside 2^-11 of themselves where a V scale does not fit fp16's 11 bits).  Key
 * scales are applied to the scores in fp32 by both; a scale may be 0.  Values (code * scale) lie
 * below 2^80.  A NaN or infinity in a value that some row of a chunk sees may reach the rows of its
 * sequence that do not (their weight for it is zero); what slots at or past a prefix's end hold
 * changes no result.  Lengths, plan, capture, aliasing and errors as for cw_step_attention; the
 * timing events are not recorded.  The plan depends on window and full_lens_h, not on the other
 * shapes.  Workspace: cw_shaped_workspace_bytes (0 if the arguments are invalid). */
size_t cw_shaped_workspace_bytes(const int32_t* prefix_lens_h, const int32_t* suffix_lens_h,
                                 int32_t num_seqs, int32_t num_kv_heads, int32_t gqa_group,
                                 int32_t head_dim, int32_t page_size, cw_kv_dtype_t kv_dtype,
                                 int32_t window, const int32_t* full_lens_h);
cw_status_t cw_shaped_attention(const void* q, const void* k_new, const void* v_new,
                                const void* k_pool, const void* v_pool, const float* k_scale,
                                const float* v_scale, const int32_t* block_table,
                                int32_t bt_stride, int32_t num_pages,
                                const int32_t* prefix_lens_h, const int32_t* suffix_lens_h,
                                int32_t num_seqs, int32_t num_kv_heads, int32_t gqa_group,
                                int32_t head_dim, int32_t page_size, float softmax_scale,
                                cw_kv_dtype_t kv_dtype, float score_cap, const float* slopes,
                                int32_t window, const int32_t* key_begins,
                                const int32_t* full_lens_h, void* out, float* lse,
                                void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Differential attention over the paged cache: the difference of two softmax maps with a
 * learned weight per head, for chunks of new tokens and single tokens mixed.
 *
 * Query pair h (query heads 2 h and 2 h + 1 of q) uses key pair j = h / G, whose two
 * maps have key heads 2 j and 2 j + 1 and whose value is 2 D wide, its halves value heads
 * 2 j and 2 j + 1:
 *   x_h = (softmax(scale q_2h K_2j^T) - lam[h] softmax(scale q_2h+1 K_2j+1^T)) [V_2j | V_2j+1]
 *   out_h = out_scale * x_h                                          (norm_weight NULL)
 *   out_h = out_scale * x_h / sqrt(mean(x_h^2) + norm_eps) * norm_weight      (else)
 * with the causal limits, packed rows, cached and new keys of cw.h.  So the pools are
 * those of cw.h with 2 * num_kv_pairs heads, and cw_kv_write_pages, cw_qk_norm_rope, the
 * swaps and the block manager serve them as they are (a new token's two value halves
 * side by side are its value heads 2 j, 2 j + 1).  The pools are only read: the page
 * write of the new K/V is cw_kv_write_pages or cw_qk_norm_rope, before or after.
 *
 *   q bf16 [T, 2 Hp, D], Hp = num_kv_pairs * G;  k_new, v_new bf16 [T, 2 num_kv_pairs, D];
 *   pools [num_pages, 2 num_kv_pairs, P, D], fp8 scales [num_pages, 2 num_kv_pairs];
 *   lam fp32 [Hp], any finite values; norm_weight fp32 [2 D] or NULL; out bf16 [T, Hp, 2 D]
 *
 * Supported: head_dim 64 or 128, page_size 16 or 64, gqa_group 1..16, num_kv_pairs
 * 1..512; out_scale finite, norm_eps finite and >= 0.  Sequences with one new token run on
 * the HBM-streaming kernel, the others on the matrix-core kernel, which over fp8 pools
 * takes q, k_new, v_new and the cached values (code * scale) in fp16: of such a call their
 * magnitudes must lie below 65504 (and are held to 2^-25 where they lie below 2^-14, beside 2^-11
 * of themselves where a V scale does not fit fp16's 11 bits).  Key scales are applied to the
 * scores in fp32 by both.  The streaming kernel has no such limit: V scales may differ as they
 * like.  A scale may be 0 (a page of zeros).  Values (code * scale) lie below 2^80, as they are
 * summed in fp32 with weights of up to 2^16; with a norm, mean(x_h^2) must be an fp32 number:
 * values below about 2^59.  A NaN or infinity in a new token's value may reach the rows of earlier
 * tokens of its sequence (their weight for it is zero); what slots at or past a prefix's end hold
 * changes no result.  Lengths, plan, capture, aliasing and errors as for
 * cw_step_attention; the timing events are not recorded.  Workspace:
 * cw_diff_workspace_bytes (0 if the arguments are invalid). */
size_t cw_diff_workspace_bytes(const int32_t* prefix_lens_h, const int32_t* suffix_lens_h,
                               int32_t num_seqs, int32_t num_kv_pairs, int32_t gqa_group,
                               int32_t head_dim, int32_t page_size, cw_kv_dtype_t kv_dtype);
cw_status_t cw_diff_attention(const void* q, const void* k_new, const void* v_new,
                              const void* k_pool, const void* v_pool, const float* k_scale,
                              const float* v_scale, const int32_t* block_table,
                              int32_t bt_stride, int32_t num_pages,
                              const int32_t* prefix_lens_h, const int32_t* suffix_lens_h,
                              int32_t num_seqs, int32_t num_kv_pairs, int32_t gqa_group,
                              int32_t head_dim, int32_t page_size, float softmax_scale,
                              cw_kv_dtype_t kv_dtype, const float* lam, const float* norm_weight,
                              float norm_eps, float out_scale, void* out, void* workspace,
                              size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CW_LAYER_H_ */
