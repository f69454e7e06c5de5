/*
 * planfront_ops.h -- the operators of one decode layer, exported by libplanfront.so beside the plan-scoring ABI.
 *
 * The serving model of planfront.h prices a decode step as, per layer, max(compute, HBM) of the attention (its
 * weights and the cached keys and values of the running sequences) and of the experts (the weights of those that a
 * token chose), at efficiencies the caller measured.  Here are the two kernels whose time it prices, and what stands
 * around them in a layer, for a caller who wants the HBM rate that they reach on this GPU or checks a ranked plan with
 * the layer itself:
 *
 *   pf_decode_attention   one query token per sequence against an 8-bit paged cache           (priced)
 *   pf_moe_forward        router, routed and shared experts of a few tokens                   (priced)
 *   pf_add_rms_norm       residual addition, root-mean-square norm, output in 8 bits with scales
 *   pf_kv_append          new keys and values into the cache, one scale per page and head
 *
 * Conventions are those of planfront.h: int32 status codes, "d_" pointers are device memory owned by the caller, the
 * library allocates nothing, all work is enqueued on `stream` and nothing synchronizes.  Every pointer must belong
 * to the device that is current.  8-bit values are e4m3 (4 exponent bits, 3 mantissa bits, largest 448, no
 * infinity), rounded to nearest even and saturated.  Workspaces are 256-byte aligned, their contents are ignored.
 * Sizes are checked on the host; what lives in device memory (lengths, page tables) is checked by the kernels, as
 * each call says.
 */
#ifndef PLANFRONT_OPS_H
#define PLANFRONT_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { PF_DT_BF16 = 0, PF_DT_F16 = 1, PF_DT_F32 = 2, PF_DT_E4M3 = 3 };
#define PF_NORM_MAX_H 16384
#define PF_SCALE_GROUP 128      /* elements of a row that share an activation scale; side of a weight-scale block */

/* a = x + residual (32 bits, not rounded in between);  y = a / sqrt(mean(a^2) + eps) * weight;
 * per group g of PF_SCALE_GROUP consecutive elements (group = 128) or per row (group = 0):
 *   scale_g = max(max|y| / 448, 2^-100), 1 where the group is zero throughout;  q = e4m3(y / scale_g).
 * d_x, d_residual, d_sum and d_y: `rows` rows of H elements of `dtype` (PF_DT_BF16, F16, F32), row strides in
 * elements; d_q: [rows, H] contiguous; d_scale: [rows, ceil(H / 128)] or [rows].
 *   d_residual NULL: a = x.  d_weight NULL: 1.  d_sum (a, rounded to dtype), d_y (y, rounded) and the pair d_q /
 *   d_scale may each be NULL.  d_sum may be d_residual or d_x themselves (with the same stride), no other overlap.
 * A NaN or an infinity makes its own row's y and q NaN or zero and no other's.  The mean square is fp32: a row whose
 * squares add up to more than 2^128 gives y = 0.
 * Any alignment is taken; pointers and strides that are multiples of 16 bytes are read 16 bytes at a time.
 * PF_EINVAL: a NULL d_x, no output at all, d_q without d_scale, another dtype or group, eps < 0 or not finite, a
 * stride below H; PF_ERANGE: H outside 1 .. PF_NORM_MAX_H, rows < 0 or >= 2^31.  rows = 0 does nothing. */
int pf_add_rms_norm(int32_t dtype, int64_t rows, int32_t H, const void *d_x, int64_t x_stride, const void *d_residual,
                    int64_t residual_stride, const void *d_weight, float eps, int32_t group, void *d_sum,
                    int64_t sum_stride, void *d_y, int64_t y_stride, uint8_t *d_q, float *d_scale, void *stream);

/* An 8-bit paged cache: keys and values [n_pages, n_kv, page, hd] of e4m3 (16-byte aligned), and their scales
 * [n_pages, n_kv], fp32; the value of an element is its byte's times its page and head's scale. */
typedef struct {
    int32_t n_pages, n_kv, page, hd; /* page: 16, 32, 64 or 128 tokens; hd: 64 or 128 */
    uint8_t *d_k, *d_v;
    float *d_k_scale, *d_v_scale;
} pf_kv_cache_t;

/* Append d_cu_new[b + 1] - d_cu_new[b] tokens to each sequence b, behind its d_len[b] cached ones: token j of b is row
 * d_cu_new[b] + j of d_k / d_v (n_new rows of [n_kv, hd], `dtype` bf16 or f16, row strides in elements, a multiple of 8,
 * the base 16-byte aligned) and goes to position d_len[b] + j, page d_table[b * table_cols + position / page].
 * A page and head's scale is the least power of two s >= 2^-100 with max|x| <= 448 s over what the call writes there
 * and, where the page holds earlier tokens of the sequence, no smaller than it was; those tokens' bytes are then brought to
 * the new scale (exactly but for e4m3's underflow).  NaN elements stay NaN and do not count for the maximum; an infinity
 * saturates, and the scale is bounded by 2^118.
 * max_new: upper bound of tokens appended to one sequence (the kernel appends no more).  Tokens whose page index is
 * outside the table, whose page is outside the cache or whose row is outside [0, n_new) are not written.  No two
 * sequences may append to the same page in one call.  d_len is not advanced.
 * PF_EINVAL: NULL or misaligned pointers, another dtype, page or hd, bad strides; PF_ERANGE: negative or too large
 * counts.  n_seq = 0, n_new = 0 or max_new = 0 does nothing. */
int pf_kv_append(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int64_t n_new, int32_t max_new, const void *d_k,
                 int64_t k_stride, const void *d_v, int64_t v_stride, const int32_t *d_cu_new, const int32_t *d_len,
                 const int32_t *d_table, int32_t table_cols, void *stream);

/* out[b, h] = sum_t softmax_t(sm_scale * q[b, h] . K[t]) V[t] over the d_len[b] cached tokens of sequence b, query head h
 * reading key / value head h / (n_heads / n_kv).  q, out: n_seq rows of [n_heads, hd], `dtype` bf16 or f16, row
 * strides in elements (multiples of 8, 16-byte aligned bases).  d_lse (may be NULL): [n_seq, n_heads] fp32,
 * log(sum_t exp(sm_scale * q . K[t])).  A sequence of length <= 0 gives zeros and -infinity, and so
 * does every one with a table of no columns (d_table may then be NULL).  Nothing beyond d_len[b] is
 * read, so what lies there may be NaN.  Tokens on a page outside the cache, or past the table's columns, are left out.
 * A query element that is not finite makes its own head's out and lse NaN (0 and -infinity where all its scores are
 * -infinity) and no other's.
 * Keys and values are exact, scores, maxima and sums fp32; a token's weight enters the values' sum with 11 bits (fewer below 2^-29 of
 * the row's largest, none below 2^-40; a page's value scale counts with the weight there), and the denominator with all of them.
 * Scales in the cache have to be positive and finite (below 2^-60 a value scale counts as 2^-60).
 * Several query tokens of one sequence are several rows with the same table row and their own lengths.
 * PF_EINVAL: NULL or misaligned pointers, another dtype, page or hd, n_heads not a multiple of n_kv, sm_scale not
 * finite; PF_ERANGE: counts out of range (n_seq <= PF_ATTN_MAX_SEQ; the table's room, n_seq * table_cols * page, below
 * 2^36 tokens and below 2^31 for one sequence); PF_EWORKSPACE. */
#define PF_ATTN_MAX_SEQ 8192
size_t pf_decode_attention_workspace(const pf_kv_cache_t *cache, int32_t n_seq, int32_t n_heads);
int pf_decode_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q,
                        int64_t q_stride, const int32_t *d_len, const int32_t *d_table, int32_t table_cols, float sm_scale,
                        void *d_out, int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes,
                        void *stream);

/* One mixture-of-experts layer as this GPU holds it: experts [first, first + n_local) of n_experts, and n_shared
 * experts that every token takes with weight 1 (indices n_local .. n_local + n_shared - 1 of the weight tensors).
 *   logits = x . router^T;  a token's top_k experts are those of the largest logits (ties: the lowest index; a NaN
 *   counts as -infinity);  w = softmax over the chosen logits;
 *   out = sum over the token's chosen local experts of w * down(silu(gate . x) * (up . x)), plus the shared experts.
 * A token none of whose experts is local, on a GPU without shared experts, gives zeros.
 * All sums are fp32.  bf16 weights: tokens as they are, the products' inner activations with 16 bits (two bf16 numbers).  e4m3
 * weights: tokens and inner activations with 11 bits (fp16 times a power of two a row; inner activations also lose what is below
 * 2^-37 |x|^2 times the product of the largest gate and up row norms of their block of 128). */
typedef struct {
    int32_t H, F;                 /* model width (multiple of 16) and expert width (any) */
    int32_t n_experts, first, n_local, n_shared, top_k;
    int32_t wtype;                /* PF_DT_BF16, or PF_DT_E4M3 with one fp32 scale per 128 x 128 block */
} pf_moe_t;
#define PF_MOE_MAX_TOKENS 512
#define PF_MOE_MAX_EXPERTS 512
#define PF_MOE_MAX_CHOICES 16   /* top_k + n_shared */

/* Lay an expert set's weights out for pf_moe_forward, once: gate and up [n_local + n_shared, F, H], down [n_local +
 * n_shared, H, F], row-major and contiguous, 16-byte aligned; with e4m3 weights their scales, d_gate_scale and d_up_scale
 * [n_local + n_shared, ceil(F / 128), ceil(H / 128)], d_down_scale [.., ceil(H / 128), ceil(F / 128)] (NULL with bf16).
 * d_packed: pf_moe_packed_bytes(m) bytes (0 where `m` is not valid), 256-byte aligned; it holds everything that
 * pf_moe_forward needs of the weights.
 * PF_EINVAL: NULL or misaligned pointers, inconsistent pf_moe_t, scales missing or not wanted. */
size_t pf_moe_packed_bytes(const pf_moe_t *m);
int pf_moe_pack(const pf_moe_t *m, const void *d_gate, const void *d_up, const void *d_down, const float *d_gate_scale,
                const float *d_up_scale, const float *d_down_scale, void *d_packed, void *stream);

/* T tokens through the layer.  d_x: T rows of H bf16 (row stride in elements, multiple of 8, 16-byte aligned), what
 * the router reads, and the experts too unless d_xq / d_xscale give the tokens in 8 bits as pf_add_rms_norm writes
 * them (group 128; e4m3 weights only).  d_router: [n_experts, H] bf16, contiguous.  d_packed: see pf_moe_pack.
 * d_out: [T, H] bf16, contiguous.  d_ids [T, top_k] and d_weights [T, top_k]: the router's choice, in order of falling
 * logits (global expert indices).
 * d_status (may be NULL): one word, 0 after a complete call, 1 if a wait inside the kernel ran out.  d_out is then NaN
 * (a part of it that was complete before may be right), with or without d_status.
 * PF_EINVAL: NULL or misaligned pointers, inconsistent pf_moe_t, d_xq without d_xscale or with bf16 weights; PF_ERANGE: T outside 0 .. PF_MOE_MAX_TOKENS; PF_EWORKSPACE; T = 0 does nothing. */
size_t pf_moe_workspace(const pf_moe_t *m, int32_t T);
int pf_moe_forward(const pf_moe_t *m, int32_t T, const void *d_x, int64_t x_stride, const uint8_t *d_xq, const float *d_xscale,
                   const void *d_router, const void *d_packed, void *d_out, int32_t *d_ids, float *d_weights, int32_t *d_status,
                   void *d_workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
