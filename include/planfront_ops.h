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
 *   pf_rope               rotary positions of query or key heads, and their gradient
 *   pf_kv_append_rope     the append with the rotation on the way
 *   pf_prefix_attention   pf_decode_attention for sequences that share long prefixes
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
 * the row's largest, none below 2^-40; a page's value scale counts with the weight there), and the denominator with all of them (weight times value scale
 * from 2^-141 of the row's largest such product on).
 * Scales in the cache have to be positive and at most 2^126 (below 2^-60 a value scale counts as 2^-60).
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

/* Rotary positions.  Pair i of a head's first `rot` elements, i < rot / 2, at position p becomes
 *   (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t),   t = p * freq[i] radians;
 * pair i is elements i and i + rot / 2 (PF_ROPE_HALF) or 2 i and 2 i + 1 (PF_ROPE_INTERLEAVED); elements from `rot` on stay as they are.
 * d_phase: rot / 2 words, freq[i] as a fraction of a turn times 2^64 (pf_rotary_phases), so that angles are exact to 2^-32 turns at every
 * 32-bit position, negative ones included; their sines and cosines carry 2^-23 of their own size (2^-21.4 of the pair's length for what is then rounded to 8 bits).
 * An element that is not finite spoils its own pair only. */
enum { PF_ROPE_HALF = 0, PF_ROPE_INTERLEAVED = 1 };
#define PF_ROPE_MAX_HD 1024
#define PF_ROPE_MAX_HEADS 65535
typedef struct {
    int32_t rot, layout;      /* rot: even, 0 .. hd */
    float amplitude;          /* finite; 1 but for some long-context scalings */
    const uint64_t *d_phase;
} pf_rotary_t;
/* Host: phase[i] = round(frac(freq[i] / (2 pi)) * 2^64), i < n.  PF_EINVAL: NULL, a frequency that is not finite; PF_ERANGE: n < 0. */
int pf_rotary_phases(int32_t n, const double *freq, uint64_t *phase);

/* y[t, h] = rotation of x[t, h] to position d_pos[t], or, where `transposed` is not 0, the transposed matrix times x[t, h]: the gradient with
 * respect to x, given the gradient with respect to y.  Heads of hd contiguous elements of `dtype` (PF_DT_BF16, F16, F32; 32-bit arithmetic, rounded once); strides of a token
 * and of a head in elements, in either order.  d_y may be d_x with the same strides, no other overlap.  Any alignment is taken; with hd and rot
 * multiples of 16, and pointers and strides multiples of 16 bytes, 16 bytes are moved at a time.
 * PF_EINVAL: NULL or misaligned pointers, another dtype or layout, rot odd or above hd, heads or tokens that overlap; PF_ERANGE: counts out of
 * range.  tokens = 0 or heads = 0 does nothing. */
int pf_rope(const pf_rotary_t *rotary, int32_t transposed, int32_t dtype, int64_t tokens, int32_t heads, int32_t hd, const void *d_x, int64_t x_token,
            int64_t x_head, const int32_t *d_pos, void *d_y, int64_t y_token, int64_t y_head, void *stream);

/* pf_kv_append with keys rotated on the way: from `dtype` to 32 bits, rotated, and rounded once, to e4m3; scales are chosen over the rotated
 * keys.  The queries of the same tokens, n_heads heads a row of d_q, are rotated into d_q_out (d_q itself, with the same stride, allowed; n_heads = 0: none).
 * Token j of sequence b has position d_pos[d_cu_new[b] + j] or, where d_pos is NULL, d_len[b] + j; its place in the cache is d_len[b] + j
 * either way.  A query row is written if its token is one of the first max_new of a sequence, whether or not the table has a place for its key;
 * other rows of d_q_out are left as they were.  rotary->rot is a multiple of 16.  d_cu_new does not decrease.
 * Otherwise as pf_kv_append, which see. */
int pf_kv_append_rope(const pf_kv_cache_t *cache, const pf_rotary_t *rotary, int32_t dtype, int32_t n_seq, int64_t n_new, int32_t max_new,
                      int32_t n_heads, const void *d_q, int64_t q_stride, void *d_q_out, int64_t q_out_stride, const void *d_k, int64_t k_stride,
                      const void *d_v, int64_t v_stride, const int32_t *d_cu_new, const int32_t *d_len, const int32_t *d_table,
                      int32_t table_cols, const int32_t *d_pos, void *stream);

/* Single-token attention of sequences that share prefixes: sequences d_cu_seqs[g] .. d_cu_seqs[g + 1] - 1 see, in front of their own d_len[b]
 * cached tokens (table row b), the d_prefix_len[g] tokens on the pages of prefix table row g.  A prefix is read once for all rows of its group that fit a
 * tile of 256 (sequences times query heads of a key head), not once a sequence.
 *   out[b, h] = softmax over both of sm_scale * q[b, h] . K[t], times V[t]
 * d_cu_seqs: n_groups + 1 offsets that do not decrease (NULL, with one group: all sequences); a sequence in no group sees its own tokens only.  Prefixes of any length, and tables, lengths,
 * missing pages, scales, q, out and lse otherwise as in pf_decode_attention.  A row that sees no token gives zeros and -infinity.
 * Weights enter the values' sum with the bits that they have there; scores of any finite size are taken.
 * A wait inside the kernel that runs out makes the rows that it concerns NaN; pf_prefix_attention_status says so too: one int32 of device memory, 0 after a
 * complete call, 1 otherwise (d_status may be NULL: pf_prefix_attention).
 * Values are added up in 32 bits over 65536 tokens at a time, more in calls of more than 4.8 million (tile of rows, 128 tokens) pairs.
 * PF_EINVAL, PF_ERANGE (also: n_groups above PF_PREFIX_MAX_GROUPS, a prefix table row with room for more than PF_PREFIX_MAX_TOKENS, n_seq * n_heads
 * of 2^30 and more), PF_EWORKSPACE as there.  n_groups = 0: no sequence has a prefix. */
#define PF_PREFIX_MAX_GROUPS 1024
#define PF_PREFIX_MAX_TOKENS 2147479552 /* 2^31 - 4096 */
size_t pf_prefix_attention_workspace(const pf_kv_cache_t *cache, int32_t n_seq, int32_t n_heads, int32_t n_groups, int32_t prefix_cols);
int pf_prefix_attention(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q, int64_t q_stride,
                        const int32_t *d_len, const int32_t *d_table, int32_t table_cols, int32_t n_groups, const int32_t *d_cu_seqs,
                        const int32_t *d_prefix_len, const int32_t *d_prefix_table, int32_t prefix_cols, float sm_scale, void *d_out,
                        int64_t out_stride, float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream);
int pf_prefix_attention_status(const pf_kv_cache_t *cache, int32_t dtype, int32_t n_seq, int32_t n_heads, const void *d_q, int64_t q_stride,
                               const int32_t *d_len, const int32_t *d_table, int32_t table_cols, int32_t n_groups, const int32_t *d_cu_seqs,
                               const int32_t *d_prefix_len, const int32_t *d_prefix_table, int32_t prefix_cols, float sm_scale, void *d_out,
                               int64_t out_stride, float *d_lse, int32_t *d_status, void *d_workspace, size_t workspace_bytes, void *stream);

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
