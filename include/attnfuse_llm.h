/*
 * attnfuse_llm.h -- operators of language models around the attention of
 * attnfuse.h, in the same library: the norm and rotation of queries and keys, at
 * positions of one axis or several, paged caches, prefixes that a batch shares, and
 * windows whose first tokens stay visible (sinks).
 *
 * The conventions of attnfuse.h hold (ownership, streams, RoPE tables, error
 * codes, validation before any HIP call), with two additions:
 *
 * Strides.  Inputs that a program takes as slices of larger tensors have a
 *           stride for each dimension but the last, in elements.  The last
 *           dimension is contiguous, every stride is >= 0 and a multiple of 16
 *           bytes, and every pointer 16-byte aligned.
 * Workspaces hold a call's intermediate results only: any memory will do from call
 *           to call, but calls that may overlap (on different streams, or replays
 *           of graphs) need one each.
 * Positions and slots are read on the device and cannot be refused by the
 *           call: each entry point says what one out of range does.
 */
#ifndef ATTNFUSE_LLM_H
#define ATTNFUSE_LLM_H

#include "attnfuse.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Norm and rotation of every head's query and key rows in one pass.  For a row
 * x of D values at position p:
 *     y = q_weight o x / sqrt(mean(x^2) + eps)   (k_weight for keys)
 *     out = R_p y                                (out = y for AF_ROPE_NONE)
 * in fp32, rounded once.
 *
 *   Q [B,H,S,D], K [B,H_kv,S,D]   inputs (dtype), with strides
 *   Qr, Kr                        outputs (dtype), contiguous; Qr may be Q and
 *                                 Kr may be K where that is contiguous.  K and
 *                                 Kr may both be NULL (H_kv is then ignored).
 *   q_weight, k_weight            [D], of weight_dtype (AF_DTYPE_*), or NULL: 1
 *   eps                           finite, >= 0
 *   positions                     device int32 [B,S], contiguous, or NULL:
 *                                 0..S-1.  A row whose position is not in [0,
 *                                 rope_table_rows) comes out as NaN.  Not read
 *                                 for AF_ROPE_NONE.
 *   rope, rope_theta, rope_table, rope_table_rows   as attnfuse_fwd (rows >= S
 *                                 without positions, >= 1 with them)
 *   B, H, H_kv >= 1 and <= 16384, 1 <= S <= 2^20; D in {64, 128} (others:
 *   UNSUPPORTED).  H need not be a multiple of H_kv.
 */
int attnfuse_qknorm_rope(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
                         int weight_dtype, float eps,
                         long long q_stride_b, long long q_stride_h, long long q_stride_s,
                         long long k_stride_b, long long k_stride_h, long long k_stride_s,
                         int B, int H, int H_kv, int S, int D, int dtype,
                         int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                         const int* positions, void* stream);

/* Bytes of workspace of attnfuse_qknorm_rope_bwd where a weight's gradient is
 * wanted (the workgroups' partial sums, at most 1025 x D fp32).  H_kv = 0: no
 * keys.  Returns 0 for invalid sizes. */
size_t attnfuse_qknorm_rope_bwd_workspace_bytes(int B, int H, int H_kv, int S, int D, int dtype);

/*
 * Backward of attnfuse_qknorm_rope.  With r = (mean(x^2) + eps)^-1/2, xh = x r,
 * dy = R_p^T dout and g = w o dy:
 *     dx = r (g - xh mean(g o xh)),   dw = sum over all rows of dy o xh
 * The sums of dw are fp32, in an order that the sizes alone fix, and rounded once.
 *
 *   Q, K, weights, eps, strides, positions, rope...   as the forward's
 *   dQr, dKr            the gradients of its outputs (dtype), contiguous
 *   dQ, dK              outputs (dtype), with strides (those of a dimension
 *                       longer than 1 at least D); must not alias inputs
 *   dq_weight, dk_weight  outputs [D] of weight_dtype, or both NULL: not wanted
 *                       (with K = NULL dk_weight is ignored).  Also where the
 *                       weights are NULL (1).
 *   workspace           of at least attnfuse_qknorm_rope_bwd_workspace_bytes
 *                       bytes, 16-byte aligned, where dq_weight is wanted
 * A row whose position is out of range gives a NaN dx and makes dw NaN.
 */
int attnfuse_qknorm_rope_bwd(const void* Q, const void* K, const void* dQr, const void* dKr, void* dQ, void* dK,
                             void* dq_weight, void* dk_weight, const void* q_weight, const void* k_weight,
                             int weight_dtype, float eps,
                             long long q_stride_b, long long q_stride_h, long long q_stride_s,
                             long long k_stride_b, long long k_stride_h, long long k_stride_s,
                             long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
                             long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
                             void* workspace, size_t workspace_bytes,
                             int B, int H, int H_kv, int S, int D, int dtype,
                             int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                             const int* positions, void* stream);

/*
 * The same for T new tokens whose keys and values go to a paged cache: Qr [T,H,
 * D] gets the normed and rotated queries, the pages of K_pages the normed and
 * rotated keys and those of V_pages the values as they are.
 *
 *   Q [T,H,D], K, V [T,H_kv,D]    inputs (dtype); strides per token and head
 *   Qr [T,H,D]                    output (dtype), contiguous; must not alias
 *   K_pages, V_pages              [num_pages, H_kv, page_size, D] (dtype), with
 *                                 strides per page, head and place (those of a
 *                                 dimension longer than 1 at least D)
 *   page_size                     a power of two, 16 .. 2^20 (others:
 *                                 UNSUPPORTED); num_pages * page_size < 2^31
 *   slots                         device int64 [T]: page * page_size + place of
 *                                 the token's key and value.  A slot outside
 *                                 [0, num_pages * page_size) is not written (-1
 *                                 for the padding of a batch).  No two tokens
 *                                 of a call may have the same slot: which of
 *                                 them is left there is then not defined.
 *   positions                     device int32 [T]; needed (and read) with RoPE
 *                                 only.  Out of range: as attnfuse_qknorm_rope
 *                                 (the cached key is NaN too).
 *   norm                          0: rotation alone (eps is ignored; weights
 *                                 must be NULL), else as attnfuse_qknorm_rope
 *   1 <= T <= 2^20; H, H_kv <= 16384.  Other slots of the pages are left as
 *   they are.  (attnfuse_decode_paged reads bf16 pages; pages of AF_DTYPE_FP32 are for
 *   the caller's own use.)
 */
int attnfuse_qknorm_rope_append(const void* Q, const void* K, const void* V, void* Qr, void* K_pages, void* V_pages,
                                const long long* slots, const void* q_weight, const void* k_weight, int weight_dtype,
                                int norm, float eps,
                                long long q_stride_t, long long q_stride_h, long long k_stride_t, long long k_stride_h,
                                long long v_stride_t, long long v_stride_h,
                                long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                                long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                                int T, int H, int H_kv, int D, int num_pages, int page_size, int dtype,
                                int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                                const int* positions, void* stream);

/*
 * Positions of several axes: the same three calls where a row has a position on
 * each of up to four axes (time, height and width of a patch of a video; text
 * has the same on all).  The D/2 pairs of a row are shared out among the axes,
 * sections[a] (>= 1) of them to axis a, D/2 in all:
 *     AF_SECTIONS_BLOCKS   the first sections[0] pairs turn by axis 0, ...
 *     AF_SECTIONS_TURNS    one pair to each axis in turn, as long as it has some
 *                          left
 * Pair i turns by positions[its axis] * w_i; the w_i are those of the table:
 *     AF_FREQUENCIES_SHARED  w_i = theta^(-2i/D) whatever the axis: the table of
 *                            attnfuse_rope_table_fill
 *     AF_FREQUENCIES_OWN     the j-th pair of axis a (from 0) has theta^(-j /
 *                            sections[a]): every axis a ladder of its own
 *
 *   rope           AF_ROPE_NEOX or AF_ROPE_INTERLEAVED: what makes a pair (NONE:
 *                  INVALID)
 *   positions      device int32 [axes, B, S] ([axes, T]), contiguous, needed.  A
 *                  row with a position on any axis that is not in [0,
 *                  rope_table_rows) comes out as NaN.
 *   axes           1 .. 4
 *   sections       [axes] in HOST memory, read during the call
 *   norm           0: rotation alone (r = 1; eps is ignored; weights must be
 *                  NULL).  The backward is then dx = R^T dout: Q, K and the
 *                  workspace are not used and may be NULL (keys are there where
 *                  dKr is), and the weights' gradients must be NULL.
 *   other arguments, workspaces and results as those of the calls above
 */
#define AF_SECTIONS_BLOCKS 0
#define AF_SECTIONS_TURNS 1
#define AF_FREQUENCIES_SHARED 0
#define AF_FREQUENCIES_OWN 1

/* Fill a table [rows, D/2] of (cos, sin) for these sections and frequencies, as
 * attnfuse_rope_table_fill does (its size is attnfuse_rope_table_bytes; one
 * launch). */
int attnfuse_axes_table_fill(float* table, int rows, int D, float rope_theta, int axes, const int* sections,
                             int section_order, int frequencies, void* stream);
int attnfuse_qknorm_axes(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
                         int weight_dtype, int norm, float eps,
                         long long q_stride_b, long long q_stride_h, long long q_stride_s,
                         long long k_stride_b, long long k_stride_h, long long k_stride_s,
                         int B, int H, int H_kv, int S, int D, int dtype,
                         int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                         const int* positions, int axes, const int* sections, int section_order, void* stream);
int attnfuse_qknorm_axes_bwd(const void* Q, const void* K, const void* dQr, const void* dKr, void* dQ, void* dK,
                             void* dq_weight, void* dk_weight, const void* q_weight, const void* k_weight,
                             int weight_dtype, int norm, float eps,
                             long long q_stride_b, long long q_stride_h, long long q_stride_s,
                             long long k_stride_b, long long k_stride_h, long long k_stride_s,
                             long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
                             long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
                             void* workspace, size_t workspace_bytes,
                             int B, int H, int H_kv, int S, int D, int dtype,
                             int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                             const int* positions, int axes, const int* sections, int section_order, void* stream);
int attnfuse_qknorm_axes_append(const void* Q, const void* K, const void* V, void* Qr, void* K_pages, void* V_pages,
                                const long long* slots, const void* q_weight, const void* k_weight, int weight_dtype,
                                int norm, float eps,
                                long long q_stride_t, long long q_stride_h, long long k_stride_t, long long k_stride_h,
                                long long v_stride_t, long long v_stride_h,
                                long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                                long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                                int T, int H, int H_kv, int D, int num_pages, int page_size, int dtype,
                                int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                                const int* positions, int axes, const int* sections, int section_order, void* stream);

/*
 * attnfuse_fwd under a sliding window whose first tokens stay visible: query i
 * sees key j when j <= i and (j > i - window or j < sinks); positions (RoPE) are
 * those in the sequence for sinks too.
 *
 *   window >= 1, sinks >= 1       any values; from window + sinks >= S on this is
 *                                 the causal mask
 *   workspace                     device memory (16-byte aligned) of at least
 *                                 attnfuse_fwd_sinks_workspace_bytes bytes for
 *                                 the rotated keys; 0 bytes, and it may be NULL,
 *                                 without RoPE and for AF_DTYPE_FP32
 *   other arguments and results as attnfuse_fwd; no ALiBi
 * As there, a pair that is not visible counts with weight 0 inside the tiles that a
 * workgroup visits: a NaN or an infinity in a row of V (in the backward of Q, K or
 * dO too) reaches queries that do not see that row.  Every row up to S is finite.
 */
size_t attnfuse_fwd_sinks_workspace_bytes(int B, int H_kv, int S, int D, int dtype, int rope);
int attnfuse_fwd_sinks(const void* Q, const void* K, const void* V, void* O, float* LSE, void* workspace,
                       size_t workspace_bytes, int B, int H, int H_kv, int S, int D, int dtype,
                       int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                       int window, int sinks, float softmax_scale, void* stream);

/* Backward of attnfuse_fwd_sinks; workspace of attnfuse_bwd_sinks_workspace_bytes
 * (0 for invalid sizes), of which the last part, as there, is not required;
 * otherwise as attnfuse_bwd.  The size does not know the type: AF_DTYPE_FP32 needs
 * it too, and uses the part that holds the row statistics. */
size_t attnfuse_bwd_sinks_workspace_bytes(int B, int H, int H_kv, int S, int D, int rope, int window, int sinks);
int attnfuse_bwd_sinks(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                       void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                       int B, int H, int H_kv, int S, int D, int dtype,
                       int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                       int window, int sinks, float softmax_scale, void* stream);

/* Bytes of device workspace of attnfuse_decode_paged and attnfuse_decode_sinks:
 * a partial (max, sum, accumulator) per (sequence, query head) and part of the
 * visible cache.  S_kv is the most keys a sequence may have (max_pages *
 * page_size); window 0 without one.  Returns 0
 * for invalid sizes. */
size_t attnfuse_decode_paged_workspace_bytes(int B, int H, int H_kv, int S_kv, int D, int window, int sinks);

/*
 * attnfuse_decode over a paged cache: one query per sequence, at position L - 1
 * of its L = cache_lens[b] cached keys, which were rotated when they were
 * written (attnfuse_qknorm_rope_append).  Key n of sequence b lies in page
 * block_table[b][n / page_size] at place n % page_size.  Under SLIDING_WINDOW
 * the query sees the last `window` keys and the first `sinks` keys.
 *
 *   Q [B,H,D]                     the newest token's queries (bf16)
 *   K_pages, V_pages              [num_pages, H_kv, page_size, D] (bf16), with
 *                                 strides per page, head and place (place: at
 *                                 most 2^24)
 *   block_table                   device int32 [B, max_pages], contiguous.  An
 *                                 entry outside [0, num_pages) holds no keys:
 *                                 they are not visible.  Entries behind a
 *                                 sequence's length, or between its sinks and
 *                                 its window, are not used.
 *   page_size                     a power of two, 16 .. 2^20 (others:
 *                                 UNSUPPORTED); max_pages * page_size <= 2^20
 *   cache_lens                    device int32 [B] or NULL (every sequence has
 *                                 max_pages * page_size keys); larger values are
 *                                 clamped to that
 *   O [B,H,D] (bf16), LSE [B,H] fp32; a sequence with no visible key gets O = 0,
 *   LSE = -inf.  A NaN in a query, or in a key that it sees, gives a NaN O and LSE.
 *   workspace                     >= attnfuse_decode_paged_workspace_bytes(B, H,
 *                                 H_kv, max_pages * page_size, D, window, sinks)
 *   mask                          NONE, CAUSAL: every cached key; or
 *                                 SLIDING_WINDOW with window >= 1
 *   sinks                         >= 0; only with SLIDING_WINDOW, and without
 *                                 ALiBi where > 0 (else AF_ERR_UNSUPPORTED)
 *   rope, rope_theta, rope_table, alibi_slopes, softmax_scale   as
 *                                 attnfuse_decode (rope_table_rows >= max_pages *
 *                                 page_size).  The rotated query is not rounded
 *                                 to fp16: keys may have any bf16 value, and the
 *                                 LSE is that of the cached keys to 2^-16 of the
 *                                 scores' magnitudes.
 *   D in {64, 128}; B < 2^16; any H <= 16384 that is a multiple of H_kv (a group of
 *   more than 32 query heads reads the cache once for each 32)
 *
 * In a call of given B, max_pages and page_size a sequence's result depends on its own
 * keys and length only, not on the other sequences.  With another B or table width the
 * keys may be shared out otherwise among workgroups: the same result to the rounding of
 * fp32 sums, not the same bits.  What lies in places that are not visible is never used,
 * whatever it is.
 */
int attnfuse_decode_paged(const void* Q, const void* K_pages, const void* V_pages, const int* block_table,
                          const int* cache_lens, void* O, float* LSE, void* workspace, size_t workspace_bytes,
                          long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                          long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                          int B, int H, int H_kv, int D, int num_pages, int page_size, int max_pages,
                          int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                          int mask, int window, int sinks,
                          const float* alibi_slopes, float softmax_scale, void* stream);

/* Bytes of device workspace of attnfuse_fwd_paged: partials (max, sum, accumulator)
 * of every (token, query head), 0 where there are none.  own_keys is max_pages *
 * page_size, prefix_keys prefix_pages * page_size (0: no prefix).  With one token of
 * each sequence T is B.  Returns 0 for invalid sizes too. */
size_t attnfuse_fwd_paged_workspace_bytes(int T, int B, int H, int H_kv, int D, int own_keys, int prefix_keys);

/*
 * Attention of new tokens over a paged cache, behind a prefix that the whole
 * batch shares and that is read once for all of it: prompts in chunks, questions
 * about one text, or one new token of each sequence.
 *
 * Sequence b has the queries of tokens q_starts[b] .. q_starts[b+1] - 1, which are
 * the last n_b of its L_b = cache_lens[b] own keys (written before, as for
 * attnfuse_decode_paged).  Its query t sees every key of the prefix and its own
 * keys 0 .. L_b - n_b + t; where that is none (no prefix, and more queries than own
 * keys), O = 0 and LSE = -inf.
 *
 *   Q [T,H,D]                     queries (bf16), already rotated
 *                                 (attnfuse_qknorm_rope_append): where the prefix
 *                                 ends, and positions of several axes, are the
 *                                 caller's
 *   K_pages, V_pages, strides, page_size   as attnfuse_decode_paged
 *   block_table                   device int32 [B, max_pages]: the pages of each
 *                                 sequence's own keys; as there
 *   q_starts                      device int32 [B + 1], not decreasing, within
 *                                 0 .. T (values outside are clamped), or NULL:
 *                                 one token of each sequence (T == B).  Rows of O
 *                                 and LSE of tokens before q_starts[0] and from
 *                                 q_starts[B] on are left as they are.
 *   cache_lens                    device int32 [B] or NULL (max_pages * page_size
 *                                 each); larger values are clamped to that
 *   prefix_table                  device int32 [prefix_pages]: the pages of the
 *                                 prefix, in order; an entry outside [0,
 *                                 num_pages) holds no keys.  prefix_pages 0, and
 *                                 NULL: no prefix
 *   prefix_len                    device int32 [1]: keys of the prefix, clamped to
 *                                 prefix_pages * page_size; NULL: all of them
 *   O [T,H,D] (bf16), LSE [T,H] fp32
 *   workspace                     >= attnfuse_fwd_paged_workspace_bytes bytes,
 *                                 16-byte aligned; may be NULL where that is 0
 *   D in {64, 128}; B < 2^16, T <= 2^20, T * H <= 2^30; prefix_pages * page_size and
 *   max_pages * page_size <= 2^20; H <= 16384, a multiple of H_kv.  Sequences of fewer
 *   than 1024 (token, head) pairs to a K/V head on average (T * H < 1024 * B * H_kv) take
 *   at least a workgroup each, of which a launch has fewer than 2^24: T * H / 64 +
 *   (B + 1) * H_kv < 2^24, and with a prefix T * H * D < 2^34 (else INVALID)
 *
 * A NaN in a query, or in a key or value that it sees, comes out as NaN.  A NaN or an
 * infinity in the value of one of the sequence's newest n_b own keys may reach queries of
 * the call that do not see it yet (with weight 0); what lies in places past a sequence's
 * length or the prefix's, and in pages of neither, is never used.  The keys are shared out by sizes alone (T, B and the tables' widths)
 * and the same call gives the same bits; in another batch a sequence's result is the same to
 * the rounding of its weights and sums.  Tables much wider than the keys they hold, and many
 * tokens of no sequence, are shared out as if they were full, which costs time.
 */
int attnfuse_fwd_paged(const void* Q, const void* K_pages, const void* V_pages, const int* block_table, const int* q_starts,
                       const int* cache_lens, const int* prefix_table, const int* prefix_len, void* O, float* LSE,
                       void* workspace, size_t workspace_bytes,
                       long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                       long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                       int T, int B, int H, int H_kv, int D, int num_pages, int page_size, int max_pages, int prefix_pages,
                       float softmax_scale, void* stream);

/*
 * attnfuse_decode (a contiguous cache [B,H_kv,S_kv,D]) with sinks: the last
 * `window` keys and the first `sinks` keys of each sequence are visible.
 * window >= 1, sinks >= 1, bf16; arguments, results and workspace otherwise as
 * attnfuse_decode_paged.
 */
int attnfuse_decode_sinks(const void* Q, const void* K, const void* V, const int* cache_lens, void* O, float* LSE,
                          void* workspace, size_t workspace_bytes, int B, int H, int H_kv, int S_kv, int D,
                          int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                          int window, int sinks, float softmax_scale, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTNFUSE_LLM_H */
