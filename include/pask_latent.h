/*
 * pask_latent.h - latent attention under the persistence table, on MI355X
 * (gfx950).
 *
 * A latent-attention layer keeps, in place of keys and values per head, one
 * vector a token shared by all heads: a latent c_t (rank elements) and a
 * rotary key r_t (rope_dim elements).  Each head's key is (W_uk c_t, r_t) and
 * its value W_uv c_t.  This header persists those vectors by the same frozen
 * table, under the same rules, statuses, flags and calling conventions as
 * pask.h (DROP / RETAIN-LOW / RETAIN-HIGH; host-side validation before any
 * HIP call; caller-owned memory; asynchronous on the caller's stream; calls on
 * one cache ordered on one stream), reads them back, and attends them in both
 * forms:
 *   absorbed  (one new token): the head's query is taken into the latent
 *             space, q_c = W_uk^T q_nope, and the head's output comes out in
 *             it; keys are (c_t, r_t) and values c_t for every head
 *             (pask_latent_decode_attn).
 *   expanded  (prompts): keys and values per head, from the expansion product
 *             of the latents: of the persisted ones, read back with their
 *             positions (pask_latent_prompt_attn_pos), or of every token
 *             (pask_latent_prompt_attn).
 * The products with W_uk and W_uv are the caller's.
 *
 * Formats:
 *   RETAIN-HIGH  bf16 latent and rotary key.
 *   RETAIN-LOW   the latent as int4 by pask.h's rule (one fp16 scale per 32
 *                elements, s = RNE_fp16(absmax / 7) saturated at 65504, code
 *                clamp(RNE(x / s), -7, 7), 0 when s == 0), the rotary key bf16.
 *                A code q stands for the value RNE_bf16(q * s): the read-back
 *                returns it and the attention uses it, so both forms see the
 *                same cache.
 *   Inputs are taken as finite; a non-finite latent kept HIGH is kept as it is.
 *
 * Numerics of both attentions: scores, softmax statistics and all sums in fp32;
 * a softmax weight is rounded once to bf16 (half a step, 2^-8 of it) for its
 * product with the value, its sum is kept of the unrounded ones.  Weights are
 * taken relative to a reference that a score may exceed by 16 in base 2 before
 * it moves, so sums of values reach 2^16 times their result: an output element
 * is certain to be finite where the query's scores, and the sums they are made
 * of, are finite in fp32 and the magnitudes of its values, over the entries that
 * the query sees, sum to less than 2^112 (5e33).
 *
 * Not here: the recent window (a policy whose recent_window is not 0 is
 * refused with PASK_E_UNSUPPORTED) and the online controller (Eq. 10 decides
 * every token; a policy's controller section is ignored).
 */
#ifndef PASK_LATENT_H
#define PASK_LATENT_H

#include "pask.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PASK_LATENT_MAX_HEADS 128

/* Geometry.  Supported: rank 128, 256 or 512; rope_dim 32 or 64; n_q_heads
 * 1..128; page_tokens 16. */
typedef struct pask_latent_geom {
  int32_t max_batch;           /* sequences the cache holds, 1..65535             */
  int32_t n_layers;            /* layers the cache holds (== policy n_layers)     */
  int32_t n_q_heads;
  int32_t rank;                /* elements of a latent                            */
  int32_t rope_dim;            /* elements of a rotary key                        */
  int32_t page_tokens;         /* 16                                              */
  int32_t max_tokens_per_seq;  /* positions per (sequence, layer)                 */
  int32_t hi_pages;            /* pages in the RETAIN-HIGH pool (all layers)      */
  int32_t lo_pages;            /* pages in the RETAIN-LOW pool (all layers)       */
} pask_latent_geom;

/* A cache: geometry plus one caller-owned device buffer of
 * pask_latent_cache_bytes(&geom) bytes, 256-byte aligned. */
typedef struct pask_latent_cache {
  pask_latent_geom geom;
  void* base;
  uint64_t bytes;
} pask_latent_cache;

/* Region offsets of a cache of this geometry, in the fields of pask.h's
 * layout (status, counters, block tables, index lists and cursors mean the
 * same; there is no window).  The pages, with q = (d mod 32) / 8 and
 * u = t XOR 12 (q mod 2) for element d of slot t:
 *   hi_page_bytes  16 (rank + rope_dim) 2: the 16-byte chunk of elements
 *                  32i + 8q .. + 7 of slot t is chunk 64 i + 16 q + u; the
 *                  rotary key follows the latent as elements rank + e
 *   lo_page_bytes  16 (rank / 2 + rank / 16 + 2 rope_dim): code words, word
 *                  (16 i + t) 4 + q holding elements 32i + 8q .. + 7 (element
 *                  j < 4 in the low nibble of byte j, element 4 + j in its
 *                  high nibble, as c + 8); fp16 scales, half 16 i + t; then
 *                  the rotary keys' chunks as in a HIGH page (i from 0)
 * PASK_E_ARG (null), PASK_E_SHAPE (unsupported). */
int pask_latent_cache_layout_query(const pask_latent_geom* geom, pask_cache_layout* out);

/* Bytes a cache of this geometry needs; 0 if the geometry is unsupported. */
size_t pask_latent_cache_bytes(const pask_latent_geom* geom);

/* Bind a caller-owned device buffer (>= pask_latent_cache_bytes, 256-byte
 * aligned) to a cache and reset it.  Errors: PASK_E_ARG, PASK_E_SHAPE,
 * PASK_E_CAPACITY, PASK_E_HIP. */
int pask_latent_cache_init(pask_latent_cache* cache, const pask_latent_geom* geom, void* base, size_t bytes,
                           hipStream_t stream);

/* Empty every sequence, as pask_cache_reset. */
int pask_latent_cache_reset(pask_latent_cache* cache, hipStream_t stream);

/* Persist new tokens for one layer, by the rules of pask_kv_append: for
 * sequence b < batch the next n_new[b] tokens (n_new_dev int32 [batch]; NULL:
 * max_new each) with tags tags_dev[b][0..n_new[b]) (u8 [batch][max_new]; may be
 * NULL in a KEEP_ALL call), latents c_dev bf16 [batch][max_new][rank] and
 * rotary keys r_dev bf16 [batch][max_new][rope_dim].  flags: 0 or
 * PASK_APPEND_KEEP_ALL.
 *
 * Errors: PASK_E_ARG (null or misaligned pointers: c_dev, r_dev 16 bytes,
 * n_new_dev 4; flags), PASK_E_SHAPE (layer, batch or max_new out of range, or
 * max_new above 2^28 - 61, whose pages are more than one launch fills;
 * policy / geometry mismatch), PASK_E_POLICY, PASK_E_UNSUPPORTED (policy with a
 * recent window), PASK_E_HIP. */
int pask_latent_append(const pask_policy* policy, pask_latent_cache* cache, int32_t layer, int32_t batch,
                       const int32_t* n_new_dev, int32_t max_new, const uint8_t* tags_dev, const void* c_dev,
                       const void* r_dev, uint32_t flags, hipStream_t stream);

/* Read the persisted entries of one layer back as dense rows, in position
 * order, packed over the batch: cu_dev int32 [batch + 1] receives the first
 * row of each sequence and the total, and the entries of sequence b go to rows
 * cu[b] .. cu[b + 1] - 1 of c_dev bf16 [rows][rank], r_dev bf16
 * [rows][rope_dim] and pos_dev int32 [rows] (their positions; nullable).
 * RETAIN-LOW latents are returned as the values they stand for.  Entries that
 * would go to row `rows` or behind it are left out (cu[batch] > rows tells),
 * and rows from cu[batch] on are left as they were.  The cache is unchanged.
 *
 * Errors: PASK_E_ARG (null or misaligned pointers: c_dev, r_dev 16 bytes,
 * pos_dev, cu_dev 4; rows < 0), PASK_E_SHAPE (layer or batch out of range;
 * batch * max_tokens_per_seq above 2^31 - 1, which cu could not hold),
 * PASK_E_HIP. */
int pask_latent_read(const pask_latent_cache* cache, int32_t layer, int32_t batch, int32_t rows, void* c_dev,
                     void* r_dev, int32_t* pos_dev, int32_t* cu_dev, hipStream_t stream);

/* Workspace bytes pask_latent_decode_attn needs for `batch` sequences when
 * none holds more than max_ctx_hint persisted entries (a larger count is still
 * correct, only less parallel; a hint below 1 or above max_tokens_per_seq
 * counts as max_tokens_per_seq); 0 for an invalid geometry or batch outside
 * 1..max_batch. */
size_t pask_latent_workspace_bytes(const pask_latent_geom* geom, int32_t batch, int32_t max_ctx_hint);

/* One decode step of one layer in the absorbed form.  Optionally persist one
 * new token per sequence first (tags_new_dev u8 [batch] != NULL; c_new_dev
 * bf16 [batch][rank], r_new_dev bf16 [batch][rope_dim]; the rules of
 * pask_latent_append), then for every head h, over the persisted entries j of
 * the layer, with q_dev bf16 [batch][n_q_heads][rank + rope_dim] holding
 * (q_c, q_r):
 *   s_j       = softmax_scale * (q_c . c_j + q_r . r_j)
 *   out[b][h] = sum_j softmax_j(s) c_j            (bf16 [batch][n_q_heads][rank])
 *   lse[b][h] = ln sum_j exp(s_j)                 (fp32 [batch][n_q_heads]; nullable)
 * A sequence with no entry gives out = 0 and lse = -inf.
 * ws_dev: device workspace of at least pask_latent_workspace_bytes(geom,
 * batch, max_ctx_hint) bytes, 256-byte aligned; calls that overlap in time
 * need workspaces of their own.
 *
 * Errors: PASK_E_ARG (null or misaligned pointers: q_dev, out_dev, c_new_dev,
 * r_new_dev 16 bytes, lse_dev 4; softmax_scale, or its product with log2 e,
 * not finite in fp32), PASK_E_SHAPE,
 * PASK_E_POLICY, PASK_E_UNSUPPORTED (policy with a recent window),
 * PASK_E_CAPACITY (workspace too small), PASK_E_HIP. */
int pask_latent_decode_attn(const pask_policy* policy, pask_latent_cache* cache, int32_t layer, int32_t batch,
                            const void* q_dev, void* out_dev, float* lse_dev, const uint8_t* tags_new_dev,
                            const void* c_new_dev, const void* r_new_dev, float softmax_scale, int32_t max_ctx_hint,
                            void* ws_dev, size_t ws_bytes, hipStream_t stream);

/* Causal attention of prompts in the expanded form, over a packed batch:
 * sequence b has the queries of rows cu_q[b] .. cu_q[b + 1] - 1 and the keys of
 * rows cu_k[b] .. cu_k[b + 1] - 1 (int32 [batch + 1] each, device).  With n_q
 * and n_k rows, query i sees the keys j <= i + (n_k - n_q): the queries are the
 * last n_q tokens of the sequence, so a prompt's later chunk follows its
 * earlier ones (with n_k < n_q the first queries see nothing).  That is so where
 * every token of the chunk has a row among the keys; over the rows of a
 * read-back, which lack the tokens the table dropped, use
 * pask_latent_prompt_attn_pos.  For head h < n_heads
 *   q_dev   bf16 [total_q][n_heads][nope_dim + rope_dim]
 *   kv_dev  bf16 [total_k][n_heads][nope_dim + v_dim]   (key part, then value)
 *   r_dev   bf16 [total_k][rope_dim]                    (shared by the heads)
 *   out[i][h] = sum_j softmax_j(softmax_scale * q_i . (k_j, r_j)) v_j
 *               (bf16 [total_q][n_heads][v_dim])
 *   lse[i][h] = ln sum exp of the scaled scores (fp32 [total_q][n_heads]; nullable)
 * A query that sees no key gives out = 0 and lse = -inf.  max_q: the most
 * queries of one sequence (queries past it are not computed).  Rows from
 * cu_q[batch] on are left as they were; offsets outside [0, total] are taken
 * as the nearest end of it.
 * Supported: nope_dim and v_dim 64 or 128, rope_dim 32 or 64, n_heads 1..128,
 * batch 1..65535.
 *
 * Errors: PASK_E_ARG (null or misaligned pointers: q_dev, kv_dev, r_dev,
 * out_dev 16 bytes, the others 4; a negative size; softmax_scale, or its
 * product with log2 e, not finite in fp32),
 * PASK_E_SHAPE (unsupported dimensions, or batch * n_heads *
 * ceil(max_q / (64 if max_q <= 64 else 256)) of 2^23 or more),
 * PASK_E_HIP.  With max_q or total_q 0 nothing is done; with total_k 0 the
 * pointers of keys are not read. */
int pask_latent_prompt_attn(int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim,
                            int32_t max_q, int32_t total_q, int32_t total_k, const int32_t* cu_q_dev,
                            const int32_t* cu_k_dev, const void* q_dev, const void* kv_dev, const void* r_dev,
                            void* out_dev, float* lse_dev, float softmax_scale, hipStream_t stream);

/* pask_latent_prompt_attn over keys at given positions, as pask_latent_read
 * returns them: pos_dev int32 [total_k], not descending within a sequence, and
 * q_first_dev int32 [batch], the position of each sequence's first query.  Query
 * i of sequence b sees the keys of the sequence at positions
 * <= q_first[b] + i: the persisted entries that a decode step at that position
 * would attend.  A token that the table dropped is seen by no query, its own
 * neither.  (With positions that do descend it is not said which keys are seen;
 * nothing outside the sequence is.)
 *
 * Errors: as pask_latent_prompt_attn; PASK_E_ARG also for q_first_dev null,
 * pos_dev null with total_k > 0, or either not 4-byte aligned. */
int pask_latent_prompt_attn_pos(int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim,
                                int32_t max_q, int32_t total_q, int32_t total_k, const int32_t* cu_q_dev,
                                const int32_t* cu_k_dev, const int32_t* pos_dev, const int32_t* q_first_dev,
                                const void* q_dev, const void* kv_dev, const void* r_dev, void* out_dev,
                                float* lse_dev, float softmax_scale, hipStream_t stream);

/* Counters of the cache, as pask_cache_stats (without per_seq_group_head). */
int pask_latent_cache_stats(const pask_policy* policy, const pask_latent_cache* cache, int32_t batch,
                            pask_stats* out, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PASK_LATENT_H */
