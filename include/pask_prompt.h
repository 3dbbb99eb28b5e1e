/*
 * pask_prompt.h - turns and prompt chunks of grouped-query layers on MI355X
 * (gfx950): the rotation of a chunk's queries and keys at the positions that
 * its tokens take, and the attention of all its queries over the mixed
 * bf16 / int4 cache of pask.h.
 *
 * A chunk goes through a layer in three calls: pask_rope_apply (queries and
 * keys), pask_kv_append (keys and values), pask_prompt_attn (queries).  The
 * same calls take a draft's few tokens, whose attention then verifies them.
 * Rows are padded as in pask_kv_append: token i < n_new[b] of sequence b is
 * row b * max_new + i.
 *
 * Statuses, validation before any HIP call, ownership, stream order and debug
 * mode are those of pask.h.
 */
#ifndef PASK_PROMPT_H
#define PASK_PROMPT_H

#include "pask.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PASK_ROPE_MAX_PAIRS 128
#define PASK_ROPE_MAX_HEAD_DIM 1024
#define PASK_ROPE_MAX_HEADS 1024

/* Which elements of the rotated part, R = rot_dim, make pair i < R / 2. */
enum {
  PASK_ROPE_HALF = 0,         /* i and R / 2 + i */
  PASK_ROPE_INTERLEAVED = 1   /* 2 i and 2 i + 1 */
};

/* Frequencies, from theta_i = base^(-2 i / R) (radians per position). */
enum {
  PASK_ROPE_PLAIN = 0,        /* theta_i */
  PASK_ROPE_LINEAR = 1,       /* theta_i / factor */
  PASK_ROPE_BASE = 2,         /* theta_i of base * factor^(R / (R - 2)): the
                                 last pair's is divided by factor, the first's
                                 kept (R = 2: plain) */
  PASK_ROPE_PARTS = 3         /* g theta_i + (1 - g) theta_i / factor, g rising
                                 from 0 to 1 as the turns of pair i over
                                 original_len positions go from low_turns to
                                 high_turns (not a ramp over i between two
                                 rounded pairs: its frequencies are written
                                 into turns) */
};

/* A rotation: plain data, filled by pask_rope_init.  Passed by value to the
 * kernels, so it needs no device memory.  A caller with frequencies of its own
 * writes them into turns. */
typedef struct pask_rope {
  int32_t head_dim;           /* elements of a head, 2..1024                    */
  int32_t rot_first;          /* the rotated ones are rot_first ..              */
  int32_t rot_dim;            /*   rot_first + rot_dim - 1; even, 2..256        */
  int32_t layout;             /* PASK_ROPE_HALF or PASK_ROPE_INTERLEAVED        */
  float magnitude;            /* multiplies the rotated elements                */
  int32_t reserved;
  double turns[PASK_ROPE_MAX_PAIRS];   /* frequency of pair i in turns (of 2 pi) per position */
} pask_rope;

/* Fill a rotation.  factor, original_len, low_turns and high_turns are read
 * only by the scalings that use them.  Host only: no HIP call.
 *
 * Errors: PASK_E_ARG (null; layout or scaling unknown; base not finite or not
 * above 0, or so far from 1 that a frequency is not; magnitude not finite; where
 * read: factor not finite or below 1, original_len below 1, low_turns not in [0, high_turns)
 * or high_turns not finite), PASK_E_SHAPE (head_dim, rot_first or rot_dim out
 * of range). */
int pask_rope_init(pask_rope* out, int32_t head_dim, int32_t rot_first, int32_t rot_dim, int32_t layout, double base,
                   int32_t scaling, double factor, int32_t original_len, double low_turns, double high_turns,
                   float magnitude);

/* Rotate queries and keys.  Row b * max_new + i, b < batch, i < n_new[b] (int32
 * [batch], device; NULL: max_new; taken into [0, max_new]) is rotated at
 * position p, pos_dev[b * max_new + i] where pos_dev is given (int32 [batch *
 * max_new], device), else first_dev[b * first_stride] + i: with first_dev the
 * n_pos word of a layer's counters (pask_cache_layout) and first_stride
 * n_layers * counter_stride, the positions that pask_kv_append is about to give
 * the rows.  For every head, pair (x, y) and a = 2 pi turns p:
 *   (x, y) -> magnitude (x cos a - y sin a, x sin a + y cos a)
 * and the elements outside the rotated part are copied.  The angle is reduced
 * in 64 bits, sines, cosines and products are of 32, results are rounded once
 * to bf16.
 *   q_in, k_in   bf16, heads of head_dim elements behind each other, rows
 *                q_in_stride (k_in_stride) elements apart: the parts of a fused
 *                projection's rows are taken where they lie
 *   q_out, k_out the same; an output may be its input (same pointer, same
 *                stride) and otherwise overlaps no input or output
 * n_q_heads or n_k_heads 0: that pair of pointers is not used.  Rows at n_new[b]
 * and behind are neither read nor written.
 *
 * Errors: PASK_E_ARG (null rope or a rope not as pask_rope_init leaves it;
 * neither or both of pos_dev and first_dev; first_stride, where it is read, below
 * 0; null pointers, pointers not aligned
 * to their elements; a stride below heads * head_dim; an output that starts at
 * its input with another stride), PASK_E_SHAPE (negative sizes, more than 1,024
 * heads, batch * max_new above 2^31 - 1), PASK_E_HIP.  With batch or max_new 0
 * nothing is done. */
int pask_rope_apply(const pask_rope* rope, int32_t batch, int32_t max_new, const int32_t* n_new_dev,
                    const int32_t* first_dev, int64_t first_stride, const int32_t* pos_dev, int32_t n_q_heads,
                    const void* q_in, int64_t q_in_stride, void* q_out, int64_t q_out_stride, int32_t n_k_heads,
                    const void* k_in, int64_t k_in_stride, void* k_out, int64_t k_out_stride, hipStream_t stream);

/* Workspace bytes pask_prompt_attn needs for these arguments (max_ctx_hint: the
 * most persisted entries of a sequence, window included; a larger count is
 * still correct, only less parallel; below 1 or above max_tokens_per_seq it
 * counts as max_tokens_per_seq).  0 where it needs none, and for an invalid
 * geometry, batch outside 1..max_batch or max_q outside 1..max_tokens_per_seq. */
size_t pask_prompt_workspace_bytes(const pask_geom* geom, int32_t batch, int32_t max_q, int32_t max_ctx_hint);

/* Attention of many query tokens of each sequence over the persisted history
 * of one layer.  Query i < n_q[b] of sequence b (int32 [batch], device; NULL:
 * max_q; taken into [0, max_q]) is at position p = first[b] + i (int32 [batch],
 * device; NULL: the queries are the last tokens appended, first[b] = the
 * sequence's positions - n_q[b]) and sees what the cache holds now at position
 * p and before: HIGH entries as stored, LOW entries as code * scale, and of the
 * recent window, at bf16, the tokens at p and before.  For query head h, reading
 * KV head h / (n_q_heads / n_kv_heads):
 *   out[b][i][h] = sum_j softmax_j(softmax_scale * q . k_j) v_j
 *   lse[b][i][h] = ln sum_j exp(softmax_scale * q . k_j)     (nullable)
 * with q_dev, out_dev bf16 [batch][max_q][n_q_heads][head_dim], lse_dev fp32
 * [batch][max_q][n_q_heads].  A query that sees nothing gives out = 0 and
 * lse = -inf.  Rows at n_q[b] and behind are left as they were.  The cache is
 * not modified.  (A token that the table dropped is seen by no query; with a
 * recent window W, one further than W back from the newest position is seen as
 * it was persisted, also by queries that are less than W behind it.)
 *
 * Numerics: scores, softmax statistics and sums in fp32, a LOW key enters its
 * score exactly; a softmax weight is rounded for its product with the value: to
 * fp16 (half a step, 2^-11 of it, and 2^-33 of the largest) where the value is
 * LOW, to two bf16 parts (2^-16 is lost, as in pask_decode_attn) where it is bf16
 * and max_q * n_q_heads / n_kv_heads is at most 32, a draft's call, and to one
 * bf16 (2^-8) in larger calls; its sum is kept of the unrounded ones; a LOW value is rounded once to fp16 (2^-11 of it, whatever else its page
 * holds); to a LOW key the queries enter as fp16, each row at a power of two
 * that leaves its elements exact down to 2^-28 of the largest.  Weights are taken relative to a reference that a score
 * may exceed by 15 in base 2 before it moves: an output element is certain to be
 * finite where the query's scores and the sums they are made of are finite in
 * fp32 and the magnitudes of its values, over the entries seen, sum to less than
 * 2^112.  A score of -Inf has weight 0 beside finite ones; one of +Inf or NaN makes
 * its query NaN; a value that is not finite reaches its own element of the queries
 * that see it, which are not finite there.
 *
 * ws_dev: device workspace of at least pask_prompt_workspace_bytes(geom, batch,
 * max_q, max_ctx_hint) bytes, 256-byte aligned (ignored where that is 0); calls
 * that overlap in time need workspaces of their own.
 *
 * Errors: PASK_E_ARG (null or misaligned pointers: q_dev, out_dev 16 bytes, the
 * others 4; softmax_scale, or its product with log2 e, not finite in fp32),
 * PASK_E_SHAPE (layer or batch out of range, max_q below 0 or above
 * max_tokens_per_seq, or more blocks than a launch holds), PASK_E_CAPACITY
 * (workspace too small), PASK_E_HIP.  With max_q 0 nothing is done. */
int pask_prompt_attn(const pask_cache* cache, int32_t layer, int32_t batch, int32_t max_q, const int32_t* n_q_dev,
                     const int32_t* first_dev, const void* q_dev, void* out_dev, float* lse_dev, float softmax_scale,
                     int32_t max_ctx_hint, void* ws_dev, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PASK_PROMPT_H */
