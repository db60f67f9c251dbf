/*
 * noble_attn.h - C ABI of libnoble, continued: the operators between the
 * grouped Q/K/V layer (noble.h) and the O layer of a transformer block on AMD
 * Instinct MI355X (gfx950).
 *
 *   noble_qk_rope_fwd / _bwd   norm of every query and key head and rotation
 *                              by position, in one pass over the layer's rows
 *   noble_kv_append            the same on the way into a paged cache
 *   noble_attn_fwd / _bwd      attention over packed sequences
 *   noble_attn_paged           attention of the newest tokens over the cache
 *   noble_rope_table           cosines and sines, scaled for long contexts
 *   noble_mask_rows            documents, prefixes and windows as the key
 *                              intervals that noble_attn_* takes
 *
 * Conventions, as in noble.h where nothing else is said: device memory owned
 * by the caller; nothing allocated, freed, synchronised or kept; work enqueued
 * on `stream`; argument checking complete before any HIP call; outputs alias
 * neither inputs nor each other; status codes of noble.h.  Storage is bf16 or
 * float32 (noble_dtype); norms, angles, softmax statistics and every sum are
 * float32, and bf16 products take bf16 operands: there the probabilities and
 * the score gradients are rounded once, as the products' operands.
 *
 * Pointers to storage are 16-byte aligned and their strides multiples of 8
 * elements, at most 2^22 for rows of a tile; the head dimension D is a
 * multiple of 8, 8 to 128; query heads are a multiple of the key heads, at
 * most 1024.  Index and float32 arrays are aligned to their element.
 */
#ifndef NOBLE_ATTN_H
#define NOBLE_ATTN_H

#include "noble.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A [rows, heads, D] tensor: element (i, h, d) at data[i row + h head + d].
 * Strides in elements; 0 is allowed for inputs (a broadcast). */
typedef struct noble_heads {
    void* data;
    int64_t row;
    int64_t head;
} noble_heads;

/* ---- norm and rotation ------------------------------------------------- */

/* Tokens t < T, rows of x: query heads, then key heads, then (noble_kv_append)
 * value heads, D elements each, rows x_row elements apart.  With weights
 * (both or none) each query and key head is normed,
 *   u = x (mean(x^2) + eps)^(-1/2) weight,
 * and then its first `rot` elements are rotated: for pair i, with c, s =
 * cos, sin[position][i],
 *   (a, b) -> (a c - b s, b c + a s),
 * where (a, b) are elements (i, i + rot / 2), or (2 i, 2 i + 1) when
 * `interleaved`.  rot is 0 or a multiple of 16, at most D.  The tables are
 * float32 [table_rows, rot / 2]; positions int32 [T] (NULL: t).  A token whose
 * position is outside the tables comes out as NaN. */
typedef struct noble_rope_desc {
    int64_t T;
    int64_t x_row;       /* elements between rows of x (and of dx) */
    int64_t table_rows;
    int32_t heads;       /* query heads; 0 is allowed */
    int32_t kv_heads;    /* key heads; 0 is allowed for fwd and bwd */
    int32_t head_dim;
    int32_t rot;
    int32_t interleaved;
    int32_t dtype;       /* noble_dtype */
    float eps;
    int32_t reserved;    /* must be 0 */
} noble_rope_desc;

/* q [T, heads, D] and k [T, kv_heads, D], dense. */
noble_status noble_qk_rope_fwd(const noble_rope_desc* desc, const void* x,
                               const float* q_weight, const float* k_weight,
                               const float* cos, const float* sin,
                               const int32_t* positions,
                               void* q, void* k, void* stream);

/* Bytes of noble_qk_rope_bwd's scratch (0 without weights): partial sums of
 * the weights' gradients, added in a fixed order. */
noble_status noble_qk_rope_scratch_size(const noble_rope_desc* desc,
                                        size_t* scratch_bytes);

/* From dq, dk (dense, as q and k): the query and key columns of dx, rows
 * desc->x_row apart (its other columns are left as they are), and with weights
 * dq_weight, dk_weight float32 [D] (overwritten). */
noble_status noble_qk_rope_bwd(const noble_rope_desc* desc,
                               const void* dq, const void* dk, const void* x,
                               const float* q_weight, const float* k_weight,
                               const float* cos, const float* sin,
                               const int32_t* positions,
                               void* dx, float* dq_weight, float* dk_weight,
                               void* scratch, size_t scratch_bytes,
                               void* stream);

/* cos and sin [length, rot / 2] of positions 0 .. length - 1, in double from
 * the frequencies base^(-2 i / rot), scaled for contexts longer than the
 * model was trained on:
 *   NOBLE_ROPE_PLAIN   as they are
 *   NOBLE_ROPE_LINEAR  positions divided by factor
 *   NOBLE_ROPE_BASE    base raised to base factor^(rot / (rot - 2)): the lowest
 *                      frequency is divided by factor, the highest kept
 *   NOBLE_ROPE_RAMP    frequencies that turn at least `fast` times over the
 *                      trained length kept, those that turn at most `slow`
 *                      times divided by factor, linear in the pair's index
 *                      between; cosines and sines times `gain`
 */
enum { NOBLE_ROPE_PLAIN = 0, NOBLE_ROPE_LINEAR = 1, NOBLE_ROPE_BASE = 2, NOBLE_ROPE_RAMP = 3 };
typedef struct noble_rope_scaling {
    int32_t kind;
    int32_t reserved;     /* must be 0 */
    double base;          /* > 1 */
    double factor;        /* >= 1 (ignored by PLAIN) */
    double trained;       /* RAMP: trained length, > 0 */
    double fast, slow;    /* RAMP: turns, fast > slow > 0 */
    double gain;          /* RAMP: > 0 */
} noble_rope_scaling;
noble_status noble_rope_table(const noble_rope_scaling* scaling, int64_t length,
                              int32_t rot, float* cos, float* sin, void* stream);

/* ---- paged cache ------------------------------------------------------- */

/* The cache is [pages, 2, kv_heads, page, D] in the storage type: keys, then
 * values, of `page` tokens, a power of two from 8 to 4096.  Slot s stands for
 * token s mod page of page s / page. */
typedef struct noble_cache_desc {
    int64_t pages;
    int32_t page;
    int32_t reserved;     /* must be 0 */
} noble_cache_desc;

/* Rows of x (desc->kv_heads key and value heads behind the query heads): the
 * keys, normed and rotated, and the values to the slots (int64 [T]) of the
 * cache, the queries, normed and rotated, to q (dense; NULL: not formed).  A
 * slot outside the cache, such as -1 for a padded row, is not written.  Slots
 * are distinct. */
noble_status noble_kv_append(const noble_rope_desc* desc,
                             const noble_cache_desc* cache_desc, const void* x,
                             const float* q_weight, const float* k_weight,
                             const float* cos, const float* sin,
                             const int32_t* positions, const int64_t* slots,
                             void* q, void* cache, void* stream);

/* ---- attention --------------------------------------------------------- */

/* Row i of query head h sees the keys j in [key_lo[i], key_hi[i]) (int32
 * [Tq], both or none; none: [0, Tk)), with `causal` only j <= i + offset.
 * Intervals are cut to [0, Tk); a row that sees no key gives o = 0,
 * lse = -inf and no gradient (one that sees keys, all with scores of -inf, gives
 * NaN, as the formula does).  With z = scale q_i.k_j:
 *   s = softcap tanh(z / softcap) (softcap 0: z) - slope[h] |i + offset - j|
 *   o_i = sum_j exp(s_j - lse_i) v_j,   lse_i = log sum_j exp(s_j)
 * (slopes float32 [heads], NULL: no bias; constants, without a gradient).
 * Query head h uses key head h / (heads / kv_heads).  Infinite and NaN values
 * reach the rows that see them and no other (such rows, and those beside
 * them, are slow, up to a key at a time, until they are all NaN). */
typedef struct noble_attn_desc {
    int64_t Tq, Tk;       /* rows of q, and of k and v: up to 2^30 - 4096 */
    int64_t offset;       /* key index of query row 0, |offset| <= 2^30 - 4096 */
    int32_t heads, kv_heads, head_dim;
    int32_t dtype;        /* noble_dtype */
    int32_t causal;
    float scale;          /* > 0, finite */
    float softcap;        /* >= 0, finite; 0: none */
    int32_t reserved;     /* must be 0 */
} noble_attn_desc;

/* o [Tq, heads, D]; lse float32 [heads, Tq], dense. */
noble_status noble_attn_fwd(const noble_attn_desc* desc, const noble_heads* q,
                            const noble_heads* k, const noble_heads* v,
                            const int32_t* key_lo, const int32_t* key_hi,
                            const float* slopes, const noble_heads* o,
                            float* lse, void* stream);

/* Bytes of noble_attn_bwd's scratch, whose contents need no
 * initialisation. */
noble_status noble_attn_bwd_scratch_size(const noble_attn_desc* desc,
                                         size_t* scratch_bytes);

/* Gradients for the upstream gradient `grad` of o, from the forward's inputs,
 * o and lse.  dq, dk, dv are overwritten; a key head's gradients are the sums
 * over its query heads.  Every output is summed in a fixed order. */
noble_status noble_attn_bwd(const noble_attn_desc* desc, const noble_heads* grad,
                            const noble_heads* q, const noble_heads* k,
                            const noble_heads* v, const noble_heads* o,
                            const float* lse,
                            const int32_t* key_lo, const int32_t* key_hi,
                            const float* slopes, const noble_heads* dq,
                            const noble_heads* dk, const noble_heads* dv,
                            void* scratch, size_t scratch_bytes, void* stream);

/* ---- attention over the cache ------------------------------------------ */

/* Sequence b holds lengths[b] tokens (int32 [B]) in the pages
 * page_table[b][0 ..] (int32 [B, table_row]), at most table_row * page.  Its
 * queries are `new_tokens` rows of q, b new_tokens ..: its last tokens, which
 * the cache holds already.  The row of token t sees the tokens 0 .. t, with a
 * window only the last `window` of them (0: all).  A token whose page is
 * outside the cache is not seen; nor is, for a row of a token before the
 * first, anything, which gives zeros.  Scores as in noble_attn_fwd.  Slots
 * past a sequence's tokens, and before every row's window, may hold anything;
 * infinite and NaN values reach the rows that see them, and no others. */
typedef struct noble_paged_desc {
    int64_t B;
    int64_t table_row;    /* entries of one sequence's page table */
    int64_t pages;
    int32_t page;
    int32_t new_tokens;   /* 1 to 2^20 */
    int32_t window;
    int32_t heads, kv_heads, head_dim;
    int32_t dtype;        /* noble_dtype */
    float scale;
    float softcap;
    int32_t reserved;     /* must be 0 */
} noble_paged_desc;

noble_status noble_attn_paged_scratch_size(const noble_paged_desc* desc,
                                           size_t* scratch_bytes);

/* o [B new_tokens, heads, D]. */
noble_status noble_attn_paged(const noble_paged_desc* desc, const noble_heads* q,
                              const void* cache, const int32_t* page_table,
                              const int32_t* lengths, const float* slopes,
                              const noble_heads* o, void* scratch,
                              size_t scratch_bytes, void* stream);

/* ---- masks ------------------------------------------------------------- */

/* Intervals of `T` packed rows: document n holds the rows starts[n] ..
 * starts[n + 1] - 1 (int32 [documents + 1], ascending).  A row sees its
 * document's rows up to itself (causal) or all of them; the first prefix[n]
 * rows (int32 [documents], NULL: none) also when they come later; with a
 * window (> 0) only the `window` rows that end with the last one it sees.
 * key_lo, key_hi, positions (int32 [T]; positions, the row's place in its
 * document, may be NULL).  A row of no document sees nothing, at position 0. */
noble_status noble_mask_rows(int64_t T, int64_t documents, const int32_t* starts,
                             const int32_t* prefix, int32_t causal, int32_t window,
                             int32_t* key_lo, int32_t* key_hi,
                             int32_t* positions, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NOBLE_ATTN_H */
