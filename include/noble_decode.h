/*
 * noble_decode.h - C ABI of libnoble, continued: decoding over the paged cache
 * of noble_attn.h beyond one token after the other.
 *
 *   noble_tree_rows        a tree of drafted tokens: who sees whom, positions
 *   noble_attn_tree        attention of such a tree's tokens over the cache
 *   noble_cache_keep       chosen tokens moved to the front of their place
 *   noble_page_means       means of the keys of the newest tokens' pages
 *   noble_block_select     the pages whose means a new token's queries favour
 *   noble_attn_blocks      attention of the newest tokens over selected pages
 *   noble_attn_weigh       attention of the newest tokens, and the weight that
 *                          every cached token receives
 *   noble_evict_select     the tokens with the most weight
 *
 * Conventions as in noble_attn.h, whose noble_paged_desc and noble_cache_desc
 * these calls take: sequence b holds lengths[b] tokens (cut to table_row *
 * page), its last new_tokens ones are the rows of q; negative lengths are
 * zero.  Tokens in pages outside the cache are not there: not seen, not
 * moved.  `window` must be 0 here.  Where a call writes to the cache or to
 * means of its pages, different sequences' pages are distinct.
 */
#ifndef NOBLE_DECODE_H
#define NOBLE_DECODE_H

#include "noble_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- a tree of drafted tokens ------------------------------------------ */

/* The last `new_tokens` (1 to NOBLE_TREE_MOST) tokens of a sequence are the
 * nodes of a tree.  parents[b][i] (int32 [B, new_tokens]) is the node's parent,
 * an earlier node, or -1: the last token before the tree.  A node with any
 * other parent, and one whose line of parents meets such a node, is no node:
 * sequences may draft fewer.  Written, for node i of sequence b:
 *   seen       int32 [B, new_tokens, NOBLE_TREE_WORDS(new_tokens)]: bit c % 32 of word
 *              c / 32 for itself and the nodes of its line of parents c (no node: none)
 *   depths     int32 [B, new_tokens]: the number of nodes above it (no node: -1)
 *   positions  int32 [B, new_tokens]: lengths[b] - new_tokens + depth (no node: 0),
 *              at least 0; NULL: not formed (lengths is not read then). */
#define NOBLE_TREE_MOST 256
#define NOBLE_TREE_WORDS(n) (((n) + 31) / 32)
noble_status noble_tree_rows(int64_t B, int32_t new_tokens, const int32_t* parents,
                             const int32_t* lengths, int32_t* seen,
                             int32_t* depths, int32_t* positions, void* stream);

/* Node i sees the tokens before the tree, the nodes of its line and itself;
 * scores as in noble_attn_paged, the bias by the difference of positions
 * (tokens before the tree stand at their place in the sequence).  No node:
 * o = 0.  seen and depths are noble_tree_rows'. */
noble_status noble_attn_tree_scratch_size(const noble_paged_desc* desc,
                                          size_t* scratch_bytes);
noble_status noble_attn_tree(const noble_paged_desc* desc, const noble_heads* q,
                             const void* cache, const int32_t* page_table,
                             const int32_t* lengths, const int32_t* seen,
                             const int32_t* depths, const float* slopes,
                             const noble_heads* o, void* scratch,
                             size_t scratch_bytes, void* stream);

/* ---- tokens that stay -------------------------------------------------- */

/* Keys and values of token start[b] + kept[b][h][i] of key head h go to the
 * place of token start[b] + i.  kept is int32 [B, kept_heads, most], ascending,
 * with kept_heads = kv_heads or 1 (for all of them); entries below their own
 * i, such as -1 at the end, are skipped.  start: int32 [B], NULL: 0.  What the
 * moved tokens' old places hold, where nothing moved to, stays. */
typedef struct noble_keep_desc {
    int64_t B;
    int64_t table_row;
    int64_t pages;
    int64_t most;         /* up to 2^31 - 4096 */
    int32_t page;
    int32_t kv_heads, head_dim;
    int32_t kept_heads;
    int32_t dtype;        /* noble_dtype */
    int32_t reserved;     /* must be 0 */
} noble_keep_desc;
noble_status noble_cache_keep(const noble_keep_desc* desc, void* cache,
                              const int32_t* page_table, const int32_t* kept,
                              const int32_t* start, void* stream);

/* ---- selected pages ---------------------------------------------------- */

/* means [pages, kv_heads, D], in the storage type: of each page that holds one
 * of a sequence's last new_tokens tokens, the mean of the keys of the tokens
 * that the sequence holds in it, summed in float64 and rounded once.  Other
 * pages' means are left as they are.  The sequence's whole cache when
 * new_tokens is its length or more (up to 2^31 - 4096).  q's fields of the
 * descriptor (heads, scale, softcap) are not used. */
noble_status noble_page_means(const noble_paged_desc* desc, const void* cache,
                              const int32_t* page_table, const int32_t* lengths,
                              void* means, void* stream);

/* For the row of token t and each key head: block c is the c-th page of the
 * sequence, its score the product of its mean and the sum of the queries that
 * share the key head (float64 sums in one order for all blocks and calls: equal
 * means have equal scores; scores no further apart than float64's rounding of
 * such a sum may rank either way).  Of the blocks up to t's own the first `sink`
 * and the last `local` are taken, then those with the highest scores (of equal
 * ones the first; NaN above all), `count` in all.  chosen: int32
 * [B new_tokens, kv_heads, count], ascending, -1 behind the last.  A block
 * outside the cache has a score of minus infinity.  count >= sink + local,
 * local >= 1. */
typedef struct noble_select_desc {
    int32_t count;        /* 1 to 65536 */
    int32_t sink;
    int32_t local;
    int32_t reserved;     /* must be 0 */
} noble_select_desc;
noble_status noble_block_select_scratch_size(const noble_paged_desc* desc,
                                             const noble_select_desc* select,
                                             size_t* scratch_bytes);
noble_status noble_block_select(const noble_paged_desc* desc,
                                const noble_select_desc* select,
                                const noble_heads* q, const void* means,
                                const int32_t* page_table,
                                const int32_t* lengths, int32_t* chosen,
                                void* scratch, size_t scratch_bytes,
                                void* stream);

/* The row of token t sees, of each key head, the tokens up to itself in the
 * blocks chosen[row][head][0 ..] (as noble_block_select writes them).  The
 * list ends before its first entry that is not larger than the one before it,
 * negative, or past t's own block. */
noble_status noble_attn_blocks_scratch_size(const noble_paged_desc* desc,
                                            int32_t count, size_t* scratch_bytes);
noble_status noble_attn_blocks(const noble_paged_desc* desc, int32_t count,
                               const noble_heads* q, const void* cache,
                               const int32_t* page_table, const int32_t* lengths,
                               const int32_t* chosen, const float* slopes,
                               const noble_heads* o, void* scratch,
                               size_t scratch_bytes, void* stream);

/* ---- accumulated weight ------------------------------------------------ */

/* o as noble_attn_paged's without a window, and for every token j that the
 * sequence holds and every key head
 *   weights_out[b][h][j] = weights[b][h][j] + sum of p_j over the rows of the
 *                          sequence's new tokens and the head's queries,
 * p being the rows' softmax; for the new tokens themselves the sum alone, so
 * what weights held there does not matter.  float32 [B, kv_heads, table_row *
 * page]; weights may be weights_out, or NULL: nothing yet.  Entries past a
 * sequence's tokens are not written.  The scratch holds the rows' scores, 4
 * bytes for each row, query head and token of the page table. */
noble_status noble_attn_weigh_scratch_size(const noble_paged_desc* desc,
                                           size_t* scratch_bytes);
noble_status noble_attn_weigh(const noble_paged_desc* desc, const noble_heads* q,
                              const void* cache, const int32_t* page_table,
                              const int32_t* lengths, const float* slopes,
                              const float* weights, float* weights_out,
                              const noble_heads* o, void* scratch,
                              size_t scratch_bytes, void* stream);

/* The `keep` tokens of each sequence and key head that stay: all, if there are
 * no more; else the first `sink`, the last `recent` and, of the others, those
 * with the most weight (of equal ones the first; NaN above all).  weights:
 * float32 [B, heads, row], of which a sequence's first min(lengths[b], row)
 * count.  kept: int32 [B, heads, keep], ascending, -1 behind the last;
 * kept_weights float32, alike: their weights, 0 behind the last (NULL: not
 * formed).  0 <= sink, recent; sink + recent <= keep. */
typedef struct noble_evict_desc {
    int64_t B;
    int64_t row;          /* up to 2^31 - 4096 */
    int32_t heads;
    int32_t keep;         /* 1 to 2^31 - 4096 */
    int32_t sink, recent;
    int32_t reserved[2];  /* must be 0 */
} noble_evict_desc;
noble_status noble_evict_select(const noble_evict_desc* desc, const float* weights,
                                const int32_t* lengths, int32_t* kept,
                                float* kept_weights, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NOBLE_DECODE_H */
