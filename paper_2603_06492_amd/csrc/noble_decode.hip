// libnoble: C ABI of decoding over the paged cache (include/noble_decode.h).
//
// Host side: argument validation (complete before any HIP call), scratch layout, launch rules and launches on the
// caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "noble_attn_host.hpp"
#include "noble_decode.h"
#include "noble_decode_attn.hpp"
#include "noble_decode_select.hpp"
#include "noble_decode_wide.hpp"

using namespace noble;

namespace {

constexpr int64_t kMaxScratch = int64_t(1) << 46;

// The fields of the cache and its sequences; new tokens up to `most`.
noble_status check_cache(const noble_paged_desc* d, int64_t most) {
    if (!d) return NOBLE_ERR_NULL_ARG;
    if (!dtype_ok(d->dtype)) return NOBLE_ERR_BAD_DTYPE;
    if (d->reserved != 0 || d->window != 0 || d->B < 0 || d->new_tokens < 1 || d->new_tokens > most) return NOBLE_ERR_BAD_SHAPE;
    if (d->page < 8 || d->page > 4096 || (d->page & (d->page - 1))) return NOBLE_ERR_BAD_SHAPE;
    if (d->B > kMaxRows || d->table_row < 0 || d->table_row > kMaxRows / d->page || d->pages < 0 || d->pages > INT32_MAX)
        return NOBLE_ERR_BAD_SHAPE;
    if (d->kv_heads < 1 || d->kv_heads > kMaxHeads || !head_dim_ok(d->head_dim)) return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}
// And those of the new tokens' queries.
noble_status check_rows(const noble_paged_desc* d, int64_t most) {
    NOBLE_TRY(check_cache(d, most));
    if (d->B > kMaxRows / d->new_tokens || d->heads < 1 || d->heads > kMaxHeads || d->heads % d->kv_heads)
        return NOBLE_ERR_BAD_SHAPE;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale) || !(d->softcap >= 0.f) || !std::isfinite(d->softcap))
        return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}
noble_status check_tables(const noble_paged_desc* d, const int32_t* page_table, const int32_t* lengths) {
    NOBLE_TRY(need_array(page_table, d->B > 0 && d->table_row > 0, 4));
    return need_array(lengths, d->B > 0, 4);
}

constexpr int64_t kMostNew = 1 << 20;

// Workgroups that cache_keep_kernel is to have, at least.
constexpr int64_t kMoving = 512;

// Rows from which weigh_kernel splits them into slices.
constexpr int kManyRows = 16, kManySlices = 16;

// Workgroups of one attention call and its scratch.
struct DecodePlan {
    int wide;                             // waves of attn_wide_kernel; 0: R groups of 16 rows of attn_decode_kernel
    bool split;                           // some pieces are joined
    int64_t R, row_tiles, slots, groups;
    size_t where, stats, z, bytes;        // offsets (the parts come first), and all of it
    int64_t chunks;
};

template <int FORM>
noble_status decode_plan(const noble_paged_desc* d, int64_t count, DecodePlan* p) {
    const int64_t share = d->heads / d->kv_heads, rows = d->new_tokens * share;
    // Little work, up to eight chunks for each wave of 256 workgroups of one group of rows, is latencies and code that runs once:
    // one group a workgroup, for all that the cache is read again.  47 trees of 8 with 8 heads to a key head over 8 to 155
    // tokens 58 -> 28 us, 64 of one head over 1000 25 -> 16, 2 of 64 over 4000 35 -> 27.  It goes by the page table: in one
    // for 4096 tokens the same 47 trees take 59.
    const int64_t chunks = d->B * (d->table_row * d->page / kKeys + 1);
    const bool little = chunks <= 8192 && chunks * d->kv_heads * cdiv(rows, kGroup) <= 8192;
    p->wide = FORM == kBlocks || d->dtype != NOBLE_BF16 || rows <= 2 * kGroup || little ? 0 : rows > 128 ? 8 : 4;
    p->R = p->wide ? 32 * p->wide / kGroup : FORM != kBlocks && rows > kGroup && !little ? 2 : 1;
    p->row_tiles = FORM == kBlocks ? d->new_tokens * cdiv(share, kGroup) : (rows + kGroup * p->R - 1) / (kGroup * p->R);
    // Workgroups that run at once: one a CU, by their LDS, or two of attn_wide_kernel's with four waves.  More of them in turn,
    // or smaller ones beside each other, read the cache more slowly: one token of 64 sequences of 16384 to 32768 tokens with
    // its weights, 256 workgroups of four waves 0.60 ms, 1280 of one wave 0.68.
    const int64_t resident = p->wide == 4 ? 512 : 256;
    const int64_t per = d->kv_heads * p->row_tiles;   // workgroups that read the same keys, or keys of other heads
    int64_t parts;
    // Of so many workgroups `one`, up to `most` of them: as many as fill those that run at once best, once, or a few times
    // where once is not near.
    const auto filling = [&](int64_t one, int64_t most) {
        int64_t slots = 1;
        double best = -1.0;
        for (int64_t turn = 1; turn <= 4 && one > 0; ++turn) {
            const int64_t n = std::clamp<int64_t>(resident * turn / one, 1, most), all = n * one;
            const double fill = (double)all / (double)((all + resident - 1) / resident * resident);
            if (fill > best + 0.1) {
                best = fill;
                slots = n;
            }
        }
        return slots;
    };
    if (FORM == kBlocks) {
        const int64_t waves = d->dtype == NOBLE_F32 && d->head_dim > 64 ? 2 : 4, lists = d->B * per;
        p->slots = filling(lists, std::clamp<int64_t>(std::min(count, d->table_row) * d->page / kKeys / waves, 1, 64));
        p->groups = lists * p->slots;
        parts = p->groups;
    } else {
        const int64_t steps = d->B * (d->table_row * d->page / (p->wide ? kPart : kKeys) + 1);
        if (steps > INT32_MAX) return NOBLE_ERR_BAD_SHAPE;   // the kernels count them in 32 bits
        p->slots = filling(per, std::max<int64_t>(steps, 1));
        p->groups = d->B > 0 ? p->slots * per : 0;
        parts = 2 * p->groups;
    }
    p->split = p->slots > 1;
    if (p->groups > kMaxGroups256 || d->B * d->new_tokens * d->heads > kMaxGroups256 * 8) return NOBLE_ERR_BAD_SHAPE;
    p->chunks = (d->table_row * d->page + kPart - 1) / kPart * (kPart / kKeys);   // whole tiles of either kernel
    p->where = p->stats = p->z = 0;
    size_t at = 0;
    if (p->split) {
        at = up256((size_t)parts * p->R * kGroup * ((d->head_dim <= 64 ? 64 : 128) + 4) * 4);
        p->where = at;
        at += up256((size_t)(FORM == kBlocks ? d->B * d->new_tokens * d->kv_heads : d->B) * sizeof(int2));
    }
    if (FORM == kWeigh) {
        const int64_t all = d->B * d->new_tokens * d->heads;
        if (p->chunks > 0 && all > kMaxScratch / 4 / kKeys / p->chunks) return NOBLE_ERR_BAD_SHAPE;
        p->stats = at;
        at += up256((size_t)all * 8);
        p->z = at;
        at += (size_t)all * p->chunks * kKeys * 4;
        if (d->B * d->kv_heads * (p->chunks * kKeys / (1024 / kManySlices) + 1) > kMaxGroups256) return NOBLE_ERR_BAD_SHAPE;
    }
    p->bytes = at;
    return NOBLE_OK;
}

DecodeArgs decode_args(const noble_paged_desc* d, const DecodePlan& p, const noble_heads* q, const void* cache,
                       const int32_t* table, const int32_t* lengths, const float* slopes, const noble_heads* o, void* scratch) {
    DecodeArgs a{};
    a.q = head_rows(q, d->dtype);
    a.o = head_rows(o, d->dtype);
    a.cache = static_cast<const char*>(cache);
    a.table = table;
    a.lengths = lengths;
    a.slopes = slopes;
    char* s = static_cast<char*>(scratch);
    a.part = reinterpret_cast<float*>(s);
    a.where = p.split ? reinterpret_cast<int2*>(s + p.where) : nullptr;
    a.stats = reinterpret_cast<float2*>(s + p.stats);
    a.z = reinterpret_cast<float*>(s + p.z);
    a.chunks = p.chunks;
    a.table_row = d->table_row;
    a.pages = d->pages;
    a.page = d->page;
    a.shift = __builtin_ctz((unsigned)d->page);
    a.page_bytes = (int64_t)2 * d->kv_heads * d->page * d->head_dim * (int64_t)elt(d->dtype);
    a.fresh = d->new_tokens;
    a.kv_heads = d->kv_heads;
    a.share = d->heads / d->kv_heads;
    a.D = d->head_dim;
    a.row_tiles = (int)p.row_tiles;
    a.slots = (int)p.slots;
    a.B = d->B;
    a.sc = score_args(d->scale, d->softcap);
    return a;
}

noble_status check_attention(const noble_paged_desc* d, const DecodePlan& p, const noble_heads* q, const void* cache,
                             const int32_t* table, const int32_t* lengths, const float* slopes, const noble_heads* o,
                             const void* scratch, size_t scratch_bytes) {
    const int64_t rows = d->B * d->new_tokens;
    NOBLE_TRY(check_heads(q, rows, d->heads, d->head_dim, false));
    NOBLE_TRY(check_heads(o, rows, d->heads, d->head_dim, true));
    NOBLE_TRY(need(cache, rows > 0 && d->pages > 0));
    NOBLE_TRY(check_tables(d, table, lengths));
    NOBLE_TRY(need_array(slopes, false, 4));
    if (scratch_bytes < p.bytes) return NOBLE_ERR_WORKSPACE_TOO_SMALL;
    return need(scratch, p.bytes > 0);
}

// The attention of one call, and the join of its pieces.
template <int FORM>
noble_status run_attention(const noble_paged_desc* d, const DecodePlan& p, const DecodeArgs& a, hipStream_t st) {
    return with_shape(d->dtype, d->head_dim, [&]<typename E, int DP>() {
        const auto kernel = [&]<int MODE>() {
            if constexpr (FORM == kBlocks) return attn_decode_kernel<E, DP, FORM, MODE, 1>;
            else {
                if constexpr (sizeof(E) == 2)
                    if (p.wide) return p.wide == 8 ? attn_wide_kernel<DP, FORM, MODE, 8> : attn_wide_kernel<DP, FORM, MODE, 4>;
                return p.R == 1 ? attn_decode_kernel<E, DP, FORM, MODE, 1> : attn_decode_kernel<E, DP, FORM, MODE, 2>;
            }
        };
        NOBLE_TRY(launch(d->softcap > 0.f ? kernel.template operator()<kCap>() : kernel.template operator()<0>(),
                         dim3((unsigned)p.groups), dim3(p.wide ? 64 * p.wide : 64 * DecodeShape<E, DP>::WAVES), st, a,
                         p.wide == 8 ? WideShape<DP, 8>::LDS : p.wide ? WideShape<DP, 4>::LDS : DecodeShape<E, DP>::LDS));
        if (!p.split) return NOBLE_OK;
        const DecodeJoinArgs j{a, d->B * d->new_tokens * d->heads, (int)p.R};
        // rows of more pieces than a set of lanes has in flight: a set for every eighth of them
        const bool many = p.slots > 8 * (FORM == kBlocks ? 1 : d->B);
        constexpr int rows = 256 / (DP / 4);   // of a workgroup, one set of lanes each
        return many ? launch(decode_join_kernel<E, DP, FORM, kJoinSlices>, dim3((unsigned)cdiv(j.items, rows / kJoinSlices)),
                             dim3(256), st, j)
                    : launch(decode_join_kernel<E, DP, FORM, 1>, dim3((unsigned)cdiv(j.items, rows)), dim3(256), st, j);
    });
}

noble_status check_select(const noble_paged_desc* d, const noble_select_desc* s) {
    NOBLE_TRY(check_rows(d, kMostNew));
    if (!s) return NOBLE_ERR_NULL_ARG;
    if (s->reserved != 0 || s->count < 1 || s->count > 65536 || s->sink < 0 || s->local < 1 || s->sink > s->count - s->local)
        return NOBLE_ERR_BAD_SHAPE;
    if (d->B * d->new_tokens * d->kv_heads > kMaxGroups256 / 4) return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}

// Blocks whose scores LDS holds: those of a sequence of up to table_row pages.
constexpr int64_t kFewestBlocks = 256, kFewBlocks = 2048, kManyBlocks = 16384;

// Few rows (times key heads) of many blocks each: workgroups of kScored blocks form their scores in a launch before the
// selection's.  One row of 4 key heads of 128 over 512, 2048 and 16250 blocks 10.7 -> 9.7, 20 -> 12 and 118 -> 30 us; 32 rows
// over 1023 16 and 16, over 4092 49 -> 42.
bool scored_apart(const noble_paged_desc* d) {
    const int64_t rows = d->B * d->new_tokens * d->kv_heads;
    return d->table_row >= 512 && rows <= std::min<int64_t>(d->table_row / 16, 128) &&
           rows * cdiv(d->table_row, kScored) <= kMaxGroups256;
}

noble_status select_scratch(const noble_paged_desc* d, size_t* bytes) {
    const int64_t rows = d->B * d->new_tokens * d->kv_heads;
    *bytes = 0;
    if (d->table_row <= kManyBlocks && !scored_apart(d)) return NOBLE_OK;
    if (rows > kMaxScratch / 8 / d->table_row) return NOBLE_ERR_BAD_SHAPE;
    *bytes = (size_t)rows * d->table_row * 8;
    return NOBLE_OK;
}

}  // namespace

extern "C" {

noble_status noble_tree_rows(int64_t B, int32_t new_tokens, const int32_t* parents, const int32_t* lengths, int32_t* seen,
                             int32_t* depths, int32_t* positions, void* stream) {
    if (B < 0 || new_tokens < 1 || new_tokens > NOBLE_TREE_MOST || B > kMaxGroups256) return NOBLE_ERR_BAD_SHAPE;
    const bool some = B > 0;
    NOBLE_TRY(need_array(parents, some, 4));
    NOBLE_TRY(need_array(lengths, some && positions, 4));
    NOBLE_TRY(need_array(seen, some, 4));
    NOBLE_TRY(need_array(depths, some, 4));
    NOBLE_TRY(need_array(positions, false, 4));
    NOBLE_TRY(check_device());
    if (!some) return NOBLE_OK;
    const TreeArgs a{parents, lengths, reinterpret_cast<uint32_t*>(seen), depths, positions, new_tokens,
                     NOBLE_TREE_WORDS(new_tokens)};
    return new_tokens <= 64 ? launch(tree_rows_wave_kernel, dim3((unsigned)B), dim3(64), (hipStream_t)stream, a)
                            : launch(tree_rows_kernel, dim3((unsigned)B), dim3(kTreeMost), (hipStream_t)stream, a);
}

noble_status noble_attn_tree_scratch_size(const noble_paged_desc* desc, size_t* scratch_bytes) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, NOBLE_TREE_MOST));
    NOBLE_TRY(decode_plan<kTree>(desc, 0, &p));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = p.bytes;
    return NOBLE_OK;
}

noble_status noble_attn_tree(const noble_paged_desc* desc, const noble_heads* q, const void* cache,
                             const int32_t* page_table, const int32_t* lengths, const int32_t* seen, const int32_t* depths,
                             const float* slopes, const noble_heads* o, void* scratch, size_t scratch_bytes, void* stream) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, NOBLE_TREE_MOST));
    NOBLE_TRY(decode_plan<kTree>(desc, 0, &p));
    NOBLE_TRY(check_attention(desc, p, q, cache, page_table, lengths, slopes, o, scratch, scratch_bytes));
    NOBLE_TRY(need_array(seen, desc->B > 0, 4));
    NOBLE_TRY(need_array(depths, desc->B > 0, 4));
    NOBLE_TRY(check_device());
    if (p.groups == 0) return NOBLE_OK;
    DecodeArgs a = decode_args(desc, p, q, cache, page_table, lengths, slopes, o, scratch);
    a.seen = reinterpret_cast<const uint32_t*>(seen);
    a.depths = depths;
    a.words = NOBLE_TREE_WORDS(desc->new_tokens);
    return run_attention<kTree>(desc, p, a, (hipStream_t)stream);
}

noble_status noble_cache_keep(const noble_keep_desc* desc, void* cache, const int32_t* page_table, const int32_t* kept,
                              const int32_t* start, void* stream) {
    if (!desc) return NOBLE_ERR_NULL_ARG;
    const noble_keep_desc& d = *desc;
    if (!dtype_ok(d.dtype)) return NOBLE_ERR_BAD_DTYPE;
    if (d.reserved != 0 || d.B < 0 || d.B > kMaxRows || d.page < 8 || d.page > 4096 || (d.page & (d.page - 1)))
        return NOBLE_ERR_BAD_SHAPE;
    if (d.table_row < 0 || d.table_row > kMaxRows / d.page || d.pages < 0 || d.pages > INT32_MAX) return NOBLE_ERR_BAD_SHAPE;
    if (d.most < 0 || d.most > kMaxRows) return NOBLE_ERR_BAD_SHAPE;
    if (d.kv_heads < 1 || d.kv_heads > kMaxHeads || !head_dim_ok(d.head_dim)) return NOBLE_ERR_BAD_SHAPE;
    if (d.kept_heads != 1 && d.kept_heads != d.kv_heads) return NOBLE_ERR_BAD_SHAPE;
    KeepArgs a{};
    a.bytes = d.head_dim * (int)elt(d.dtype);
    const int64_t groups = d.B * d.kv_heads * 2;
    // shares of a head's 16-byte parts: one, unless that leaves CUs without a workgroup
    a.lanes = a.bytes / 16;
    while (a.lanes > 1 && groups * cdiv(a.bytes / 16, a.lanes) < kMoving) a.lanes = (a.lanes + 1) / 2;
    a.slices = cdiv(a.bytes / 16, a.lanes);
    if (groups > kMaxGroups256 / a.slices) return NOBLE_ERR_BAD_SHAPE;
    const bool some = d.B > 0 && d.most > 0;
    NOBLE_TRY(need(cache, some && d.pages > 0));
    NOBLE_TRY(need_array(page_table, some, 4));
    NOBLE_TRY(need_array(kept, some, 4));
    NOBLE_TRY(need_array(start, false, 4));
    NOBLE_TRY(check_device());
    if (!some || d.pages == 0) return NOBLE_OK;
    a.cache = static_cast<char*>(cache);
    a.table = page_table;
    a.kept = kept;
    a.start = start;
    a.table_row = d.table_row;
    a.pages = d.pages;
    a.most = d.most;
    a.page = d.page;
    a.shift = __builtin_ctz((unsigned)d.page);
    a.kv_heads = d.kv_heads;
    a.kept_heads = d.kept_heads;
    const hipStream_t st = (hipStream_t)stream;
    if (d.kept_heads == 1 && d.most <= kFewMoves) {
        a.slices = (int)std::clamp<int64_t>(kMoving / 2 / d.B, 1, 2 * d.kv_heads);
        return launch(cache_move_few_kernel, dim3((unsigned)(d.B * a.slices)), dim3(256), st, a);
    }
    return launch(d.most <= 2 * (256 / a.lanes) ? cache_keep_kernel<1> : cache_keep_kernel<8>,
                  dim3((unsigned)(groups * a.slices)), dim3(256), st, a);
}

noble_status noble_page_means(const noble_paged_desc* desc, const void* cache, const int32_t* page_table,
                              const int32_t* lengths, void* means, void* stream) {
    NOBLE_TRY(check_cache(desc, kMaxRows));
    PageArgs a{};
    a.touched = (int)std::min<int64_t>(((int64_t)desc->new_tokens + desc->page - 2) / desc->page + 1, desc->table_row);
    if (a.touched > 0 && desc->B > kMaxGroups256 / desc->kv_heads / a.touched) return NOBLE_ERR_BAD_SHAPE;
    const bool some = desc->B > 0 && a.touched > 0 && desc->pages > 0;
    NOBLE_TRY(need(cache, some));
    NOBLE_TRY(need(means, some));
    NOBLE_TRY(check_tables(desc, page_table, lengths));
    NOBLE_TRY(check_device());
    if (!some) return NOBLE_OK;
    a.cache = static_cast<const char*>(cache);
    a.table = page_table;
    a.lengths = lengths;
    a.means = static_cast<char*>(means);
    a.table_row = desc->table_row;
    a.pages = desc->pages;
    a.fresh = desc->new_tokens;
    a.page = desc->page;
    a.kv_heads = desc->kv_heads;
    a.D = desc->head_dim;
    return launch(desc->dtype == NOBLE_BF16 ? page_means_kernel<uint16_t> : page_means_kernel<float>,
                  dim3((unsigned)(desc->B * desc->kv_heads * a.touched)), dim3(256), (hipStream_t)stream, a);
}

noble_status noble_block_select_scratch_size(const noble_paged_desc* desc, const noble_select_desc* select,
                                             size_t* scratch_bytes) {
    NOBLE_TRY(check_select(desc, select));
    size_t n;
    NOBLE_TRY(select_scratch(desc, &n));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = n;
    return NOBLE_OK;
}

noble_status noble_block_select(const noble_paged_desc* desc, const noble_select_desc* select, const noble_heads* q,
                                const void* means, const int32_t* page_table, const int32_t* lengths, int32_t* chosen,
                                void* scratch, size_t scratch_bytes, void* stream) {
    NOBLE_TRY(check_select(desc, select));
    size_t n;
    NOBLE_TRY(select_scratch(desc, &n));
    const int64_t rows = desc->B * desc->new_tokens;
    NOBLE_TRY(check_heads(q, rows, desc->heads, desc->head_dim, false));
    NOBLE_TRY(need(means, rows > 0 && desc->pages > 0));
    NOBLE_TRY(check_tables(desc, page_table, lengths));
    NOBLE_TRY(need_array(chosen, rows > 0, 4));
    if (scratch_bytes < n) return NOBLE_ERR_WORKSPACE_TOO_SMALL;
    NOBLE_TRY(need(scratch, n > 0));
    NOBLE_TRY(check_device());
    if (rows == 0) return NOBLE_OK;
    SelectArgs a{};
    a.q = head_rows(q, desc->dtype);
    a.means = static_cast<const char*>(means);
    a.table = page_table;
    a.lengths = lengths;
    a.chosen = chosen;
    a.keys = static_cast<uint64_t*>(scratch);
    a.table_row = desc->table_row;
    a.pages = desc->pages;
    a.page = desc->page;
    a.shift = __builtin_ctz((unsigned)desc->page);
    a.fresh = desc->new_tokens;
    a.kv_heads = desc->kv_heads;
    a.share = desc->heads / desc->kv_heads;
    a.D = desc->head_dim;
    a.count = select->count;
    a.sink = select->sink;
    a.local = select->local;
    const dim3 grid((unsigned)(rows * desc->kv_heads));
    const hipStream_t st = (hipStream_t)stream;
    if (scored_apart(desc)) a.parts = cdiv(desc->table_row, kScored);
    const auto run = [&]<typename E>() {
        if (a.parts) NOBLE_TRY(launch(block_keys_kernel<E>, dim3(grid.x * (unsigned)a.parts), dim3(256), st, a));
        if (desc->table_row <= kFewestBlocks) return launch(block_select_kernel<E, kFewestBlocks, 256>, grid, dim3(256), st, a);
        return desc->table_row <= kFewBlocks ? launch(block_select_kernel<E, kFewBlocks, 1024>, grid, dim3(1024), st, a)
                                             : launch(block_select_kernel<E, kManyBlocks, 1024>, grid, dim3(1024), st, a);
    };
    return desc->dtype == NOBLE_BF16 ? run.template operator()<uint16_t>() : run.template operator()<float>();
}

noble_status noble_attn_blocks_scratch_size(const noble_paged_desc* desc, int32_t count, size_t* scratch_bytes) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, kMostNew));
    if (count < 1 || count > 65536) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(decode_plan<kBlocks>(desc, count, &p));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = p.bytes;
    return NOBLE_OK;
}

noble_status noble_attn_blocks(const noble_paged_desc* desc, int32_t count, const noble_heads* q, const void* cache,
                               const int32_t* page_table, const int32_t* lengths, const int32_t* chosen, const float* slopes,
                               const noble_heads* o, void* scratch, size_t scratch_bytes, void* stream) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, kMostNew));
    if (count < 1 || count > 65536) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(decode_plan<kBlocks>(desc, count, &p));
    NOBLE_TRY(check_attention(desc, p, q, cache, page_table, lengths, slopes, o, scratch, scratch_bytes));
    NOBLE_TRY(need_array(chosen, desc->B > 0, 4));
    NOBLE_TRY(check_device());
    if (p.groups == 0) return NOBLE_OK;
    DecodeArgs a = decode_args(desc, p, q, cache, page_table, lengths, slopes, o, scratch);
    a.chosen = chosen;
    a.count = count;
    return run_attention<kBlocks>(desc, p, a, (hipStream_t)stream);
}

noble_status noble_attn_weigh_scratch_size(const noble_paged_desc* desc, size_t* scratch_bytes) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, kMostNew));
    NOBLE_TRY(decode_plan<kWeigh>(desc, 0, &p));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = p.bytes;
    return NOBLE_OK;
}

noble_status noble_attn_weigh(const noble_paged_desc* desc, const noble_heads* q, const void* cache,
                              const int32_t* page_table, const int32_t* lengths, const float* slopes, const float* weights,
                              float* weights_out, const noble_heads* o, void* scratch, size_t scratch_bytes, void* stream) {
    DecodePlan p;
    NOBLE_TRY(check_rows(desc, kMostNew));
    NOBLE_TRY(decode_plan<kWeigh>(desc, 0, &p));
    NOBLE_TRY(check_attention(desc, p, q, cache, page_table, lengths, slopes, o, scratch, scratch_bytes));
    NOBLE_TRY(need_array(weights, false, 4));
    NOBLE_TRY(need_array(weights_out, desc->B > 0 && desc->table_row > 0, 4));
    NOBLE_TRY(check_device());
    if (p.groups == 0) return NOBLE_OK;
    const DecodeArgs a = decode_args(desc, p, q, cache, page_table, lengths, slopes, o, scratch);
    const hipStream_t st = (hipStream_t)stream;
    NOBLE_TRY(run_attention<kWeigh>(desc, p, a, st));
    const bool many = desc->new_tokens * a.share > kManyRows;
    const WeighArgs w{a, weights, weights_out, cdiv(desc->table_row * desc->page, many ? 1024 / kManySlices : 1024),
                      aligned16(weights) && aligned16(weights_out)};
    if (w.parts == 0) return NOBLE_OK;
    return launch(many ? weigh_kernel<kManySlices> : weigh_kernel<1>, dim3((unsigned)(desc->B * desc->kv_heads * w.parts)),
                  dim3(256), st, w);
}

noble_status noble_evict_select(const noble_evict_desc* desc, const float* weights, const int32_t* lengths, int32_t* kept,
                                float* kept_weights, void* stream) {
    if (!desc) return NOBLE_ERR_NULL_ARG;
    const noble_evict_desc& d = *desc;
    if (d.reserved[0] != 0 || d.reserved[1] != 0 || d.B < 0 || d.B > kMaxRows || d.row < 0 || d.row > kMaxRows || d.heads < 1 || d.heads > kMaxHeads)
        return NOBLE_ERR_BAD_SHAPE;
    // the kernel counts places in 32 bits, 1024 beyond the last
    if (d.keep < 1 || d.keep > kMaxRows || d.sink < 0 || d.recent < 0 || d.sink > d.keep - d.recent) return NOBLE_ERR_BAD_SHAPE;
    if (d.B * d.heads > kMaxGroups256 / 4) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(need_array(weights, d.B > 0 && d.row > 0, 4));
    NOBLE_TRY(need_array(lengths, d.B > 0, 4));
    NOBLE_TRY(need_array(kept, d.B > 0, 4));
    NOBLE_TRY(need_array(kept_weights, false, 4));
    NOBLE_TRY(check_device());
    if (d.B == 0) return NOBLE_OK;
    const EvictArgs a{weights, lengths, kept, kept_weights, d.row, d.heads, d.keep, d.sink, d.recent};
    const dim3 grid((unsigned)(d.B * d.heads)), block(1024);
    return d.row <= 8192 ? launch(evict_select_kernel<8192>, grid, block, (hipStream_t)stream, a)
                         : launch(evict_select_kernel<32768>, grid, block, (hipStream_t)stream, a);
}

}  // extern "C"
