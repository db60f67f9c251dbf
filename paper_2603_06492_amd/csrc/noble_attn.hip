// libnoble: C ABI of the operators between the Q/K/V layer and the O layer (include/noble_attn.h).
//
// Host side: argument validation (complete before any HIP call), scratch layout, launch rules and launches on the
// caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "noble_attn.h"
#include "noble_attn_host.hpp"
#include "noble_attn_paged.hpp"
#include "noble_attn_tile.hpp"
#include "noble_host.hpp"
#include "noble_rope.hpp"

using namespace noble;

namespace {

// ------------------------------------------------------------------- rope --

noble_status check_rope(const noble_rope_desc* d, bool values) {
    if (!d) return NOBLE_ERR_NULL_ARG;
    if (!dtype_ok(d->dtype)) return NOBLE_ERR_BAD_DTYPE;
    if (d->reserved != 0 || d->T < 0 || d->T > kMaxRows || d->table_rows < 0 || d->table_rows > kMaxRows)
        return NOBLE_ERR_BAD_SHAPE;
    if (d->heads < 0 || d->heads > kMaxHeads || d->kv_heads < (values ? 1 : 0) || d->kv_heads > kMaxHeads)
        return NOBLE_ERR_BAD_SHAPE;
    if (!head_dim_ok(d->head_dim) || d->rot < 0 || d->rot % 16 || d->rot > d->head_dim) return NOBLE_ERR_BAD_SHAPE;
    const int64_t cols = (int64_t)(d->heads + d->kv_heads * (values ? 2 : 1)) * d->head_dim;
    if (d->x_row % 8 || d->x_row < cols || d->x_row > kMaxStride / 256) return NOBLE_ERR_BAD_SHAPE;
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}

int rope_group(int D) { return D <= 64 ? 8 : 16; }   // lanes of a head

// Lane groups that share a token's heads: a wave's, so that it reads neighbouring heads (32768 tokens of 32 heads of 128:
// forward 139 -> 95 us, backward 200 -> 170), and more as long as a CU has less than eight workgroups.
int rope_split(const noble_rope_desc* d, int heads) {
    const int64_t groups = 256 * 8 * (256 / rope_group(d->head_dim));
    const int64_t want = d->T > 0 ? (groups + d->T - 1) / d->T : 1;
    return (int)std::clamp<int64_t>(want, std::min(64 / rope_group(d->head_dim), std::max(heads, 1)), std::max(heads, 1));
}

noble_status check_rope_args(const noble_rope_desc* d, const void* x, const float* wq, const float* wk,
                             const float* cos, const float* sin, const int32_t* positions) {
    const bool some = d->T > 0;
    NOBLE_TRY(need(x, some));
    if (!wq != !wk) return NOBLE_ERR_NULL_ARG;
    NOBLE_TRY(need_array(wq, false, 4));
    NOBLE_TRY(need_array(wk, false, 4));
    NOBLE_TRY(need(cos, some && d->rot > 0 && d->table_rows > 0));
    NOBLE_TRY(need(sin, some && d->rot > 0 && d->table_rows > 0));
    return need_array(positions, false, 4);
}

RopeArgs rope_args(const noble_rope_desc* d, const void* x, const float* wq, const float* wk, const float* cos,
                   const float* sin, const int32_t* positions) {
    RopeArgs a{};
    a.x = static_cast<const char*>(x);
    a.x_row = d->x_row * (int64_t)elt(d->dtype);
    a.wq = wq;
    a.wk = wk;
    a.cos = cos;
    a.sin = sin;
    a.positions = positions;
    a.table_rows = d->table_rows;
    a.T = (int)d->T;
    a.heads = d->heads;
    a.kv_heads = d->kv_heads;
    a.D = d->head_dim;
    a.rot = d->rot;
    a.eps = d->eps;
    return a;
}

// Calls fn.template operator()<E, lanes of a head, interleaved>().
template <typename Fn>
noble_status with_rope(const noble_rope_desc* d, Fn&& fn) {
    return with_shape(d->dtype, d->head_dim, [&]<typename E, int DP>() {
        return d->interleaved ? fn.template operator()<E, DP / 8, true>() : fn.template operator()<E, DP / 8, false>();
    });
}

// Workgroups of the backward: it keeps its sums of the weights' gradients over the tokens that it steps through.
int rope_bwd_groups(const noble_rope_desc* d) {
    const int64_t items = d->T * rope_split(d, d->heads + d->kv_heads), per = 256 / rope_group(d->head_dim);
    return (int)std::min<int64_t>((items + per - 1) / per, 256 * 4);
}

// -------------------------------------------------------------- attention --

noble_status check_attn(const noble_attn_desc* d) {
    if (!d) return NOBLE_ERR_NULL_ARG;
    if (!dtype_ok(d->dtype)) return NOBLE_ERR_BAD_DTYPE;
    if (d->reserved != 0 || d->Tq < 0 || d->Tq > kMaxAttnRows || d->Tk < 0 || d->Tk > kMaxAttnRows) return NOBLE_ERR_BAD_SHAPE;
    if (d->offset < -kMaxAttnRows || d->offset > kMaxAttnRows) return NOBLE_ERR_BAD_SHAPE;
    if (d->heads < 1 || d->heads > kMaxHeads || d->kv_heads < 1 || d->heads % d->kv_heads) return NOBLE_ERR_BAD_SHAPE;
    if (!head_dim_ok(d->head_dim)) return NOBLE_ERR_BAD_SHAPE;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale) || !(d->softcap >= 0.f) || !std::isfinite(d->softcap))
        return NOBLE_ERR_BAD_SHAPE;
    // every launch within one dispatch
    const int64_t longest = std::max(d->Tq, d->Tk);
    if ((longest + 31) / 32 * d->heads > kMaxGroups256 - 64)
        return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}

noble_status check_mask(const noble_attn_desc* d, const int32_t* lo, const int32_t* hi, const float* slopes) {
    if (!lo != !hi) return NOBLE_ERR_NULL_ARG;
    NOBLE_TRY(need_array(lo, false, 4));
    NOBLE_TRY(need_array(hi, false, 4));
    return need_array(slopes, false, 4);
}

AttnArgs attn_args(const noble_attn_desc* d, const int32_t* lo, const int32_t* hi, const float* slopes) {
    AttnArgs a{};
    a.lo = lo;
    a.hi = hi;
    a.slopes = slopes;
    a.Tq = (int)d->Tq;
    a.Tk = (int)d->Tk;
    a.heads = d->heads;
    a.share = d->heads / d->kv_heads;
    a.D = d->head_dim;
    a.causal = d->causal != 0;
    a.off = (int)d->offset;
    a.scale = d->scale;
    a.sc = score_args(d->scale, d->softcap);
    return a;
}

// Whether a launch over `rows` rows of `heads` heads runs split workgroups (TileShape): float32 always, bf16 as long as
// workgroups of 128 rows are too few for the 256 CUs.  Split and not split (us), bf16, 8 heads over all keys, forward and
// backward: heads of 128, 64 workgroups (1024 rows) 15.9 + 43 and 25.7 + 90, 128 workgroups 47.6 + 130 and 47.1 + 167, 192
// workgroups 91.7 + 259 and 66.5 + 231; heads of 64, 128 workgroups 22.3 + 65 and 35.4 + 107, 192 workgroups 53.6 + 141 and
// 51.2 + 142, 256 workgroups 71.7 + 205 and 66.1 + 197.  Float32, the same way and with the same tiles of 32 rows for
// both: heads of 64, 8 x 2048 rows 94 + 291 and 165 + 505, 8 x 4096 rows 347 + 1101 and 319 + 1002, 16 x 4096 rows 691 +
// 2195 and 534 + 1771; heads of 128, 8 x 4096 rows 617 + 2196 and 658 + 2288, 24 x 5516 rows 3496 + 12661 and 3781 + 16351.
// So float32 heads of up to 64 over 8 x 4096 rows and more would take 8 to 23% less time unsplit: another set of float32
// kernels for those calls alone, which is not built.
template <typename E, int DP>
bool split_rows(int64_t rows, int64_t heads) {
    return sizeof(E) == 4 || cdiv(rows, kOwn) * heads < (DP == 64 ? 192 : 128);
}

// Whether the dk/dv launch runs split workgroups.
bool split_keys(const noble_attn_desc* d) {
    return d->dtype == NOBLE_F32 || (d->head_dim <= 64 ? split_rows<uint16_t, 64>(d->Tk, d->kv_heads)
                                                       : split_rows<uint16_t, 128>(d->Tk, d->kv_heads));
}

// The query heads that share a key head are dealt to parts in the dk/dv launch, each with workgroups and sums of its own,
// which attn_dkv_join_kernel adds: the fewest parts that give as many workgroups as run at once, one a CU (split) or two,
// or fewer than twice as many that are of one size.  dk/dv of one part, and of these with the join (us, bf16): 8 heads of
// 96 over 1, 7 x 4357 rows of documents 1083 and 341 (four parts); 16 heads of 128 over 2, 8 x 2048 causal 674 and 397;
// 4 heads of 64 over 1, 8 x 379 rows 60 and 29; 8 heads of 128 over 2, 2 x 1001 50 and 36; over 1, 200 x 150 causal 137
// and 123.  Where documents are that short and heads small the sums cost more than they give: 8 heads of 64 over 2,
// 200 x 150 62 and 86.  Twice as many parts: 302, 418, 30, 36, 172.
int64_t dkv_parts(const noble_attn_desc* d) {
    const bool split = split_keys(d);
    const int64_t share = d->heads / d->kv_heads, groups = cdiv(d->Tk, split ? 32 : kOwn) * d->kv_heads;
    const int64_t least = std::clamp<int64_t>(groups > 0 ? cdiv(split ? 256 : 512, groups) : 1, 1, share);
    for (int64_t parts = least; parts < 2 * least && parts <= share; ++parts)
        if (share % parts == 0) return parts;
    return least;
}

// The backward's scratch: lse in units of log2 and delta [heads, Tq padded to tiles], the rows' intervals [Tq], their
// spans, and the parts' sums.
struct BwdScratch {
    size_t lse2, delta, lo, keys, span, part, bytes;
    static int64_t pad(int64_t rows) { return (rows + kPart - 1) / kPart * kPart; }
    explicit BwdScratch(const noble_attn_desc* d) {
        const size_t per_head = up256((size_t)d->heads * pad(d->Tq) * 4), per_row = up256((size_t)d->Tq * 4);
        lse2 = 0;
        delta = lse2 + per_head;
        lo = delta + per_head;
        keys = lo + per_row;
        span = keys + per_row;
        part = span + up256((size_t)((d->Tq + kPart - 1) / kPart) * sizeof(int4));
        const int64_t parts = dkv_parts(d);
        bytes = part + (parts > 1 ? (size_t)parts * 2 * d->kv_heads * d->Tk * d->head_dim * 4 : 0);
    }
};

// ------------------------------------------------------------------ paged --

struct PagedPlan {
    int64_t row_tiles, pieces, groups;   // groups: workgroups of the first launch
    size_t scratch;
};

int paged_waves(int dtype, int D) { return dtype == NOBLE_F32 && D > 64 ? 2 : 4; }

// Pieces of a sequence: enough workgroups for eight turns of the CUs, which evens out sequences of different lengths, as far
// as the longest sequence that the page table can hold gives every wave of them a chunk.  A shorter sequence is cut
// into fewer (Chunks).  Two, four, eight and sixteen turns (us): 64 sequences of 16384 to 32768 tokens 576, 538, 506 and
// 516; 16 sequences of 130 to 8192 tokens 120, 111, 115 and 133.
PagedPlan paged_plan(const noble_paged_desc* d) {
    PagedPlan p;
    const int64_t share = d->heads / d->kv_heads;
    p.row_tiles = (d->new_tokens * share + kRows16 - 1) / kRows16;
    const int64_t base = d->B * d->kv_heads * p.row_tiles;
    const int64_t chunks = (d->table_row * d->page + kChunk - 1) / kChunk;
    const int64_t most = std::max<int64_t>(chunks / paged_waves(d->dtype, d->head_dim), 1);
    p.pieces = std::clamp<int64_t>(base > 0 ? (2048 + base - 1) / base : 1, 1, std::min<int64_t>(most, 64));
    p.groups = base * p.pieces;
    p.scratch = p.pieces > 1 ? (size_t)p.groups * kRows16 * ((d->head_dim <= 64 ? 64 : 128) + 4) * 4 : 0;
    return p;
}

noble_status check_paged(const noble_paged_desc* d) {
    if (!d) return NOBLE_ERR_NULL_ARG;
    if (!dtype_ok(d->dtype)) return NOBLE_ERR_BAD_DTYPE;
    if (d->reserved != 0 || d->B < 0 || d->new_tokens < 1 || d->new_tokens > (1 << 20) || d->window < 0 ||
        d->B > kMaxRows / d->new_tokens)
        return NOBLE_ERR_BAD_SHAPE;
    if (d->page < 8 || d->page > 4096 || (d->page & (d->page - 1))) return NOBLE_ERR_BAD_SHAPE;
    if (d->table_row < 0 || d->table_row > kMaxRows / d->page || d->pages < 0 || d->pages > INT32_MAX)
        return NOBLE_ERR_BAD_SHAPE;
    if (d->heads < 1 || d->heads > kMaxHeads || d->kv_heads < 1 || d->heads % d->kv_heads || !head_dim_ok(d->head_dim))
        return NOBLE_ERR_BAD_SHAPE;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale) || !(d->softcap >= 0.f) || !std::isfinite(d->softcap))
        return NOBLE_ERR_BAD_SHAPE;
    const PagedPlan p = paged_plan(d);
    if (p.groups > kMaxGroups256 || d->B * d->new_tokens * d->heads > kMaxGroups256 * 8) return NOBLE_ERR_BAD_SHAPE;
    return NOBLE_OK;
}

}  // namespace

extern "C" {

noble_status noble_qk_rope_fwd(const noble_rope_desc* desc, const void* x, const float* q_weight, const float* k_weight,
                               const float* cos, const float* sin, const int32_t* positions, void* q, void* k,
                               void* stream) {
    NOBLE_TRY(check_rope(desc, false));
    NOBLE_TRY(check_rope_args(desc, x, q_weight, k_weight, cos, sin, positions));
    NOBLE_TRY(need(q, desc->T > 0 && desc->heads > 0));
    NOBLE_TRY(need(k, desc->T > 0 && desc->kv_heads > 0));
    const int total = desc->heads + desc->kv_heads;
    RopeArgs a = rope_args(desc, x, q_weight, k_weight, cos, sin, positions);
    a.q = static_cast<char*>(q);
    a.k = static_cast<char*>(k);
    a.split = rope_split(desc, total);
    const int64_t per = 256 / rope_group(desc->head_dim), groups = (desc->T * a.split + per - 1) / per;
    if (groups > kMaxGroups256) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(check_device());
    if (groups == 0 || total == 0) return NOBLE_OK;
    return with_rope(desc, [&]<typename E, int G, bool INTER>() {
        return launch(qk_rope_kernel<E, G, INTER, false>, dim3((unsigned)groups), dim3(256), (hipStream_t)stream, a);
    });
}

noble_status noble_qk_rope_scratch_size(const noble_rope_desc* desc, size_t* scratch_bytes) {
    NOBLE_TRY(check_rope(desc, false));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = (size_t)rope_bwd_groups(desc) * 2 * 128 * 4;
    return NOBLE_OK;
}

noble_status noble_qk_rope_bwd(const noble_rope_desc* desc, const void* dq, const void* dk, const void* x,
                               const float* q_weight, const float* k_weight, const float* cos, const float* sin,
                               const int32_t* positions, void* dx, float* dq_weight, float* dk_weight, void* scratch,
                               size_t scratch_bytes, void* stream) {
    NOBLE_TRY(check_rope(desc, false));
    NOBLE_TRY(check_rope_args(desc, x, q_weight, k_weight, cos, sin, positions));
    NOBLE_TRY(need(dq, desc->T > 0 && desc->heads > 0));
    NOBLE_TRY(need(dk, desc->T > 0 && desc->kv_heads > 0));
    NOBLE_TRY(need(dx, desc->T > 0));
    NOBLE_TRY(need_array(dq_weight, q_weight != nullptr, 4));
    NOBLE_TRY(need_array(dk_weight, q_weight != nullptr, 4));
    const int total = desc->heads + desc->kv_heads, groups = total > 0 ? rope_bwd_groups(desc) : 0;
    const size_t bytes = q_weight ? (size_t)groups * 2 * 128 * 4 : 0;
    if (scratch_bytes < bytes) return NOBLE_ERR_WORKSPACE_TOO_SMALL;
    NOBLE_TRY(need(scratch, bytes > 0));
    NOBLE_TRY(check_device());
    RopeArgs a = rope_args(desc, x, q_weight, k_weight, cos, sin, positions);
    a.q = static_cast<char*>(const_cast<void*>(dq));
    a.k = static_cast<char*>(const_cast<void*>(dk));
    a.dx = static_cast<char*>(dx);
    a.partial = static_cast<float*>(scratch);
    a.split = rope_split(desc, total);
    if (groups > 0)
        NOBLE_TRY(with_rope(desc, [&]<typename E, int G, bool INTER>() {
            return launch(qk_rope_bwd_kernel<E, G, INTER>, dim3((unsigned)groups), dim3(256), (hipStream_t)stream, a);
        }));
    if (!q_weight) return NOBLE_OK;
    const RopeDwArgs w{a.partial, dq_weight, dk_weight, groups, desc->head_dim};
    return launch(rope_dw_kernel, dim3((unsigned)cdiv(desc->head_dim, 16), 2), dim3(1024), (hipStream_t)stream, w);
}

noble_status noble_kv_append(const noble_rope_desc* desc, const noble_cache_desc* cache_desc, const void* x,
                             const float* q_weight, const float* k_weight, const float* cos, const float* sin,
                             const int32_t* positions, const int64_t* slots, void* q, void* cache, void* stream) {
    NOBLE_TRY(check_rope(desc, true));
    if (!cache_desc) return NOBLE_ERR_NULL_ARG;
    const noble_cache_desc& c = *cache_desc;
    if (c.reserved != 0 || c.pages < 0 || c.pages > INT32_MAX || c.page < 8 || c.page > 4096 || (c.page & (c.page - 1)))
        return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(check_rope_args(desc, x, q_weight, k_weight, cos, sin, positions));
    NOBLE_TRY(need_array(slots, desc->T > 0, 8));
    NOBLE_TRY(need(q, false));
    NOBLE_TRY(need(cache, desc->T > 0 && c.pages > 0));
    RopeArgs a = rope_args(desc, x, q_weight, k_weight, cos, sin, positions);
    a.q = static_cast<char*>(q);
    a.slots = slots;
    a.cache = static_cast<char*>(cache);
    a.page = c.page;
    a.page_shift = __builtin_ctz((unsigned)c.page);
    a.slot_count = c.pages * c.page;
    a.split = rope_split(desc, (q ? desc->heads : 0) + desc->kv_heads);
    const int64_t per = 256 / rope_group(desc->head_dim), groups = (desc->T * a.split + per - 1) / per;
    if (groups > kMaxGroups256) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(check_device());
    if (groups == 0) return NOBLE_OK;
    return with_rope(desc, [&]<typename E, int G, bool INTER>() {
        return launch(qk_rope_kernel<E, G, INTER, true>, dim3((unsigned)groups), dim3(256), (hipStream_t)stream, a);
    });
}

noble_status noble_rope_table(const noble_rope_scaling* scaling, int64_t length, int32_t rot, float* cos, float* sin,
                              void* stream) {
    if (!scaling) return NOBLE_ERR_NULL_ARG;
    const noble_rope_scaling& s = *scaling;
    if (s.reserved != 0 || s.kind < NOBLE_ROPE_PLAIN || s.kind > NOBLE_ROPE_RAMP || length < 0 || length > kMaxRows ||
        rot < 16 || rot > 128 || rot % 16 || !(s.base > 1.0) || !std::isfinite(s.base))
        return NOBLE_ERR_BAD_SHAPE;
    if (s.kind != NOBLE_ROPE_PLAIN && !(s.factor >= 1.0 && std::isfinite(s.factor))) return NOBLE_ERR_BAD_SHAPE;
    if (s.kind == NOBLE_ROPE_RAMP &&
        !(s.trained > 0.0 && std::isfinite(s.trained) && s.slow > 0.0 && s.fast > s.slow && std::isfinite(s.fast) &&
          s.gain > 0.0 && std::isfinite(s.gain)))
        return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(need(cos, length > 0));
    NOBLE_TRY(need(sin, length > 0));
    RopeTableArgs a{};
    a.cos = cos;
    a.sin = sin;
    a.pairs = rot / 2;
    a.n = length * a.pairs;
    a.kind = s.kind;
    a.rot = rot;
    a.base = s.kind == NOBLE_ROPE_BASE ? s.base * std::pow(s.factor, (double)rot / (rot - 2)) : s.base;
    a.factor = s.factor;
    a.gain = 1.0;
    if (s.kind == NOBLE_ROPE_RAMP) {
        // the pair whose frequency turns n times over the trained length
        const auto pair = [&](double n) { return a.pairs * std::log(s.trained / (2.0 * M_PI * n)) / std::log(s.base); };
        a.ramp_lo = pair(s.fast);
        a.ramp_hi = pair(s.slow);
        a.gain = s.gain;
    }
    const int64_t groups = (a.n + 255) / 256;
    if (groups > kMaxGroups256) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(check_device());
    if (groups == 0) return NOBLE_OK;
    return launch(rope_table_kernel, dim3((unsigned)groups), dim3(256), (hipStream_t)stream, a);
}

noble_status noble_mask_rows(int64_t T, int64_t documents, const int32_t* starts, const int32_t* prefix, int32_t causal,
                             int32_t window, int32_t* key_lo, int32_t* key_hi, int32_t* positions, void* stream) {
    if (T < 0 || T > kMaxRows || documents < 0 || documents >= INT32_MAX || window < 0) return NOBLE_ERR_BAD_SHAPE;
    NOBLE_TRY(need_array(starts, T > 0 && documents > 0, 4));
    NOBLE_TRY(need_array(prefix, false, 4));
    NOBLE_TRY(need_array(key_lo, T > 0, 4));
    NOBLE_TRY(need_array(key_hi, T > 0, 4));
    NOBLE_TRY(need_array(positions, false, 4));
    NOBLE_TRY(check_device());
    if (T == 0) return NOBLE_OK;
    const MaskArgs a{starts, prefix, key_lo, key_hi, positions, (int)T, (int)documents, causal != 0, window};
    return launch(mask_rows_kernel, dim3((unsigned)cdiv(T, 256)), dim3(256), (hipStream_t)stream, a);
}

noble_status noble_attn_bwd_scratch_size(const noble_attn_desc* desc, size_t* scratch_bytes) {
    NOBLE_TRY(check_attn(desc));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = BwdScratch(desc).bytes;
    return NOBLE_OK;
}

noble_status noble_attn_fwd(const noble_attn_desc* desc, const noble_heads* q, const noble_heads* k,
                            const noble_heads* v, const int32_t* key_lo, const int32_t* key_hi, const float* slopes,
                            const noble_heads* o, float* lse, void* stream) {
    NOBLE_TRY(check_attn(desc));
    NOBLE_TRY(check_heads(q, desc->Tq, desc->heads, desc->head_dim, false));
    NOBLE_TRY(check_heads(k, desc->Tk, desc->kv_heads, desc->head_dim, false));
    NOBLE_TRY(check_heads(v, desc->Tk, desc->kv_heads, desc->head_dim, false));
    NOBLE_TRY(check_heads(o, desc->Tq, desc->heads, desc->head_dim, true));
    NOBLE_TRY(check_mask(desc, key_lo, key_hi, slopes));
    NOBLE_TRY(need_array(lse, desc->Tq > 0, 4));
    NOBLE_TRY(check_device());
    if (desc->Tq == 0) return NOBLE_OK;
    AttnArgs a = attn_args(desc, key_lo, key_hi, slopes);
    a.q = head_rows(q, desc->dtype);
    a.k = head_rows(k, desc->dtype);
    a.v = head_rows(v, desc->dtype);
    a.o = head_rows(o, desc->dtype);
    a.lse = lse;
    return with_shape(desc->dtype, desc->head_dim, [&]<typename E, int DP>() {
        return with_mode(desc->softcap > 0.f, slopes != nullptr, [&]<int MODE>() {
            const bool split = split_rows<E, DP>(desc->Tq, desc->heads);
            const int64_t tiles = cdiv(desc->Tq, split ? 32 : kOwn);
            return launch(split ? attn_fwd_kernel<E, DP, MODE, true> : attn_fwd_kernel<E, DP, MODE, sizeof(E) == 4>,
                          dim3((unsigned)HeadOrder::grid(desc->kv_heads, tiles * a.share)), dim3(256), (hipStream_t)stream, a);
        });
    });
}

noble_status noble_attn_bwd(const noble_attn_desc* desc, const noble_heads* grad, const noble_heads* q,
                            const noble_heads* k, const noble_heads* v, const noble_heads* o, const float* lse,
                            const int32_t* key_lo, const int32_t* key_hi, const float* slopes, const noble_heads* dq,
                            const noble_heads* dk, const noble_heads* dv, void* scratch, size_t scratch_bytes,
                            void* stream) {
    NOBLE_TRY(check_attn(desc));
    const int D = desc->head_dim;
    NOBLE_TRY(check_heads(grad, desc->Tq, desc->heads, D, false));
    NOBLE_TRY(check_heads(q, desc->Tq, desc->heads, D, false));
    NOBLE_TRY(check_heads(k, desc->Tk, desc->kv_heads, D, false));
    NOBLE_TRY(check_heads(v, desc->Tk, desc->kv_heads, D, false));
    NOBLE_TRY(check_heads(o, desc->Tq, desc->heads, D, false));
    NOBLE_TRY(check_heads(dq, desc->Tq, desc->heads, D, true));
    NOBLE_TRY(check_heads(dk, desc->Tk, desc->kv_heads, D, true));
    NOBLE_TRY(check_heads(dv, desc->Tk, desc->kv_heads, D, true));
    NOBLE_TRY(check_mask(desc, key_lo, key_hi, slopes));
    NOBLE_TRY(need_array(lse, desc->Tq > 0, 4));
    const BwdScratch ws(desc);
    if (scratch_bytes < ws.bytes) return NOBLE_ERR_WORKSPACE_TOO_SMALL;
    NOBLE_TRY(need(scratch, ws.bytes > 0));
    NOBLE_TRY(check_device());
    AttnArgs a = attn_args(desc, key_lo, key_hi, slopes);
    a.q = head_rows(q, desc->dtype);
    a.k = head_rows(k, desc->dtype);
    a.v = head_rows(v, desc->dtype);
    a.o = head_rows(o, desc->dtype);
    a.g = head_rows(grad, desc->dtype);
    a.dq = head_rows(dq, desc->dtype);
    a.dk = head_rows(dk, desc->dtype);
    a.dv = head_rows(dv, desc->dtype);
    a.lse = const_cast<float*>(lse);
    a.Tpad = (int)BwdScratch::pad(desc->Tq);
    char* s = static_cast<char*>(scratch);
    a.lse2 = reinterpret_cast<float*>(s + ws.lse2);
    a.delta = reinterpret_cast<float*>(s + ws.delta);
    a.row_lo = reinterpret_cast<int*>(s + ws.lo);
    a.row_keys = reinterpret_cast<int*>(s + ws.keys);
    a.span = reinterpret_cast<int4*>(s + ws.span);
    a.part = reinterpret_cast<float*>(s + ws.part);
    a.parts = (int)dkv_parts(desc);
    const hipStream_t st = (hipStream_t)stream;
    return with_shape(desc->dtype, D, [&]<typename E, int DP>() {
        return with_mode(desc->softcap > 0.f, slopes != nullptr, [&]<int MODE>() {
            if (desc->Tq > 0) {
                const bool split = split_rows<E, DP>(desc->Tq, desc->heads);
                const int64_t tiles = cdiv(desc->Tq, split ? 32 : kOwn);
                NOBLE_TRY(launch(split ? attn_dq_kernel<E, DP, MODE, true> : attn_dq_kernel<E, DP, MODE, sizeof(E) == 4>,
                                 dim3((unsigned)HeadOrder::grid(desc->kv_heads, tiles * a.share)), dim3(256), st, a));
            }
            if (desc->Tk > 0) {
                const bool split = split_keys(desc);
                const int64_t tiles = cdiv(desc->Tk, split ? 32 : kOwn);
                const auto kernel = [&]<bool PARTS>() {
                    return split ? attn_dkv_kernel<E, DP, MODE, true, PARTS>
                                 : attn_dkv_kernel<E, DP, MODE, sizeof(E) == 4, PARTS>;
                };
                NOBLE_TRY(launch(a.parts > 1 ? kernel.template operator()<true>() : kernel.template operator()<false>(),
                                 dim3((unsigned)HeadOrder::grid(desc->kv_heads, tiles * a.parts)), dim3(256), st, a));
                if (a.parts > 1)
                    NOBLE_TRY(launch(attn_dkv_join_kernel<E>,
                                     dim3((unsigned)cdiv(desc->kv_heads * desc->Tk * (D / 4), 256), 2), dim3(256), st, a));
            }
            return NOBLE_OK;
        });
    });
}

noble_status noble_attn_paged_scratch_size(const noble_paged_desc* desc, size_t* scratch_bytes) {
    NOBLE_TRY(check_paged(desc));
    if (!scratch_bytes) return NOBLE_ERR_NULL_ARG;
    *scratch_bytes = paged_plan(desc).scratch;
    return NOBLE_OK;
}

noble_status noble_attn_paged(const noble_paged_desc* desc, const noble_heads* q, const void* cache,
                              const int32_t* page_table, const int32_t* lengths, const float* slopes,
                              const noble_heads* o, void* scratch, size_t scratch_bytes, void* stream) {
    NOBLE_TRY(check_paged(desc));
    const int64_t rows = desc->B * desc->new_tokens;
    NOBLE_TRY(check_heads(q, rows, desc->heads, desc->head_dim, false));
    NOBLE_TRY(check_heads(o, rows, desc->heads, desc->head_dim, true));
    NOBLE_TRY(need(cache, rows > 0 && desc->pages > 0));
    NOBLE_TRY(need_array(page_table, rows > 0 && desc->table_row > 0, 4));
    NOBLE_TRY(need_array(lengths, rows > 0, 4));
    NOBLE_TRY(need_array(slopes, false, 4));
    const PagedPlan plan = paged_plan(desc);
    if (scratch_bytes < plan.scratch) return NOBLE_ERR_WORKSPACE_TOO_SMALL;
    NOBLE_TRY(need(scratch, plan.scratch > 0));
    NOBLE_TRY(check_device());
    if (plan.groups == 0) return NOBLE_OK;
    PagedArgs a{};
    a.q = head_rows(q, desc->dtype);
    a.o = head_rows(o, desc->dtype);
    a.cache = static_cast<const char*>(cache);
    a.table = page_table;
    a.lengths = lengths;
    a.slopes = slopes;
    a.part = static_cast<float*>(scratch);
    a.table_row = desc->table_row;
    a.pages = desc->pages;
    a.page = desc->page;
    a.shift = __builtin_ctz((unsigned)desc->page);
    a.page_bytes = (int64_t)2 * desc->kv_heads * desc->page * desc->head_dim * (int64_t)elt(desc->dtype);
    a.fresh = desc->new_tokens;
    a.window = desc->window;
    a.heads = desc->heads;
    a.kv_heads = desc->kv_heads;
    a.share = desc->heads / desc->kv_heads;
    a.D = desc->head_dim;
    a.row_tiles = (int)plan.row_tiles;
    a.pieces = (int)plan.pieces;
    a.sc = score_args(desc->scale, desc->softcap);
    const hipStream_t st = (hipStream_t)stream;
    return with_shape(desc->dtype, desc->head_dim, [&]<typename E, int DP>() {
        NOBLE_TRY(with_mode(desc->softcap > 0.f, slopes != nullptr, [&]<int MODE>() {
            return launch(a.fresh > 1 ? attn_paged_kernel<E, DP, MODE, true> : attn_paged_kernel<E, DP, MODE, false>,
                          dim3((unsigned)plan.groups), dim3(64 * PagedShape<E, DP>::WAVES), st, a);
        }));
        if (plan.pieces == 1) return NOBLE_OK;
        const JoinArgs j{a, rows * desc->heads};
        return launch(attn_join_kernel<E, DP>, dim3((unsigned)cdiv(j.items, 256 / (DP / 4))), dim3(256), st, j);
    });
}

}  // extern "C"
