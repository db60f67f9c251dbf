// Attention of each sequence's newest tokens over the paged cache where a row does not simply see every token before it:
// a tree of drafted tokens (kTree), pages that were selected for each row and key head (kBlocks), and the plain order with
// the scores kept, from which the weight of every cached token is formed (kWeigh).
//
// As in attn_paged_kernel, a workgroup takes rows (new tokens x query heads that share a key head) of one sequence and key
// head; its waves take turns at chunks of 32 keys, which come to LDS without passing through registers, through a ring of
// each wave's own, and their results meet in LDS.  Here a workgroup has R groups of 16 rows, the columns of R sets of 16x16x32
// MFMAs that share every operand read from LDS, so that a tree of eight tokens with four heads to a key head reads its cache
// once; a workgroup goes through several sequences in turn; and chunks that every row sees, nearly all, run without masks.
//
// Probabilities are rounded to the storage type as the operand of their product with the values, so that bf16 values meet the
// bf16 matrix instructions (large products 1250 TFLOP/s, float32's 155); their sums, and the weights of kWeigh, are of
// unrounded ones.  Each is off by half a step, 2^-8 of itself, at most, and o with it by 2^-8 sum p |v|: over the performance
// cases o lies 0.0020 to 0.0024 (norms) from 64 bits, where its own rounding to bf16 alone makes 0.0017.
//
// What bounds it: reading the cache, once.  16 sequences of 130 to 8192 tokens, 16 key heads of 128 (0.55 GB): one drafted
// token 5.6 TB/s, 32 of them (R = 2) 4.7: the step of two groups is long enough that four waves a CU leave gaps.  One token
// of 64 sequences of 16384 to 32768 tokens over 4 key heads (3.2 GB): 6.3 TB/s, and 5.4 with the scores of kWeigh stored,
// 0.1 GB of writes among the reads that cost 95 us (in whatever layout, non-temporal or not, waited for or not).
// float32, 8 sequences of 4096 to 8192 tokens, 32 drafted ones, 8 key heads of 128: 155 us for one query head to each (0.40 GB,
// 2.6 TB/s), and 270 for two, whose 64 rows read the cache twice.
#pragma once

#include "noble_attn_common.hpp"

namespace noble {

enum { kTree = 0, kBlocks = 1, kWeigh = 2 };

struct DecodeArgs {
    HeadRows q, o;
    const char* cache;
    const int* table;
    const int* lengths;
    const float* slopes;
    float* part;          // [part][row tile][kv_heads][16 R][DP + 4] float32: product, maximum, sum
    int2* where;          // [B]: the slot that begins a sequence, and its pieces (kBlocks: [B fresh, kv_heads])
    int64_t table_row, pages, page_bytes;   // page_bytes: of one page, keys and values of all heads
    int page, shift, fresh, kv_heads, share, D;
    int64_t B;
    int row_tiles, slots;   // slots: workgroups of one key head and row tile, for all sequences (kBlocks: for each list)
    ScoreArgs sc;
    const uint32_t* seen;   // kTree: [B, fresh, words]
    const int* depths;      // [B, fresh]
    int words;
    int count;              // kBlocks: entries of a list
    const int* chosen;      // [B fresh, kv_heads, count]
    float* z;               // kWeigh: scores, times log2 e: [B, kv_heads, chunks of 32 tokens, fresh share, 32]
    float2* stats;          // [B, kv_heads, fresh share]: maximum, 1 / sum
    int64_t chunks;

    __device__ __forceinline__ int held(int b) const {
        return (int)min((int64_t)max(lengths[b], 0), table_row * page);
    }
    __device__ __forceinline__ bool there(int b, int block) const {
        const int n = table[b * table_row + block];
        return n >= 0 && n < pages;
    }
    __device__ __forceinline__ const uint32_t* line(int b, int tok) const {
        return seen + ((int64_t)b * fresh + tok) * words;
    }
    __device__ __forceinline__ const int* list(int b, int tok, int kv) const {
        return chosen + (((int64_t)b * fresh + tok) * kv_heads + kv) * count;
    }
};

// Bits c .. c + 31 of a node's line; places before the tree are all seen.
__device__ __forceinline__ uint32_t line_bits(const uint32_t* line, int words, int c) {
    if (c <= -32) return ~0u;
    if (c < 0) return (line[0] << -c) | ((1u << -c) - 1u);
    const int i = c >> 5, s = c & 31;
    const uint32_t lo = i < words ? line[i] : 0u, hi = i + 1 < words ? line[i + 1] : 0u;
    return s ? (lo >> s) | (hi << (32 - s)) : lo;
}
__device__ __forceinline__ bool line_holds(const uint32_t* line, int c) { return line[c >> 5] >> (c & 31) & 1u; }

constexpr int kKeys = 32;        // keys of a wave's step
constexpr int kGroup = 16;       // rows of a group

// Entries of a row's list up to the first that is not larger than the one before it, negative or past the row's own block.
__device__ __forceinline__ int list_length(const int* list, int count, int last, int lane) {
    int n = 0;
    for (int i0 = 0; i0 < count; i0 += 64) {
        const int i = i0 + lane;
        const bool in = i < count;
        const int e = in ? list[i] : -1, before = in && i > 0 ? list[i - 1] : -1;
        const uint64_t end = ~__ballot(in && e > before && e <= last);
        const int run = end ? __builtin_ctzll(end) : 64;
        n += run;
        if (run < 64) break;
    }
    return n;
}

// What a row's sum of products is multiplied by where its sum of probabilities is zero: it sees no key in the cache (0), or its
// scores are all minus infinity, and 0 / 0 is not a number.
template <int FORM>
__device__ float decode_empty(const DecodeArgs& a, int b, int kv, int tok) {
    const int first = a.held(b) - a.fresh, at = first + tok;
    if constexpr (FORM == kBlocks) {
        const int* list = a.list(b, tok, kv);
        const int last = at >= 0 ? at >> a.shift : -1;
        for (int i = 0, before = -1; i < a.count && list[i] > before && list[i] <= last; ++i) {
            before = list[i];
            if (a.there(b, before)) return NAN;
        }
        return 0.f;
    } else {
        const int end = FORM == kTree ? first : at + 1;
        for (int j = 0; j < end; j += a.page)
            if (a.there(b, j >> a.shift)) return NAN;
        if constexpr (FORM == kTree) {
            const uint32_t* line = a.line(b, tok);
            for (int c = max(-first, 0); c <= tok; ++c)
                if (line_holds(line, c) && a.there(b, (first + c) >> a.shift)) return NAN;
        }
        return 0.f;
    }
}

// Four elements of a row of o from the row's sums.
template <typename E, int FORM>
__device__ __forceinline__ void decode_store(const DecodeArgs& a, int b, int kv, int tok, int in_tok, int d, f32x4 sum,
                                             float total) {
    const float inv = total != 0.f ? 1.f / total : decode_empty<FORM>(a, b, kv, tok);
    if (FORM == kTree && !line_holds(a.line(b, tok), tok)) sum = f32x4{0.f, 0.f, 0.f, 0.f};   // no node, whatever it met
    else sum *= inv;
    if (d < a.D)
        store4<E>(a.o.ptr + (int64_t)(kv * a.share + in_tok) * a.o.head + ((int64_t)b * a.fresh + tok) * a.o.row +
                      d * (int)sizeof(E),
                  sum[0], sum[1], sum[2], sum[3]);
}

// The sum of a wave's values up to this lane's, by row shifts and broadcasts (see wave_fold).
__device__ __forceinline__ uint32_t wave_upto(uint32_t v) {
    int x = (int)v;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
    return (uint32_t)x;
}

// The steps (of `keys` keys) of all sequences in a row are dealt to the slots in equal ranges, so that a batch of sequences of
// different lengths keeps every workgroup busy to the end: a slot has the end of one sequence, whole ones, and the beginning
// of one, at most.  Every wave works its range out for itself from the lengths.  16 sequences of 130 to 8192 tokens, 16 key
// heads of 128, whole calls: 1024 workgroups over pieces of their own sequence each, 106 us for one new token and 113 for 16;
// 256 workgroups over slots 100 and 106.
struct Slots {
    int b = 0, begin = 0, steps = 0;   // the sequence, the slot's first step in it, the sequence's steps
    int left = 0;                      // steps of the slot from there on
    uint32_t from = 0;                 // steps before the sequence
    uint32_t per = 0, more = 0;        // a slot's steps; slots that have one more
    Slots() = default;
    // A sequence without keys has a step too, in which its rows are written.
    static __device__ __forceinline__ int steps_of(const DecodeArgs& a, int64_t b, int keys) {
        return b < a.B ? max((a.held((int)b) + keys - 1) / keys, 1) : 0;
    }
    __device__ __forceinline__ uint32_t first(uint32_t slot) const { return slot * per + min(slot, more); }
    // The slot that has a step.
    __device__ __forceinline__ uint32_t of(uint32_t step) const {
        const uint32_t longer = more * (per + 1);
        return step < longer ? step / (per + 1) : more + (step - longer) / per;
    }
    // least: steps of a slot, but for the last ones of calls that have fewer
    __device__ __forceinline__ Slots(const DecodeArgs& a, int slot, int keys, int least, int lane) {
        const int one = steps_of(a, lane, keys);   // of the first 64 sequences, a lane each
        const uint32_t ones = wave_upto(one);
        uint32_t total = __builtin_amdgcn_readlane(ones, 63);
        for (int64_t n = 64; n < a.B; n += 64)
            total += __builtin_amdgcn_readlane(wave_upto(steps_of(a, n + lane, keys)), 63);
        // short sequences side by side: 23 of up to 34 tokens, 7 drafted ones with 16 heads over 2, 37 us one after the other
        const uint32_t used = min((uint32_t)a.slots, max((total + least - 1) / least, (uint32_t)a.B));
        if ((uint32_t)slot >= used) return;
        per = total / used;
        more = total - per * used;
        const uint32_t at = first(slot);
        left = (int)(first(slot + 1) - at);
        for (int64_t n = 0; n < a.B; n += 64) {
            const uint32_t mine = n ? steps_of(a, n + lane, keys) : one;
            const uint32_t upto = n ? wave_upto(mine) : ones;
            const uint64_t here = __ballot(at - from < upto);
            if (here) {
                const int l = __builtin_ctzll(here);
                b = (int)n + l;
                steps = __builtin_amdgcn_readlane(mine, l);
                from += __builtin_amdgcn_readlane(upto, l) - steps;
                begin = (int)(at - from);
                break;
            }
            from += __builtin_amdgcn_readlane(upto, 63);
        }
        b = __builtin_amdgcn_readfirstlane(b);
        begin = __builtin_amdgcn_readfirstlane(begin);
        steps = __builtin_amdgcn_readfirstlane(steps);
        from = __builtin_amdgcn_readfirstlane(from);
        left = __builtin_amdgcn_readfirstlane(left);
        per = __builtin_amdgcn_readfirstlane(per);
        more = __builtin_amdgcn_readfirstlane(more);
    }
    __device__ __forceinline__ int stop() const { return min(steps, begin + left); }
    __device__ __forceinline__ bool whole() const { return begin == 0 && left >= steps; }
    __device__ __forceinline__ int pieces(int slot) const { return (int)(of(from + steps - 1) - slot) + 1; }
    // The next sequence; false: the slot is done.
    __device__ __forceinline__ bool next(const DecodeArgs& a, int keys) {
        left -= stop() - begin;
        if (left <= 0) return false;
        from += steps;
        ++b;
        begin = 0;
        steps = __builtin_amdgcn_readfirstlane(steps_of(a, b, keys));
        return true;
    }
};

template <typename E, int DP>
struct DecodeShape {
    static constexpr int STAGE = 2 * kKeys * DP * (int)sizeof(E);             // keys and values of a chunk
    static constexpr int LDS = 128 * 1024;
    static constexpr int WAVES = LDS / (2 * STAGE) < 4 ? 2 : 4;
    static constexpr int STAGES = LDS / (WAVES * STAGE);
};

template <typename E, int DP, int FORM, int MODE, int R>
__global__ __launch_bounds__((64 * DecodeShape<E, DP>::WAVES), (sizeof(E) * DP > 256 ? 1 : 2)) void attn_decode_kernel(DecodeArgs a) {
    using T = Tile<E, DP>;
    using S = DecodeShape<E, DP>;
    constexpr int ES = T::ES, NS = DP / 32, ND = DP / 16, W = S::WAVES, NST = S::STAGES;
    constexpr int RPI = 1024 / T::RB, PER = kKeys / RPI;   // rows of a request, requests of a chunk's keys
    // As much as S::LDS, from the launch: were it declared, the compiler would reckon with one wave a SIMD and 512 registers,
    // and keep sums in accumulation registers, from and to which every step would move them.
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;
    // pieces of one (sequence, key head) apart, key heads of a sequence side by side: their pages are the same
    int w = blockIdx.x;
    const int kv = w % a.kv_heads;
    w /= a.kv_heads;
    const int rt = w % a.row_tiles, slot = w / a.row_tiles, db = a.D * ES;
    Slots sl;
    int b, piece = 0;
    if constexpr (FORM == kBlocks) {
        b = slot / a.slots;
        piece = slot % a.slots;
    } else {
        sl = Slots(a, slot, kKeys, W, lane);
        if (sl.left <= 0) return;
        b = sl.b;
    }
    for (;;) {
        // this lane's row of each group.  kBlocks: a tile's rows are one token's; else tokens x heads, one after the other
        const int per_tok = FORM == kBlocks ? (a.share + kGroup - 1) / kGroup : 1;
        const int rows = FORM == kBlocks ? a.share : a.fresh * a.share;
        const int row0 = (FORM == kBlocks ? rt % per_tok : rt * R) * kGroup;
        const int tok0 = FORM == kBlocks ? rt / per_tok : row0 / a.share;
        const int tok1 = FORM == kBlocks ? tok0 : (min(rows, row0 + R * kGroup) - 1) / a.share;
        bool live[R];
        int tok[R], head[R];
        Frag<E> q[R][NS];
#pragma unroll
        for (int g = 0; g < R; ++g) {
            const int r = row0 + g * kGroup + n16;
            live[g] = r < rows;
            tok[g] = FORM == kBlocks ? tok0 : live[g] ? r / a.share : tok1;
            head[g] = live[g] ? kv * a.share + r - (FORM == kBlocks ? 0 : tok[g] * a.share) : 0;
            const char* qp = a.q.ptr + (int64_t)head[g] * a.q.head + ((int64_t)b * a.fresh + tok[g]) * a.q.row;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int d = 32 * s + 8 * g4;
                q[g][s] = global_frag<E>(qp + d * ES, live[g] && d < a.D);
            }
        }
        const int len = a.held(b), first = len - a.fresh;   // first: place of the first new token
        const int* list = FORM == kBlocks ? a.list(b, tok0, kv) : nullptr;
        // the keys are [0, end): tokens of the sequence, or (kBlocks) of the listed pages in a row
        int end, listed = 0;
        if constexpr (FORM == kBlocks) {
            const int at = first + tok0;
            listed = __builtin_amdgcn_readfirstlane(list_length(list, a.count, at >= 0 ? at >> a.shift : -1, lane));
            end = listed > 0 ? (listed - 1) * a.page + min(a.page, at + 1 - list[listed - 1] * a.page) : 0;
            end = __builtin_amdgcn_readfirstlane(end);
        } else {
            end = max(first + tok1 + 1, 0);
        }
        const int chunks = (end + kKeys - 1) / kKeys;
        int c0, c1, part;   // part: where the sums go, unless they are all of the rows'
        bool whole;
        if constexpr (FORM == kBlocks) {
            // lists are of one length but for those of short sequences, which are cut into fewer pieces
            const int pieces = max(1, min(a.slots, chunks / W));
            if (piece >= pieces) return;
            c0 = (int)((int64_t)chunks * piece / pieces) + wave;
            c1 = (int)((int64_t)chunks * (piece + 1) / pieces);
            whole = pieces == 1;
            part = slot;
            if (a.where && piece == 0 && threadIdx.x == 0)
                a.where[((int64_t)b * a.fresh + tok0) * a.kv_heads + kv] = int2{slot, pieces};
        } else {
            c0 = sl.begin + wave;
            c1 = min(chunks, sl.stop());
            whole = sl.whole();
            part = 2 * slot + (sl.begin == 0 ? 1 : 0);
            if (a.where && sl.begin == 0 && kv == 0 && rt == 0 && threadIdx.x == 0) a.where[b] = int2{slot, sl.pieces(slot)};
        }
        float slope[R];
        const int* depths = FORM == kTree ? a.depths + (int64_t)b * a.fresh : nullptr;
        int at[R];   // a row's position, which the bias goes by
#pragma unroll
        for (int g = 0; g < R; ++g) {
            slope[g] = a.slopes ? a.slopes[head[g]] * kLog2e / a.sc.unit : 0.f;
            at[g] = first + (FORM == kTree ? depths[tok[g]] : tok[g]);
        }

        char* ring = lds + wave * NST * S::STAGE;
        typedef const __attribute__((address_space(4))) int* table_ptr;
        const table_ptr table = (table_ptr)(a.table + b * a.table_row);
        const table_ptr blocks = (table_ptr)list;
        // a lane's place in each request of a chunk, from the chunk's first key on
        uint32_t vo[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int row = i * RPI + lane / T::NC, ch = (lane % T::NC) ^ T::swz(row);
            vo[i] = 16 * ch < db ? (uint32_t)(row * db + 16 * ch) : kOOB;
        }
        const char* heads = a.cache + (int64_t)kv * a.page * db;
        const int64_t values = (int64_t)a.kv_heads * a.page * db;   // from a key to its value
        // Requests a chunk's keys and values; returns which keys have no page in the cache (they come as zeros).
        const auto request = [&](int c, char* dst) {
            const int k0 = c * kKeys;
            uint32_t bad = 0;
            bool ok = false;
            i32x4 dk, dv;
#pragma unroll
            for (int x = 0; x < kKeys / 8; ++x) {
                const int key = k0 + 8 * x;
                if (x == 0 || (key & (a.page - 1)) == 0) {   // a page starts here, or the chunk does
                    int page = -1;
                    if (key < end) page = table[FORM == kBlocks ? blocks[key >> a.shift] : key >> a.shift];
                    ok = page >= 0 && page < a.pages;
                    const char* base = heads + (int64_t)(ok ? page : 0) * a.page_bytes + (int64_t)((key & (a.page - 1)) - 8 * x) * db;
                    const int bytes = ok ? min(end - k0, kKeys) * db : 0;
                    dk = wave_desc(base, bytes);
                    dv = wave_desc(base + values, bytes);
                }
                if (!ok) bad |= 0xffu << (8 * x);
#pragma unroll
                for (int i = 8 * x / RPI; i < 8 * (x + 1) / RPI; ++i) {
                    dma16(dk, dst + i * 1024, vo[i], 0);
                    dma16(dv, dst + S::STAGE / 2 + i * 1024, vo[i], 0);
                }
            }
            return bad;
        };
        // That again, for a chunk that is here.
        const auto missing = [&](int c) {
            uint32_t bad = 0;
            bool ok = false;
#pragma unroll
            for (int x = 0; x < kKeys / 8; ++x) {
                const int key = c * kKeys + 8 * x;
                if (x == 0 || (key & (a.page - 1)) == 0) {
                    const int page = key < end ? table[key >> a.shift] : -1;
                    ok = page >= 0 && page < a.pages;
                }
                if (!ok) bad |= 0xffu << (8 * x);
            }
            return bad;
        };
        // Which of this lane's eight keys of the chunk at k0 (places 16 (i / 4) + 4 g4 + i % 4) the row of a token sees.
        const auto sees = [&](int t, int k0) {
            uint32_t mask;
            if constexpr (FORM == kTree) {
                mask = line_bits(a.line(b, t), a.words, k0 - first);
            } else {
                const int n = (FORM == kBlocks ? end : first + t + 1) - k0;   // keys up to the token
                mask = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
            }
            return mask;
        };
        const auto mine = [&](uint32_t mask) { return (mask >> (4 * g4) & 15u) | (mask >> (16 + 4 * g4) & 15u) << 4; };

        f32x4 acc[R][ND];
        float m[R], l[R];
#pragma unroll
        for (int g = 0; g < R; ++g) {
            m[g] = -INFINITY;
            l[g] = 0.f;
#pragma unroll
            for (int d = 0; d < ND; ++d) acc[g][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const auto step = [&]<bool EDGE>(const char* kt, int k0, uint32_t bad) {
            const char* vt = kt + S::STAGE / 2;
            float z[R][8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4 sv[R];
#pragma unroll
                for (int g = 0; g < R; ++g) sv[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < NS; ++x) {
                    const Frag<E> kf = T::along(kt, 16 * u + n16, 4 * x + g4);
#pragma unroll
                    for (int g = 0; g < R; ++g) mma16x16(sv[g], kf, q[g][x]);
                }
#pragma unroll
                for (int g = 0; g < R; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[g][4 * u + i] = sv[g][i];
            }
            // keys that some of the rows do not see
            const bool edge = EDGE || (FORM == kBlocks && k0 + kKeys > end);
            int block[4];   // kBlocks: the chunk's pages, whose places the bias goes by
            if (FORM == kBlocks && a.slopes) {
#pragma unroll
                for (int x = 0; x < 4; ++x) block[x] = blocks[min((k0 + 8 * x) >> a.shift, listed - 1)] << a.shift;
            }
            Frag<E> p[R];
#pragma unroll
            for (int g = 0; g < R; ++g) {
                scores<E, MODE, 8>(a.sc, z[g], z[g], nullptr);
                if (a.slopes) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int o = 16 * (i >> 2) + 4 * g4 + (i & 3);
                        int pos = k0 + o;
                        if constexpr (FORM == kBlocks) {
                            const int x = o >> 3;
                            pos = (x == 0 ? block[0] : x == 1 ? block[1] : x == 2 ? block[2] : block[3]) + (pos & (a.page - 1));
                        } else if (FORM == kTree && EDGE && pos >= first) {
                            const int node = pos - first;
                            pos = node < a.fresh ? first + depths[(uint32_t)node] : pos;
                        }
                        z[g][i] = fmaf(-slope[g], fabsf((float)(pos - at[g])), z[g][i]);
                    }
                }
                if (edge || bad) {
                    const uint32_t mask = mine(sees(tok[g], k0) & ~bad);
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[g][i] = mask >> i & 1u ? z[g][i] : -INFINITY;
                }
                if constexpr (FORM == kWeigh) {
                    if (live[g]) {
                        const int r = row0 + g * kGroup + n16;
                        const float unit = MODE & kCap ? 1.f : a.sc.unit;
                        float* zp = a.z + ((((int64_t)b * a.kv_heads + kv) * a.chunks + k0 / kKeys) * rows + r) * kKeys + 4 * g4;
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            *reinterpret_cast<f32x4*>(zp + 16 * u) = f32x4{z[g][4 * u] * unit, z[g][4 * u + 1] * unit,
                                                                           z[g][4 * u + 2] * unit, z[g][4 * u + 3] * unit};
                    }
                }
                float top = z[g][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, z[g][i]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32)) * (MODE & kCap ? 1.f : a.sc.unit);
                if (__any(top > m[g] + 8.f)) {   // see attn_fwd_kernel
                    const float to = fmaxf(m[g], top);
                    const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[g] - to);
                    m[g] = to;
                    l[g] *= f;
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[g][d] *= f;
                }
                const float base = m[g] == -INFINITY ? 0.f : m[g];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[g][i] = exp_score<MODE>(a.sc, z[g][i], base);
                    l[g] += z[g][i];
                }
                p[g] = to_frag<E>(z[g]);
            }
            // a value that a row does not see meets a probability of zero, which an infinite or NaN one would outlive: then
            // each token's rows are multiplied by the values that this token sees, with zeros for the others
            bool odd = false;
            if (EDGE && a.fresh > 1) {
#pragma unroll
                for (int d = 0; d < ND; ++d) odd |= not_finite(T::across16(vt, d, lane));
            }
            if (EDGE) asm volatile("" ::: "memory");   // the operands are read again: they are too many to be kept
            if (EDGE && __any(odd)) {
                for (int t = tok0; t <= tok1; ++t) {
                    asm volatile("" ::: "memory");
                    const uint32_t mask = mine(sees(t, k0));
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const Frag<E> vf = only(T::across16(vt, d, lane), mask);
#pragma unroll
                        for (int g = 0; g < R; ++g) {
                            f32x4 sum = acc[g][d];
                            mma16x16(sum, vf, p[g]);
                            acc[g][d] = tok[g] == t ? sum : acc[g][d];
                        }
                    }
                }
            } else {
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const Frag<E> vf = T::across16(vt, d, lane);
#pragma unroll
                    for (int g = 0; g < R; ++g) mma16x16(acc[g][d], vf, p[g]);
                }
            }
        };
        operands_here();
        int ahead = c0;   // next chunk to request
        uint32_t bads[NST];
#pragma unroll
        for (int s = 0; s < NST; ++s) {
            bads[s] = 0;
            if (s < NST - 1) {
                if (ahead < c1) bads[s] = request(ahead, ring + s * S::STAGE);
                ahead += W;
            }
        }
        // The next chunk into the stage of the step before, whose reads have been waited for; waits for this step's.
        const auto next = [&](char* free) {
            uint32_t bad = 0;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (ahead < c1) {
                bad = request(ahead, free);
                wait_vmcnt<2 * PER * (NST - 1)>();
            } else {
                wait_vmcnt<0>();
            }
            asm volatile("" ::: "memory");
            ahead += W;
            return bad;
        };
        // Chunks that every row sees whole, and then the others, whose masks and whose care for values that are not seen would
        // cost the first loop registers: it would move its sums from and to the accumulation ones in every step.
        const int plain = FORM == kBlocks ? c1 : min(c1, max(first + (FORM == kWeigh ? tok0 + 1 : 0), 0) / kKeys);
        int ch = c0, stage = 0;
        for (bool more = ch < plain; more;) {
#pragma unroll
            for (int s = 0; s < NST; ++s) {
                bads[(s + NST - 1) % NST] = next(ring + (s + NST - 1) % NST * S::STAGE);
                step.template operator()<false>(ring + s * S::STAGE, ch * kKeys, bads[s]);
                ch += W;
                stage = (s + 1) % NST;
                if (ch >= plain) {
                    more = false;
                    break;
                }
            }
        }
        if constexpr (FORM != kBlocks) {
            for (; ch < c1; ch += W) {
                next(ring + (stage + NST - 1) % NST * S::STAGE);
                step.template operator()<true>(ring + stage * S::STAGE, ch * kKeys, missing(ch));
                stage = (stage + 1) % NST;
            }
        }

        // the waves' results meet, a group at a time: [wave][16 rows][DP + 4] float32
        constexpr int LD = DP + 4;
        static_assert(W * kGroup * LD * 4 <= W * NST * S::STAGE, "fits the ring");
#pragma unroll
        for (int g = 0; g < R; ++g) {
            l[g] += __shfl_xor(l[g], 16);
            l[g] += __shfl_xor(l[g], 32);
            __syncthreads();
            float* dst = reinterpret_cast<float*>(lds) + (wave * kGroup + n16) * LD;
#pragma unroll
            for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(dst + 16 * d + 4 * g4) = acc[g][d];
            if (g4 == 0) {
                dst[DP] = m[g];
                dst[DP + 1] = l[g];
            }
            __syncthreads();
            const int take = min(rows - row0 - g * kGroup, kGroup);
            for (int e = threadIdx.x; e < take * (DP / 4); e += 64 * W) {
                const int row = e / (DP / 4), d = e % (DP / 4) * 4;
                const float* src = reinterpret_cast<const float*>(lds) + row * LD;
                float top = -INFINITY;
#pragma unroll
                for (int x = 0; x < W; ++x) top = fmaxf(top, src[x * kGroup * LD + DP]);
                const float base = top == -INFINITY ? 0.f : top;
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
                float total = 0.f;
#pragma unroll
                for (int x = 0; x < W; ++x) {
                    const float* p = src + x * kGroup * LD;
                    const float f = __builtin_amdgcn_exp2f(p[DP] - base);
                    sum += *reinterpret_cast<const f32x4*>(p + d) * f;
                    total += p[DP + 1] * f;
                }
                if (!whole) {
                    float* out = a.part + ((((int64_t)part * a.row_tiles + rt) * a.kv_heads + kv) * R + g) * kGroup * LD + row * LD;
                    *reinterpret_cast<f32x4*>(out + d) = sum;
                    if (d == 0) {
                        out[DP] = top;
                        out[DP + 1] = total;
                    }
                } else {
                    const int rr = row0 + g * kGroup + row, t = FORM == kBlocks ? tok0 : rr / a.share;
                    if (FORM == kWeigh && d == 0)
                        a.stats[((int64_t)b * a.kv_heads + kv) * rows + rr] = make_float2(top, 1.f / total);
                    decode_store<E, FORM>(a, b, kv, t, rr - (FORM == kBlocks ? 0 : t * a.share), d, sum, total);
                }
            }
        }
        if constexpr (FORM == kBlocks) return;
        if (!sl.next(a, kKeys)) return;
        b = sl.b;
        __syncthreads();   // the ring is free
    }
}

// Joins the pieces of every row, in their order.  A row's DP / 4 lanes each take four elements; the pieces of rows with many are
// dealt to SLICES sets of such lanes, whose sums meet in LDS in the sets' order (one token after 32768, 4 key heads, 64
// pieces, the whole call: 28 us for one set, 22 for eight).  kWeigh: and keeps the rows' maxima and sums for weigh_kernel.
struct DecodeJoinArgs {
    DecodeArgs a;
    int64_t items;   // rows of all heads
    int groups;      // R
};
constexpr int kJoinSlices = 8;
template <typename E, int DP, int FORM, int SLICES>
__global__ __launch_bounds__(256) void decode_join_kernel(DecodeJoinArgs j) {
    const DecodeArgs& a = j.a;
    constexpr int LANES = DP / 4, LD = DP + 4, ITEMS = 256 / LANES / SLICES;
    const int lane = threadIdx.x % LANES, slice = threadIdx.x / LANES % SLICES;
    const int64_t here = (int64_t)blockIdx.x * ITEMS + threadIdx.x / LANES / SLICES, item = min(here, j.items - 1);
    const int d = lane * 4, rows = a.fresh * a.share;
    const int row = (int)(item % rows), kv = (int)(item / rows % a.kv_heads), b = (int)(item / rows / a.kv_heads);
    const int tok = row / a.share, in_tok = row - tok * a.share;
    int rt, slot;   // the row's tile and place in it
    if constexpr (FORM == kBlocks) {
        rt = tok * ((a.share + kGroup - 1) / kGroup) + in_tok / kGroup;
        slot = in_tok % kGroup;
    } else {
        rt = row / (kGroup * j.groups);
        slot = row % (kGroup * j.groups);
    }
    const int2 where = a.where[FORM == kBlocks ? ((int64_t)b * a.fresh + tok) * a.kv_heads + kv : b];
    const int pieces = where.y;
    const bool mine = here < j.items && pieces > 1;
    if (SLICES == 1 && !mine) return;
    const int64_t tile = (int64_t)j.groups * kGroup * LD, step = (int64_t)a.row_tiles * a.kv_heads * tile;   // from piece to piece
    // piece n of a list is part n from its first on; of a sequence, its first piece is its slot's second part, the others the
    // next slots' first ones
    const int64_t place = ((int64_t)rt * a.kv_heads + kv) * tile + (int64_t)slot * LD;
    const float* p = a.part + place + (FORM == kBlocks ? where.x : 2 * where.x + 1) * step;
    const auto at = [&](int n) { return p + (FORM == kBlocks ? n : n ? 2 * n - 1 : 0) * step; };
    // eight pieces at a time, their loads all in flight
    constexpr int N = 8;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f, top = -INFINITY;
    const int n0 = pieces * slice / SLICES, n1 = mine ? pieces * (slice + 1) / SLICES : 0;
    for (int x0 = n0; x0 < n1; x0 += N) {
        f32x4 v[N];
        float m[N], l[N], next = top;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float* q = at(min(x0 + n, n1 - 1));
            v[n] = *reinterpret_cast<const f32x4*>(q + d);
            m[n] = x0 + n < n1 ? q[DP] : -INFINITY;
            l[n] = q[DP + 1];
        }
#pragma unroll
        for (int n = 0; n < N; ++n) next = fmaxf(next, m[n]);
        const float base = next == -INFINITY ? 0.f : next, keep = __builtin_amdgcn_exp2f(top - base);
        sum *= keep;
        total *= keep;
        top = next;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (x0 + n >= n1) break;
            const float f = __builtin_amdgcn_exp2f(m[n] - base);
            sum += v[n] * f;
            total += l[n] * f;
        }
    }
    if constexpr (SLICES > 1) {
        __shared__ f32x4 sums[256];
        __shared__ float2 stats[256];
        sums[threadIdx.x] = sum;
        stats[threadIdx.x] = make_float2(top, total);
        __syncthreads();
        if (slice > 0 || !mine) return;
        for (int x = 1; x < SLICES; ++x) top = fmaxf(top, stats[threadIdx.x + x * LANES].x);
        const float base = top == -INFINITY ? 0.f : top;
        sum = {0.f, 0.f, 0.f, 0.f};
        total = 0.f;
#pragma unroll
        for (int x = 0; x < SLICES; ++x) {
            const float2 one = stats[threadIdx.x + x * LANES];
            const float f = __builtin_amdgcn_exp2f(one.x - base);
            sum += sums[threadIdx.x + x * LANES] * f;
            total += one.y * f;
        }
    }
    if (FORM == kWeigh && d == 0) a.stats[item] = make_float2(top, 1.f / total);
    decode_store<E, FORM>(a, b, kv, tok, in_tok, d, sum, total);
}

// The weight that every token received: of the rows that see it, exp2(score - maximum) / sum, added in the rows' order.  A
// thread takes four tokens that follow each other, and one of SLICES ranges of the rows, whose sums meet in LDS: 496 rows of
// 388 tokens, 108 us with the attention for one range, 24 for sixteen.
struct WeighArgs {
    DecodeArgs a;
    const float* in;   // [B, kv_heads, table_row page], nullptr: nothing
    float* out;
    int parts;         // workgroups of one (sequence, key head)
    bool wide;         // in and out may be read and written 16 bytes at a time
};
template <int SLICES>
__global__ __launch_bounds__(256) void weigh_kernel(WeighArgs w) {
    const DecodeArgs& a = w.a;
    constexpr int LANES = 256 / SLICES;
    const int head = blockIdx.x / w.parts, b = head / a.kv_heads;   // (sequence, key head)
    const int len = a.held(b), first = len - a.fresh, rows = a.fresh * a.share;
    const int lane = threadIdx.x % LANES, slice = threadIdx.x / LANES;
    const int j0 = (int)(blockIdx.x % w.parts) * LANES * 4, j = j0 + lane * 4;
    if (j0 >= len) return;
    const int64_t base = (int64_t)head * a.table_row * a.page + j;
    f32x4 old = {0.f, 0.f, 0.f, 0.f};
    if (slice == 0 && w.in && j < first) {   // rows of weights are multiples of eight tokens
        if (w.wide) old = *reinterpret_cast<const f32x4*>(w.in + base);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) old[i] = w.in[base + i];
    }
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (j < len && a.there(b, j >> a.shift)) {
        const float2* stats = a.stats + (int64_t)head * rows;
        const float* z = a.z + (((int64_t)head * a.chunks + j / kKeys) * rows) * kKeys + j % kKeys;
        const int r1 = (int)((int64_t)rows * (slice + 1) / SLICES);
        constexpr int N = SLICES > 1 ? 8 : 4;   // rows whose scores are requested together
        for (int r0 = (int)((int64_t)rows * slice / SLICES); r0 < r1; r0 += N) {
            f32x4 v[N];
            float2 st[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                v[n] = *reinterpret_cast<const f32x4*>(z + (int64_t)min(r0 + n, rows - 1) * kKeys);
                if (SLICES > 1) st[n] = stats[min(r0 + n, rows - 1)];   // else one row for the whole wave, read where it is used
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int r = r0 + n;
                if (r >= r1) break;
                if (SLICES == 1) st[n] = stats[r];
                const int at = first + r / a.share - j;   // of the four tokens, those up to it are seen
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += i <= at ? __builtin_amdgcn_exp2f(v[n][i] - st[n].x) * st[n].y : 0.f;
            }
        }
    }
    if constexpr (SLICES > 1) {
        __shared__ f32x4 sums[SLICES][LANES];
        sums[slice][lane] = sum;
        __syncthreads();
        if (slice > 0) return;
        for (int x = 1; x < SLICES; ++x) sum += sums[x][lane];
    }
    if (j >= len) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += j + i < first ? old[i] : 0.f;
    if (w.wide && j + 4 <= len) {
        *reinterpret_cast<f32x4*>(w.out + base) = sum;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i < len) w.out[base + i] = sum[i];
    }
}

}  // namespace noble
