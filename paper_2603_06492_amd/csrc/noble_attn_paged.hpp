// Attention of the newest tokens of each sequence over a paged cache.
//
// A workgroup takes 16 rows (new tokens x query heads that share a key head) of one sequence and key head, and one
// piece of its keys; its waves take turns at chunks of 32 keys, each with a running maximum, sum and product of its
// own, which meet in LDS at the end.  Keys and values go to LDS without passing through registers, through a ring
// that only its wave uses: no barrier in the loop, and every wave has the next chunks in flight while it multiplies.
// The 16 rows are the columns of 16x16x32 MFMAs, so one read of a key serves every query head that shares it.
// Pieces of one sequence are joined by attn_join_kernel, in their order.
//
// What bounds it: reading the cache, once.  64 sequences of 16384 to 32768 tokens, 16 heads of 128 over 4 key heads: 3.2 GB
// in 514 us, 6.3 TB/s; 16 sequences of 130 to 8192 tokens, 16 key heads: 0.55 GB in 109 us, 5.0 TB/s.  One token over 1000
// keys takes 6 us and 3 for the join: the latencies of lengths, page table, cache and partial results in a row.  It is made for
// few new tokens: a prompt reads its keys once for every 16 rows (4096 tokens, 16 heads over 4: 0.65 ms, attn_fwd_kernel 0.10).
#pragma once

#include "noble_attn_common.hpp"

namespace noble {

struct PagedArgs {
    HeadRows q, o;
    const char* cache;
    const int* table;
    const int* lengths;
    const float* slopes;
    float* part;          // [workgroup][16][DP + 4] float32: product, maximum, sum
    int64_t table_row, pages, page_bytes;   // page_bytes: of one page, keys and values of all heads
    int page, shift, fresh, window, heads, kv_heads, share, D;
    int row_tiles, pieces;
    ScoreArgs sc;
    // The first token that the row of token `at` sees.  A row before the first token sees none, and its number, down to
    // -2^20, would take the window's difference past 32 bits.
    __device__ __forceinline__ int oldest(int at) const { return window > 0 ? max(max(at, -1) - window + 1, 0) : 0; }
    // What a row's sum of products is multiplied by.  A sum of probabilities of zero: the row sees no key in the cache, or its
    // scores are all minus infinity, and 0 / 0 is not a number.
    __device__ float inverse(float total, int b, int at) const {
        if (total != 0.f) return 1.f / total;
        for (int j = oldest(at); j <= at; j = (j | (page - 1)) + 1) {
            const int n = table[b * table_row + (j >> shift)];
            if (n >= 0 && n < pages) return NAN;
        }
        return 0.f;
    }
};

constexpr int kChunk = 32;       // keys of a wave's step
constexpr int kRows16 = 16;      // rows of a workgroup

// A sequence's keys as a row tile sees them, in chunks, and the pieces that they are split into: at least one chunk for
// every wave of a piece.
struct Chunks {
    int len, first, count, start, end, pieces, at0, at1;   // chunks [first, first + count) of the keys [start, end)
    __device__ __forceinline__ Chunks(const PagedArgs& a, int b, int row_tile, int waves) {
        const int64_t held = a.table_row * a.page;
        len = (int)min((int64_t)max(a.lengths[b], 0), held);
        const int rows = a.fresh * a.share, r1 = min(rows, (row_tile + 1) * kRows16) - 1;
        at0 = len - a.fresh + row_tile * kRows16 / a.share;
        at1 = len - a.fresh + r1 / a.share;
        end = max(at1 + 1, 0);
        start = a.oldest(at0);
        first = start / kChunk;
        count = end > start ? (end + kChunk - 1) / kChunk - first : 0;
        pieces = max(1, min(a.pieces, count / waves));
    }
    __device__ __forceinline__ int bound(int piece) const { return first + (int)((int64_t)count * piece / pieces); }
};

template <typename E, int DP>
struct PagedShape {
    static constexpr int WAVES = sizeof(E) * DP > 256 ? 2 : 4;
    static constexpr int STAGE = 2 * kChunk * DP * (int)sizeof(E);             // keys and values of a chunk
    static constexpr int STAGES = 128 * 1024 / (WAVES * STAGE);
};

// SEVERAL: more than one new token a sequence, whose rows may see different keys of a tile.  Calls of single tokens do
// without: with the general kernel 16 sequences of 130 to 8192 tokens, cap, take 114 us and not 109, one of 1000 6.7 and
// not 6.4.
template <typename E, int DP, int MODE, bool SEVERAL>
__global__ __launch_bounds__((64 * PagedShape<E, DP>::WAVES)) void attn_paged_kernel(PagedArgs a) {
    using T = Tile<E, DP>;
    using S = PagedShape<E, DP>;
    constexpr int ES = T::ES, NS = DP / 32, ND = DP / 16, W = S::WAVES, NST = S::STAGES;
    constexpr int RPI = 1024 / T::RB, PER = kChunk / RPI;   // rows of a request, requests of a chunk's keys
    __shared__ __attribute__((aligned(1024))) char lds[W * NST * S::STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;
    // pieces of one (sequence, key head) apart, key heads of a sequence side by side: their pages are the same
    int w = blockIdx.x;
    const int kv = w % a.kv_heads;
    w /= a.kv_heads;
    const int rt = w % a.row_tiles;
    w /= a.row_tiles;
    const int piece = w % a.pieces, b = w / a.pieces, db = a.D * ES;
    // this lane's row, whose loads go out before anything that waits for the lengths
    const int r = rt * kRows16 + n16, rows = a.fresh * a.share;
    const bool live = r < rows;
    const int tok = SEVERAL ? r / a.share : 0, head = kv * a.share + r - tok * a.share;
    Frag<E> q[NS];
    const char* qp = a.q.ptr + (int64_t)(live ? head : 0) * a.q.head + ((int64_t)b * a.fresh + (live ? tok : 0)) * a.q.row;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int d = 32 * s + 8 * g4;
        q[s] = global_frag<E>(qp + d * ES, live && d < a.D);
    }
    const float slope = MODE & kBias ? a.slopes[live ? head : 0] * kLog2e / a.sc.unit : 0.f;
    const Chunks ck(a, b, rt, W);
    if (piece >= ck.pieces) return;
    const int at = live ? ck.len - a.fresh + tok : ck.at1;
    const int c0 = ck.bound(piece) + wave, c1 = ck.bound(piece + 1);

    char* ring = lds + wave * NST * S::STAGE;
    typedef const __attribute__((address_space(4))) int* table_ptr;
    const table_ptr table = (table_ptr)(a.table + b * a.table_row);
    uint32_t bad = 0;   // keys of the next chunk without a page in the cache
    uint32_t bads[NST];
    const auto request = [&](int c, int stage) {
        const int k0 = c * kChunk;
        char* dst = ring + stage * S::STAGE;
        const int in_page = k0 & (a.page - 1);
        const char* base = a.cache + (int64_t)kv * a.page * db + (int64_t)in_page * db;
        int page = -1;
        bad = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int key = k0 + i * RPI, left = max(min(ck.end - key, RPI), 0);
            // a new page starts here, or the chunk does; pages hold at least a request's rows
            if (i == 0 || ((in_page + i * RPI) & (a.page - 1)) == 0) {
                page = left > 0 ? table[key >> a.shift] : -1;
                if (i > 0) base = a.cache + (int64_t)kv * a.page * db - (int64_t)i * RPI * db;
            }
            const bool ok = page >= 0 && page < a.pages;
            if (!ok) bad |= ((1u << RPI) - 1u) << (i * RPI);
            const char* src = base + (int64_t)(ok ? page : 0) * a.page_bytes + (int64_t)i * RPI * db;
            const int row = i * RPI + lane / T::NC, ch = (lane % T::NC) ^ T::swz(row);
            // a key before every row's window is not read either: what it holds may be anything
            const uint32_t vo = 16 * ch < db && (k0 >= ck.start || k0 + row >= ck.start) ? (uint32_t)((lane / T::NC) * db + 16 * ch) : kOOB;
            const int64_t bytes = ok ? (int64_t)left * db : 0;
            dma16(wave_desc(src, bytes), dst + i * 1024, vo, 0);
            dma16(wave_desc(src + (int64_t)a.kv_heads * a.page * db, bytes), dst + S::STAGE / 2 + i * 1024, vo, 0);
        }
    };


    f32x4 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    operands_here();
    int ahead = c0;   // next chunk to request
#pragma unroll
    for (int s = 0; s < NST - 1; ++s) {
        if (ahead < c1) request(ahead, s);
        bads[s] = bad;
        ahead += W;
    }
    bads[NST - 1] = 0;
    for (int c = c0; c < c1; c += NST * W) {
#pragma unroll
        for (int s = 0; s < NST; ++s) {
            const int ch = c + s * W;
            if (ch >= c1) break;
            // the stage of the step before is free: its reads have been waited for
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (ahead < c1) {
                request(ahead, (s + NST - 1) % NST);
                bads[(s + NST - 1) % NST] = bad;
                wait_vmcnt<2 * PER * (NST - 1)>();
            } else {
                wait_vmcnt<0>();
            }
            asm volatile("" ::: "memory");
            ahead += W;
            const int k0 = ch * kChunk;
            const char* kt = ring + s * S::STAGE;
            const char* vt = kt + S::STAGE / 2;
            float z[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4 sv = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < NS; ++x) mma16x16(sv, T::along(kt, 16 * u + n16, 4 * x + g4), q[x]);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * u + i] = sv[i];
            }
            scores<E, MODE, 8>(a.sc, z, z, nullptr);
            if constexpr (MODE & kBias) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    z[i] = fmaf(-slope, fabsf((float)(k0 + 4 * g4 - at) + (float)(16 * (i >> 2) + (i & 3))), z[i]);
            }
            // keys that some of the rows do not see
            const bool edge = k0 + kChunk > ck.at0 + 1 || k0 < a.oldest(ck.at1);
            if (edge || bads[s]) {
                const int from = a.oldest(at);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int o = 16 * (i >> 2) + 4 * g4 + (i & 3), j = k0 + o;
                    z[i] = j <= at && j >= from && !((bads[s] >> o) & 1u) ? z[i] : -INFINITY;
                }
            }
            float top = z[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, z[i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32)) * (MODE & kCap ? 1.f : a.sc.unit);
            if (__any(top > m + 8.f)) {   // see attn_fwd_kernel
                const float to = fmaxf(m, top);
                const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[d] *= f;
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[i] = exp_score<MODE>(a.sc, z[i], base);
                l += z[i];
            }
            const Frag<E> p = to_frag<E>(z);
            // a value that a row does not see meets a probability of zero, which an infinite or NaN one would outlive: then
            // each token's rows are multiplied by the values that this token sees, with zeros for the others
            bool odd = false;
            if (SEVERAL && edge && ck.at0 < ck.at1) {
#pragma unroll
                for (int d = 0; d < ND; ++d) odd |= not_finite(T::across16(vt, d, lane));
            }
            if (SEVERAL && __any(odd)) {
                for (int t = ck.at0; t <= ck.at1; ++t) {
                    uint32_t seen = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = k0 + 16 * (i >> 2) + 4 * g4 + (i & 3);
                        seen |= (uint32_t)(j <= t && j >= a.oldest(t)) << i;
                    }
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        f32x4 sum = acc[d];
                        mma16x16(sum, only(T::across16(vt, d, lane), seen), p);
                        acc[d] = at == t ? sum : acc[d];
                    }
                }
            } else {
#pragma unroll
                for (int d = 0; d < ND; ++d) mma16x16(acc[d], T::across16(vt, d, lane), p);
            }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // the waves' results meet: [wave][16 rows][DP + 4] float32
    constexpr int LD = DP + 4;
    static_assert(W * kRows16 * LD * 4 <= W * NST * S::STAGE, "fits the ring");
    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds) + (wave * kRows16 + n16) * LD;
#pragma unroll
    for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(mine + 16 * d + 4 * g4) = acc[d];
    if (g4 == 0) {
        mine[DP] = m;
        mine[DP + 1] = l;
    }
    __syncthreads();
    const int take = min(rows - rt * kRows16, kRows16);
    for (int e = threadIdx.x; e < take * (DP / 4); e += 64 * W) {
        const int row = e / (DP / 4), d = e % (DP / 4) * 4;
        const float* src = reinterpret_cast<const float*>(lds) + row * LD;
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < W; ++x) top = fmaxf(top, src[x * kRows16 * LD + DP]);
        const float base = top == -INFINITY ? 0.f : top;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int x = 0; x < W; ++x) {
            const float* p = src + x * kRows16 * LD;
            const float f = __builtin_amdgcn_exp2f(p[DP] - base);
            sum += *reinterpret_cast<const f32x4*>(p + d) * f;
            total += p[DP + 1] * f;
        }
        if (ck.pieces == 1) {
            const int rr = rt * kRows16 + row;
            const float inv = a.inverse(total, b, ck.len - a.fresh + rr / a.share);
            if (d < a.D)
                store4<E>(a.o.ptr + (int64_t)(kv * a.share + rr % a.share) * a.o.head +
                              ((int64_t)b * a.fresh + rr / a.share) * a.o.row + d * ES,
                          sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
        } else {
            float* out = a.part + ((int64_t)blockIdx.x * kRows16 + row) * LD;
            *reinterpret_cast<f32x4*>(out + d) = sum;
            if (d == 0) {
                out[DP] = top;
                out[DP + 1] = total;
            }
        }
    }
}

// Joins the pieces of every row that was split, in their order.  A row's DP / 4 lanes each take four elements.
struct JoinArgs {
    PagedArgs a;
    int64_t items;   // rows of all heads
};
template <typename E, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(JoinArgs j) {
    const PagedArgs& a = j.a;
    constexpr int ES = sizeof(E), LANES = DP / 4, LD = DP + 4;
    const int64_t item = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (item >= j.items) return;
    const int d = threadIdx.x % LANES * 4, rows = a.fresh * a.share;
    const int row = (int)(item % rows), kv = (int)(item / rows % a.kv_heads), b = (int)(item / rows / a.kv_heads);
    const int rt = row / kRows16;
    const Chunks ck(a, b, rt, PagedShape<E, DP>::WAVES);
    if (ck.pieces == 1) return;
    const int64_t step = (int64_t)a.row_tiles * a.kv_heads * kRows16 * LD;   // from piece to piece
    const float* p = a.part + ((((int64_t)b * a.pieces * a.row_tiles + rt) * a.kv_heads + kv) * kRows16 + row % kRows16) * LD;
    // eight pieces at a time, their loads all in flight
    constexpr int N = 8;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f, top = -INFINITY;
    for (int x0 = 0; x0 < ck.pieces; x0 += N) {
        f32x4 v[N];
        float m[N], l[N], next = top;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float* q = p + min(x0 + n, ck.pieces - 1) * step;
            v[n] = *reinterpret_cast<const f32x4*>(q + d);
            m[n] = x0 + n < ck.pieces ? q[DP] : -INFINITY;
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
            const float f = __builtin_amdgcn_exp2f(m[n] - base);
            sum += v[n] * f;
            total += l[n] * f;
        }
    }
    const float inv = a.inverse(total, b, ck.len - a.fresh + row / a.share);
    if (d < a.D)
        store4<E>(a.o.ptr + (int64_t)(kv * a.share + row % a.share) * a.o.head +
                      ((int64_t)b * a.fresh + row / a.share) * a.o.row + d * ES,
                  sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
}

}  // namespace noble
