// Attention of many new rows over the paged cache, bf16: trees (kTree) and prompts or long drafts whose scores are kept
// (kWeigh), see noble_decode_attn.hpp.
//
// As in attn_fwd_kernel, each of a workgroup's waves owns 32 rows (new tokens x query heads of one key head), the columns of
// 32x32x16 MFMAs, and all share tiles of 64 keys in LDS.  Here the keys come by the page table and from memory, not from a
// cache that other workgroups have filled: three tiles are on their way while one is multiplied, in a ring of four that takes
// a CU's LDS, and up to 256 rows share each.  Tiles that every row sees run without masks; the last ones, which hold the new
// tokens, in a loop of their own.  Probabilities are rounded to bf16 for their product with the values, as there.
//
// What bounds it: issue.  8 sequences of 16384 to 32768 tokens, 64 drafted tokens each, 16 heads of 128 over 4: calls of 156
// us, 0.66 PFLOP/s (0.40 GB, 2.6 TB/s; the kernel, traced, 165 us in the first twenty calls and 150 after a hundred); the
// matrix cores are busy for a third of the time, vector and scalar operations for half, and waves of one workgroup, which
// pass the same barriers, do not fill each other's gaps as two workgroups would.  With four waves and two stages, two
// workgroups a CU, which then read the cache twice, 188 us.  Up to 128 rows four waves and two stages are faster: 16 drafted
// tokens 113 us, and 125 with one workgroup a CU and four stages.
#pragma once

#include "noble_attn_tile.hpp"
#include "noble_decode_attn.hpp"

namespace noble {

// Eight waves take a CU's LDS, workgroups of four half of it.
template <int DP, int NW>
struct WideShape {
    static constexpr int STAGE = 2 * Tile<uint16_t, DP>::bytes(kPart), STAGES = NW == 8 ? 4 : 2, LDS = STAGES * STAGE;
};

// NW: waves, of 32 rows each.
template <int DP, int FORM, int MODE, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_wide_kernel(DecodeArgs a) {
    using E = uint16_t;
    using T = Tile<E, DP>;
    using S = WideShape<DP, NW>;
    constexpr int ES = T::ES, TB = S::STAGE / 2, NS = DP / 16, ND = DP / 32, KEYS = kPart, NST = S::STAGES, kWideRows = 32 * NW;
    constexpr int MINE = KEYS / NW, RPI = 1024 / T::RB, PER = MINE / RPI;   // a wave's share of a tile's keys, of a request, requests
    extern __shared__ __attribute__((aligned(1024))) char lds[];   // S::LDS, see attn_decode_kernel
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    int w = blockIdx.x;
    const int kv = w % a.kv_heads;
    w /= a.kv_heads;
    const int rt = w % a.row_tiles, slot = w / a.row_tiles, db = a.D * ES;
    Slots sl(a, slot, KEYS, 2, lane);
    if (sl.left <= 0) return;
    for (;;) {
        const int b = sl.b;
        const int rows = a.fresh * a.share, row0 = rt * kWideRows, wave_row = row0 + 32 * wave, row = wave_row + (lane & 31);
        const bool live = row < rows, any = wave_row < rows;
        const int tok = (live ? row : rows - 1) / a.share, head = live ? kv * a.share + row - tok * a.share : 0;
        Frag<E> q[NS];
        const char* qp = a.q.ptr + (int64_t)head * a.q.head + ((int64_t)b * a.fresh + tok) * a.q.row + 8 * h * ES;
#pragma unroll
        for (int s = 0; s < NS; ++s) q[s] = global_frag<E>(qp + 16 * s * ES, live && 16 * s + 8 * h < a.D);
        const int len = a.held(b), first = len - a.fresh;
        const int end = max(first + (min(rows, row0 + kWideRows) - 1) / a.share + 1, 0);   // keys that a row here may see
        const int t1 = min((end + KEYS - 1) / KEYS, sl.stop()), t0 = min(t1, sl.begin);
        if (a.where && sl.begin == 0 && kv == 0 && rt == 0 && threadIdx.x == 0) a.where[b] = int2{slot, sl.pieces(slot)};
        // tokens of the wave's rows
        const int tok0 = min(wave_row, rows - 1) / a.share, tok1 = (min(rows, wave_row + 32) - 1) / a.share;
        const float slope = a.slopes ? a.slopes[head] * kLog2e / a.sc.unit : 0.f;
        const int* depths = FORM == kTree ? a.depths + (int64_t)b * a.fresh : nullptr;
        const int at = first + (FORM == kTree ? depths[tok] : tok);

        typedef const __attribute__((address_space(4))) int* table_ptr;
        const table_ptr table = (table_ptr)(a.table + b * a.table_row);
        uint32_t vo[PER];   // a lane's place in each request of the wave's share of a tile
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = wave * MINE + i * RPI + lane / T::NC, ch = (lane % T::NC) ^ T::swz(r);
            vo[i] = 16 * ch < db ? (uint32_t)((lane / T::NC) * db + 16 * ch) : kOOB;
        }
        const char* heads = a.cache + (int64_t)kv * a.page * db;
        const int64_t values = (int64_t)a.kv_heads * a.page * db;   // from a key to its value
        // Requests the wave's share of a tile; returns which of the tile's keys have no page in the cache.
        const auto request = [&](int n) {
            const int k0 = (t0 + n) * KEYS;
            char* dst = lds + (n & (NST - 1)) * S::STAGE + wave * MINE * T::RB;
            uint64_t bad = 0;
            int page = -1, own[MINE / 8];
            if (a.page >= KEYS) {   // one page holds the tile
                page = table[k0 >> a.shift];
                if (page >= a.pages) page = -1;
                if (page < 0) bad = ~0ull;
#pragma unroll
                for (int x = 0; x < MINE / 8; ++x) own[x] = page;
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int key = k0 + 8 * x;
                    if (x == 0 || (key & (a.page - 1)) == 0) {
                        page = -1;
                        if (key < end) page = table[key >> a.shift];
                        if (page >= a.pages) page = -1;
                    }
                    if (page < 0) bad |= 0xffull << (8 * x);
                    if (x / (MINE / 8) == wave) own[x % (MINE / 8)] = page;
                }
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int key = k0 + wave * MINE + i * RPI, pg = own[i * RPI >> 3];
                const int bytes = pg >= 0 ? max(min(end - key, RPI), 0) * db : 0;
                const char* src = heads + (int64_t)max(pg, 0) * a.page_bytes + (int64_t)(key & (a.page - 1)) * db;
                dma16(wave_desc(src, bytes), dst + i * 1024, vo[i], 0);
                dma16(wave_desc(src + values, bytes), dst + TB + i * 1024, vo[i], 0);
            }
            return bad;
        };
        const int count = t1 - t0;

        f32x16 acc[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
        float m = -INFINITY, l = 0.f;
        const Reader<E, DP> rd(lds, lane);
        operands_here();
        uint64_t bad = 0, bad1 = 0, bad2 = 0, bad3 = 0;   // of this tile and the next three
        if (count > 0) bad1 = request(0);
        if (NST > 2 && count > 1) bad2 = request(1);
        if (NST > 2 && count > 2) bad3 = request(2);

        // bits 32 u + 8 (i / 4) + i % 4 of the lane's 32 scores: of the tile's keys those that the row of a token sees
        const auto sees = [&](int t, int k0) {
            if constexpr (FORM == kTree) {
                const uint32_t* line = a.line(b, t);
                return (uint64_t)line_bits(line, a.words, k0 - first) | (uint64_t)line_bits(line, a.words, k0 + 32 - first) << 32;
            } else {
                const int n = first + t + 1 - k0;
                return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
            }
        };
        const auto step = [&]<bool EDGE>(int n) {
            const int k0 = (t0 + n) * KEYS;
            // this wave's share of the tile is here, and every wave's; and every wave has read the tile before
            const int newer = count - 1 - n;
            if (NST > 2 && newer >= 2) wait_vmcnt<4 * PER>();
            else if (NST > 2 && newer == 1) wait_vmcnt<2 * PER>();
            else wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            bad = bad1;
            if constexpr (NST > 2) {
                bad1 = bad2;
                bad2 = bad3;
                if (newer >= 3) bad3 = request(n + 3);
            } else {
                if (newer >= 1) bad1 = request(n + 1);
            }
            if (!any) return;
            const Reader<E, DP> at_tile = rd.at((n & (NST - 1)) * S::STAGE);
            float z[32];
            f32x16 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < NS; ++x)
#pragma unroll
                for (int u = 0; u < 2; ++u) mma32x32(s[u], at_tile.along(x, 32 * u * T::RB), q[x]);
            if constexpr (!EDGE) read_ahead<2 * NS, 1, 1, 4>();
            __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                raw(s[u], z + 16 * u);
                scores<E, MODE, 16>(a.sc, z + 16 * u, z + 16 * u, nullptr);
            }
            if (a.slopes) {
                if constexpr (EDGE && FORM == kTree) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        int pos = k0 + 8 * (i >> 2) + 4 * h + (i & 3);
                        const int node = pos - first;
                        if (node >= 0 && node < a.fresh) pos = first + depths[(uint32_t)node];
                        z[i] = fmaf(-slope, fabsf((float)(pos - at)), z[i]);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < 2; ++u) bias16(z + 16 * u, slope, (float)(k0 + 4 * h - at) + 32.f * u);
                }
            }
            if (EDGE || bad) {
                const uint64_t mask = (EDGE ? sees(tok, k0) : ~0ull) & ~bad;
                const uint32_t half[2] = {(uint32_t)(mask >> (4 * h)), (uint32_t)(mask >> (32 + 4 * h))};
#pragma unroll
                for (int i = 0; i < 32; ++i) z[i] = half[i >> 4] >> (8 * (i >> 2 & 3) + (i & 3)) & 1u ? z[i] : -INFINITY;
            }
            if constexpr (FORM == kWeigh) {
                if (live) {
                    const float unit = MODE & kCap ? 1.f : a.sc.unit;
                    float* zp = a.z + ((((int64_t)b * a.kv_heads + kv) * a.chunks + k0 / kKeys) * rows + row) * kKeys + 4 * h;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<f32x4*>(zp + (int64_t)(i >> 2) * rows * kKeys + 8 * (i & 3)) =
                            f32x4{z[4 * i] * unit, z[4 * i + 1] * unit, z[4 * i + 2] * unit, z[4 * i + 3] * unit};
                }
            }
            float top = z[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = fmaxf(top, z[i]);
            top = max_halves(top) * (MODE & kCap ? 1.f : a.sc.unit);
            if (__any(top > m + 8.f)) {   // see attn_fwd_kernel
                const float to = fmaxf(m, top);
                const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[d][i] *= f;
            }
            const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                z[i] = exp_score<MODE>(a.sc, z[i], from);
                l += z[i];
            }
            if constexpr (EDGE) {
                // a value that a row does not see meets a probability of zero, which an infinite or NaN one would outlive: then
                // each token's rows are multiplied by the values that this token sees, with zeros for the others
                bool odd = false;
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int d = 0; d < ND; ++d) odd |= not_finite(at_tile.across(d, TB + 16 * x * T::RB));
                asm volatile("" ::: "memory");   // the operands are read again: they are too many to be kept
                if (__any(odd)) {
                    for (int t = tok0; t <= tok1; ++t) {
                        asm volatile("" ::: "memory");
                        const uint64_t mask = sees(t, k0);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const uint32_t keys = (uint32_t)(mask >> (16 * x + 4 * h)), set = (keys & 15u) | (keys >> 4 & 0xf0u);
                            const Frag<E> p = to_frag<E>(z + 8 * x);
#pragma unroll
                            for (int d = 0; d < ND; ++d) {
                                f32x16 sum = acc[d];
                                mma32x32(sum, only(at_tile.across(d, TB + 16 * x * T::RB), set), p);
#pragma unroll
                                for (int i = 0; i < 16; ++i) acc[d][i] = tok == t ? sum[i] : acc[d][i];
                            }
                        }
                    }
                    return;
                }
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const Frag<E> p = to_frag<E>(z + 8 * x);
#pragma unroll
                for (int d = 0; d < ND; ++d) mma32x32(acc[d], at_tile.across(d, TB + 16 * x * T::RB), p);
            }
            if constexpr (!EDGE) read_ahead<4 * ND, 1, 2, 4>();
            __builtin_amdgcn_s_setprio(0);
        };
        // keys that every row of the workgroup sees
        const int all = max(FORM == kTree ? first : first + row0 / a.share + 1, 0);
        const int seen = min(max(all / KEYS - t0, 0), count);
        int n = 0;
        for (; n < seen; ++n) step.template operator()<false>(n);
        for (; n < count; ++n) step.template operator()<true>(n);
        l = sum_halves(l);

        if (!live) {
        } else if (!sl.whole()) {
            float* out = a.part + ((((int64_t)2 * slot + (sl.begin == 0 ? 1 : 0)) * a.row_tiles + rt) * a.kv_heads + kv) * (kWideRows * (DP + 4)) +
                         (row - row0) * (DP + 4);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(out + 32 * d + 8 * i + 4 * h) =
                        f32x4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
            if (h == 0) {
                out[DP] = m;
                out[DP + 1] = l;
            }
        } else {
            if (FORM == kWeigh && h == 0) a.stats[((int64_t)b * a.kv_heads + kv) * rows + row] = make_float2(m, 1.f / l);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    decode_store<E, FORM>(a, b, kv, tok, row - tok * a.share, 32 * d + 8 * i + 4 * h,
                                          f32x4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]}, l);
        }
        if (!sl.next(a, KEYS)) return;
        __syncthreads();   // the tiles' places are free
    }
}

}  // namespace noble
