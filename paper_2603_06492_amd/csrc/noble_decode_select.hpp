// The operators around attention over a cache that is not read, or not kept, as a whole: rows of a tree, means of pages,
// selection of pages and of tokens, and the move of the tokens that stay.
#pragma once

#include <type_traits>

#include "noble_decode_attn.hpp"

namespace noble {

// ------------------------------------------------------------------- tree --

struct TreeArgs {
    const int* parents;
    const int* lengths;
    uint32_t* seen;
    int* depths;
    int* positions;
    int n, words;
};

// One workgroup a tree, one thread a node.  A node's line is its own bit and its parent's line: after round k a node has the
// bits of the nodes up to 2^k steps above it and the place 2^k steps above it (-1: the root, -2: no node), so a tree of n
// nodes takes log2 n rounds, however deep it is.
constexpr int kTreeMost = 256, kTreeWords = kTreeMost / 32;
__global__ __launch_bounds__(kTreeMost) void tree_rows_kernel(TreeArgs a) {
    __shared__ uint32_t bits[2][kTreeMost][kTreeWords + 1];
    __shared__ int up[2][kTreeMost];
    const int i = threadIdx.x;
    const int64_t b = blockIdx.x;
    if (i < a.n) {
        const int p = a.parents[b * a.n + i];
        up[0][i] = p >= -1 && p < i ? p : -2;
        for (int w = 0; w < a.words; ++w) bits[0][i][w] = w == i >> 5 ? 1u << (i & 31) : 0u;
    }
    int cur = 0;
    for (int step = 1; step < a.n; step *= 2) {
        __syncthreads();
        if (i < a.n) {
            const int u = up[cur][i];
            up[cur ^ 1][i] = u < 0 ? u : up[cur][u];
            for (int w = 0; w < a.words; ++w) bits[cur ^ 1][i][w] = bits[cur][i][w] | (u < 0 ? 0u : bits[cur][u][w]);
        }
        cur ^= 1;
    }
    if (i >= a.n) return;
    // n rounds' steps of at least n - 1 reach the root or none
    const bool node = up[cur][i] == -1;
    int depth = -1;
    for (int w = 0; w < a.words; ++w) {
        const uint32_t v = node ? bits[cur][i][w] : 0u;
        depth += __popc(v);
        a.seen[(b * a.n + i) * a.words + w] = v;
    }
    a.depths[b * a.n + i] = depth;
    if (a.positions) a.positions[b * a.n + i] = node ? max(max(a.lengths[b], 0) - a.n + depth, 0) : 0;
}

// Up to 64 nodes: one wave a tree, the lines in registers.
__global__ __launch_bounds__(64) void tree_rows_wave_kernel(TreeArgs a) {
    const int i = threadIdx.x;
    const int64_t b = blockIdx.x;
    int up = -2;
    if (i < a.n) {
        const int p = a.parents[b * a.n + i];
        up = p >= -1 && p < i ? p : -2;
    }
    const int first = a.positions ? max(a.lengths[b], 0) - a.n : 0;
    uint32_t lo = i < 32 ? 1u << i : 0u, hi = i < 32 ? 0u : 1u << (i - 32);
    for (int step = 1; step < a.n; step *= 2) {
        const int from = max(up, 0);
        const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
        const int next = __shfl(up, from);
        if (up >= 0) {
            lo |= l;
            hi |= h;
            up = next;
        }
    }
    if (i >= a.n) return;
    const bool node = up == -1;
    const int depth = node ? __popc(lo) + __popc(hi) - 1 : -1;
    uint32_t* seen = a.seen + (b * a.n + i) * a.words;
    seen[0] = node ? lo : 0u;
    if (a.words > 1) seen[1] = node ? hi : 0u;
    a.depths[b * a.n + i] = depth;
    if (a.positions) a.positions[b * a.n + i] = node ? max(first + depth, 0) : 0;
}

// ------------------------------------------------------------------ pages --

struct PageArgs {
    const char* cache;
    const int* table;
    const int* lengths;
    char* means;
    int64_t table_row, pages, fresh;
    int page, kv_heads, D, touched;   // touched: workgroups of one (sequence, key head)
    __device__ __forceinline__ int64_t held(int b) const { return min((int64_t)max(lengths[b], 0), table_row * page); }
};

template <typename E>
__device__ __forceinline__ float element(const char* p) {
    if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
    else return *reinterpret_cast<const float*>(p);
}
// Eight consecutive elements.
template <typename E>
__device__ __forceinline__ void elements8(const Frag<E>& f, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(E) == 2) x[i] = __uint_as_float(i & 1 ? f.v[i >> 1] & 0xffff0000u : f.v[i >> 1] << 16);
        else x[i] = __uint_as_float(f.v[i >> 2][i & 3]);
    }
}

// A float64 value rounded once to bf16, to nearest even: the float32 in between takes the side of the value where it
// would be a tie.
__device__ __forceinline__ uint16_t double_to_bf16(double x) {
    const float f = (float)x;
    uint32_t u = __float_as_uint(f);
    if ((u & 0xffffu) == 0x8000u && x == x) u += fabs(x) > fabs((double)f) ? 1 : fabs(x) < fabs((double)f) ? -1 : 0;
    return (uint16_t)(pack_bf16(__uint_as_float(u), 0.f) & 0xffffu);
}

// The mean of one page's keys of one head.  Eight elements a lane, D / 8 lanes a token, the workgroup's other lanes on other
// tokens; float64 sums in one order, by the head's size and the tokens held, and one rounding to the storage type.
template <typename E>
__global__ __launch_bounds__(256) void page_means_kernel(PageArgs a) {
    __shared__ double sums[256][9];
    const int per = a.D / 8, groups = 256 / per;
    int w = blockIdx.x;
    const int kv = w % a.kv_heads;
    w /= a.kv_heads;
    const int t = w % a.touched, b = w / a.touched;
    const int64_t len = a.held(b), from = max(len - a.fresh, (int64_t)0);
    const int64_t block = from / a.page + t;
    if (block * a.page >= len) return;
    const int page = a.table[b * a.table_row + block];
    if (page < 0 || page >= a.pages) return;
    const int n = (int)min(len - block * a.page, (int64_t)a.page), ES = (int)sizeof(E);
    const char* k = a.cache + ((int64_t)page * 2 * a.kv_heads + kv) * a.page * a.D * ES;
    const int g = threadIdx.x / per, x = threadIdx.x % per;
    double s[8] = {};
    if (g < groups)
        for (int r = g; r < n; r += groups) {
            float v[8];
            elements8(global_frag<E>(k + ((int64_t)r * a.D + 8 * x) * ES, true), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += (double)v[i];
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = s[i];
    __syncthreads();
    for (int e = threadIdx.x; e < a.D; e += 256) {
        double total = 0.0;
        for (int r = 0; r < min(groups, n); ++r) total += sums[r * per + e / 8][e % 8];
        total /= n;
        char* out = a.means + (((int64_t)page * a.kv_heads + kv) * a.D + e) * ES;
        if constexpr (sizeof(E) == 2) *reinterpret_cast<uint16_t*>(out) = double_to_bf16(total);
        else *reinterpret_cast<float*>(out) = (float)total;
    }
}

// -------------------------------------------------------------- selection --

// A lane's value from the lane that a DPP control pairs it with.
template <int CTRL>
__device__ __forceinline__ double from_pair(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xf, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, false);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
// Of 2 N sums a lane keeps half, the upper one if `upper`, and gives its pair, which keeps the other, the rest.
template <int CTRL, int N>
__device__ __forceinline__ void halve(double* s, bool upper) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double mine = upper ? s[N + i] : s[i], other = upper ? s[i] : s[N + i];
        s[i] = mine + from_pair<CTRL>(other);
    }
}
// Eight sums over eight lanes, or sixteen, with 7 additions (8) in a lane where each by itself takes 24 (32): returns that of
// place `which`, a lane's own.  All are added in one order, so that equal blocks have equal sums.
__device__ __forceinline__ double lanes_sums(double (&s)[8], int x, bool sixteen, int& which) {
    if (sixteen) {
        halve<0x140, 4>(s, x & 8);   // row_mirror: lanes i and 15 - i
        halve<0x141, 2>(s, x & 4);   // row_half_mirror: i and 7 - i
        halve<0x4e, 1>(s, x & 2);    // quad_perm: i and i ^ 2
        which = x >> 1;
        return s[0] + from_pair<0xb1>(s[0]);   // i and i ^ 1
    }
    halve<0x141, 4>(s, x & 4);
    halve<0x4e, 2>(s, x & 2);
    halve<0xb1, 1>(s, x & 1);
    which = x;
    return s[0];
}

// Whole numbers in the order of the values, NaN above all, -0 with 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    if (x != x) return ~0u;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double x) {
    if (x != x) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(x == 0.0 ? 0.0 : x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// The `need` largest of the keys key(lo) .. key(hi - 1), of equal ones the first, between places that are taken in any case:
// out(i, taken, j) for four places j .. j + 3 of [0, n), a bit for each that is taken, the i-th of all taken.  The least key taken is found from its highest 11
// bits down, by counting the keys that agree with it so far; places are then counted off by waves that each own a range.
// Digits of 11 bits hold all of a float32's exponent and two bits more: with 8, nearly all weights fall into a few counts,
// whose additions wait for each other.
template <typename K, int THREADS>
struct Pick {
    static constexpr int WAVES = THREADS / 64, BITS = 11, BINS = 1 << BITS, COPIES = 2, PER = BINS / THREADS;
    uint32_t hist[COPIES][BINS];
    __attribute__((aligned(16))) uint32_t sums[WAVES];
    __attribute__((aligned(16))) uint32_t above[WAVES], equal[WAVES];
    K prefix, mask;
    uint32_t left, done;

    template <typename Key, typename Out>
    __device__ int run(int n, int lo, int hi, int need, Key key, Out out) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        K pre = 0, msk = 0;
        uint32_t want = (uint32_t)need;
        for (int i = tid; i < COPIES * BINS; i += THREADS) hist[0][i] = 0;
        for (int shift = 8 * (int)sizeof(K) - BITS; want > 0; shift = max(shift - BITS, 0)) {
            __syncthreads();
            for (int j = (lo & ~3) + 4 * tid; j < hi; j += 4 * THREADS) {
                K k[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) k[i] = key(j + i);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (j + i >= lo && j + i < hi && (k[i] & msk) == pre)
                        atomicAdd(&hist[wave % COPIES][(uint32_t)(k[i] >> shift) & (BINS - 1)], 1u);
            }
            __syncthreads();
            // a thread has PER counts, the first thread the largest keys'; they are zero again for the next digit
            uint32_t c[PER], sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = 0;
#pragma unroll
                for (int x = 0; x < COPIES; ++x) {
                    c[i] += hist[x][BINS - 1 - PER * tid - i];
                    hist[x][BINS - 1 - PER * tid - i] = 0;
                }
                sum += c[i];
            }
            uint32_t upto = wave_upto(sum);   // of this thread's counts and those before them
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
#pragma unroll
            for (int x = 0; x < WAVES; ++x) upto += x < wave ? sums[x] : 0u;
            uint32_t before = upto - sum;
            if (before < want && upto >= want) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (before + c[i] >= want) {
                        prefix = pre | (K)(BINS - 1 - PER * tid - i) << shift;
                        mask = msk | (K)(BINS - 1) << shift;
                        left = want - before;
                        done = shift == 0 || c[i] == want - before;   // or the whole bin is taken
                        break;
                    }
                    before += c[i];
                }
            }
            __syncthreads();
            pre = prefix;
            msk = mask;
            want = left;
            if (done) break;
        }
        // places in order: those above the least key or taken in any case, and the first `want` of the least.  Waves own
        // ranges, a lane four places that follow each other.
        const int span = ((n + 4 * THREADS - 1) / (4 * THREADS)) * 256, j0 = min(wave * span, n), j1 = min(j0 + span, n);
        const auto state = [&](int j, uint32_t& is_above, uint32_t& is_equal) {   // of the lane's four places, a bit each
            is_above = is_equal = 0;
            K k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = need > 0 && j < j1 ? key(j + i) & msk : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = j + i < j1, any = in && (j + i < lo || j + i >= hi);
                is_above |= (any || (in && need > 0 && k[i] > pre) ? 1u : 0u) << i;
                is_equal |= (!any && in && need > 0 && k[i] == pre ? 1u : 0u) << i;
            }
        };
        // of the counts up to four of the lanes: those of the lanes below, and all
        const uint64_t below = (1ull << lane) - 1;
        const auto add = [&](uint32_t c, uint32_t& upto, uint32_t& sum) {
            const uint64_t b0 = __ballot(c & 1), b1 = __ballot(c & 2), b2 = __ballot(c & 4);
            upto = __popcll(b0 & below) + 2 * __popcll(b1 & below) + 4 * __popcll(b2 & below);
            sum = __popcll(b0) + 2 * __popcll(b1) + 4 * __popcll(b2);
        };
        uint32_t na = 0, ne = 0, unused, c;
        uint64_t states = 0;   // of the first eight steps, all there are where LDS holds the keys of a wave's range
        int step = 0;
        for (int j = j0; j < j1; j += 256, ++step) {
            uint32_t u, e;
            state(j + 4 * lane, u, e);
            states |= step < 8 ? (uint64_t)(u | e << 4) << (8 * step) : 0ull;
            add(__popc(u), unused, c);
            na += c;
            add(__popc(e), unused, c);
            ne += c;
        }
        if (lane == 0) {
            above[wave] = na;
            equal[wave] = ne;
        }
        __syncthreads();
        uint32_t at = 0, same = 0, all = 0, every = 0;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            at += x < wave ? above[x] : 0u;
            same += x < wave ? equal[x] : 0u;
            all += above[x];
            every += equal[x];
        }
        step = 0;
        for (int j = j0; j < j1; j += 256, ++step) {
            uint32_t u, e, ua, ea, us, es;
            if (step < 8) {
                u = (uint32_t)(states >> (8 * step)) & 15u;
                e = (uint32_t)(states >> (8 * step + 4)) & 15u;
            } else {
                state(j + 4 * lane, u, e);
            }
            add(__popc(u), ua, us);
            add(__popc(e), ea, es);
            ua += at;
            ea += same;
            int places[4];
            uint32_t taken = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool iu = u >> i & 1u, ie = e >> i & 1u;
                places[i] = (int)(ua + min(ea, want));
                taken |= (iu || (ie && ea < want) ? 1u : 0u) << i;
                ua += iu;
                ea += ie;
            }
            out(places, taken, j + 4 * lane);
            at += us;
            same += es;
        }
        return (int)(all + min(every, want));
    }
};

struct EvictArgs {
    const float* weights;
    const int* lengths;
    int* kept;
    float* kept_weights;
    int64_t row;
    int heads, keep, sink, recent;
};

// One workgroup a sequence and key head.  LDS holds the weights of up to N tokens; longer rows are read again each time.  Bound
// by its passes over LDS and by additions to the same count: 256 rows of 4096 weights 10 us, of 32768 39 us, the same ones time
// after time, and 44 for 16384 to 32768 beside the moves of their cache, which leave the weights in memory; of equal weights,
// whose counts all fall into one, 19 and 109.
template <int N>
__global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t keys[N];
    __shared__ Pick<uint32_t, 1024> pick;
    const int b = blockIdx.x / a.heads;
    const int n = (int)min((int64_t)max(a.lengths[b], 0), a.row);
    const float* w = a.weights + (int64_t)blockIdx.x * a.row;
    int* kept = a.kept + (int64_t)blockIdx.x * a.keep;
    float* kw = a.kept_weights ? a.kept_weights + (int64_t)blockIdx.x * a.keep : nullptr;
    const auto out = [&](const int (&i)[4], uint32_t taken, int j) {
        float v[4];   // the weights themselves: keys do not tell -0 from 0, nor one NaN from another
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = kw && taken >> x & 1u ? w[j + x] : 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (taken >> x & 1u) {
                kept[i[x]] = j + x;
                if (kw) kw[i[x]] = v[x];
            }
    };
    int total = n;
    if (n <= a.keep) {
        for (int j = threadIdx.x; j < n; j += 1024) {
            kept[j] = j;
            if (kw) kw[j] = w[j];
        }
    } else {
        const int lo = a.sink, hi = n - a.recent, need = a.keep - a.sink - a.recent;
        if (n <= N) {
            constexpr int U = 8;   // loads in flight: one at a time, 32768 weights take 8 us more
            for (int j0 = threadIdx.x; j0 < n; j0 += U * 1024) {
                float v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = w[min(j0 + u * 1024, n - 1)];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j0 + u * 1024 < n) keys[j0 + u * 1024] = ordered(v[u]);
            }
            __syncthreads();
            total = pick.run(n, lo, hi, need, [&](int j) { return keys[j]; }, out);
        } else {
            total = pick.run(n, lo, hi, need, [&](int j) { return ordered(w[min(j, n - 1)]); }, out);
        }
    }
    for (int i = total + threadIdx.x; i < a.keep; i += 1024) {
        kept[i] = -1;
        if (kw) kw[i] = 0.f;
    }
}

struct SelectArgs {
    HeadRows q;
    const char* means;
    const int* table;
    const int* lengths;
    int* chosen;
    uint64_t* keys;     // [B fresh, kv_heads, table_row] where LDS does not hold them, or other workgroups form them
    int64_t table_row, pages;
    int page, shift, fresh, kv_heads, share, D, count, sink, local;
    int parts;          // workgroups that form a row's keys, 0: the one that selects

    // Blocks up to the row's own.
    __device__ __forceinline__ int blocks(int row) const {
        const int64_t held = min((int64_t)max(lengths[row / fresh], 0), table_row * page), at = held - fresh + row % fresh;
        return at >= 0 ? (int)(at >> shift) + 1 : 0;
    }
};

// keys[lo .. hi - 1] of a row and key head, eight elements of a mean a lane.
template <typename E, int THREADS>
__device__ __forceinline__ void block_keys(const SelectArgs& a, int row, int kv, int lo, int hi, uint64_t* keys) {
    const int ES = (int)sizeof(E), lanes = a.D <= 64 ? 8 : 16;
    const int x = threadIdx.x % lanes, g = threadIdx.x / lanes;
    const bool in = 8 * x < a.D;
    double q[8] = {};
    const char* qp = a.q.ptr + (int64_t)row * a.q.row + (int64_t)kv * a.share * a.q.head + 8 * x * ES;
    for (int h0 = 0; h0 < a.share; h0 += 4) {
        Frag<E> f[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) f[h] = global_frag<E>(qp + (h0 + h) * a.q.head, in && h0 + h < a.share);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            float v[8];
            elements8(f[h], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] += (double)v[i];
        }
    }
    // eight blocks at a time: their pages, then their means, all in flight
    constexpr int U = 8;
    const int step = THREADS / lanes;
    const uint32_t stride = (uint32_t)(a.kv_heads * a.D * ES);   // from a page's mean to the next one's
    const char* means = a.means + (kv * a.D + 8 * x) * ES;
    for (int j0 = lo + g; j0 < hi; j0 += U * step) {
        int page[U];
        uint32_t there = 0;   // a bit each
        Frag<E> mean[U];
#pragma unroll
        for (int n = 0; n < U; ++n) page[n] = j0 + n * step < hi ? a.table[(int64_t)(row / a.fresh) * a.table_row + j0 + n * step] : -1;
#pragma unroll
        for (int n = 0; n < U; ++n) {
            const bool ok = page[n] >= 0 && page[n] < a.pages;
            there |= (uint32_t)ok << n;
            mean[n] = global_frag<E>(means + (uint64_t)(ok ? (uint32_t)page[n] : 0u) * stride, in && a.pages > 0);
        }
        double s[U];
#pragma unroll
        for (int n = 0; n < U; ++n) {
            float v[8];
            elements8(mean[n], v);
            s[n] = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[n] = fma(q[i], (double)v[i], s[n]);
        }
        int n;
        const double sum = lanes_sums(s, x, lanes == 16, n);
        const int j = j0 + n * step;
        if (j < hi) keys[j] = ordered(there >> n & 1u ? sum : -(double)INFINITY);
    }
}

constexpr int kScored = 128;   // blocks of a workgroup
// The keys of a row's blocks by several workgroups, for block_select_kernel to select from (see scored_apart).
template <typename E>
__global__ __launch_bounds__(256) void block_keys_kernel(SelectArgs a) {
    const int list = blockIdx.x / a.parts, row = list / a.kv_heads, n = a.blocks(row);
    const int hi = n - a.local, j0 = a.sink + (int)(blockIdx.x % a.parts) * kScored;
    if (n <= a.count || j0 >= hi) return;
    block_keys<E, 256>(a, row, list % a.kv_heads, j0, min(j0 + kScored, hi), a.keys + (int64_t)list * a.table_row);
}

// One workgroup a row and key head: the scores of the row's blocks, eight elements a lane, then the selection.  LDS holds the
// scores of up to N blocks; those of longer sequences lie in global memory.  Bound by latencies in a row (length, page, mean,
// then some seven barriers) and by float64's arithmetic: 512 blocks of heads of 128, 10 us for one row of 4 key heads, 14 for
// 64 (with the means read one at a time 18 and 28, each block's sum over the lanes by itself 11 and 15; with the next means
// under way during the sums 12.7 and 16).
template <typename E, int N, int THREADS>
__global__ __launch_bounds__(THREADS) void block_select_kernel(SelectArgs a) {
    __shared__ __attribute__((aligned(16))) uint64_t local_keys[N];
    __shared__ Pick<uint64_t, THREADS> pick;
    const int kv = blockIdx.x % a.kv_heads, row = blockIdx.x / a.kv_heads, n = a.blocks(row);
    int* chosen = a.chosen + (int64_t)blockIdx.x * a.count;
    const auto out = [&](const int (&i)[4], uint32_t taken, int j) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (taken >> x & 1u) chosen[i[x]] = j + x;
    };
    int total = n;
    if (n <= a.count) {
        for (int j = threadIdx.x; j < n; j += THREADS) chosen[j] = j;
    } else {
        const int lo = a.sink, hi = n - a.local, need = a.count - a.sink - a.local;
        uint64_t* keys = n <= N ? local_keys : a.keys + (int64_t)blockIdx.x * a.table_row;
        if (need > 0) {
            if (!a.parts) block_keys<E, THREADS>(a, row, kv, lo, hi, keys);
            else if (n <= N)
                for (int j = lo + threadIdx.x; j < hi; j += THREADS) local_keys[j] = a.keys[(int64_t)blockIdx.x * a.table_row + j];
            __syncthreads();
        }
        // two copies, so that the one over LDS is compiled for it
        if (n <= N) total = pick.run(n, lo, hi, need, [&](int j) { return local_keys[j]; }, out);
        else total = pick.run(n, lo, hi, need, [&](int j) { return keys[min(j, hi - 1)]; }, out);
    }
    for (int i = total + threadIdx.x; i < a.count; i += THREADS) chosen[i] = -1;
}

// ------------------------------------------------------------------- move --

struct KeepArgs {
    char* cache;
    const int* table;
    const int* kept;
    const int* start;
    int64_t table_row, pages, most;
    int page, shift, kv_heads, kept_heads;
    int bytes, slices, lanes;   // of a token's head; shares of it that workgroups take; lanes of a share
};

// One workgroup moves a share of one sequence's and key head's keys (or values), tokens in ascending order, a tile of them
// through registers at a time, U a lane.  A token never moves up, so what a tile writes no later tile reads: the next tile is
// requested, and the one after it looked up, while this one is on its way.  What a tile writes and an earlier lane of the same
// tile reads, the barrier keeps.  Bound by memory: 64 x 4 heads of 128, 8192 of 16384 to 32768 tokens each, 2.1 GB read and
// written in 440 us, 4.9 TB/s (3.2 without the next tile under way).
template <int U>
__global__ __launch_bounds__(256) void cache_keep_kernel(KeepArgs a) {
    int w = blockIdx.x;
    const int slice = w % a.slices;
    w /= a.slices;
    const int half = w & 1;   // keys or values
    w >>= 1;
    const int kv = w % a.kv_heads, b = w / a.kv_heads;
    const int per = 256 / a.lanes, r = threadIdx.x / a.lanes;
    const int byte = 16 * (slice * a.lanes + threadIdx.x % a.lanes);
    const bool in = r < per && byte < a.bytes;
    const int* kept = a.kept + ((int64_t)b * a.kept_heads + (a.kept_heads > 1 ? kv : 0)) * a.most;
    const int* table = a.table + b * a.table_row;
    const int64_t start = a.start ? a.start[b] : 0, held = a.table_row * a.page, head = (int64_t)a.page * a.bytes;
    char* base = a.cache + ((int64_t)half * a.kv_heads + kv) * head + (in ? byte : 0);
    const int64_t page_bytes = 2 * a.kv_heads * head;
    struct Look {
        int from[U];          // the token that goes to place i0 + u per + r; -1: none
        int src[U], dst[U];   // its page and that place's
    };
    const auto tokens = [&](int64_t i0, Look& l) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * per + r;
            l.from[u] = in && i < a.most ? kept[i] : -1;
        }
    };
    const auto pages = [&](int64_t i0, Look& l) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * per + r, s = start + l.from[u], d = start + i;
            const bool ok = l.from[u] > i && s >= 0 && s < held && d >= 0 && d < held;
            l.src[u] = ok ? table[s >> a.shift] : -1;
            l.dst[u] = ok ? table[d >> a.shift] : -1;
        }
    };
    struct Tile {
        u32x4 v[U];
        char* to[U];   // nullptr: nothing moves
    };
    const auto load = [&](int64_t i0, const Look& l, Tile& t) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t s = start + l.from[u], d = start + i0 + u * per + r;
            const bool ok = l.src[u] >= 0 && l.src[u] < a.pages && l.dst[u] >= 0 && l.dst[u] < a.pages;
            t.to[u] = ok ? base + (int64_t)l.dst[u] * page_bytes + (d & (a.page - 1)) * a.bytes : nullptr;
            // in any case: the compiler then knows how many loads are behind this tile's
            t.v[u] = *reinterpret_cast<const u32x4*>(ok ? base + (int64_t)l.src[u] * page_bytes + (s & (a.page - 1)) * a.bytes : base);
        }
    };
    const int64_t step = (int64_t)per * U;
    Look l;
    Tile t[2];
    tokens(0, l);
    pages(0, l);
    load(0, l, t[0]);
    if (step < a.most) {
        tokens(step, l);
        pages(step, l);
    }
    for (int64_t i0 = 0; i0 < a.most;) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (i0 + step < a.most) {
                load(i0 + step, l, t[x ^ 1]);
                tokens(i0 + 2 * step, l);
            }
            // this lane's loads of the tile have arrived, and every lane's: then any may store
#pragma unroll
            for (int u = 0; u < U; ++u) asm volatile("" : "+v"(t[x].v[u]));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (t[x].to[u]) *reinterpret_cast<u32x4*>(t[x].to[u]) = t[x].v[u];
            pages(i0 + 2 * step, l);
            i0 += step;
            if (i0 >= a.most) break;
        }
    }
}


// Lists that all key heads share, such as a tree's accepted branch: a workgroup takes some of the heads' keys and values of
// one sequence.  Most entries move nothing; those that do are listed in LDS, and their parts dealt to the lanes.
constexpr int kFewMoves = 256;
__global__ __launch_bounds__(256) void cache_move_few_kernel(KeepArgs a) {
    __shared__ int64_t from[kFewMoves], to[kFewMoves];
    __shared__ int moves[4];
    const int shares = a.slices;   // workgroups of a sequence
    const int share = blockIdx.x % shares, b = blockIdx.x / shares;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = threadIdx.x;
    const int64_t head = (int64_t)a.page * a.bytes, page_bytes = 2 * a.kv_heads * head, held = a.table_row * a.page;
    const int64_t start = a.start ? a.start[b] : 0;
    const int* table = a.table + b * a.table_row;
    int64_t src = 0, dst = 0;
    bool ok = false;
    if (i < a.most) {
        const int k = a.kept[b * a.most + i];
        const int64_t s = start + k, d = start + i;
        if (k > i && s >= 0 && s < held && d >= 0 && d < held) {
            const int ps = table[s >> a.shift], pd = table[d >> a.shift];
            ok = ps >= 0 && ps < a.pages && pd >= 0 && pd < a.pages;
            src = (int64_t)ps * page_bytes + (s & (a.page - 1)) * a.bytes;
            dst = (int64_t)pd * page_bytes + (d & (a.page - 1)) * a.bytes;
        }
    }
    const uint64_t some = __ballot(ok);
    if (lane == 0) moves[wave] = __popcll(some);
    __syncthreads();
    int at = __popcll(some & ((1ull << lane) - 1)), n = 0;
    for (int x = 0; x < 4; ++x) {
        at += x < wave ? moves[x] : 0;
        n += moves[x];
    }
    if (ok) {
        from[at] = src;
        to[at] = dst;
    }
    __syncthreads();
    // parts of 16 bytes: of a token's head, of the heads' keys and values that are this workgroup's, of the moves.  A tile of
    // moves at a time, in ascending order, each part by the same lane for every move: it reads what no earlier move writes.
    const int parts = a.bytes / 16, all = 2 * a.kv_heads, h0 = all * share / shares, h1 = all * (share + 1) / shares;
    constexpr int U = 4;
    for (int p = i; p < (h1 - h0) * parts; p += 256) {
        char* base = a.cache + (int64_t)(h0 + p / parts) * head + p % parts * 16;
        for (int m = 0; m < n; m += U) {
            u32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const u32x4*>(base + from[min(m + u, n - 1)]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (m + u < n) *reinterpret_cast<u32x4*>(base + to[m + u]) = v[u];
        }
    }
}

}  // namespace noble
