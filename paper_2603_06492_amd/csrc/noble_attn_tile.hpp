// Attention over rows of packed sequences: forward, dq, and dk with dv.
//
// Row i of query head h sees the keys [lo_i, hi_i).  With z = scale q.k, s = cap tanh(z / cap) (or z) minus
// slope |at_i - j|, the forward keeps a running maximum m and sum l over the keys (float32, units of log2):
//   o = sum_j exp(s_j - m) v_j / l,   lse = m + log l,
// and the backward forms p = exp(s - lse) again:
//   dp = do.v,  delta = do.o,  dz = p (dp - delta) (1 - tanh^2) scale,
//   dq_i = sum_j dz k_j,  dk_j = sum_i dz q_i,  dv_j = sum_i p do_i.
// dq and dk/dv are separate launches, each of which owns its outputs: two of the seven products are formed twice, and
// in exchange no output is summed by atomics, so results do not depend on the order in which workgroups run.
#pragma once

#include "noble_attn_common.hpp"

namespace noble {

struct AttnArgs {
    HeadRows q, k, v, o, g;      // g: the upstream gradient
    HeadRows dq, dk, dv;
    const int* lo;               // the caller's intervals (nullable)
    const int* hi;
    const float* slopes;         // [heads], with the bias
    float* lse;                  // [heads, Tq], natural logarithm
    float* lse2;                 // backward: lse log2 e, +inf for a row that sees no key, and delta: [heads, Tpad]
    float* delta;
    int* row_lo;                 // backward: the rows' first keys and numbers of keys, and of each 64 rows the bounds
    int* row_keys;
    int4* span;
    float* part;                 // backward, parts > 1: dk and dv of each part, [parts][2][key heads][Tk][D]
    int parts;                   // that the query heads of a key head are dealt to
    int Tq, Tk, heads, share, D;   // share: query heads of a key head
    int Tpad;                      // Tq rounded up to a tile: rows past the end have probability zero in lse2
    int causal, off;               // key index of row 0
    float scale;
    ScoreArgs sc;
};

constexpr int kOwn = 128;   // rows of a workgroup: 32 for each of four waves
constexpr int kPart = 64;   // partner rows of a tile

// How a workgroup of four waves divides its work.  Each wave owns 32 rows of its own and all four share tiles of 64 partner
// rows (two stages in LDS, a barrier a tile); or, split, the four share 32 own rows and take turns at tiles of 32
// partner rows, each through stages of its own without a barrier, and their sums meet at the end.  Split workgroups are
// four times as many with a quarter of the steps one after the other: for calls that do not fill the CUs, and for
// float32, whose products are 16 times the bf16 ones' time and leave the reading of tiles out of account.
template <typename E, int DP, bool SPLIT>
struct TileShape {
    static constexpr int OWN = SPLIT ? 32 : kOwn, PART = SPLIT ? 32 : kPart, U = PART / 32;
    static constexpr int TB = Tile<E, DP>::bytes(PART), STAGE = 2 * TB;
    static constexpr int STAGES = SPLIT && 8 * STAGE > 131072 ? 1 : 2;
    static constexpr int LDS = (SPLIT ? 4 : 1) * STAGES * STAGE;
    static constexpr int REQUESTS = STAGE / 1024;   // of a split wave and stage
};

// Where a wave's tiles are and when: the n-th of `count`.  request(n, address) asks for one; at(n) waits until it is there
// and has the next one asked for; done(n) says that it has been read.
template <typename E, int DP, bool SPLIT, typename Request>
struct Tiles {
    using S = TileShape<E, DP, SPLIT>;
    char* lds;
    int count;
    const Request& request;
    __device__ __forceinline__ Tiles(char* lds_, int wave, int count_, const Request& r)
        : lds(SPLIT ? lds_ + wave * S::STAGES * S::STAGE : lds_), count(count_), request(r) {
        if (count > 0) request(0, lds);
    }
    __device__ __forceinline__ int offset(int n) const { return S::STAGES == 2 ? (n & 1) * S::STAGE : 0; }
    __device__ __forceinline__ void at(int n) const {
        if constexpr (!SPLIT) {
            arrive_all();
            if (n + 1 < count) request(n + 1, lds + offset(n + 1));
        } else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other stage has been read
            if (S::STAGES == 2 && n + 1 < count) {
                request(n + 1, lds + offset(n + 1));
                wait_vmcnt<S::REQUESTS>();
            } else {
                wait_vmcnt<0>();
            }
            asm volatile("" ::: "memory");
        }
    }
    __device__ __forceinline__ void done(int n) const {
        if constexpr (S::STAGES == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (n + 1 < count) request(n + 1, lds);
        }
    }
};

// The four waves' sums of the same 32 rows, acc of lane l's row l % 32, as [wave][32][DP + 4] float32 in LDS.
template <int DP>
struct Meeting {
    static constexpr int LD = DP + 4, BYTES = 4 * 32 * LD * 4;
    float* at;
    int wave, lane;
    __device__ __forceinline__ Meeting(char* lds, int wave_, int lane_)
        : at(reinterpret_cast<float*>(lds)), wave(wave_), lane(lane_) {}
    __device__ __forceinline__ void put(const f32x16 (&acc)[DP / 32], float x, float y) const {
        float* p = at + (wave * 32 + (lane & 31)) * LD;
        const int h = lane >> 5;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(p + 32 * d + 8 * i + 4 * h) =
                    f32x4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
        if (h == 0) {
            p[DP] = x;
            p[DP + 1] = y;
        }
    }
    __device__ __forceinline__ const float* get(int w, int row) const { return at + (w * 32 + row) * LD; }
};

// The keys that row i sees, within [0, Tk): {0, 0} for a row that sees none.
__device__ __forceinline__ int2 row_interval(const AttnArgs& a, int i) {
    int lo = 0, hi = a.Tk;
    if (a.lo) {
        lo = max(a.lo[i], 0);
        hi = min(a.hi[i], a.Tk);
    }
    if (a.causal) hi = (int)min((int64_t)hi, (int64_t)i + a.off + 1);
    return lo < hi ? int2{lo, hi} : int2{0, 0};
}

__device__ __forceinline__ void raw(const f32x16& s, float* z) {
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = s[i];
}

// Workgroup -> (head, own tile): the last tiles (the longest ones under a causal mask) of a key head first, the query
// heads that share it side by side.
struct OwnTile {
    int head = 0, tile = 0;
    bool work;
    __device__ __forceinline__ OwnTile(const AttnArgs& a, int rows) {
        const int tiles = (a.Tq + rows - 1) / rows;
        int kv = 0, at = 0;
        work = HeadOrder{a.heads / a.share, tiles * a.share}.place(blockIdx.x, kv, at);
        head = kv * a.share + at % a.share;
        tile = tiles - 1 - at / a.share;
    }
};

// The own rows' intervals as the kernels that own queries use them: of this lane's row, of the wave's rows and of the
// workgroup's.
struct OwnRows {
    int lo, hi;             // this lane's row
    int wave_lo, wave_hi;   // the keys that any row of the wave sees
    int full_lo, full_hi;   // the keys that every row of the wave sees
    int all_lo, all_hi;     // the keys that any row of the workgroup sees
    // j - lo, unsigned, is below this for the keys that the row sees
    __device__ __forceinline__ uint32_t width() const { return (uint32_t)(hi - lo); }
    // `all`: also the workgroup's, which has the 128 rows from row0; the wave has the 32 from wave_row.
    __device__ __forceinline__ OwnRows(const AttnArgs& a, int row0, int wave_row, bool all, int lane) {
        const int i = wave_row + (lane & 31);
        const bool in = i < a.Tq;
        const int2 r = in ? row_interval(a, i) : int2{0, 0};
        lo = r.x;
        hi = r.y;
        wave_hi = wave_max(hi);
        wave_lo = min(wave_min(lo < hi ? lo : INT32_MAX), wave_hi);
        // rows past the end do not count: their queries are zeros and nothing of them is stored
        full_lo = wave_max(in ? lo : 0);
        full_hi = wave_min(in ? hi : INT32_MAX);
        all_lo = wave_lo;
        all_hi = wave_hi;
        if (!all) return;
        int least = INT32_MAX, most = 0;
#pragma unroll
        for (int k = 0; k < kOwn / 64; ++k) {
            const int n = row0 + 64 * k + lane;
            const int2 t = n < a.Tq ? row_interval(a, n) : int2{0, 0};
            if (t.x < t.y) {
                least = min(least, t.x);
                most = max(most, t.y);
            }
        }
        all_hi = wave_max(most);
        all_lo = min(wave_min(least), all_hi);
    }
};

// ---- rows whose sums came out infinite or NaN ------------------------------------------------------------------------
// A product over a tile multiplies a key (or row) that is not seen by a probability of zero, and zero times an infinite
// or NaN element is NaN.  So a wave that finds such a result forms these rows again, one after the other and over the
// seen partners alone, with two elements of the head a lane: unseen values do not reach a row, seen ones do.  A row whose
// elements are all NaN stays that and is done, so a training step that has turned into NaN or infinities is not slow:
// 2048 rows of 8 heads of 128, forward and backward, 74 to 102 -> 0.3 ms (0.2 without).  One infinite value that every row sees
// is: its rows' other elements are sums over all their keys, 60 ms for 4096 causal rows of 16 heads (0.44 without).

// The sums' zeroes: NaN if any element is infinite or NaN.
template <int ND>
__device__ __forceinline__ float zero_of(const f32x16 (&acc)[ND], float t) {
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) t = fmaf(acc[d][i], 0.f, t);
    return t;
}
// The own rows (bit r: row r of 32) that the lanes l and l + 32 say no to.
__device__ __forceinline__ uint32_t rows_of(bool bad) {
    const uint64_t b = __ballot(bad);
    return (uint32_t)b | (uint32_t)(b >> 32);
}
struct Pair {
    float x = 0.f, y = 0.f;
};
// Elements 2 lane and 2 lane + 1 of one row (zeros past the head).
template <typename E>
__device__ __forceinline__ Pair load_pair(const HeadRows& t, int head, int64_t row, int D, int lane) {
    Pair p;
    if (2 * lane < D) {
        const char* at = t.ptr + head * t.head + row * t.row + 2 * lane * (int)sizeof(E);
        if constexpr (sizeof(E) == 2) {
            const uint32_t v = *reinterpret_cast<const uint32_t*>(at);
            p.x = __uint_as_float(v << 16);
            p.y = __uint_as_float(v & 0xffff0000u);
        } else {
            p.x = reinterpret_cast<const float*>(at)[0];
            p.y = reinterpret_cast<const float*>(at)[1];
        }
    }
    return p;
}
template <typename E>
__device__ __forceinline__ void store_pair(const HeadRows& t, int head, int64_t row, int D, int lane, float x, float y) {
    if (2 * lane >= D) return;
    char* at = t.ptr + head * t.head + row * t.row + 2 * lane * (int)sizeof(E);
    if constexpr (sizeof(E) == 2) {
        *reinterpret_cast<uint32_t*>(at) = pack_bf16(x, y);
    } else {
        reinterpret_cast<float*>(at)[0] = x;
        reinterpret_cast<float*>(at)[1] = y;
    }
}
__device__ __forceinline__ float wave_dot(const Pair& a, const Pair& b) {
    float s = a.x * b.x + a.y * b.y;
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    return s;
}
// Whether a row's elements are all NaN.
__device__ __forceinline__ bool all_nan(const Pair& p, int D, int lane) {
    return __all(2 * lane >= D || (p.x != p.x && p.y != p.y));
}
// The probability of key j for row i of one head, and the cap's slope.
template <typename E, int MODE>
__device__ __forceinline__ float one_probability(const AttnArgs& a, const Pair& q, const Pair& k, float slope, int i, int j,
                                                 float lse2, float& cap_slope) {
    const float s = wave_dot(q, k);
    float z;
    cap_slope = 1.f;
    scores<E, MODE, 1>(a.sc, &s, &z, MODE & kCap ? &cap_slope : nullptr);
    if constexpr (MODE & kBias) z = fmaf(-slope, fabsf((float)((int64_t)i + a.off - j)), z);
    return exp_score<MODE>(a.sc, z, lse2);
}

// Forward.  What bounds it at long rows: the issue slots that a score's 5 to 12 vector operations take (its exponential
// counts for four) beside the matrix cores, at the clock that both together leave: a prompt of 16384 tokens, 16 heads of
// 128 over 4 key heads, prefix mask and bias, 1.26 ms, 0.97 PFLOP/s; a large library product reaches 1.25 on this card.
// Packed short rows are bound by the steps that follow each other in one workgroup: 8 x 1024 tokens, 8 heads of 128,
// causal, 32.6 us (0.53 PFLOP/s of seen pairs), 128 images of 197 tokens, 12 heads of 64, 53 us (2.9 TB/s).
template <typename E, int DP, int MODE, bool SPLIT>
__global__ __launch_bounds__(256, SPLIT ? 1 : 2) void attn_fwd_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    using S = TileShape<E, DP, SPLIT>;
    constexpr int ES = T::ES, TB = S::TB, NS = DP / 16, ND = DP / 32, U = S::U, PART = S::PART;
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const OwnTile w(a, S::OWN);
    if (!w.work) return;
    const int row0 = w.tile * S::OWN, wave_row = SPLIT ? row0 : row0 + 32 * wave, row = wave_row + (lane & 31);
    const int kv = w.head / a.share, db = a.D * ES;
    Frag<E> q[NS];
    const char* qp = a.q.ptr + w.head * a.q.head + (int64_t)row * a.q.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = global_frag<E>(qp + 16 * s * ES, row < a.Tq && 16 * s + 8 * h < a.D);
    const OwnRows own(a, row0, wave_row, !SPLIT, lane);

    const int tiles = (own.all_hi - own.all_lo + PART - 1) / PART;
    const auto key_of = [&](int n) { return own.all_lo + (SPLIT ? 4 * n + wave : n) * PART; };
    const auto request = [&](int n, char* dst) {
        const int k0 = key_of(n), who = SPLIT ? 0 : wave;
        constexpr int NW = SPLIT ? 1 : 4;
        T::template request<NW, PART>(rows_desc(a.k, kv, k0, own.all_hi, db), dst, (int)a.k.row, db, who, lane);
        T::template request<NW, PART>(rows_desc(a.v, kv, k0, own.all_hi, db), dst + TB, (int)a.v.row, db, who, lane);
    };
    const Tiles<E, DP, SPLIT, decltype(request)> ts(lds, wave, SPLIT ? (tiles - wave + 3) >> 2 : tiles, request);

    const float slope = MODE & kBias ? a.slopes[w.head] * kLog2e / a.sc.unit : 0.f;
    const int at = row + a.off;

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    const Reader<E, DP> rd(ts.lds, lane);
    operands_here();

    for (int n = 0; n < ts.count; ++n) {
        ts.at(n);
        const int k0 = key_of(n);
        if (!SPLIT && (k0 >= own.wave_hi || k0 + PART <= own.wave_lo)) continue;
        const Reader<E, DP> at_tile = rd.at(ts.offset(n));
        float z[16 * U];
        f32x16 s[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int x = 0; x < NS; ++x)
#pragma unroll
            for (int u = 0; u < U; ++u) mma32x32(s[u], at_tile.along(x, 32 * u * T::RB), q[x]);
        if constexpr (ES == 2) read_ahead<U * NS, 1, 1, 4>();
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw(s[u], z + 16 * u);
            scores<E, MODE, 16>(a.sc, z + 16 * u, z + 16 * u, nullptr);
            if constexpr (MODE & kBias) bias16(z + 16 * u, slope, (float)(k0 + 4 * h - at) + 32.f * u);
        }
        if (k0 < own.full_lo || k0 + PART > own.full_hi) {
#pragma unroll
            for (int i = 0; i < 16 * U; ++i) {
                const int j = k0 + 8 * (i >> 2) + 4 * h + (i & 3);
                z[i] = (uint32_t)(j - own.lo) < own.width() ? z[i] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 16 * U; ++i) top = fmaxf(top, z[i]);
        top = max_halves(top) * (MODE & kCap ? 1.f : a.sc.unit);
        // The maximum that the exponents are taken from need only be near: it follows once a row's own has grown by
        // 2^8, which leaves sums and products far inside their range, and most tiles leave acc as it is.
        if (__any(top > m + 8.f)) {
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
        for (int i = 0; i < 16 * U; ++i) {
            z[i] = exp_score<MODE>(a.sc, z[i], from);
            l += z[i];
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int x = 0; x < 2 * U; ++x) {
            const Frag<E> p = to_frag<E>(z + 8 * x);
#pragma unroll
            for (int d = 0; d < ND; ++d) mma32x32(acc[d], at_tile.across(d, TB + 16 * x * T::RB), p);
        }
        if constexpr (ES == 2) read_ahead<2 * U * ND, 1, 2, 4>();
        __builtin_amdgcn_s_setprio(0);
        ts.done(n);
    }

    l = sum_halves(l);
    const bool ok = zero_of(acc, 0.f) == 0.f;
    uint32_t again = rows_of(row < a.Tq && !ok);
    // A sum of zero: a row that sees no key, or one whose scores are all minus infinity, and 0 / 0 is not a number.
    if constexpr (!SPLIT) {
        const float inv = l != 0.f ? 1.f / l : own.lo < own.hi ? NAN : 0.f;
        if (row < a.Tq && !((again >> (lane & 31)) & 1u)) {
            char* op = a.o.ptr + w.head * a.o.head + (int64_t)row * a.o.row;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = 32 * d + 8 * i + 4 * h;
                    if (e < a.D)
                        store4<E>(op + e * ES, acc[d][4 * i] * inv, acc[d][4 * i + 1] * inv, acc[d][4 * i + 2] * inv,
                                  acc[d][4 * i + 3] * inv);
                }
        }
    } else {
        const Meeting<DP> meet(lds, wave, lane);
        static_assert(Meeting<DP>::BYTES + 16 <= S::LDS, "the sums fit the stages");
        uint32_t* flags = reinterpret_cast<uint32_t*>(lds + Meeting<DP>::BYTES);
        __syncthreads();   // the stages have been read
        meet.put(acc, m, l);
        if (lane == 0) flags[wave] = again;
        __syncthreads();
        again = flags[0] | flags[1] | flags[2] | flags[3];
        const uint32_t sees = rows_of(own.lo < own.hi);
        // every lane's statistics of its row, over the waves
        float top = -INFINITY, total = 0.f, f[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) top = fmaxf(top, meet.get(x, lane & 31)[DP]);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            total += meet.get(x, lane & 31)[DP + 1] * __builtin_amdgcn_exp2f(meet.get(x, lane & 31)[DP] - (top == -INFINITY ? 0.f : top));
        m = top;
        l = total;
        for (int e = threadIdx.x; e < 32 * (DP / 4); e += 256) {
            const int r = e / (DP / 4), d = e % (DP / 4) * 4;
            float most = -INFINITY, sum = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) most = fmaxf(most, meet.get(x, r)[DP]);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                f[x] = __builtin_amdgcn_exp2f(meet.get(x, r)[DP] - (most == -INFINITY ? 0.f : most));
                sum += meet.get(x, r)[DP + 1] * f[x];
            }
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 4; ++x) v += *reinterpret_cast<const f32x4*>(meet.get(x, r) + d) * f[x];
            const float inv = sum != 0.f ? 1.f / sum : (sees >> r) & 1u ? NAN : 0.f;
            if (d < a.D && row0 + r < a.Tq && !((again >> r) & 1u))
                store4<E>(a.o.ptr + w.head * a.o.head + (int64_t)(row0 + r) * a.o.row + d * ES, v[0] * inv, v[1] * inv,
                          v[2] * inv, v[3] * inv);
        }
        again &= 0x11111111u << wave;   // a quarter of the rows for each wave
    }
    const float lse2 = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    if (h == 0 && row < a.Tq && (!SPLIT || wave == 0))
        a.lse[(int64_t)w.head * a.Tq + row] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
    for (; again; again &= again - 1) {
        const int r = __builtin_ctz(again), i = wave_row + r;
        const int lo = __shfl(own.lo, r), hi = __shfl(own.hi, r);
        const float from = __shfl(lse2, r);
        const Pair qi = load_pair<E>(a.q, w.head, i, a.D, lane);
        Pair sum;
        for (int j = lo; j < hi && !all_nan(sum, a.D, lane); ++j) {
            float unused;
            const float p = one_probability<E, MODE>(a, qi, load_pair<E>(a.k, kv, j, a.D, lane), slope, i, j, from, unused);
            const Pair v = load_pair<E>(a.v, kv, j, a.D, lane);
            sum.x += p * v.x;
            sum.y += p * v.y;
        }
        store_pair<E>(a.o, w.head, i, a.D, lane, sum.x, sum.y);
    }
}

// The sum over eight elements of two fragments' products.
template <typename E>
__device__ __forceinline__ float dot8(const Frag<E>& a, const Frag<E>& b) {
    float sum = 0.f;
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sum = fmaf(bf2f(a.v[j] & 0xffffu), bf2f(b.v[j] & 0xffffu), sum);
            sum = fmaf(__uint_as_float(a.v[j] & 0xffff0000u), __uint_as_float(b.v[j] & 0xffff0000u), sum);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum = fmaf(__uint_as_float(a.v[j >> 2][j & 3]), __uint_as_float(b.v[j >> 2][j & 3]), sum);
    }
    return sum;
}

// The intervals of 64 rows, one a lane, and what they span.
__device__ __forceinline__ void write_spans(const AttnArgs& a, int tile, int lane) {
    const int i = kPart * tile + lane;
    const bool in = i < a.Tq;
    const int2 r = in ? row_interval(a, i) : int2{0, 0};
    if (in) {
        a.row_lo[i] = r.x;
        a.row_keys[i] = r.y - r.x;
    }
    const int most = wave_max(r.y), least = min(wave_min(r.x < r.y ? r.x : INT32_MAX), most);
    const int from = wave_max(in ? r.x : 0), to = wave_min(in ? r.y : INT32_MAX);
    if (lane == 0 && kPart * tile < a.Tq) a.span[tile] = int4{least, most, from, to};
}

// dq, and what the dk/dv launch after it reads: delta (do is here already, o is read once for it), lse in units of log2,
// the rows' intervals and what 64 of them span.  delta is do.o of the rounded o, plus what is left of sum p (dp - delta)
// after the row's keys, which an exact one would make zero: so dk does not carry o's rounding.
// Three products a tile where the forward has two: 8 x 1024 tokens 48 us, the images 71 us.
template <typename E, int DP, int MODE, bool SPLIT>
__global__ __launch_bounds__(256, SPLIT ? 1 : 2) void attn_dq_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    using S = TileShape<E, DP, SPLIT>;
    constexpr int ES = T::ES, TB = S::TB, NS = DP / 16, ND = DP / 32, U = S::U, PART = S::PART;
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const OwnTile w(a, S::OWN);
    if (!w.work) return;
    const int row0 = w.tile * S::OWN, wave_row = SPLIT ? row0 : row0 + 32 * wave, row = wave_row + (lane & 31);
    const int kv = w.head / a.share, db = a.D * ES;
    Frag<E> q[NS], g[NS];
    const char* qp = a.q.ptr + w.head * a.q.head + (int64_t)row * a.q.row + 8 * h * ES;
    const char* gp = a.g.ptr + w.head * a.g.head + (int64_t)row * a.g.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const bool ok = row < a.Tq && 16 * s + 8 * h < a.D;
        q[s] = global_frag<E>(qp + 16 * s * ES, ok);
        g[s] = global_frag<E>(gp + 16 * s * ES, ok);
    }
    const OwnRows own(a, row0, wave_row, !SPLIT, lane);

    const int tiles = (own.all_hi - own.all_lo + PART - 1) / PART;
    const auto key_of = [&](int n) { return own.all_lo + (SPLIT ? 4 * n + wave : n) * PART; };
    const auto request = [&](int n, char* dst) {
        const int k0 = key_of(n), who = SPLIT ? 0 : wave;
        constexpr int NW = SPLIT ? 1 : 4;
        T::template request<NW, PART>(rows_desc(a.k, kv, k0, own.all_hi, db), dst, (int)a.k.row, db, who, lane);
        T::template request<NW, PART>(rows_desc(a.v, kv, k0, own.all_hi, db), dst + TB, (int)a.v.row, db, who, lane);
    };
    const Tiles<E, DP, SPLIT, decltype(request)> ts(lds, wave, SPLIT ? (tiles - wave + 3) >> 2 : tiles, request);

    const float slope = MODE & kBias ? a.slopes[w.head] * kLog2e / a.sc.unit : 0.f;
    const int at = row + a.off;
    float delta = 0.f, lse2 = INFINITY;
    {
        const char* op = a.o.ptr + w.head * a.o.head + (int64_t)row * a.o.row + 8 * h * ES;
#pragma unroll
        for (int s = 0; s < NS; ++s)
            delta += dot8(global_frag<E>(op + 16 * s * ES, row < a.Tq && 16 * s + 8 * h < a.D), g[s]);
        delta = sum_halves(delta);
        const float lse = row < a.Tq ? a.lse[(int64_t)w.head * a.Tq + row] : -INFINITY;
        if (lse != -INFINITY) lse2 = lse * kLog2e;
        else if (own.lo < own.hi) lse2 = NAN;   // its scores are all minus infinity
        if (h == 0 && row < a.Tpad && (!SPLIT || wave == 0)) a.lse2[(int64_t)w.head * a.Tpad + row] = lse2;
    }
    if (w.head == 0 && row0 % kPart == 0 && wave < (S::OWN + kPart - 1) / kPart) write_spans(a, row0 / kPart + wave, lane);
    if (SPLIT && wave == 0 && h == 0 && row0 + 32 == a.Tpad - 32 && row0 + 32 >= a.Tq) {
        // a last tile of 64 rows whose second half no workgroup owns
        a.lse2[(int64_t)w.head * a.Tpad + row + 32] = INFINITY;
        a.delta[(int64_t)w.head * a.Tpad + row + 32] = 0.f;
    }
    float rest = 0.f;   // sum of p (dp - delta): what delta lacks, o having been rounded

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

    const Reader<E, DP> rd(ts.lds, lane);
    operands_here();
    for (int n = 0; n < ts.count; ++n) {
        ts.at(n);
        const int k0 = key_of(n);
        if (!SPLIT && (k0 >= own.wave_hi || k0 + PART <= own.wave_lo)) continue;
        const Reader<E, DP> at_tile = rd.at(ts.offset(n));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int ku = k0 + 32 * u;
            if (U > 1 && (ku >= own.wave_hi || ku + 32 <= own.wave_lo)) continue;
            const bool part = ku < own.full_lo || ku + 32 > own.full_hi;
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
            __builtin_amdgcn_s_setprio(1);
            // S and dP in turn for heads of 128 (8 x 1024 tokens: 50.2 -> 47.4 us), one after the other for heads of 64, whose
            // sums are half as long (ViT-B images: 74.7 us, in turn 76.5)
            if constexpr (DP == 128) {
#pragma unroll
                for (int x = 0; x < NS; ++x) {
                    mma32x32(s, at_tile.along(x, 32 * u * T::RB), q[x]);
                    mma32x32(dp, at_tile.along(x, TB + 32 * u * T::RB), g[x]);
                }
            } else {
#pragma unroll
                for (int x = 0; x < NS; ++x) mma32x32(s, at_tile.along(x, 32 * u * T::RB), q[x]);
#pragma unroll
                for (int x = 0; x < NS; ++x) mma32x32(dp, at_tile.along(x, TB + 32 * u * T::RB), g[x]);
            }
            if constexpr (ES == 2) read_ahead<2 * NS, 1, 1, 4>();
            __builtin_amdgcn_s_setprio(0);
            float z[16], dz[16], cap_slope[16];
            raw(s, z);
            scores<E, MODE, 16>(a.sc, z, z, MODE & kCap ? cap_slope : nullptr);
            if constexpr (MODE & kBias) bias16(z, slope, (float)(k0 + 4 * h - at) + 32.f * u);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                dz[i] = exp_score<MODE>(a.sc, z[i], lse2) * (dp[i] - delta);
            }
            if (part) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = k0 + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3);
                    dz[i] = (uint32_t)(j - own.lo) < own.width() ? dz[i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                rest += dz[i];
                if constexpr (MODE & kCap) dz[i] *= cap_slope[i];
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<E> f = to_frag<E>(dz + 8 * x);
#pragma unroll
                for (int d = 0; d < ND; ++d) mma32x32(acc[d], at_tile.across(d, (32 * u + 16 * x) * T::RB), f);
            }
            if constexpr (ES == 2) read_ahead<2 * ND, 1, 2, 4>();
            __builtin_amdgcn_s_setprio(0);
        }
        ts.done(n);
    }

    rest = sum_halves(rest);
    uint32_t again = rows_of(row < a.Tq && !(zero_of(acc, 0.f) == 0.f));
    if constexpr (!SPLIT) {
        if (row < a.Tq && !((again >> (lane & 31)) & 1u)) {
            char* op = a.dq.ptr + w.head * a.dq.head + (int64_t)row * a.dq.row;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = 32 * d + 8 * i + 4 * h;
                    if (e < a.D)
                        store4<E>(op + e * ES, acc[d][4 * i] * a.scale, acc[d][4 * i + 1] * a.scale,
                                  acc[d][4 * i + 2] * a.scale, acc[d][4 * i + 3] * a.scale);
                }
        }
    } else {
        const Meeting<DP> meet(lds, wave, lane);
        static_assert(Meeting<DP>::BYTES + 16 <= S::LDS, "the sums fit the stages");
        uint32_t* flags = reinterpret_cast<uint32_t*>(lds + Meeting<DP>::BYTES);
        __syncthreads();   // the stages have been read
        meet.put(acc, rest, 0.f);
        if (lane == 0) flags[wave] = again;
        __syncthreads();
        again = flags[0] | flags[1] | flags[2] | flags[3];
        rest = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) rest += meet.get(x, lane & 31)[DP];
        for (int e = threadIdx.x; e < 32 * (DP / 4); e += 256) {
            const int r = e / (DP / 4), d = e % (DP / 4) * 4;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 4; ++x) v += *reinterpret_cast<const f32x4*>(meet.get(x, r) + d);
            if (d < a.D && row0 + r < a.Tq && !((again >> r) & 1u))
                store4<E>(a.dq.ptr + w.head * a.dq.head + (int64_t)(row0 + r) * a.dq.row + d * ES, v[0] * a.scale,
                          v[1] * a.scale, v[2] * a.scale, v[3] * a.scale);
        }
        again &= 0x11111111u << wave;   // a quarter of the rows for each wave
    }
    if (h == 0 && row < a.Tpad && (!SPLIT || wave == 0)) a.delta[(int64_t)w.head * a.Tpad + row] = delta + rest;
    for (; again; again &= again - 1) {
        const int r = __builtin_ctz(again), i = wave_row + r;
        const int lo = __shfl(own.lo, r), hi = __shfl(own.hi, r);
        const float from = __shfl(lse2, r), less = __shfl(delta, r);
        const Pair qi = load_pair<E>(a.q, w.head, i, a.D, lane), gi = load_pair<E>(a.g, w.head, i, a.D, lane);
        Pair sum;
        for (int j = lo; j < hi && !all_nan(sum, a.D, lane); ++j) {
            float cap_slope;
            const Pair k = load_pair<E>(a.k, kv, j, a.D, lane);
            const float p = one_probability<E, MODE>(a, qi, k, slope, i, j, from, cap_slope);
            const float dz = p * (wave_dot(gi, load_pair<E>(a.v, kv, j, a.D, lane)) - less) * cap_slope * a.scale;
            sum.x += dz * k.x;
            sum.y += dz * k.y;
        }
        store_pair<E>(a.dq, w.head, i, a.D, lane, sum.x, sum.y);
    }
}

// The query heads [at, end) of a key head's that part p of them has.
struct HeadPart {
    int at, end;
    __device__ __forceinline__ HeadPart(int share, int p, int parts) : at(share * p / parts), end(share * (p + 1) / parts) {}
};

// The 64-row tiles of queries that see a workgroup's keys, in order, over query heads that share the key head.
// 64 tiles are looked at together, one a lane.
struct Partners {
    int end, tiles;
    const int4* span;
    int k0, k1, w0, w1;      // the workgroup's keys, and the wave's
    int head, base = -64, lane;
    uint64_t any = 0, mine = 0, full = 0;
    __device__ __forceinline__ Partners(const AttnArgs& a, HeadPart heads, int key0, int keys, int wave_key, int wave_keys, int lane_)
        : end(heads.end), tiles((a.Tq + kPart - 1) / kPart), span(a.span), k0(key0), k1(min(key0 + keys, a.Tk)),
          w0(wave_key), w1(min(wave_key + wave_keys, a.Tk)), head(heads.at), lane(lane_) {}
    // The next (head, tile), and whether the wave's keys are seen by any or by all of its rows; false at the end.
    __device__ __forceinline__ bool next(int& hd, int& tile, bool& seen, bool& whole) {
        while (!any) {
            base += 64;
            if (base >= tiles) {
                base = 0;
                if (++head >= end) return false;
            }
            int4 s = {0, 0, 0, 0};
            if (base + lane < tiles) s = span[base + lane];
            any = __ballot(s.x < k1 && s.y > k0);
            mine = __ballot(s.x < w1 && s.y > w0);
            full = __ballot(s.z <= w0 && s.w >= w1);
        }
        const int b = __builtin_ctzll(any);
        any &= any - 1;
        hd = head;
        tile = base + b;
        seen = (mine >> b) & 1;
        whole = (full >> b) & 1;
        return true;
    }
};

// dk and dv of 128 keys, 32 a wave: S and dP, then their products with the rows' gradients and queries.
// bf16 heads of 128: the two sums (128 registers), the keys (32), S and dP (32) and the operands read ahead leave no room
// for the values in the 256 registers that a wave has when two share a SIMD, so the values are read from LDS for every
// tile, and tiles are 32 rows, so that two workgroups fit a CU's LDS.  With the values in registers and one wave a SIMD
// 8 x 1024 tokens took 104 us, with 64 keys a wave 94, this way 65 to 67; 128 images of 12 heads of 64 take 89.
template <typename E, int DP, bool SPLIT>
struct DkvShape {
    static constexpr bool VALUES_IN_LDS = !SPLIT && sizeof(E) == 2 && DP == 128;
    static constexpr int OWN = SPLIT ? 32 : kOwn, ROWS = VALUES_IN_LDS || SPLIT ? 32 : kPart;
    static constexpr int TB = Tile<E, DP>::bytes(ROWS), INFO = 4 * kPart * 4, STAGE = 2 * TB + INFO;
    static constexpr int STAGES = SPLIT && 8 * STAGE > 160 * 1024 ? 1 : 2;
    static constexpr int LDS = (SPLIT ? 4 : 1) * STAGES * STAGE + (VALUES_IN_LDS ? Tile<E, DP>::bytes(kOwn) : 0);
    static constexpr int REQUESTS = 2 * TB / 1024 + 4;   // of a split wave and stage
};

// Where a part's sums for dk (which 0) or dv (1) go.
__device__ __forceinline__ HeadRows part_rows(const AttnArgs& a, int part, int which) {
    HeadRows r;
    r.row = (int64_t)a.D * 4;
    r.head = a.Tk * r.row;
    r.ptr = reinterpret_cast<char*>(a.part) + (2 * part + which) * (a.heads / a.share) * r.head;
    return r;
}

// PARTS: more than one part; with the choice made inside one kernel, forward and backward of 128 images of
// 12 heads of 64 took 246 us and not 225.
template <typename E, int DP, int MODE, bool SPLIT, bool PARTS>
__global__ __launch_bounds__(256, SPLIT ? 1 : 2) void attn_dkv_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    using S = DkvShape<E, DP, SPLIT>;
    constexpr int ES = T::ES, TB = S::TB, NS = DP / 16, ND = DP / 32, ROWS = S::ROWS, STAGE = S::STAGE;
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    int kv = 0, key_tile = 0;   // the first keys (which the most rows see under a causal mask) first
    const int parts = PARTS ? a.parts : 1;
    if (!HeadOrder{a.heads / a.share, (a.Tk + S::OWN - 1) / S::OWN * parts}.place(blockIdx.x, kv, key_tile)) return;
    const int part_of = key_tile % parts;
    key_tile /= parts;
    const HeadPart heads(a.share, part_of, parts);
    const int key0 = key_tile * S::OWN, wkey = SPLIT ? key0 : key0 + 32 * wave, key = wkey + (lane & 31), db = a.D * ES;

    // Tiles of ROWS rows: of all waves, or every fourth one (`turn`) for each
    Partners it(a, heads, key0, S::OWN, wkey, 32, lane);
    char* stages = SPLIT ? lds + wave * S::STAGES * STAGE : lds;
    int gi = 0, tile = 0, sub = 0, turn = -1;   // sub: the part of ROWS rows of a 64-row tile
    bool seen = false, whole = false, more = it.next(gi, tile, seen, whole);
    const auto step = [&] {
        if (++sub == kPart / ROWS || tile * kPart + sub * ROWS >= a.Tq) {
            sub = 0;
            more = it.next(gi, tile, seen, whole);
        }
    };
    const auto advance = [&] {   // to this wave's next tile
        if constexpr (!SPLIT) {
            step();
        } else {
            const int steps = turn < 0 ? wave : 4;
            turn = 0;
            for (int x = 0; x < steps && more; ++x) step();
        }
    };
    if constexpr (SPLIT) advance();
    const auto request = [&](int stage) {
        char* dst = stages + stage * STAGE;
        const int head = kv * a.share + gi, r0 = tile * kPart + sub * ROWS;
        constexpr int NW = SPLIT ? 1 : 4;
        const int who = SPLIT ? 0 : wave;
        T::template request<NW, ROWS>(rows_desc(a.q, head, r0, a.Tq, db), dst, (int)a.q.row, db, who, lane);
        T::template request<NW, ROWS>(rows_desc(a.g, head, r0, a.Tq, db), dst + TB, (int)a.g.row, db, who, lane);
        const int64_t rh = (int64_t)head * a.Tpad + r0;
#pragma unroll
        for (int x = 0; x < 4 / NW; ++x) {
            const int n = SPLIT ? x : wave;
            const void* src = n == 0 ? static_cast<const void*>(a.lse2 + rh) : n == 1 ? a.delta + rh :
                              n == 2 ? static_cast<const void*>(a.row_lo + r0) : a.row_keys + r0;
            dma4(wave_desc(static_cast<const char*>(src), (int64_t)(n < 2 ? ROWS : min(a.Tq - r0, ROWS)) * 4),
                 dst + 2 * TB + n * kPart * 4, lane);
        }
    };
    if (more) request(0);
    if constexpr (S::VALUES_IN_LDS)
        T::template request<4, kOwn>(rows_desc(a.v, kv, key0, a.Tk, db), lds + 2 * STAGE, (int)a.v.row, db, wave, lane);

    Frag<E> k[NS], v[S::VALUES_IN_LDS ? 1 : NS];
    const char* kp = a.k.ptr + kv * a.k.head + (int64_t)key * a.k.row + 8 * h * ES;
    const char* vp = a.v.ptr + kv * a.v.head + (int64_t)key * a.v.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const bool ok = key < a.Tk && 16 * s + 8 * h < a.D;
        k[s] = global_frag<E>(kp + 16 * s * ES, ok);
        if constexpr (!S::VALUES_IN_LDS) v[s] = global_frag<E>(vp + 16 * s * ES, ok);
    }

    f32x16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;

    const Reader<E, DP> rd(stages, lane);
    const Reader<E, DP> values = rd.at(2 * STAGE + 32 * wave * T::RB);
    operands_here();
    for (int n = 0; more; ++n) {
        const int r0 = tile * kPart + sub * ROWS, head = kv * a.share + gi;
        const int stage = S::STAGES == 2 ? (n & 1) * STAGE : 0;
        const bool mine = seen, part = !whole;
        if constexpr (!SPLIT) {
            arrive_all();
            advance();
            if (more) request((n + 1) & 1);
        } else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other stage has been read
            advance();
            if (S::STAGES == 2 && more) {
                request((n + 1) & 1);
                wait_vmcnt<S::REQUESTS>();
            } else {
                wait_vmcnt<0>();
            }
            asm volatile("" ::: "memory");
        }
        if (!SPLIT && !mine) continue;
        const float slope = MODE & kBias ? a.slopes[head] * kLog2e / a.sc.unit : 0.f;
#pragma unroll 1
        for (int u = 0; u < ROWS / 32; ++u) {
            // 32 rows: S and dP, p, dv, dz, dk
            const Reader<E, DP> at = rd.at(stage + 32 * u * T::RB);
            const char* rows = stages + stage + 2 * TB + 4 * (32 * u + 4 * h);   // lse2, delta, first key, keys of rows 4 h ..
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(s, at.along(x, 0), k[x]);
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                if constexpr (S::VALUES_IN_LDS) mma32x32(dp, at.along(x, TB), values.along(x, 0));
                else mma32x32(dp, at.along(x, TB), v[x]);
            }
            if constexpr (S::VALUES_IN_LDS) {
                read_ahead<NS, 1, 1, 3>();
                read_ahead<NS, 1, 2, 2>();
            } else if constexpr (ES == 2) {
                read_ahead<2 * NS, 1, 1, 4>();
            }
            __builtin_amdgcn_s_setprio(0);
            float p[16], cap_slope[16];
            raw(s, p);
            scores<E, MODE, 16>(a.sc, p, p, MODE & kCap ? cap_slope : nullptr);
            if constexpr (MODE & kBias) bias16(p, slope, (float)(r0 + 4 * h + a.off - key) + 32.f * u);
            if (part) {
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const i32x4 lo = *reinterpret_cast<const i32x4*>(rows + 8 * kPart + 32 * i4);
                    const i32x4 keys = *reinterpret_cast<const i32x4*>(rows + 12 * kPart + 32 * i4);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        p[4 * i4 + e] = (uint32_t)(key - lo[e]) < (uint32_t)keys[e] ? p[4 * i4 + e] : -INFINITY;
                }
            }
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const f32x4 lse2 = *reinterpret_cast<const f32x4*>(rows + 32 * i4);
                const f32x4 delta = *reinterpret_cast<const f32x4*>(rows + 4 * kPart + 32 * i4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * i4 + e;
                    p[i] = exp_score<MODE>(a.sc, p[i], lse2[e]);
                    dp[i] = p[i] * (dp[i] - delta[e]);
                    if constexpr (MODE & kCap) dp[i] *= cap_slope[i];
                }
            }
            float dz[16];
            raw(dp, dz);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<E> fp = to_frag<E>(p + 8 * x), fz = to_frag<E>(dz + 8 * x);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    mma32x32(dv[d], at.across(d, TB + 16 * x * T::RB), fp);
                    mma32x32(dk[d], at.across(d, 16 * x * T::RB), fz);
                }
            }
            if constexpr (ES == 2) read_ahead<4 * ND, 1, 2, 3>();
            __builtin_amdgcn_s_setprio(0);
        }
        if constexpr (S::STAGES == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) request(0);
        }
    }

    // the keys whose dk (0) or dv (1) has to be formed again
    uint32_t again[2] = {rows_of(key < a.Tk && !(zero_of(dk, 0.f) == 0.f)), rows_of(key < a.Tk && !(zero_of(dv, 0.f) == 0.f))};
    // the outputs, or this part's sums of float32
    using Out = std::conditional_t<PARTS, float, E>;
    const HeadRows to_dk = PARTS ? part_rows(a, part_of, 0) : a.dk, to_dv = PARTS ? part_rows(a, part_of, 1) : a.dv;
    if constexpr (!SPLIT) {
        const bool store_k = key < a.Tk && !((again[0] >> (lane & 31)) & 1u), store_v = key < a.Tk && !((again[1] >> (lane & 31)) & 1u);
        char* okp = to_dk.ptr + kv * to_dk.head + (int64_t)key * to_dk.row;
        char* ovp = to_dv.ptr + kv * to_dv.head + (int64_t)key * to_dv.row;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 32 * d + 8 * i + 4 * h, at = e * (int)sizeof(Out);
                if (store_k && e < a.D)
                    store4<Out>(okp + at, dk[d][4 * i] * a.scale, dk[d][4 * i + 1] * a.scale, dk[d][4 * i + 2] * a.scale,
                                dk[d][4 * i + 3] * a.scale);
                if (store_v && e < a.D)
                    store4<Out>(ovp + at, dv[d][4 * i], dv[d][4 * i + 1], dv[d][4 * i + 2], dv[d][4 * i + 3]);
            }
    } else {
        const Meeting<DP> meet(lds, wave, lane);
        static_assert(Meeting<DP>::BYTES + 32 <= S::LDS, "the sums fit the stages");
        uint32_t* flags = reinterpret_cast<uint32_t*>(lds + Meeting<DP>::BYTES);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const HeadRows& to = which ? to_dv : to_dk;
            const float scale = which ? 1.f : a.scale;
            __syncthreads();   // the stages, and then dk's sums, have been read
            meet.put(which ? dv : dk, 0.f, 0.f);
            if (lane == 0) flags[4 * which + wave] = again[which];
            __syncthreads();
            const uint32_t* f = flags + 4 * which;
            again[which] = f[0] | f[1] | f[2] | f[3];
            for (int e = threadIdx.x; e < 32 * (DP / 4); e += 256) {
                const int r = e / (DP / 4), d = e % (DP / 4) * 4;
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < 4; ++x) v += *reinterpret_cast<const f32x4*>(meet.get(x, r) + d);
                if (d < a.D && key0 + r < a.Tk && !((again[which] >> r) & 1u))
                    store4<Out>(to.ptr + kv * to.head + (int64_t)(key0 + r) * to.row + d * (int)sizeof(Out), v[0] * scale,
                                v[1] * scale, v[2] * scale, v[3] * scale);
            }
            again[which] &= 0x11111111u << wave;   // a quarter of the keys for each wave
        }
    }
    for (uint32_t left = again[0] | again[1]; left; left &= left - 1) {
        const int r = __builtin_ctz(left), j = wkey + r;
        const bool need_k = (again[0] >> r) & 1u, need_v = (again[1] >> r) & 1u;
        const Pair kj = load_pair<E>(a.k, kv, j, a.D, lane), vj = load_pair<E>(a.v, kv, j, a.D, lane);
        Pair sk, sv;
        const auto done = [&] { return (!need_k || all_nan(sk, a.D, lane)) && (!need_v || all_nan(sv, a.D, lane)); };
        const int tiles = (a.Tq + kPart - 1) / kPart;
        for (int head = kv * a.share + heads.at; head < kv * a.share + heads.end && !done(); ++head) {
            const float slope = MODE & kBias ? a.slopes[head] * kLog2e / a.sc.unit : 0.f;
            // of 64 tiles those, and of their 64 rows those that see the key: one a lane
            for (int t0 = 0; t0 < tiles && !done(); t0 += 64) {
                int4 span = {0, 0, 0, 0};
                if (t0 + lane < tiles) span = a.span[t0 + lane];
                for (uint64_t of = __ballot(span.x <= j && j < span.y); of && !done(); of &= of - 1) {
                    const int i0 = (t0 + __builtin_ctzll(of)) * kPart;
                    const bool sees = i0 + lane < a.Tq && (uint32_t)(j - a.row_lo[i0 + lane]) < (uint32_t)a.row_keys[i0 + lane];
                    for (uint64_t rows = __ballot(sees); rows && !done(); rows &= rows - 1) {
                        const int i = i0 + __builtin_ctzll(rows);
                        const int64_t at = (int64_t)head * a.Tpad + i;
                        float cap_slope;
                        const Pair q = load_pair<E>(a.q, head, i, a.D, lane), g = load_pair<E>(a.g, head, i, a.D, lane);
                        const float p = one_probability<E, MODE>(a, q, kj, slope, i, j, a.lse2[at], cap_slope);
                        const float dz = p * (wave_dot(g, vj) - a.delta[at]) * cap_slope * a.scale;
                        sv.x += p * g.x;
                        sv.y += p * g.y;
                        sk.x += dz * q.x;
                        sk.y += dz * q.y;
                    }
                }
            }
        }
        if (need_k) store_pair<Out>(to_dk, kv, j, a.D, lane, sk.x, sk.y);
        if (need_v) store_pair<Out>(to_dv, kv, j, a.D, lane, sv.x, sv.y);
    }
}

// dk and dv from the parts' sums, in their order: four elements a thread.
template <typename E>
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(AttnArgs a) {
    const int quads = a.D / 4, which = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)(a.heads / a.share) * a.Tk;
    if (i >= rows * quads) return;
    const float* p = a.part + which * rows * a.D + 4 * i;
    f32x4 sum = *reinterpret_cast<const f32x4*>(p);
    for (int n = 1; n < a.parts; ++n) sum += *reinterpret_cast<const f32x4*>(p + 2 * n * rows * a.D);
    const int64_t row = i / quads;
    const HeadRows& to = which ? a.dv : a.dk;
    store4<E>(to.ptr + row / a.Tk * to.head + row % a.Tk * to.row + i % quads * 4 * (int)sizeof(E), sum[0], sum[1], sum[2], sum[3]);
}

}  // namespace noble
