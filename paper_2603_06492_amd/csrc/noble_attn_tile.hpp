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
    float* lse2;                 // backward: lse log2 e, +inf for a row that sees nothing, and delta: [heads, Tpad]
    float* delta;
    int* row_lo;                 // backward: the rows' intervals, and of each 64 rows the least and largest bounds
    int* row_hi;
    int4* span;
    int Tq, Tk, heads, share, D;   // share: query heads of a key head
    int Tpad;                      // Tq rounded up to a tile: rows past the end have probability zero in lse2
    int causal, off;               // key index of row 0
    float scale;
    ScoreArgs sc;
};

constexpr int kOwn = 128;   // rows of a workgroup: 32 for each of four waves
constexpr int kPart = 64;   // partner rows of a tile

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

// Workgroup -> (head, own tile): one key head's workgroups in a row, the last tiles (the longest ones under a causal
// mask) first, the query heads that share the key head side by side.
struct OwnTile {
    int head, tile;
    __device__ __forceinline__ OwnTile(int tiles, int heads, int share) {
        const int w = xcd_order(blockIdx.x, gridDim.x);
        const int per = tiles * share, kv = w / per, r = w - kv * per;
        head = kv * share + r % share;
        tile = tiles - 1 - r / share;
    }
};

// The own rows' intervals as the kernels that own queries use them: of this lane's row, of the wave's rows and of the
// workgroup's.
struct OwnRows {
    int lo, hi;             // this lane's row
    int wave_lo, wave_hi;   // the keys that any row of the wave sees
    int full_lo, full_hi;   // the keys that every row of the wave sees
    int all_lo, all_hi;     // the keys that any row of the workgroup sees
    __device__ __forceinline__ OwnRows(const AttnArgs& a, int row0, int wave, int lane) {
        int least = INT32_MAX, most = 0;
#pragma unroll
        for (int k = 0; k < kOwn / 64; ++k) {
            const int i = row0 + 64 * k + lane;
            const int2 r = i < a.Tq ? row_interval(a, i) : int2{0, 0};
            if (r.x < r.y) {
                least = min(least, r.x);
                most = max(most, r.y);
            }
        }
        all_hi = wave_max(most);
        all_lo = min(wave_min(least), all_hi);
        const int i = row0 + 32 * wave + (lane & 31);
        const bool in = i < a.Tq;
        const int2 r = in ? row_interval(a, i) : int2{0, 0};
        lo = r.x;
        hi = r.y;
        wave_hi = wave_max(hi);
        wave_lo = min(wave_min(lo < hi ? lo : INT32_MAX), wave_hi);
        // rows past the end do not count: their queries are zeros and nothing of them is stored
        full_lo = wave_max(in ? lo : 0);
        full_hi = wave_min(in ? hi : INT32_MAX);
    }
};

// What bounds it: the matrix cores and the exponentials, about evenly, at long rows.
template <typename E, int DP, int MODE>
__global__ __launch_bounds__(256, sizeof(E) == 2 ? 2 : 1) void attn_fwd_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    constexpr int ES = T::ES, TB = T::bytes(kPart), NS = DP / 16, ND = DP / 32;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const OwnTile w((a.Tq + kOwn - 1) / kOwn, a.heads, a.share);
    const int row0 = w.tile * kOwn, row = row0 + 32 * wave + (lane & 31), kv = w.head / a.share, db = a.D * ES;
    const OwnRows own(a, row0, wave, lane);

    const auto request = [&](int t) {
        char* dst = lds + (t & 1) * 2 * TB;
        const int k0 = own.all_lo + t * kPart;
        T::template request<4, kPart>(rows_desc(a.k, kv, k0, own.all_hi, db), dst, (int)a.k.row, db, wave, lane);
        T::template request<4, kPart>(rows_desc(a.v, kv, k0, own.all_hi, db), dst + TB, (int)a.v.row, db, wave, lane);
    };
    const int tiles = (own.all_hi - own.all_lo + kPart - 1) / kPart;
    if (tiles > 0) request(0);

    Frag<E> q[NS];
    const char* qp = a.q.ptr + w.head * a.q.head + (int64_t)row * a.q.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = global_frag<E>(qp + 16 * s * ES, row < a.Tq && 16 * s + 8 * h < a.D);
    const float slope2 = MODE & kBias ? a.slopes[w.head] * kLog2e : 0.f;
    const int at = row + a.off;

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    for (int t = 0; t < tiles; ++t) {
        arrive_all();
        if (t + 1 < tiles) request(t + 1);
        const int k0 = own.all_lo + t * kPart;
        if (k0 >= own.wave_hi || k0 + kPart <= own.wave_lo) continue;
        const char* kt = lds + (t & 1) * 2 * TB;
        const char* vt = kt + TB;
        float z[32];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(s, T::along(kt, 32 * u + (lane & 31), 2 * x + h), q[x]);
            raw(s, z + 16 * u);
            scores<E, MODE, 16>(a.sc, z + 16 * u, z + 16 * u, nullptr);
            if constexpr (MODE & kBias) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    z[16 * u + i] -= slope2 * (float)abs(at - (k0 + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3)));
            }
        }
        if (k0 < own.full_lo || k0 + kPart > own.full_hi) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int j = k0 + 8 * (i >> 2) + 4 * h + (i & 3);
                z[i] = j >= own.lo && j < own.hi ? z[i] : -INFINITY;
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, z[i]);
        top = max_halves(top);
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
        for (int i = 0; i < 32; ++i) {
            z[i] = __builtin_amdgcn_exp2f(z[i] - from);
            l += z[i];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const Frag<E> p = to_frag<E>(z + 8 * x);
#pragma unroll
            for (int d = 0; d < ND; ++d) mma32x32(acc[d], T::across(vt, 16 * x, d, lane), p);
        }
    }

    l = sum_halves(l);
    if (row >= a.Tq) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
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
    if (h == 0) a.lse[(int64_t)w.head * a.Tq + row] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

// Before the backward's products: delta = do.o and lse in units of log2 for every row and head, the rows' intervals and
// what 64 of them span.  Sixteen lanes a row; bound by reading do and o.
template <typename E>
__global__ __launch_bounds__(256) void attn_bwd_prep_kernel(AttnArgs a) {
    constexpr int ES = sizeof(E);
    const int tile = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = lane & 15;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = 64 * tile + 16 * k + 4 * wave + (lane >> 4);
        const bool ok = row < a.Tq && 8 * c < a.D;
        const Frag<E> o = global_frag<E>(a.o.ptr + head * a.o.head + row * a.o.row + 8 * c * ES, ok);
        const Frag<E> g = global_frag<E>(a.g.ptr + head * a.g.head + row * a.g.row + 8 * c * ES, ok);
        float sum = 0.f;
        if constexpr (ES == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum += bf2f(o.v[j] & 0xffffu) * bf2f(g.v[j] & 0xffffu);
                sum += __uint_as_float(o.v[j] & 0xffff0000u) * __uint_as_float(g.v[j] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += __uint_as_float(o.v[j >> 2][j & 3]) * __uint_as_float(g.v[j >> 2][j & 3]);
        }
#pragma unroll
        for (int x = 8; x; x >>= 1) sum += __shfl_xor(sum, x);
        if (c == 0) {
            const float lse = row < a.Tq ? a.lse[(int64_t)head * a.Tq + row] : -INFINITY;
            const int64_t at = (int64_t)head * a.Tpad + row;
            a.lse2[at] = lse == -INFINITY ? INFINITY : lse * kLog2e;
            a.delta[at] = sum;
        }
    }
    if (head == 0 && wave == 0) {
        const int i = 64 * tile + lane;
        const bool in = i < a.Tq;
        const int2 r = in ? row_interval(a, i) : int2{0, 0};
        if (in) {
            a.row_lo[i] = r.x;
            a.row_hi[i] = r.y;
        }
        const int most = wave_max(r.y), least = min(wave_min(r.x < r.y ? r.x : INT32_MAX), most);
        const int from = wave_max(in ? r.x : 0), to = wave_min(in ? r.y : INT32_MAX);
        if (lane == 0) a.span[tile] = int4{least, most, from, to};
    }
}

template <typename E, int DP, int MODE>
__global__ __launch_bounds__(256, sizeof(E) == 2 ? 2 : 1) void attn_dq_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    constexpr int ES = T::ES, TB = T::bytes(kPart), NS = DP / 16, ND = DP / 32;
    __shared__ __attribute__((aligned(1024))) char lds[4 * TB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const OwnTile w((a.Tq + kOwn - 1) / kOwn, a.heads, a.share);
    const int row0 = w.tile * kOwn, row = row0 + 32 * wave + (lane & 31), kv = w.head / a.share, db = a.D * ES;
    const OwnRows own(a, row0, wave, lane);

    const auto request = [&](int t) {
        char* dst = lds + (t & 1) * 2 * TB;
        const int k0 = own.all_lo + t * kPart;
        T::template request<4, kPart>(rows_desc(a.k, kv, k0, own.all_hi, db), dst, (int)a.k.row, db, wave, lane);
        T::template request<4, kPart>(rows_desc(a.v, kv, k0, own.all_hi, db), dst + TB, (int)a.v.row, db, wave, lane);
    };
    const int tiles = (own.all_hi - own.all_lo + kPart - 1) / kPart;
    if (tiles > 0) request(0);

    Frag<E> q[NS], g[NS];
    const char* qp = a.q.ptr + w.head * a.q.head + (int64_t)row * a.q.row + 8 * h * ES;
    const char* gp = a.g.ptr + w.head * a.g.head + (int64_t)row * a.g.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const bool ok = row < a.Tq && 16 * s + 8 * h < a.D;
        q[s] = global_frag<E>(qp + 16 * s * ES, ok);
        g[s] = global_frag<E>(gp + 16 * s * ES, ok);
    }
    const float slope2 = MODE & kBias ? a.slopes[w.head] * kLog2e : 0.f;
    const int at = row + a.off;
    const int64_t rh = (int64_t)w.head * a.Tpad + row;
    const float lse2 = row < a.Tq ? a.lse2[rh] : INFINITY, delta = row < a.Tq ? a.delta[rh] : 0.f;

    f32x16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

    for (int t = 0; t < tiles; ++t) {
        arrive_all();
        if (t + 1 < tiles) request(t + 1);
        const int k0 = own.all_lo + t * kPart;
        if (k0 >= own.wave_hi || k0 + kPart <= own.wave_lo) continue;
        const char* kt = lds + (t & 1) * 2 * TB;
        const char* vt = kt + TB;
        const bool part = k0 < own.full_lo || k0 + kPart > own.full_hi;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(s, T::along(kt, 32 * u + (lane & 31), 2 * x + h), q[x]);
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(dp, T::along(vt, 32 * u + (lane & 31), 2 * x + h), g[x]);
            float z[16], dz[16], slope[16];
            raw(s, z);
            scores<E, MODE, 16>(a.sc, z, z, MODE & kCap ? slope : nullptr);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (MODE & kBias)
                    z[i] -= slope2 * (float)abs(at - (k0 + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3)));
                dz[i] = __builtin_amdgcn_exp2f(z[i] - lse2) * (dp[i] - delta);
                if constexpr (MODE & kCap) dz[i] *= slope[i];
            }
            if (part) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = k0 + 32 * u + 8 * (i >> 2) + 4 * h + (i & 3);
                    dz[i] = j >= own.lo && j < own.hi ? dz[i] : 0.f;
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<E> f = to_frag<E>(dz + 8 * x);
#pragma unroll
                for (int d = 0; d < ND; ++d) mma32x32(acc[d], T::across(kt, 32 * u + 16 * x, d, lane), f);
            }
        }
    }

    if (row >= a.Tq) return;
    char* op = a.dq.ptr + w.head * a.dq.head + (int64_t)row * a.dq.row;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = 32 * d + 8 * i + 4 * h;
            if (e < a.D)
                store4<E>(op + e * ES, acc[d][4 * i] * a.scale, acc[d][4 * i + 1] * a.scale, acc[d][4 * i + 2] * a.scale,
                          acc[d][4 * i + 3] * a.scale);
        }
}

// The 64-row tiles of queries that see a workgroup's keys, in order, over the query heads that share the key head.
// 64 tiles are looked at together, one a lane.
struct Partners {
    int share, tiles;
    const int4* span;
    int k0, k1, w0, w1;      // the workgroup's keys, and the wave's
    int head = 0, base = -64, lane;
    uint64_t any = 0, mine = 0, full = 0;
    __device__ __forceinline__ Partners(const AttnArgs& a, int key0, int wave, int lane_)
        : share(a.share), tiles((a.Tq + kPart - 1) / kPart), span(a.span), k0(key0), k1(min(key0 + kOwn, a.Tk)),
          w0(key0 + 32 * wave), w1(min(key0 + 32 * wave + 32, a.Tk)), lane(lane_) {}
    // The next (head, tile), and whether the wave's keys are seen by any or by all of its rows; false at the end.
    __device__ __forceinline__ bool next(int& hd, int& tile, bool& seen, bool& whole) {
        while (!any) {
            base += 64;
            if (base >= tiles) {
                base = 0;
                if (++head >= share) return false;
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

template <typename E, int DP, int MODE>
__global__ __launch_bounds__(256, sizeof(E) == 2 ? 2 : 1) void attn_dkv_kernel(AttnArgs a) {
    using T = Tile<E, DP>;
    constexpr int ES = T::ES, TB = T::bytes(kPart), NS = DP / 16, ND = DP / 32, STAGE = 2 * TB + 4 * kPart * 4;
    __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int tiles = (a.Tk + kOwn - 1) / kOwn, wg = xcd_order(blockIdx.x, gridDim.x);
    const int kv = wg / tiles, key0 = (wg - kv * tiles) * kOwn, key = key0 + 32 * wave + (lane & 31), db = a.D * ES;

    Partners it(a, key0, wave, lane);
    const auto request = [&](int stage, int gi, int tile) {
        char* dst = lds + stage * STAGE;
        const int head = kv * a.share + gi, r0 = tile * kPart;
        T::template request<4, kPart>(rows_desc(a.q, head, r0, a.Tq, db), dst, (int)a.q.row, db, wave, lane);
        T::template request<4, kPart>(rows_desc(a.g, head, r0, a.Tq, db), dst + TB, (int)a.g.row, db, wave, lane);
        const int64_t rh = (int64_t)head * a.Tpad + r0;
        const char* src = reinterpret_cast<const char*>(wave == 0 ? a.lse2 + rh : wave == 1 ? a.delta + rh :
                                                        reinterpret_cast<const float*>(wave == 2 ? a.row_lo + r0 : a.row_hi + r0));
        dma4(wave_desc(src, (int64_t)(wave < 2 ? kPart : a.Tq - r0) * 4), dst + 2 * TB + wave * kPart * 4, lane);
    };
    int gi = 0, tile = 0;
    bool seen = false, whole = false, more = it.next(gi, tile, seen, whole);
    if (more) request(0, gi, tile);

    Frag<E> k[NS], v[NS];
    const char* kp = a.k.ptr + kv * a.k.head + (int64_t)key * a.k.row + 8 * h * ES;
    const char* vp = a.v.ptr + kv * a.v.head + (int64_t)key * a.v.row + 8 * h * ES;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const bool ok = key < a.Tk && 16 * s + 8 * h < a.D;
        k[s] = global_frag<E>(kp + 16 * s * ES, ok);
        v[s] = global_frag<E>(vp + 16 * s * ES, ok);
    }

    f32x16 dk[ND], dv[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.f;

    for (int n = 0; more; ++n) {
        const int r0 = tile * kPart, head = kv * a.share + gi;
        const bool do_it = seen, part = !whole;
        arrive_all();
        more = it.next(gi, tile, seen, whole);
        if (more) request((n + 1) & 1, gi, tile);
        if (!do_it) continue;
        const char* qt = lds + (n & 1) * STAGE;
        const char* gt = qt + TB;
        const char* rows = gt + TB;
        const float slope2 = MODE & kBias ? a.slopes[head] * kLog2e : 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(s, T::along(qt, 32 * u + (lane & 31), 2 * x + h), k[x]);
#pragma unroll
            for (int x = 0; x < NS; ++x) mma32x32(dp, T::along(gt, 32 * u + (lane & 31), 2 * x + h), v[x]);
            float p[16], dz[16], slope[16];
            raw(s, p);
            scores<E, MODE, 16>(a.sc, p, p, MODE & kCap ? slope : nullptr);
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const int r = 32 * u + 8 * i4 + 4 * h;   // four rows of the tile
                const f32x4 lse2 = *reinterpret_cast<const f32x4*>(rows + 4 * r);
                const f32x4 delta = *reinterpret_cast<const f32x4*>(rows + 4 * kPart + 4 * r);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * i4 + e;
                    if constexpr (MODE & kBias) p[i] -= slope2 * (float)abs(r0 + r + e + a.off - key);
                    p[i] = __builtin_amdgcn_exp2f(p[i] - lse2[e]);
                    dz[i] = p[i] * (dp[i] - delta[e]);
                    if constexpr (MODE & kCap) dz[i] *= slope[i];
                }
            }
            if (part) {
                typedef int i32x4_ __attribute__((ext_vector_type(4)));
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const int r = 32 * u + 8 * i4 + 4 * h;
                    const i32x4_ lo = *reinterpret_cast<const i32x4_*>(rows + 8 * kPart + 4 * r);
                    const i32x4_ hi = *reinterpret_cast<const i32x4_*>(rows + 12 * kPart + 4 * r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool ok = key >= lo[e] && key < hi[e];
                        p[4 * i4 + e] = ok ? p[4 * i4 + e] : 0.f;
                        dz[4 * i4 + e] = ok ? dz[4 * i4 + e] : 0.f;
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Frag<E> fp = to_frag<E>(p + 8 * x), fz = to_frag<E>(dz + 8 * x);
#pragma unroll
                for (int d = 0; d < ND; ++d) mma32x32(dv[d], T::across(gt, 32 * u + 16 * x, d, lane), fp);
#pragma unroll
                for (int d = 0; d < ND; ++d) mma32x32(dk[d], T::across(qt, 32 * u + 16 * x, d, lane), fz);
            }
        }
    }

    if (key >= a.Tk) return;
    char* okp = a.dk.ptr + kv * a.dk.head + (int64_t)key * a.dk.row;
    char* ovp = a.dv.ptr + kv * a.dv.head + (int64_t)key * a.dv.row;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = 32 * d + 8 * i + 4 * h;
            if (e < a.D) {
                store4<E>(okp + e * ES, dk[d][4 * i] * a.scale, dk[d][4 * i + 1] * a.scale, dk[d][4 * i + 2] * a.scale,
                          dk[d][4 * i + 3] * a.scale);
                store4<E>(ovp + e * ES, dv[d][4 * i], dv[d][4 * i + 1], dv[d][4 * i + 2], dv[d][4 * i + 3]);
            }
        }
}

}  // namespace noble
