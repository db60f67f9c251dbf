// Norm of query and key heads and rotation by position, forward, backward, and on the way into a paged cache.
//
// One pass over the Q/K/V layer's rows.  Sixteen lanes (eight for D <= 64) hold a head, eight elements each: the
// head's mean square is four (three) lane exchanges away, a half-layout pair's other element one.  A lane group stays
// at one token and steps over its heads, so the token's cosines and sines are read once.  Bound by memory: 32768 tokens of
// 16 + 16 heads of 128 in bf16, forward 95 us (5.6 TB/s), backward 167 to 182 us (4.4 to 4.8 TB/s) and 5 us for the weights' sums;
// 3108 prompt tokens of 16 + 4 heads into the cache 11 us, 16 single tokens 4 us, which is a launch.
#pragma once

#include "noble_attn_common.hpp"

namespace noble {

struct RopeArgs {
    const char* x;
    int64_t x_row;                 // bytes
    const float* wq;
    const float* wk;
    const float* cos;
    const float* sin;
    const int* positions;
    char* q;                       // dense [T, heads, D] (fwd, append), or dq
    char* k;                       // dense [T, kv_heads, D] (fwd), or dk
    const int64_t* slots;          // append
    char* cache;
    char* dx;                      // bwd
    float* partial;                // bwd: [workgroups][2][128] float32
    int64_t table_rows, slot_count;
    int T, heads, kv_heads, D, rot;
    int page, page_shift;
    int split;                     // lane groups that share a token's heads
    float eps;
};

template <typename E>
__device__ __forceinline__ void to_f32(const Frag<E>& f, float* x) {
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(f.v[j] << 16);
            x[2 * j + 1] = __uint_as_float(f.v[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(f.v[j >> 2][j & 3]);
    }
}
template <typename E>
__device__ __forceinline__ void store_frag(char* p, const Frag<E>& f) {
    if constexpr (sizeof(E) == 2) {
        *reinterpret_cast<u32x4*>(p) = f.v;
    } else {
        *reinterpret_cast<u32x4*>(p) = f.v[0];
        *reinterpret_cast<u32x4*>(p + 16) = f.v[1];
    }
}

// This lane's eight cosines and sines: of elements 8 c .. 8 c + 7 (half layout: pair index 8 (c mod rot / 16) ..,
// interleaved: four pairs, 4 c ..).  Elements past the rotated ones get 1 and 0, a position outside the table NaN.
template <bool INTER>
struct Angles {
    float c[INTER ? 4 : 8], s[INTER ? 4 : 8];
    __device__ __forceinline__ Angles(const RopeArgs& a, int64_t pos, int chunk) {
        constexpr int N = INTER ? 4 : 8;
        const bool turned = 8 * chunk < a.rot, known = pos >= 0 && pos < a.table_rows;
        const int half = a.rot >> 4, first = INTER ? 4 * chunk : 8 * (chunk < half ? chunk : chunk - half);
        const float fill = turned ? NAN : 1.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            c[i] = fill;
            s[i] = turned ? NAN : 0.f;
        }
        if (turned && known) {
            const f32x4* pc = reinterpret_cast<const f32x4*>(a.cos + pos * (a.rot >> 1) + first);
            const f32x4* ps = reinterpret_cast<const f32x4*>(a.sin + pos * (a.rot >> 1) + first);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const f32x4 vc = pc[i], vs = ps[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    c[4 * i + e] = vc[e];
                    s[4 * i + e] = vs[e];
                }
            }
        }
    }
    // The elements turned forward (dir 1) or back (dir -1), in place.  Those past the rotated ones are kept, not turned by
    // nothing: an infinite one would become NaN, or make its neighbour that.
    __device__ __forceinline__ void turn(float* x, int rot, int chunk, float dir) const {
        const bool turned = 8 * chunk < rot;
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = x[2 * i], q = x[2 * i + 1], t = dir * s[i];
                x[2 * i] = turned ? p * c[i] - q * t : p;
                x[2 * i + 1] = turned ? q * c[i] + p * t : q;
            }
        } else {
            // the pair's other element: rot / 16 lanes on for the first half, back for the second
            const int half = rot >> 4;
            const bool first = chunk < half;
            const int lane = threadIdx.x & 63, from = chunk < 2 * half ? (first ? lane + half : lane - half) : lane;
            const float sign = first ? -dir : dir;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float other = __shfl(x[i], from);
                x[i] = turned ? x[i] * c[i] + other * (sign * s[i]) : x[i];
            }
        }
    }
};

template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int o = G / 2; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Eight weights of this lane's elements (ones where there are none).
__device__ __forceinline__ void load_weight(const float* w, int chunk, bool in, float* out) {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = w && in ? w[8 * chunk + i] : 1.f;
}

// Lane groups of a workgroup of 256 are (token, part of its heads); the loop bounds of the groups of a wave differ
// only in the tail, where a group repeats its last head and stores nothing: the lane exchanges need every lane.
template <typename E, int G, bool INTER, bool APPEND>
__global__ __launch_bounds__(256) void qk_rope_kernel(RopeArgs a) {
    constexpr int ES = sizeof(E), PER = 256 / G;
    const int c = threadIdx.x % G;
    const int64_t item = (int64_t)blockIdx.x * PER + threadIdx.x / G;
    const int64_t tok = item / a.split;
    const int part = (int)(item - tok * a.split);
    const bool live = tok < a.T, in = 8 * c < a.D;
    const int64_t t = live ? tok : a.T - 1;
    const int total = a.heads + a.kv_heads;
    const Angles<INTER> ang(a, a.positions ? a.positions[t] : t, c);
    float wq[8], wk[8];
    load_weight(a.wq, c, in, wq);
    load_weight(a.wk, c, in, wk);
    const bool norm = a.wq != nullptr;
    const int64_t db = (int64_t)a.D * ES;
    const char* xr = a.x + t * a.x_row + (int64_t)8 * c * ES;
    const int64_t slot = APPEND ? a.slots[t] : 0;
    const bool keep = !APPEND || (slot >= 0 && slot < a.slot_count);
    char* row = nullptr;
    if constexpr (APPEND)   // keys of the slot's page; values a.kv_heads page rows further
        row = a.cache + ((slot >> a.page_shift) * 2 * a.kv_heads * a.page + (slot & (a.page - 1))) * db;
    const int first = APPEND && !a.q ? a.heads : 0;   // no queries wanted
    const int steps = (total - first + a.split - 1) / a.split;
    // the next head is on its way while this one is worked on
    const auto head_at = [&](int n) { return min(first + part + n * a.split, total - 1); };
    Frag<E> next{};
    if (steps > 0) next = global_frag<E>(xr + head_at(0) * db, in);
    for (int n = 0; n < steps; ++n) {
        const bool have = first + part + n * a.split < total;
        const int h = head_at(n);
        const bool isq = h < a.heads;
        float x[8];
        to_f32(next, x);
        if (n + 1 < steps) next = global_frag<E>(xr + head_at(n + 1) * db, in);
        if (norm) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
            const float r = rsqrtf(group_sum<G>(sum) / (float)a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (isq ? wq[i] : wk[i]);
        }
        if (a.rot) ang.turn(x, a.rot, c, 1.f);
        if (!live || !have || !in) continue;
        const int64_t off = (int64_t)8 * c * ES;
        if (isq) store_frag<E>(a.q + (t * a.heads + h) * db + off, to_frag<E>(x));
        else if constexpr (!APPEND) store_frag<E>(a.k + (t * a.kv_heads + h - a.heads) * db + off, to_frag<E>(x));
        else if (keep) store_frag<E>(row + (int64_t)(h - a.heads) * a.page * db + off, to_frag<E>(x));
    }
    if constexpr (APPEND) {
        if (!live || !in || !keep) return;
        for (int h = part; h < a.kv_heads; h += a.split)
            store_frag<E>(row + (int64_t)(a.kv_heads + h) * a.page * db + (int64_t)8 * c * ES,
                          global_frag<E>(xr + (total + h) * db, true));
    }
}

// Backward.  With n = x r and du the gradient turned back: dx = r (w du - n mean(n w du)), dw = sum n du.  Each lane
// sums its eight elements' dw over the tokens of its group, the workgroup's groups meet in LDS and the workgroups'
// sums in rope_dw_kernel, each in a fixed order.
template <typename E, int G, bool INTER>
__global__ __launch_bounds__(256) void qk_rope_bwd_kernel(RopeArgs a) {
    constexpr int ES = sizeof(E), PER = 256 / G;
    __shared__ float part_q[PER][8 * G + 4], part_k[PER][8 * G + 4];
    const int c = threadIdx.x % G, grp = threadIdx.x / G;
    const bool in = 8 * c < a.D, norm = a.wq != nullptr;
    const int total = a.heads + a.kv_heads;
    float wq[8], wk[8], sq[8], sk[8];
    load_weight(a.wq, c, in, wq);
    load_weight(a.wk, c, in, wk);
#pragma unroll
    for (int i = 0; i < 8; ++i) sq[i] = sk[i] = 0.f;
    const int64_t db = (int64_t)a.D * ES, off = (int64_t)8 * c * ES;
    const int64_t items = (int64_t)a.T * a.split, stride = (int64_t)gridDim.x * PER;
    // every group of the workgroup makes the same number of passes: the lane exchanges need every lane
    for (int64_t base = (int64_t)blockIdx.x * PER; base < items; base += stride) {
        const int64_t item = base + grp, tok = item / a.split;
        const bool live = item < items;
        const int64_t t = live ? tok : a.T - 1;
        const int part = (int)(item - tok * a.split);
        const Angles<INTER> ang(a, a.positions ? a.positions[t] : t, c);
        const int steps = (total + a.split - 1) / a.split;
        const auto head_at = [&](int n) { return min(part + n * a.split, total - 1); };
        const auto grad = [&](int n) {
            const int h = head_at(n);
            const char* gp = h < a.heads ? a.q + (t * a.heads + h) * db : a.k + (t * a.kv_heads + h - a.heads) * db;
            return global_frag<E>(gp + off, in);
        };
        const auto value = [&](int n) { return global_frag<E>(a.x + t * a.x_row + head_at(n) * db + off, in && norm); };
        Frag<E> next_g = grad(0), next_x = value(0);
        for (int n = 0; n < steps; ++n) {
            const bool have = live && part + n * a.split < total;
            const int h = head_at(n);
            const bool isq = h < a.heads;
            float x[8], du[8];
            to_f32(next_g, du);
            to_f32(next_x, x);
            if (n + 1 < steps) {
                next_g = grad(n + 1);
                next_x = value(n + 1);
            }
            if (a.rot) ang.turn(du, a.rot, c, -1.f);
            if (norm) {
                float sum = 0.f, dot = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
                const float r = rsqrtf(group_sum<G>(sum) / (float)a.D + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= r;
                    const float w = isq ? wq[i] : wk[i], nd = x[i] * du[i];
                    if (have) (isq ? sq[i] : sk[i]) += nd;
                    du[i] *= w;
                    dot += w * nd;
                }
                const float mean = group_sum<G>(dot) / (float)a.D;
#pragma unroll
                for (int i = 0; i < 8; ++i) du[i] = r * (du[i] - x[i] * mean);
            }
            if (have && in) store_frag<E>(a.dx + t * a.x_row + h * db + off, to_frag<E>(du));
        }
    }
    if (!norm) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        part_q[grp][8 * c + i] = sq[i];
        part_k[grp][8 * c + i] = sk[i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * 8 * G; e += 256) {
        const bool isq = e < 8 * G;
        const int d = isq ? e : e - 8 * G;
        float s = 0.f;
        for (int g = 0; g < PER; ++g) s += isq ? part_q[g][d] : part_k[g][d];
        a.partial[((int64_t)blockIdx.x * 2 + (isq ? 0 : 1)) * 128 + d] = s;
    }
}

// The workgroups' sums of the weights' gradients, 64 lanes a column, in a fixed order.
struct RopeDwArgs {
    const float* partial;
    float* dwq;
    float* dwk;
    int parts, D;
};
static __global__ __launch_bounds__(1024) void rope_dw_kernel(RopeDwArgs a) {
    constexpr int ROWS = 64;
    __shared__ float part[ROWS][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, col = blockIdx.x * 16 + x, which = blockIdx.y;
    float s = 0.f;
    // eight loads in flight: one by one, 2048 partial sums took 50 us, a quarter of the backward
#pragma unroll 8
    for (int p = y; p < a.parts; p += ROWS) s += a.partial[((int64_t)p * 2 + which) * 128 + col];
    part[y][x] = s;
    __syncthreads();
    if (y == 0 && col < a.D) {
        float t = 0.f;
        for (int i = 0; i < ROWS; ++i) t += part[i][x];
        (which ? a.dwk : a.dwq)[col] = t;
    }
}

// cos and sin of position x frequency in double, rounded once.
struct RopeTableArgs {
    float* cos;
    float* sin;
    int64_t n;
    int pairs, kind, rot;
    double base, factor, ramp_lo, ramp_hi, gain;
};
static __global__ __launch_bounds__(256) void rope_table_kernel(RopeTableArgs a) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= a.n) return;
    const int64_t p = e / a.pairs;
    const int i = (int)(e - p * a.pairs);
    double f = pow(a.base, -2.0 * i / a.rot);
    if (a.kind == 1) f /= a.factor;
    if (a.kind == 3) {
        const double w = fmin(fmax((i - a.ramp_lo) / fmax(a.ramp_hi - a.ramp_lo, 1e-3), 0.0), 1.0);
        f = f * (1.0 - w) + f / a.factor * w;
    }
    double s, c;
    sincos((double)p * f, &s, &c);
    a.cos[e] = (float)(c * a.gain);
    a.sin[e] = (float)(s * a.gain);
}

// Key intervals of packed documents: each row finds its document by bisection.
struct MaskArgs {
    const int* starts;
    const int* prefix;
    int* lo;
    int* hi;
    int* positions;
    int T, documents, causal, window;
};
static __global__ __launch_bounds__(256) void mask_rows_kernel(MaskArgs a) {
    const int64_t i64 = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i64 >= a.T) return;
    const int i = (int)i64;
    int below = -1, above = a.documents;   // the last n with starts[n] <= i
    while (above - below > 1) {
        const int mid = below + (above - below) / 2;
        if (a.starts[mid] <= i) below = mid;
        else above = mid;
    }
    int lo = 0, hi = 0, at = 0;
    if (below >= 0 && i < a.starts[below + 1]) {
        const int first = a.starts[below], end = min(a.starts[below + 1], a.T);
        lo = max(first, 0);
        hi = a.causal ? i + 1 : end;
        if (a.causal && a.prefix) hi = max(hi, (int)min((int64_t)end, (int64_t)first + a.prefix[below]));
        if (a.window > 0) lo = max(lo, hi - a.window);
        at = i - first;
    }
    a.lo[i] = lo;
    a.hi[i] = hi;
    if (a.positions) a.positions[i] = at;
}

}  // namespace noble
