// Host code that the attention side's entry points share: limits, argument checks, the kernels' forms by type and size.
#pragma once

#include <algorithm>
#include <cmath>

#include "noble_attn.h"
#include "noble_attn_common.hpp"
#include "noble_host.hpp"

namespace noble {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 4096;
constexpr int64_t kMaxAttnRows = (int64_t(1) << 30) - 4096;   // and offsets: the kernels' row and key numbers are 32 bits
constexpr int64_t kMaxRowStride = int64_t(1) << 22;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxGroups256 = (int64_t)UINT32_MAX / 256;   // workgroups of 256 that one dispatch holds
constexpr int kMaxHeads = 1024;

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline size_t elt(int dtype) { return dtype == NOBLE_BF16 ? 2 : 4; }
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A float32 or index array: aligned to its element, present unless it holds nothing.
inline noble_status need_array(const void* p, bool nonempty, size_t size) {
    if (!p) return nonempty ? NOBLE_ERR_NULL_ARG : NOBLE_OK;
    return aligned_to(p, size) ? NOBLE_OK : NOBLE_ERR_MISALIGNED;
}

inline bool head_dim_ok(int D) { return D >= 8 && D <= 128 && D % 8 == 0; }
inline bool dtype_ok(int t) { return t == NOBLE_BF16 || t == NOBLE_F32; }

// Calls fn.template operator()<E, DP>(): heads of up to 64 elements run on tiles of 64, others on tiles of 128.
template <typename Fn>
noble_status with_shape(int dtype, int D, Fn&& fn) {
    if (dtype == NOBLE_BF16) return D <= 64 ? fn.template operator()<uint16_t, 64>() : fn.template operator()<uint16_t, 128>();
    return D <= 64 ? fn.template operator()<float, 64>() : fn.template operator()<float, 128>();
}
// Calls fn.template operator()<MODE>() for the cap and the bias of a call.
template <typename Fn>
noble_status with_mode(bool cap, bool bias, Fn&& fn) {
    if (cap) return bias ? fn.template operator()<kCap | kBias>() : fn.template operator()<kCap>();
    return bias ? fn.template operator()<kBias>() : fn.template operator()<0>();
}

// Strides and pointer of one tensor; an output's elements are distinct.
inline noble_status check_heads(const noble_heads* t, int64_t rows, int heads, int D, bool output) {
    if (!t) return NOBLE_ERR_NULL_ARG;
    if (t->row < 0 || t->row % 8 || t->row > kMaxRowStride || t->head < 0 || t->head % 8 || t->head > kMaxStride)
        return NOBLE_ERR_BAD_SHAPE;
    if (output && rows > 0) {
        const bool rows_outer = (heads == 1 || t->head >= D) && (rows == 1 || t->row >= (heads - 1) * t->head + D);
        const bool heads_outer = (rows == 1 || t->row >= D) && (heads == 1 || t->head >= (rows - 1) * t->row + D);
        if (!rows_outer && !heads_outer) return NOBLE_ERR_BAD_SHAPE;
    }
    return need(t->data, rows > 0);
}

inline HeadRows head_rows(const noble_heads* t, int dtype) {
    const int64_t es = (int64_t)elt(dtype);
    return HeadRows{static_cast<char*>(t->data), t->row * es, t->head * es};
}

// Scores from raw products, in units of log2 (float32 from double; a cap of 0 is none).  Caps below 1e-18 and above 1e18 are
// taken as these: scores under the first are alike to a float32 exponential, and scores of up to 1e14 are within 3e-9 of
// themselves under the second.
inline ScoreArgs score_args(float scale, float softcap) {
    ScoreArgs k{};
    const double log2e = 1.4426950408889634, cap = softcap > 0.f ? std::clamp((double)softcap, 1e-18, 1e18) : 0.0;
    k.unit = cap > 0.0 ? 1.f : (float)(scale * log2e);
    if (cap > 0.0) {
        const double x = scale / cap;
        k.cap_in = (float)x;
        k.cap_e = (float)(2.0 * x * log2e);
        k.cap_out = (float)(cap * log2e);
        k.inv2 = (float)(1.0 / (cap * log2e * cap * log2e));
        // tanh(x) / x as a polynomial in x^2 on [0, 1/4].  From the first coefficient on that no normal float32 holds, the
        // scale being that far from the cap, the terms are left out, and the polynomial ends where they would be 3e-8.
        const double fit[5] = {1.0, -0.3333307206630707, 0.13324828445911407, -0.05298924073576927, 0.017141319811344147};
        double end = 0.5;
        for (int i = 0; i < 5; ++i) {
            k.p[i] = (float)(fit[i] * scale * log2e * std::pow(x, 2 * i));
            if (i > 0 && !std::isnormal(k.p[i])) {
                end = std::pow(3e-8 / std::fabs(fit[i]), 0.5 / i);
                for (; i < 5; ++i) k.p[i] = 0.f;
            }
        }
        k.small = (float)(end / x);
    }
    return k;
}

}  // namespace noble
