// Building blocks of the attention kernels on gfx950: a tile of 64 partner rows in LDS (keys and values in the forward
// and the dq product, queries and upstream gradients in the dk/dv product), read both along its rows and across them,
// for products whose other operand stays in registers.
//
// Every product is written with the wave's own 32 rows as the MFMA's columns (operand B) and the partner rows, or
// the head's elements, as its rows (operand A).  Then each lane holds, for ONE own row, 16 of 32 partner rows of the
// scores: the softmax statistics need one exchange between lane l and l + 32, and the probabilities feed the next
// product as its operand B without leaving their lane.  The order of the summed index inside one MFMA is free as
// long as both operands share it, so that product takes the partner rows in the order in which the scores lie:
// step s of a lane half h covers rows 16 s + 4 h + {0..3} and 16 s + 8 + 4 h + {0..3}.
#pragma once

#include "noble_gemm_dma.hpp"

namespace noble {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Rows of one [rows, heads, D] tensor; strides in bytes.
struct HeadRows {
    char* ptr;
    int64_t row, head;
};

// Eight consecutive elements of the summed index: one 32x32x16 bf16 MFMA, or eight 32x32x2 float32 ones that each
// take one element of every lane.
template <typename E> struct Frag;
template <> struct Frag<uint16_t> { u32x4 v; };
template <> struct Frag<float> { u32x4 v[2]; };

__device__ __forceinline__ void mma32x32(f32x16& c, const Frag<uint16_t>& a, const Frag<uint16_t>& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0,
                                                0, 0);
}
__device__ __forceinline__ void mma32x32(f32x16& c, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.v[j >> 2][j & 3]), __uint_as_float(b.v[j >> 2][j & 3]),
                                                 c, 0, 0, 0);
}
__device__ __forceinline__ void mma16x16(f32x4& c, const Frag<uint16_t>& a, const Frag<uint16_t>& b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v), __builtin_bit_cast(bf16x8, b.v), c, 0,
                                                0, 0);
}
__device__ __forceinline__ void mma16x16(f32x4& c, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.v[j >> 2][j & 3]), __uint_as_float(b.v[j >> 2][j & 3]),
                                                 c, 0, 0, 0);
}

// Whether any element is infinite or NaN: its exponent's bits are all ones.
__device__ __forceinline__ bool not_finite(const Frag<uint16_t>& f) {
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) odd |= (f.v[j] & 0x7f800000u) == 0x7f800000u || (f.v[j] & 0x7f80u) == 0x7f80u;
    return odd;
}
__device__ __forceinline__ bool not_finite(const Frag<float>& f) {
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) odd |= (f.v[j >> 2][j & 3] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
// The elements whose bits are set; the others as zeros.
__device__ __forceinline__ Frag<uint16_t> only(Frag<uint16_t> f, uint32_t set) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        f.v[j] &= (set >> (2 * j) & 1u ? 0xffffu : 0u) | (set >> (2 * j + 1) & 1u ? 0xffff0000u : 0u);
    return f;
}
__device__ __forceinline__ Frag<float> only(Frag<float> f, uint32_t set) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = set >> j & 1u ? f.v[j >> 2][j & 3] : 0u;
    return f;
}

// Two float32 values as bf16 in one register, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
}

// Eight float32 values as a fragment.  On the bf16 path probabilities and score gradients are rounded here, like the
// operands of every bf16 product; their sums stay in float32.
template <typename E>
__device__ __forceinline__ Frag<E> to_frag(const float* p) {
    Frag<E> f;
    if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f.v[j] = pack_bf16(p[2 * j], p[2 * j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = __float_as_uint(p[j]);
    }
    return f;
}

// Eight elements from global memory, zeros where !ok.
template <typename E>
__device__ __forceinline__ Frag<E> global_frag(const char* p, bool ok) {
    Frag<E> f;
    if constexpr (sizeof(E) == 2) {
        f.v = ok ? *reinterpret_cast<const u32x4*>(p) : u32x4{0, 0, 0, 0};
    } else {
        f.v[0] = ok ? *reinterpret_cast<const u32x4*>(p) : u32x4{0, 0, 0, 0};
        f.v[1] = ok ? *reinterpret_cast<const u32x4*>(p + 16) : u32x4{0, 0, 0, 0};
    }
    return f;
}

// Four consecutive elements to global memory, each rounded once.
template <typename E>
__device__ __forceinline__ void store4(char* p, float a, float b, float c, float d) {
    if constexpr (sizeof(E) == 2)
        *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(a, b), pack_bf16(c, d)};
    else
        *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
}

// A tile of rows of DP elements in LDS: RB bytes a row, in chunks of 16 bytes; chunk c of row r lies at chunk
// c ^ swz(r).  bf16: with swz stepping by 4 over four consecutive rows, both reads cover the 64 banks once a pass:
// 16 rows at one chunk (fragments along the rows), and 4 rows at 4 chunks (ds_read_b64_tr_b16, fragments across).
template <typename E, int DP>
struct Tile {
    static constexpr int ES = sizeof(E), RB = DP * ES, NC = RB / 16;
    static constexpr int bytes(int rows) { return rows * RB; }
    static __device__ __forceinline__ int swz(int row) {
        if constexpr (ES == 4) return row & 15;
        else if constexpr (NC == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
        else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * RB + ((chunk ^ swz(row)) << 4); }

    // 8 elements of the row: 8 k .. 8 k + 7.
    static __device__ __forceinline__ Frag<E> along(const char* t, int row, int k) {
        Frag<E> f;
        if constexpr (ES == 2) {
            f.v = *reinterpret_cast<const u32x4*>(t + at(row, k));
        } else {
            f.v[0] = *reinterpret_cast<const u32x4*>(t + at(row, 2 * k));
            f.v[1] = *reinterpret_cast<const u32x4*>(t + at(row, 2 * k + 1));
        }
        return f;
    }
    // Elements 32 dt + lane % 32 of the rows row0 + 4 h + {0..3} and row0 + 8 + 4 h + {0..3}, h = lane / 32: operand A
    // of a product over these rows.
    static __device__ __forceinline__ Frag<E> across(const char* t, int row0, int dt, int lane) {
        Frag<E> f;
        const int h = lane >> 5;
        if constexpr (ES == 2) {
            const int j = lane & 15, r = row0 + 4 * h + (j >> 2);
            const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((j & 3) >> 1), b = 8 * (j & 1);
            const uint64_t lo = ds_read_tr(t + at(r, c) + b), hi = ds_read_tr(t + at(r + 8, c) + b);
            f.v = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
        } else {
            const int d = 32 * dt + (lane & 31);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = row0 + 4 * h + (j & 3) + 8 * (j >> 2);
                f.v[j >> 2][j & 3] = *reinterpret_cast<const uint32_t*>(t + at(r, d >> 2) + 4 * (d & 3));
            }
        }
        return f;
    }

    // Elements 16 dt + lane % 16 of the rows 4 g + {0..3} and 16 + 4 g + {0..3}, g = lane / 16: operand A of a 16x16
    // product over 32 rows.
    static __device__ __forceinline__ Frag<E> across16(const char* t, int dt, int lane) {
        Frag<E> f;
        const int g = lane >> 4, j = lane & 15;
        if constexpr (ES == 2) {
            const int r = 4 * g + (j >> 2), c = 2 * dt + ((j & 3) >> 1), b = 8 * (j & 1);
            const uint64_t lo = ds_read_tr(t + at(r, c) + b), hi = ds_read_tr(t + at(r + 16, c) + b);
            f.v = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
        } else {
            const int d = 16 * dt + j;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = 4 * g + (e & 3) + 16 * (e >> 2);
                f.v[e >> 2][e & 3] = *reinterpret_cast<const uint32_t*>(t + at(r, d >> 2) + 4 * (d & 3));
            }
        }
        return f;
    }

    // Requests `rows` rows for the tile at lds, shared by NW waves, from a descriptor whose base is the first row's and
    // whose size ends behind the last row that may be read: rows past it, and elements past the head's `db` bytes, come
    // as zeros.
    template <int NW, int ROWS>
    static __device__ __forceinline__ void request(i32x4 desc, char* lds, int stride, int db, int wave, int lane) {
        constexpr int PER = ROWS * RB / 1024 / NW, RPI = 1024 / RB;
        static_assert(PER * NW * 1024 == ROWS * RB, "whole requests");
        // Request i holds rows RPI i .. of the tile: RPI i in the scalar offset, the row inside it in the lane's
        const int in = lane / NC, near = in * stride;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int first = (wave * PER + i) * RPI, c = (lane % NC) ^ swz(first + in);
            dma16(desc, lds + (wave * PER + i) * 1024, 16 * c < db ? (uint32_t)(near + 16 * c) : kOOB,
                  (uint32_t)(first * stride));
        }
    }
};

// Fragments of tiles from one lane's place in them.  With the swizzle as it is, the places of a row's fragments differ
// from the first one's by an exclusive or of a constant, and rows by a constant in the instruction's offset field: two
// registers stand for all of them.  `off` is a whole number of rows.
template <typename E, int DP>
struct Reader {
    using T = Tile<E, DP>;
    const char* lds;
    int lane;
    __device__ __forceinline__ Reader(const char* base, int lane_) : lds(base), lane(lane_) {}
    __device__ __forceinline__ Reader at(int off) const { return Reader(lds + off, lane); }
    // Elements 16 x + 8 (lane / 32) .. of row lane % 32 of the 32 rows at `off`.
    __device__ __forceinline__ Frag<E> along(int x, int off) const {
        return T::along(lds + off, lane & 31, 2 * x + (lane >> 5));
    }
    // Elements 32 d + lane % 32 of the 16 rows at `off` (see Tile::across).
    __device__ __forceinline__ Frag<E> across(int d, int off) const { return T::across(lds + off, 0, d, lane); }
};
template <int DP>
struct Reader<uint16_t, DP> {
    using T = Tile<uint16_t, DP>;
    uint32_t al, ac;   // LDS addresses
    __device__ __forceinline__ Reader(const char* base, int lane) {
        const uint32_t b = (uint32_t)reinterpret_cast<uintptr_t>(NOBLE_LDS(base));
        const int h = lane >> 5, j = lane & 15;
        al = b + T::at(lane & 31, h);
        ac = b + T::at(4 * h + (j >> 2), 2 * ((lane >> 4) & 1) + ((j & 3) >> 1)) + 8 * (j & 1);
    }
    __device__ __forceinline__ Reader at(int off) const {
        Reader r = *this;
        r.al += off;
        r.ac += off;
        return r;
    }
    __device__ __forceinline__ Frag<uint16_t> along(int x, int off) const {
        typedef const __attribute__((address_space(3))) u32x4* ptr;
        return {*(ptr)(uintptr_t)((al ^ (32 * x)) + off)};
    }
    __device__ __forceinline__ Frag<uint16_t> across(int d, int off) const {
        typedef __attribute__((address_space(3))) s16x4* ptr;
        const uint64_t lo = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)((ac ^ (64 * d)) + off)));
        const uint64_t hi = __builtin_bit_cast(
            uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)((ac ^ (64 * d) ^ 32) + off + 8 * T::RB)));
        return {u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)}};
    }
};

// A descriptor in scalar registers, whichever way its words (the same in every lane) were computed.
__device__ __forceinline__ i32x4 wave_desc(const char* base, int64_t bytes) {
    i32x4 d = make_desc(base, bytes);
#pragma unroll
    for (int i = 0; i < 3; ++i) d[i] = __builtin_amdgcn_readfirstlane(d[i]);
    return d;
}

// Descriptor of rows [row0, row_end) of one head.
__device__ __forceinline__ i32x4 rows_desc(const HeadRows& x, int head, int row0, int row_end, int db) {
    return wave_desc(x.ptr + head * x.head + row0 * x.row, row_end > row0 ? (row_end - 1 - row0) * x.row + db : 0);
}

// 64 consecutive 4-byte values into LDS at dst, zeros past the descriptor's end.
__device__ __forceinline__ void dma4(i32x4 desc, char* lds_dst, int lane) {
    const uint32_t m0 = (uint32_t)reinterpret_cast<uintptr_t>(NOBLE_LDS(lds_dst));
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "buffer_load_dword %1, %2, 0 offen lds"
        :
        : "s"(m0), "v"((uint32_t)(4 * lane)), "s"(desc)
        : "memory", "m0");
}

// Order of a run of MFMAs whose operand A comes from LDS, READS reads for each PER MFMAs: AHEAD operands are read before
// the first MFMA and each operand's registers are read again as soon as its MFMAs have been issued.  Without it every
// MFMA waits for a read that was issued right before it.
template <int MFMAS, int PER, int READS, int AHEAD>
__device__ __forceinline__ void read_ahead() {
    constexpr int N = MFMAS / PER, A = AHEAD < N ? AHEAD : N;
    __builtin_amdgcn_sched_group_barrier(0x100, READS * A, 0);
#pragma unroll
    for (int i = 0; i < N - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, PER * A, 0);
}

// All requests of this wave have arrived and its LDS reads are done, and so it is for every wave.
__device__ __forceinline__ void arrive_all() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The wave's own operands, loaded before a loop, are here.  By the builtin, which the compiler counts: without it, it waits
// for them at their first use in every turn of the loop, and with them for the tile that was requested right before.
__device__ __forceinline__ void operands_here() {
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
}

// The larger (or the sum) of a value and that of lane ^ 32.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The least or largest of a wave's values, by row shifts and broadcasts (in lane 63 at the end): six dependent VALU
// operations, where six exchanges through LDS take ten times as long and stand before a kernel's first request.
template <typename F>
__device__ __forceinline__ int wave_fold(int x, int none, F f) {
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));   // row_shr:1, 2, 4, 8
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));   // row_bcast:15 into rows 1 and 3
    x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));   // row_bcast:31 into rows 2 and 3
    return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_min(int x) {
    return wave_fold(x, INT32_MAX, [](int a, int b) { return min(a, b); });
}
__device__ __forceinline__ int wave_max(int x) {
    return wave_fold(x, INT32_MIN, [](int a, int b) { return max(a, b); });
}

// Workgroups run round robin over the 8 XCDs, each with an L2 of its own.  Key heads are dealt to XCDs so that the
// workgroups that share keys and values share an L2: with g the common divisor of the key heads and 8, each 8 / g XCDs
// take heads / g key heads together, every one of them each (8 / g)th workgroup of these heads.  Contiguous ranges
// would give one XCD the long rows of a causal mask and another the short ones.
struct HeadOrder {
    int heads, per;   // key heads, workgroups of one
    __host__ __device__ static int common(int heads) { return heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1; }
    // Workgroups to launch: those without work end at once.
    __host__ static int64_t grid(int heads, int64_t per) {
        const int g = common(heads), m = 8 / g;
        return (heads / g * per + m - 1) / m * 8;
    }
    // The key head and the place among its workgroups; false: no work.
    __device__ __forceinline__ bool place(int b, int& head, int& at) const {
        const int g = common(heads), m = 8 / g, x = b & 7, mine = heads / g;
        // An XCD's 32 CUs each get one workgroup of 32 in a row and one of the next 32: every other 32 run backwards,
        // so that a CU's two are not the same place of two documents (all long ones or all short ones).  Forward and dq
        // of 8 documents of 1024 rows: 40 -> 37 and 54 -> 49 us.
        int slot = b >> 3;
        if ((slot & 32) && (slot | 31) < (int)(gridDim.x >> 3)) slot ^= 31;
        const int item = slot * m + x % m;
        if (item >= mine * per) return false;
        head = x / m * mine + item / per;
        at = item % per;
        return true;
    }
};

constexpr int kCap = 1, kBias = 2;   // bits of a kernel's MODE

// From raw products q.k to scores: z in units in which z `unit` is the score times log2 e.  Without a cap z is the product
// and unit = scale log2 e, which the exponential's multiply-add takes along; with one unit is 1.  From the host.
struct ScoreArgs {
    float unit;
    float cap_in;     // scale / cap
    float cap_e;      // 2 scale log2 e / cap: exp2 of it is e^2x
    float cap_out;    // cap log2 e
    float inv2;       // 1 / cap_out^2
    float small;      // |s| up to which the polynomial is taken: x = s scale / cap up to 1/2, or less (score_args)
    float p[5];       // there: score = s (p0 + p1 s^2 + .. + p4 s^8)
};

// exp of a score less `from` (both times log2 e).
template <int MODE>
__device__ __forceinline__ float exp_score(const ScoreArgs& k, float z, float from) {
    return __builtin_amdgcn_exp2f(MODE & kCap ? z - from : fmaf(z, k.unit, -from));
}

// The distance bias on z, slope in the same units, of the keys or rows `first` + 8 (i / 4) + i % 4 for i < 16.  Distances
// are exact in float32 up to 2^24.
__device__ __forceinline__ void bias16(float* z, float slope, float first) {
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = fmaf(-slope, fabsf(first + (float)(8 * (i >> 2) + (i & 3))), z[i]);
}

// N scores of one lane.  tanh by two formulas: up to 1/2 an odd polynomial of degree 9 (fitted to tanh(x) / x on
// [0, 1/4] in x^2: relative error 3e-8), above it 1 - 2 / (e^2x + 1), whose absolute error of 1e-7 is relative there.
// With the caps in use nearly every score is below, and a wave without a larger one runs the polynomial alone: 6
// multiplications and additions for each score, where exp and reciprocal take as long as 10.  The float32 path
// takes the library's tanh.  z may be s.  `slope` (given or nullptr): the cap's derivative, 1 - tanh^2.
template <typename E, int MODE, int N>
__device__ __forceinline__ void scores(const ScoreArgs& k, const float* s, float* z, float* slope) {
    if constexpr (!(MODE & kCap)) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = s[i];
    } else if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = tanhf(s[i] * k.cap_in);
            z[i] = t * k.cap_out;
            if (slope) slope[i] = 1.f - t * t;
        }
    } else {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(s[i]));
        const auto near = [&](float x) {
            const float y = x * x;
            return x * fmaf(fmaf(fmaf(fmaf(k.p[4], y, k.p[3]), y, k.p[2]), y, k.p[1]), y, k.p[0]);
        };
        if (__any(top > k.small)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = s[i];   // z may be s
                const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * k.cap_e) + 1.f);
                z[i] = fabsf(x) > k.small ? t * k.cap_out : near(x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = near(s[i]);
        }
        if (slope) {
#pragma unroll
            for (int i = 0; i < N; ++i) slope[i] = fmaf(-(z[i] * z[i]), k.inv2, 1.f);
        }
    }
}

}  // namespace noble
