// A row of reals in the registers of one workgroup, and sums over it: what the norms and the quantisation of rows share.
#pragma once

#include "gemm_staging.h"
#include "quant_rows.h"
#include "real_types.h"

namespace bnn {

constexpr int64_t kMaxRowHeld = 16384;       // elements of the longest row that a workgroup holds in registers

__device__ inline float sum_of_wave(float v) {
    v = sum_of_32(v);
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Sums of a and of b over the workgroup of up to WAVES wavefronts, the same in every thread.  Two buffers in turn: a thread writes
// one again only after the barrier of the sum between, by which everyone has read it.
template <int WAVES>
struct Sums {
    float2* lds;             // [2][WAVES]; zero where there is no such wavefront
    int turn = 0;
    __device__ inline explicit Sums(float2* p) : lds(p) {
        if constexpr (WAVES > 1) {
            if (threadIdx.x < 2 * WAVES) lds[threadIdx.x] = make_float2(0.0f, 0.0f);
            __syncthreads();
        }
    }
    __device__ inline float2 operator()(float a, float b) {
        a = sum_of_wave(a);
        b = sum_of_wave(b);
        if constexpr (WAVES > 1) {
            float2* const p = lds + turn * WAVES;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = make_float2(a, b);
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                a += p[w].x;
                b += p[w].y;
            }
        }
        return make_float2(a, b);
    }
};

// The largest of what the threads of the workgroup have, the same in every thread; buffers and turns as above.
template <int WAVES>
struct Largest {
    uint32_t* lds;           // [2][WAVES]
    int turn = 0;
    __device__ inline explicit Largest(uint32_t* p) : lds(p) {
        if constexpr (WAVES > 1) {
            if (threadIdx.x < 2 * WAVES) lds[threadIdx.x] = 0;
            __syncthreads();
        }
    }
    __device__ inline uint32_t operator()(uint32_t v) {
        auto from = [&](auto control) { return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), decltype(control)::value, 0xF, 0xF, true)); };
        v = largest_of_quad(v);
        v = max(v, from(std::integral_constant<int, 0x141>{}));      // row_half_mirror
        v = max(v, from(std::integral_constant<int, 0x140>{}));      // row_mirror
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(p[0], p[1]);
        const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(q[0], q[1]);
        if constexpr (WAVES > 1) {
            uint32_t* const w = lds + turn * WAVES;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = v;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v = max(v, w[i]);
        }
        return v;
    }
};

// A row's layout over a workgroup: CH groups of G elements a thread, in a workgroup of no more wavefronts than the row needs (WAVES
// at most).  Group i of a thread begins with column first_col(i).
template <int W, int GROUP, int GROUPS, bool IS_SHORT>
struct Layout {
    static constexpr int WAVES = W, G = GROUP, CH = GROUPS;
    static constexpr bool SHORT = IS_SHORT;      // rows of fewer than G elements
    static constexpr bool FULL = W == 1 || (W == 16);
    static inline int threads(int64_t D) { return FULL ? 64 * W : 64 * int(ceil_div(D, 64 * G * CH)); }
    __device__ static inline int first_col(int i) { return (i * (FULL ? 64 * W : int(blockDim.x)) + int(threadIdx.x)) * G; }
};

template <typename L>
using Values = float[L::CH][L::G];

template <typename L, typename F>
__device__ inline void each(F&& f) {
#pragma unroll
    for (int i = 0; i < L::CH; ++i)
#pragma unroll
        for (int e = 0; e < L::G; ++e) f(i, e);
}

// A row's part of this thread, as it lies in memory.  Loads ask no questions, so that the compiler knows how many are on their way:
// what lies past the row's end is loaded from its last group (SHORT: an element at a time), and put right by `widened`.
template <typename E, typename L>
struct Row {
    typename Group<E, L::G>::type v[L::CH];
    __device__ inline void load(const void* matrix, int64_t m, int64_t ld, int D) {
        const E* const row = static_cast<const E*>(matrix) + m * ld;
#pragma unroll
        for (int i = 0; i < L::CH; ++i) {
            const int c = L::first_col(i);
            if constexpr (L::SHORT) v[i] = load_group<E, L::G>(row + c, D - c);
            else v[i] = *reinterpret_cast<const typename Group<E, L::G>::any*>(row + min(c, D - L::G));
        }
    }
    // As floats, zero past the row's end.
    __device__ inline void widened(int D, Values<L>& to) const {
#pragma unroll
        for (int i = 0; i < L::CH; ++i) {
            const int c = L::first_col(i);
            typename Group<E, L::G>::type q = v[i];
            // The wavefront's last group lies past the row's end: some of them have to be moved.
            if (!L::SHORT && __builtin_amdgcn_readfirstlane(c) + 64 * L::G > D) q = row_end<E, L::G>(q, D - c);
#pragma unroll
            for (int e = 0; e < L::G; ++e) to[i][e] = float(q[e]);
        }
    }
};

// Zero past the row's end: the unit checks the bound (333 x 2049 float16 with layer norms 9.0 us instead of 9.4 with row_end for vectors too).
// AS_ROW: as a row instead, for a kernel that has too few registers either way and keeps fewer in scratch memory so.
template <typename L, bool AS_ROW = false>
__device__ inline void load_vector(const float* p, int D, float otherwise, Values<L>& v) {
    if (!p) return each<L>([&](int i, int e) { v[i][e] = otherwise; });
    if constexpr (AS_ROW) {
        Row<float, L> row;
        row.load(p, 0, 0, D);
        return row.widened(D, v);
    }
    constexpr int kWords = 0x00027000;               // data format: 32 bits
    const auto vector = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), 0, D * 4, kWords);
#pragma unroll
    for (int i = 0; i < L::CH; ++i)
#pragma unroll
        for (int q = 0; q < L::G / 4; ++q) {
            const auto words = __builtin_amdgcn_raw_buffer_load_b128(vector, (L::first_col(i) + 4 * q) * 4, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][4 * q + e] = __uint_as_float(words[e]);
        }
}

template <typename E, typename L, bool PAST = false>
__device__ inline void store_row(E* row, int D, const Values<L>& v) {
#pragma unroll
    for (int i = 0; i < L::CH; ++i) {
        const int c = L::first_col(i);
        if (c < D) store_group<E, L::G, PAST>(row + c, v[i], D - c);
    }
}

template <typename L>
__device__ inline float sum_of(const Values<L>& v) {
    float s = 0.0f;
    each<L>([&](int i, int e) { s += v[i][e]; });
    return s;
}

template <typename L>
__device__ inline float sum_of_squares(const Values<L>& v) {
    float s = 0.0f;
    each<L>([&](int i, int e) { s = fmaf(v[i][e], v[i][e], s); });
    return s;
}

// Elements past the row's end are, and stay, zero.
template <typename L>
__device__ inline void trim(Values<L>& v, int D) {
#pragma unroll
    for (int i = 0; i < L::CH; ++i) {
        const int c = L::first_col(i);
        if (__builtin_amdgcn_readfirstlane(c) + 64 * L::G <= D) continue;      // for a whole wavefront
#pragma unroll
        for (int e = 0; e < L::G; ++e) v[i][e] = c + e < D ? v[i][e] : 0.0f;
    }
}

// Codes, scale and x^ of a row whose elements past its end are zero.
template <typename E, typename L, bool PAST = true>
__device__ inline void store_row_i8(const QuantOut& o, int64_t m, int D, const Values<L>& v, Largest<L::WAVES>& largest) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < L::CH; ++i) most = max(most, largest_of_8(v[i]));
    const float s = i8_scale(largest(most));
    if (threadIdx.x == 0) static_cast<float*>(o.scales)[m] = s;
#pragma unroll
    for (int i = 0; i < L::CH; ++i) {
        const int c = L::first_col(i);
        if ((c & ~31) < D) quantise_i8<E, PAST>(o, m, c, v[i], s, D);
    }
}

template <typename E, typename L, bool PAST = true>
__device__ inline void store_row_mx4(const QuantOut& o, int64_t m, int D, const Values<L>& v) {
#pragma unroll
    for (int i = 0; i < L::CH; ++i) {
        const int c = L::first_col(i);
        if ((c & ~31) < D) quantise_mx4<E, PAST>(o, m, c, v[i], D);
    }
}

// Calls f(layout) for rows of D elements.
template <typename F>
inline void with_row(int64_t D, F&& f) {
    if (D < 8) f(Layout<1, 8, 1, true>{});
    else if (D <= 512) f(Layout<1, 8, 1, false>{});
    else if (D <= 1024) f(Layout<1, 8, 2, false>{});
    else if (D <= 4096) f(Layout<4, 8, 2, false>{});
    else if (D <= 8192) f(Layout<8, 8, 2, false>{});
    else f(Layout<16, 8, 2, false>{});
}

}  // namespace bnn
