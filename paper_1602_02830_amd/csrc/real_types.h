// What the operators on real activations share: element types, loads and stores of eight elements at any alignment,
// activations with their derivatives, and the widening of packed weights to +-1 operands of the matrix engine.
#pragma once

#include <type_traits>

#include "bnn_internal.h"

namespace bnn {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float v16f_t __attribute__((ext_vector_type(16)));
typedef uint32_t v4u_t __attribute__((ext_vector_type(4)));

template <typename E>
inline constexpr bool is_f32 = std::is_same<E, float>::value;

// The type that the matrix engine multiplies for activations of type E: float32 ones are split into three bfloat16 terms.
template <typename E>
using Operand = typename std::conditional<is_f32<E>, bf16_t, E>::type;

template <typename E, int G>
struct Group {
    typedef E type __attribute__((ext_vector_type(G)));
    typedef E any __attribute__((ext_vector_type(G), aligned(sizeof(E))));      // the same at the type's own alignment
};
template <typename E>
using Vec8 = Group<E, 8>;

// Calls `f` with a value of the C++ type of a bnn_type; false for a type that does not exist.
template <typename F>
inline bool with_type(int type, F&& f) {
    switch (type) {
        case BNN_BF16: f(bf16_t{}); return true;
        case BNN_F16: f(f16_t{}); return true;
        case BNN_F32: f(float{}); return true;
        default: return false;
    }
}

inline int64_t type_bytes(int type) { return type == BNN_F32 ? 4 : type == BNN_BF16 || type == BNN_F16 ? 2 : 0; }

// G elements from p on, of which the first `valid` exist; zero for the others, which are not read.  p is aligned to
// its element: a whole group is one or two 16-byte loads, which need no more than that.  The elements of a part of a group are
// loaded all at once (the last one again for those that are not there): one by one, each would wait for the one before.
template <typename E, int G>
__device__ inline typename Group<E, G>::type load_group(const E* p, int64_t valid) {
    typename Group<E, G>::type v = {};
    if (valid >= G) {
        v = *reinterpret_cast<const typename Group<E, G>::any*>(p);
    } else if (valid > 0) {
        const int last = int(valid) - 1;
        E e[G - 1];
#pragma unroll
        for (int i = 0; i < G - 1; ++i) e[i] = p[min(i, last)];
#pragma unroll
        for (int i = 0; i < G - 1; ++i) v[i] = i <= last ? e[i] : E(0.0f);
    }
    return v;
}

template <typename E>
__device__ inline typename Vec8<E>::type load8(const E* p, int64_t valid) {
    return load_group<E, 8>(p, valid);
}

// What is left of a row from a group's first element on, `left` elements: the group as it is for G or more, and for fewer the
// last ones of v - the row's last G elements, loaded in the group's place - moved down, with zeros after them.
template <typename E, int G = 8>
__device__ inline typename Group<E, G>::type row_end(typename Group<E, G>::type v, int left) {
    const int by = G - left;
#pragma unroll
    for (int step = G / 2; step > 0; step >>= 1) {
        typename Group<E, G>::type moved = v;
#pragma unroll
        for (int i = 0; i < G; ++i) moved[i] = i + step < G ? v[i + step] : E(0.0f);
        if (by > 0 && (by & step)) v = moved;
    }
    return left > 0 ? v : typename Group<E, G>::type{};
}

// PAST: whole groups go past the cache.
template <typename E, int G, bool PAST = false>
__device__ inline void store_group(E* p, const float (&v)[G], int64_t valid) {
    typedef typename Group<E, G>::any any;
    typename Group<E, G>::type o;
#pragma unroll
    for (int i = 0; i < G; ++i) o[i] = E(v[i]);
    if (valid >= G) {
        if constexpr (PAST) __builtin_nontemporal_store(o, reinterpret_cast<any*>(p));
        else *reinterpret_cast<any*>(p) = o;
    } else {
#pragma unroll
        for (int i = 0; i < G - 1; ++i)
            if (i < valid) p[i] = o[i];
    }
}

template <typename E>
__device__ inline void store8(E* p, const float (&v)[8], int64_t valid) {
    store_group<E, 8>(p, v, valid);
}

template <typename E, int W>
__device__ inline void load_some(const E* p, int64_t valid, float (&v)[W]) {
    const auto q = load_group<E, W>(p, valid);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = float(q[i]);
}

// ---- activations, float32 --------------------------------------------------------------------------------------
// For results of 16 bits the exponential and the reciprocal are the hardware's (1 ulp each, and the exponent's product
// with log2 e rounded once: relative error below 1e-6 for |z| < 16, far under half a unit of 16 bits); for float32
// results they are the library's.

template <bool FAST>
__device__ inline float exp_of(float z) {
    return FAST ? __expf(z) : expf(z);
}

template <bool FAST>
__device__ inline float over(float a, float b) {
    return FAST ? a * __builtin_amdgcn_rcpf(b) : a / b;
}

constexpr float kSqrtHalf = 0.70710678118654752f;        // sqrt(1 / 2)
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kInvSqrt2Pi = 0.3989422804014327f;       // 1 / sqrt(2 pi)

// W values at a time, so that one is chosen once for them.
template <bool FAST, int W>
__device__ inline void activate(int act, const float (&z)[W], float (&f)[W]) {
    auto all = [&](auto&& one) {
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = one(z[i]);
    };
    switch (act) {
        case BNN_ACT_RELU: return all([](float v) { return v > 0.0f ? v : v != v ? v : 0.0f; });
        case BNN_ACT_SILU: return all([](float v) { return over<FAST>(v, 1.0f + exp_of<FAST>(-v)); });
        case BNN_ACT_SIGMOID: return all([](float v) { return over<FAST>(1.0f, 1.0f + exp_of<FAST>(-v)); });
        // 1 + erf(u) = erfc(-u): below zero the sum would cancel (at z = -5, 4 % of the result, and nothing is left from -5.5 on).
        // The sum was faster where the epilogue counts: 4096 x 784 -> 2 x 4096 bfloat16 73 us, 77 with this.
        case BNN_ACT_GELU: return all([](float v) { return 0.5f * v * erfcf(-v * kSqrtHalf); });
        // 0.5 z (1 + tanh u) = z / (1 + e^(-2u))
        case BNN_ACT_GELU_TANH:
            return all([](float v) { return over<FAST>(v, 1.0f + exp_of<FAST>(-kTwoSqrt2OverPi * (v + 0.044715f * v * v * v))); });
        default: return all([](float v) { return v; });
    }
}

// The activation and its derivative (of relu at 0: 0).
template <bool FAST, int W>
__device__ inline void activate_both(int act, const float (&z)[W], float (&f)[W], float (&df)[W]) {
    auto all = [&](auto&& one) {
#pragma unroll
        for (int i = 0; i < W; ++i) one(z[i], f[i], df[i]);
    };
    switch (act) {
        case BNN_ACT_RELU:
            return all([](float v, float& y, float& dy) {
                y = v > 0.0f ? v : v != v ? v : 0.0f;
                dy = v > 0.0f ? 1.0f : 0.0f;
            });
        case BNN_ACT_SILU:
            return all([](float v, float& y, float& dy) {
                const float s = over<FAST>(1.0f, 1.0f + exp_of<FAST>(-v));
                y = v * s;
                dy = s * (1.0f + v * (1.0f - s));
            });
        case BNN_ACT_SIGMOID:
            return all([](float v, float& y, float& dy) {
                // 1 - s = e s, which keeps its digits where s is almost 1, and is infinity times 0 far below zero.
                const float e = exp_of<FAST>(-v);
                y = over<FAST>(1.0f, 1.0f + e);
                dy = y * (v > 0.0f ? e * y : 1.0f - y);
            });
        case BNN_ACT_GELU:
            return all([](float v, float& y, float& dy) {
                const float c = 0.5f * erfcf(-v * kSqrtHalf);
                y = v * c;
                dy = c + v * kInvSqrt2Pi * exp_of<FAST>(-0.5f * v * v);
            });
        case BNN_ACT_GELU_TANH:
            return all([](float v, float& y, float& dy) {
                const float s = over<FAST>(1.0f, 1.0f + exp_of<FAST>(-kTwoSqrt2OverPi * (v + 0.044715f * v * v * v)));
                y = v * s;
                // s (1 - s) is 0 long before the polynomial overflows, but 0 * inf is not.
                const float slope = s * (1.0f - s);
                dy = slope == 0.0f ? s : s + v * slope * kTwoSqrt2OverPi * (1.0f + 0.134145f * v * v);
            });
        default:
            return all([](float v, float& y, float& dy) {
                y = v;
                dy = 1.0f;
            });
    }
}

// Sum over each half wavefront of 32 lanes, in every lane of it: inside rows of 16 lanes by data-parallel permutes, then the rows'.
__device__ inline float sum_of_32(float v) {
    auto from = [&](auto control) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xF, 0xF, true));
    };
    v += from(std::integral_constant<int, 0xB1>{});       // quad_perm [1,0,3,2]
    v += from(std::integral_constant<int, 0x4E>{});       // quad_perm [2,3,0,1]
    v += from(std::integral_constant<int, 0x141>{});      // row_half_mirror
    v += from(std::integral_constant<int, 0x140>{});      // row_mirror
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Sum over the lanes that are 4, 8, ... apart, in every one of them.
__device__ inline float sum_of_every_fourth(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xF, 0xF, true));       // row_ror:4
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, true));       // row_ror:8
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// ---- packed weights as operands of the matrix engine --------------------------------------------------------------
// A lane takes 32 elements of a row from one word: element e is bit e.  Of 16 bits b, the word y = b | b << 15 has bit 2j
// at 2j and bit 2j + 1 at 2j + 16, so that one shift brings a pair of elements to the signs of two 16-bit floats, and one
// operation puts 1.0 under them: 2 operations a pair, 18 for 16 elements.  A sign is set where the bit is: the operand is
// MINUS the weight, and who reads the sums negates them.

template <typename O>
inline constexpr uint32_t kOnes = std::is_same<O, bf16_t>::value ? 0x3F803F80u : 0x3C003C00u;

// The two constants in registers: with both in sight the compiler makes two operations with literals of the one.
template <typename O>
struct Widening {
    uint32_t signs = 0x80008000u, ones = kOnes<O>;
    __device__ inline Widening() { asm("" : "+s"(signs), "+v"(ones)); }
    __device__ inline typename Vec8<O>::type operator()(uint32_t y, int s) const {       // elements from 8 * s on, s = 0 or 1
        v4u_t d;
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = ((y << (15 - 8 * s - 2 * j)) & signs) | ones;
        return __builtin_bit_cast(typename Vec8<O>::type, d);
    }
};

__device__ inline uint32_t spread_low(uint32_t w) {
    const uint32_t b = w & 0xFFFFu;
    return b | (b << 15);
}

__device__ inline uint32_t spread_high(uint32_t w) {
    const uint32_t b = w >> 16;
    return b | (b << 15);
}

__device__ inline v16f_t mfma16(Vec8<bf16_t>::type a, Vec8<bf16_t>::type b, v16f_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ inline v16f_t mfma16(Vec8<f16_t>::type a, Vec8<f16_t>::type b, v16f_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

typedef float v4f_t __attribute__((ext_vector_type(4)));

__device__ inline v4f_t mfma32(Vec8<bf16_t>::type a, Vec8<bf16_t>::type b, v4f_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ inline v4f_t mfma32(Vec8<f16_t>::type a, Vec8<f16_t>::type b, v4f_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ inline float cut_off(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }

// The upper halves of two words, the first one's below.
__device__ inline uint32_t upper_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Eight activations as operands: one term of a 16-bit type, three of float32.
template <typename E>
inline constexpr int kTermsOf = is_f32<E> ? 3 : 1;

// A float32 is the sum of three bfloat16 exactly (24 significant bits, 8 each).  Each term is what is left cut off after 8
// bits: all have the sign of the value, so no sum of some of them is larger than it and overflows where it does not.  An infinity
// stays in the first term alone, and so does a NaN (whose upper half is kept from being an infinity's).
//
// NONZERO: for products of such terms with one another, where a term of zero would make a NaN of the other factor's infinity: no term of
// a value that is not zero is.  A first or second term that leaves nothing is one unit smaller in its last place, so that the third
// is below 2^-14 of the value, and an infinity has ones of its sign in its other terms.
template <typename E, bool NONZERO = false>
__device__ inline void terms_of(const typename Vec8<E>::type& v, typename Vec8<Operand<E>>::type (&t)[kTermsOf<E>]) {
    if constexpr (is_f32<E>) {
        v4u_t d[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float top[2], rest[2], middle[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = v[2 * i + e];
                top[e] = cut_off(x);
                if constexpr (NONZERO) {
                    const bool finite = __builtin_fabsf(x) < __builtin_inff();
                    if (finite && top[e] == x && x != 0.0f) top[e] = __uint_as_float(__float_as_uint(x) - 0x10000u);
                    rest[e] = finite ? x - top[e] : __builtin_copysignf(2.0f, x);
                    top[e] = x != x ? x + x : top[e];
                    middle[e] = cut_off(rest[e]);
                    if (middle[e] == rest[e] && x != 0.0f) middle[e] = finite ? __uint_as_float(__float_as_uint(rest[e]) - 0x10000u) : 0.5f * rest[e];
                } else {
                    rest[e] = __builtin_fabsf(x) < __builtin_inff() ? x - top[e] : 0.0f;
                    top[e] = x != x ? x + x : top[e];
                    middle[e] = cut_off(rest[e]);
                }
            }
            d[0][i] = upper_halves(top[0], top[1]);
            d[1][i] = upper_halves(middle[0], middle[1]);
            d[2][i] = upper_halves(rest[0] - middle[0], rest[1] - middle[1]);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) t[p] = __builtin_bit_cast(typename Vec8<Operand<E>>::type, d[p]);
    } else {
        t[0] = v;
    }
}

// Row of a 32-row operand block that lane a of the first operand loads, so that accumulator register i of lane half h is
// row 16 h + i of the block: register i belongs to operand row 8 (i / 4) + 4 h + i % 4.
__device__ inline int consecutive_rows(int a) { return 16 * ((a >> 2) & 1) + 4 * (a >> 3) + (a & 3); }

}  // namespace bnn
