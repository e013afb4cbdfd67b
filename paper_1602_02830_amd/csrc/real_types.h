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

template <typename E>
struct Vec8 {
    typedef E type __attribute__((ext_vector_type(8)));
    typedef E any __attribute__((ext_vector_type(8), aligned(sizeof(E))));      // the same at the type's own alignment
};

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

// Eight elements from p on, of which the first `valid` exist; zero for the others, which are not read.  p is aligned to
// its element: a whole group is one or two 16-byte loads, which need no more than that.
template <typename E>
__device__ inline typename Vec8<E>::type load8(const E* p, int64_t valid) {
    typename Vec8<E>::type v = {};
    if (valid >= 8) {
        v = *reinterpret_cast<const typename Vec8<E>::any*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < valid) v[i] = p[i];
    }
    return v;
}

template <typename E>
__device__ inline void store8(E* p, const float (&v)[8], int64_t valid) {
    typename Vec8<E>::type o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = E(v[i]);
    if (valid >= 8) {
        *reinterpret_cast<typename Vec8<E>::any*>(p) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < valid) p[i] = o[i];
    }
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

template <bool FAST>
__device__ inline float activate(int act, float z) {
    switch (act) {
        case BNN_ACT_RELU: return z > 0.0f ? z : z != z ? z : 0.0f;
        case BNN_ACT_SILU: return over<FAST>(z, 1.0f + exp_of<FAST>(-z));
        case BNN_ACT_SIGMOID: return over<FAST>(1.0f, 1.0f + exp_of<FAST>(-z));
        case BNN_ACT_GELU: return 0.5f * z * (1.0f + erff(z * kSqrtHalf));
        // 0.5 z (1 + tanh u) = z / (1 + e^(-2u))
        case BNN_ACT_GELU_TANH: return over<FAST>(z, 1.0f + exp_of<FAST>(-kTwoSqrt2OverPi * (z + 0.044715f * z * z * z)));
        default: return z;
    }
}

// The activation and its derivative (of relu at 0: 0).
template <bool FAST>
__device__ inline void activate_both(int act, float z, float& f, float& df) {
    switch (act) {
        case BNN_ACT_RELU:
            f = z > 0.0f ? z : z != z ? z : 0.0f;
            df = z > 0.0f ? 1.0f : 0.0f;
            break;
        case BNN_ACT_SILU: {
            const float s = over<FAST>(1.0f, 1.0f + exp_of<FAST>(-z));
            f = z * s;
            df = s * (1.0f + z * (1.0f - s));
            break;
        }
        case BNN_ACT_SIGMOID: {
            const float s = over<FAST>(1.0f, 1.0f + exp_of<FAST>(-z));
            f = s;
            df = s * (1.0f - s);
            break;
        }
        case BNN_ACT_GELU: {
            const float c = 0.5f * (1.0f + erff(z * kSqrtHalf));
            f = z * c;
            df = c + z * kInvSqrt2Pi * exp_of<FAST>(-0.5f * z * z);
            break;
        }
        case BNN_ACT_GELU_TANH: {
            const float u2 = kTwoSqrt2OverPi * (z + 0.044715f * z * z * z);
            const float s = over<FAST>(1.0f, 1.0f + exp_of<FAST>(-u2));
            f = z * s;
            // s (1 - s) is 0 long before the polynomial overflows, but 0 * inf is not.
            const float slope = s * (1.0f - s);
            df = slope == 0.0f ? s : s + z * slope * kTwoSqrt2OverPi * (1.0f + 0.134145f * z * z);
            break;
        }
        default:
            f = z;
            df = 1.0f;
    }
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

// v = t[0] + t[1] + t[2] exactly, each a bfloat16 (8 significant bits; a float32 has 24).  Each term is what is left cut off
// after 8 bits: all have the sign of v, so no sum of some of them is larger than v and overflows where v does not.  An
// infinity or a NaN stays in the first term alone.
__device__ inline float cut_off(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }

__device__ inline void split3(float v, bf16_t (&t)[3]) {
    const bool finite = __builtin_fabsf(v) < __builtin_inff();
    const float top = cut_off(v), r1 = finite ? v - top : 0.0f, middle = cut_off(r1);
    t[0] = bf16_t(finite ? top : v);
    t[1] = bf16_t(middle);
    t[2] = bf16_t(r1 - middle);
}

// Row of a 32-row operand block that lane a of the first operand loads, so that accumulator register i of lane half h is
// row 16 h + i of the block: register i belongs to operand row 8 (i / 4) + 4 h + i % 4.
__device__ inline int consecutive_rows(int a) { return 16 * ((a >> 2) & 1) + 4 * (a >> 3) + (a & 3); }

}  // namespace bnn
