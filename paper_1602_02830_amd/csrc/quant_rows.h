// Rows of reals as codes of 8 or 4 bits with scales (bnn_rows), and back: what quantisation, norms and products share.
//
// BNN_ROWS_I8   q = x / s to the nearest whole number, s = the row's largest magnitude / 127 in float32
// BNN_ROWS_MX4  c = x / 2^e to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, e for each 32 elements the smallest
//               exponent with which the largest magnitude does not round past 6
//
// Of two codes as near the even one is taken.  Codes of a block of 32 elements lie in the order in which a word of 32 weights is
// widened (q_bits.h): nibble 8 i + j of the 16 bytes is element 4 j + i, byte 4 i + j of the 32 is element 8 j + i.  A row of
// activations lives for one product, so that this order costs nobody anything, and the product saves the operations that would bring
// weights into another one: for codes of 4 bits 27 instead of 7 for each 32 weights.
//
// Four neighbouring lanes have a block between them, eight consecutive elements each, here and in the epilogues of products.
#pragma once

#include "real_types.h"

namespace bnn {

inline int64_t block_bytes(int rows) { return rows == BNN_ROWS_I8 ? 32 : 16; }
inline bool rows_kind(int rows) { return rows == BNN_ROWS_I8 || rows == BNN_ROWS_MX4; }

constexpr float kLeastRowScale = 1.1754943508222875e-38f;       // 2^-126
constexpr uint32_t kNoScale = 255;                              // of a block with an infinity or a NaN

// Codes and scales of one matrix; hat: the values that they stand for, in the activations' type, or null.
struct QuantOut {
    uint8_t* codes;          // [M][ld_c]
    void* scales;            // float [M] or bytes [M][ld_s]
    void* hat;               // [M][ld_h]
    int64_t ld_c, ld_s, ld_h;
};

// A magnitude's bits: as whole numbers they are ordered like the magnitudes, infinities and NaNs above all others.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ inline bool finite_bits(uint32_t magnitude) { return magnitude < 0x7F800000u; }

__device__ inline uint32_t largest_of_8(const float (&v)[8]) {
    uint32_t m = magnitude(v[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) m = max(m, magnitude(v[e]));
    return m;
}

// The value of lane Q of each quad, in its four lanes.
template <int Q>
__device__ inline uint32_t quad_lane(uint32_t v) {
    return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), Q * 0x55, 0xF, 0xF, true));
}

__device__ inline uint32_t largest_of_quad(uint32_t v) {
    v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, true)));        // quad_perm [1,0,3,2]
    return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, true)));     // quad_perm [2,3,0,1]
}

// ---- 4 bits, a power of two for each 32 elements -------------------------------------------------------------------

// The scale's byte, e + 127, from the block's largest magnitude: 7 * 2^e and more round past 6, so a mantissa from 1.75 on
// counts as the next power of two.  1 at least: a float32 of its own in every case (it is 2^-126, blocks below 2^-124 lose
// digits).
__device__ inline uint32_t mx4_scale(uint32_t largest) {
    if (!finite_bits(largest)) return kNoScale;
    return uint32_t(max(int((largest + 0x200000u) >> 23) - 2, 1));
}

// The power of two of a scale's byte; of kNoScale NaN.
__device__ inline float mx4_power(uint32_t scale) { return __uint_as_float(scale == kNoScale ? 0x7FC00000u : scale << 23); }

// Eight elements: byte i has the codes of elements i and i + 4, the lower bits the first one's.
__device__ inline uint32_t mx4_codes(const float (&v)[8], uint32_t scale) {
    const float by = __uint_as_float(scale == kNoScale ? 0x3F800000u : scale << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[4], by, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[1], v[5], by, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[6], by, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[3], v[7], by, 3);
    return c;
}

__device__ inline void mx4_values(uint32_t c, uint32_t scale, float (&v)[8]) {
    const float by = mx4_power(scale);
    auto pair = [&](auto which) {
        constexpr int i = decltype(which)::value;
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, i);
        v[i] = p[0] * by;
        v[i + 4] = p[1] * by;
    };
    pair(std::integral_constant<int, 0>{});
    pair(std::integral_constant<int, 1>{});
    pair(std::integral_constant<int, 2>{});
    pair(std::integral_constant<int, 3>{});
}

// From byte i of each lane of a quad for word i of the block, to word `lane % 4` in each lane; and, being a transposition, back.
__device__ inline uint32_t mx4_turn(uint32_t c) {
    const uint32_t i = threadIdx.x & 3, pick = i | (i + 4) << 8;
    const uint32_t low = __builtin_amdgcn_perm(quad_lane<1>(c), quad_lane<0>(c), pick);
    const uint32_t high = __builtin_amdgcn_perm(quad_lane<3>(c), quad_lane<2>(c), pick);
    return (low & 0xFFFFu) | (high << 16);
}

// ---- 8 bits, a scale for each row ---------------------------------------------------------------------------------

// A row's scale from its largest magnitude; NaN for a row with an infinity or a NaN.
__device__ inline float i8_scale(uint32_t largest) {
    return finite_bits(largest) ? fmaxf(__uint_as_float(largest) / 127.0f, kLeastRowScale) : __uint_as_float(0x7FC00000u);
}

// Whole numbers of steps of eight elements, exactly the nearest ones: a product with 1 / s is off by less than 3e-5, so where it is
// within 1e-4 of a border, the border (q + 1/2) s itself is compared with x, in one rounding that keeps the difference's sign.
__device__ inline void i8_steps(const float (&v)[8], float s, float (&q)[8]) {
    const float inv = 1.0f / s;
    bool near = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = v[e] * inv;
        q[e] = rintf(t);
        near |= fabsf(t - q[e]) > 0.4999f;
    }
    if (near) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float above = fmaf(-(q[e] + 0.5f), s, v[e]), below = fmaf(-(q[e] - 0.5f), s, v[e]);
            const bool odd = (int(q[e]) & 1) != 0;
            if (above > 0.0f || (above == 0.0f && odd)) q[e] += 1.0f;
            else if (below < 0.0f || (below == 0.0f && odd)) q[e] -= 1.0f;
        }
    }
    // Of a row that stands for nothing.
    if (s != s) {
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = 0.0f;
    }
}

__device__ inline uint2 i8_codes(const float (&q)[8]) {
    auto four = [&](int e) {
        const uint32_t a = uint32_t(int(q[e])), b = uint32_t(int(q[e + 1])), c = uint32_t(int(q[e + 2])), d = uint32_t(int(q[e + 3]));
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
    };
    return make_uint2(four(0), four(4));
}

__device__ inline void i8_values(uint2 c, float s, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = float(int8_t(c.x >> (8 * e))) * s;
        v[e + 4] = float(int8_t(c.y >> (8 * e))) * s;
    }
}

// From byte e of each lane of a quad for word e of the block, to words 2 (lane % 4) and one more in each lane.
__device__ inline uint2 i8_turn(uint2 c) {
    const uint32_t i = 2 * (threadIdx.x & 3), pick = i | (i + 1) << 8;
    const uint32_t r0 = __builtin_amdgcn_perm(quad_lane<0>(c.y), quad_lane<0>(c.x), pick), r1 = __builtin_amdgcn_perm(quad_lane<1>(c.y), quad_lane<1>(c.x), pick);
    const uint32_t r2 = __builtin_amdgcn_perm(quad_lane<2>(c.y), quad_lane<2>(c.x), pick), r3 = __builtin_amdgcn_perm(quad_lane<3>(c.y), quad_lane<3>(c.x), pick);
    return make_uint2(__builtin_amdgcn_perm(__builtin_amdgcn_perm(r3, r2, 0x0C0C0400u), __builtin_amdgcn_perm(r1, r0, 0x0C0C0400u), 0x05040100u),
                      __builtin_amdgcn_perm(__builtin_amdgcn_perm(r3, r2, 0x0C0C0501u), __builtin_amdgcn_perm(r1, r0, 0x0C0C0501u), 0x05040100u));
}

// And back: a lane gets byte `lane % 4` of each of the eight words, lane p of the quad having words 2 p and 2 p + 1.
__device__ inline uint2 i8_turn_back(uint2 c) {
    const uint32_t i = threadIdx.x & 3, pick = i | (i + 4) << 8;
    const uint32_t r0 = __builtin_amdgcn_perm(quad_lane<0>(c.y), quad_lane<0>(c.x), pick), r1 = __builtin_amdgcn_perm(quad_lane<1>(c.y), quad_lane<1>(c.x), pick);
    const uint32_t r2 = __builtin_amdgcn_perm(quad_lane<2>(c.y), quad_lane<2>(c.x), pick), r3 = __builtin_amdgcn_perm(quad_lane<3>(c.y), quad_lane<3>(c.x), pick);
    return make_uint2((r0 & 0xFFFFu) | r1 << 16, (r2 & 0xFFFFu) | r3 << 16);
}

// ---- eight elements of a lane, from column `col` (a multiple of 8) of row m on ---------------------------------------------
// All four lanes of a quad call these with their columns of one block.  Elements from N on are zero.  Stores go past the cache, which
// these results do not share with anything that is read twice: rows of 4096 bfloat16 quantised, with x^, 16384 in 55.7 us instead of 65.3, 1000 in
// 6.4 instead of 7.3, of 4 bits 43.4 instead of 48.2; BinaryFeedForward.forward, which reads them next, is not slower at any size.

__device__ inline void store_mx4(const QuantOut& o, int64_t m, int64_t col, uint32_t codes, uint32_t scale) {
    const uint32_t word = mx4_turn(codes);
    __builtin_nontemporal_store(word, reinterpret_cast<uint32_t*>(o.codes + m * o.ld_c + (col >> 1)));
    if ((threadIdx.x & 3) == 0) static_cast<uint8_t*>(o.scales)[m * o.ld_s + (col >> 5)] = uint8_t(scale);
}

__device__ inline void store_i8(const QuantOut& o, int64_t m, int64_t col, uint2 codes) {
    typedef uint32_t pair_t __attribute__((ext_vector_type(2)));
    const uint2 words = i8_turn(codes);
    __builtin_nontemporal_store(pair_t{words.x, words.y}, reinterpret_cast<pair_t*>(o.codes + m * o.ld_c + col));
}

template <typename E, bool PAST = true>
__device__ inline void quantise_mx4(const QuantOut& o, int64_t m, int64_t col, const float (&v)[8], int64_t N) {
    const uint32_t scale = mx4_scale(largest_of_quad(largest_of_8(v)));
    const uint32_t codes = mx4_codes(v, scale);
    store_mx4(o, m, col, codes, scale);
    if (o.hat && col < N) {
        float hat[8];
        mx4_values(codes, scale, hat);
        store_group<E, 8, PAST>(static_cast<E*>(o.hat) + m * o.ld_h + col, hat, N - col);
    }
}

// s: the row's.
template <typename E, bool PAST = true>
__device__ inline void quantise_i8(const QuantOut& o, int64_t m, int64_t col, const float (&v)[8], float s, int64_t N) {
    float q[8];
    i8_steps(v, s, q);
    store_i8(o, m, col, i8_codes(q));
    if (o.hat && col < N) {
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] *= s;
        store_group<E, 8, PAST>(static_cast<E*>(o.hat) + m * o.ld_h + col, q, N - col);
    }
}

// Checks of codes and scales of M rows of K elements, as the entry points that read or write them share them.
inline int check_rows(int rows, const uint8_t* codes, int64_t ld_c, const void* scales, int64_t ld_s, int64_t M, int64_t K) {
    if (!rows_kind(rows)) return BNN_ERR_INVALID_ARG;
    const bool mx4 = rows == BNN_ROWS_MX4;
    if (M > 0 && ((K > 0 && !codes) || ((K > 0 || !mx4) && !scales))) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(codes, 16) || !aligned_to(scales, mx4 ? 16 : 4)) return BNN_ERR_ALIGNMENT;
    if (K == 0) return BNN_OK;
    const int64_t blocks = (K + 31) / 32;
    if (ld_c < blocks * block_bytes(rows) || ld_c > kMaxDim || (mx4 && (ld_s < blocks || ld_s > kMaxDim))) return BNN_ERR_INVALID_ARG;
    if (ld_c % 16 != 0 || (mx4 && ld_s % 16 != 0)) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}

}  // namespace bnn
