// The power of two by which float16 gradients are multiplied while they lie in memory.
//
// Backward passes round ds = scale * dz to 16 bits between the product that makes it and the two that read it.  A channel's scale
// is about 1 / sqrt(K): gradients that float16 holds as normal numbers, and whose dx and dw it holds too, have a ds among
// its subnormals (stored as it is, 512 to 4096 channels with a scale of 1/64: dx 0.2 - 1 % off for dy of 1e-3, 2 - 11 % for 1e-4, 15 - 90 %
// for 1e-5).  So ds is stored times 2^e and the float32 sums of dx and dw are divided by it again.  e follows from a bound of |ds|,
// made of the largest finite magnitudes of dy, x, scale and bias:
//
//   linear:  |ds| <= max|dy| 1.2 max|scale|                                         (slopes of all activations are below 1.2)
//   gated:   |ds| <= max|dh| max(1.2 Z, 1 for a sigmoid) max|scale|,  Z = max|scale| K max|x| + max|bias| >= |z|
//
// 2^e brings the bound to between 2^14 and 2^15, half of float16's largest and 2^28 above its smallest normal number.  The bound is loose,
// for Gaussian operands by 2^6 to 2^12 and with outliers by 2^10 more; what it leaves is still normal, or rounded to 2^-24 of values of
// 2^-12.  bfloat16 has float32's exponents and needs none of it.  Looking costs a pass over dy, gated over x too, beside the transposition of
// the weights: 500 x 784 -> 2 x 1531 42.0 us with it and 40.4 without, 3762 x 911 -> 2 x 256 66.5 and 63.0.
#pragma once

#include "real_types.h"

namespace bnn {

// The largest finite magnitudes: of the scale (1 without one), of the bias, then what each workgroup found that looked at dy, and at x.
struct GradientBounds {
    const float* parts;
    int of_dy, of_x;           // workgroups; of_dy == 0: ds is stored as it is
};

constexpr int kMostLookers = 256;       // workgroups that look at one of the matrices
constexpr int kMostBoundParts = 2 + 2 * kMostLookers;

// |v|, or 0 where that is infinite or no number: such an element spoils what it reaches at any factor, and must not spoil the rest.
__device__ inline float finite_magnitude(float v) {
    const float a = __builtin_fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}

__device__ inline float largest_of_wave(float m) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    return m;
}

// The factor in two halves: loads that go out before a kernel's others do, and the factor, the same in every lane, of what they bring.
// All lanes of the wavefront take part in both.
template <bool GATED>
class StoredFactor {
    static constexpr int kLoads = kMostLookers / 64;
    float scale = 1.0f, bias = 0.0f, dy[kLoads] = {}, x[GATED ? kLoads : 1] = {};

public:
    __device__ inline explicit StoredFactor(const GradientBounds& b) {
        if (b.of_dy == 0) return;
        const int lane = threadIdx.x & 63;
        scale = b.parts[0];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) dy[i] = b.parts[2 + min(lane + 64 * i, b.of_dy - 1)];
        if constexpr (GATED) {
            bias = b.parts[1];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) x[i] = b.parts[2 + b.of_dy + min(lane + 64 * i, b.of_x - 1)];
        }
    }
    __device__ inline float operator()(int K, int act) const {
        float bound = dy[0], z = 1.2f;
#pragma unroll
        for (int i = 1; i < kLoads; ++i) bound = fmaxf(bound, dy[i]);
        if constexpr (GATED) {
            float xs = x[0];
#pragma unroll
            for (int i = 1; i < kLoads; ++i) xs = fmaxf(xs, x[i]);
            z = 1.2f * (scale * (float(K) * largest_of_wave(xs)) + bias);
            if (act == BNN_ACT_SIGMOID) z = fmaxf(z, 1.0f);
        }
        bound = largest_of_wave(bound) * z * scale;
        if (!(bound > 0.0f && bound < __builtin_inff())) return 1.0f;
        const int e = 14 - (int(__float_as_uint(bound) >> 23) - 127);
        return __uint_as_float(uint32_t(127 + min(max(e, -100), 100)) << 23);
    }
};

// One over the factor, once for each channel of a product that reads stored gradients.  By all workgroups together, one along y.
__device__ inline void leave_units(float* units, int count, float factor) {
    if (blockIdx.y != 0) return;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < count; i += int64_t(gridDim.x) * blockDim.x) units[i] = 1.0f / factor;
}

// The largest finite magnitude of the groups of eight elements from `first` on, `step` apart, counted row by row.
template <typename E>
__device__ inline float largest_of_matrix(const E* p, int64_t ld, int64_t rows, int cols, uint32_t first, uint32_t step) {
    const uint32_t per_row = uint32_t(cols + 7) / 8;
    float m = 0.0f;
    int64_t row = first / per_row;
    uint32_t c = first % per_row;
    const uint32_t rows_on = step / per_row, on = step % per_row;
    while (row < rows) {
        typename Vec8<E>::type v[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // The row's end from its last eight elements: some are looked at twice.
            const int at = min(int(c * 8), max(cols - 8, 0));
            if (row < rows) v[i] = load8<E>(p + row * ld + at, cols - at);
            row += rows_on;
            c += on;
            if (c >= per_row) {
                c -= per_row;
                ++row;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_magnitude(float(v[i][e])));
    }
    return m;
}

}  // namespace bnn
