// The power of two by which float16 gradients are multiplied while they lie in memory.
//
// Backward passes round ds = scale * dz to 16 bits between the product that makes it and the two that read it.  A channel's scale
// is about 1 / sqrt(K): gradients that float16 holds as normal numbers, and whose dx and dw it holds too, have a ds among
// its subnormals (stored as it is, 512 to 4096 channels with a scale of 1/64: dx 0.2 - 1 % off for dy of 1e-3, 2 - 11 % for 1e-4, 15 - 90 %
// for 1e-5).  So ds is stored times 2^e and the float32 sums of dx and dw are divided by it again.  e follows from a bound of |ds|,
// made of the largest finite magnitudes of dy, x, scale and bias:
//
//   linear:  |ds| <= max|dy| 1.2 max|scale|                                         (slopes of all activations are below 1.2)
//   gated:   |ds| <= max over rows m of |dh_m| max(1.2 Z_m, 1 for a sigmoid) max|scale|,  Z_m = max|scale| sum_k |x_mk| + max|bias| >= |z_m|
//
// 2^e brings the bound to between 2^14 and 2^15, half of float16's largest and 2^28 above its smallest normal number.  The bound is loose, for
// Gaussian operands of 4096 columns by about 2^9; with outliers a thousand times as large in some rows of x and of dh, the other rows' ds are
// normal numbers still (with max|x| K in the place of the row's sum they were not, and lost digits).  bfloat16 has float32's exponents and needs
// none of it.  Powers of two change no digit of a normal number.  Looking costs a pass over dy, gated over x too, beside the transposition of
// the weights: 500 x 784 -> 2 x 1531 43.2 us with it and 40.4 without, 3762 x 911 -> 2 x 256 68.8 and 63.0.
#pragma once

#include "real_types.h"

namespace bnn {

// The largest finite magnitudes: of the scale (1 without one), of the bias, then what each workgroup found that looked at rows of dy, and
// (gated) what each found of a row's dy times the sum of its x.
struct GradientBounds {
    const float* parts;
    int lookers;               // workgroups; 0: ds is stored as it is
};

constexpr int kMostLookers = 256;
constexpr int kMostBoundParts = 2 + 2 * kMostLookers;

// |v|, or 0 where that is infinite or no number: such an element spoils what it reaches at any factor, and must not spoil the rest.
__device__ inline float finite_magnitude(float v) {
    const float a = __builtin_fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}

// What `join` makes of the values of each aligned group of 8, 16, 32 or 64 lanes, in every lane of it, by lane permutes.
template <typename F>
__device__ inline float over_group(float v, int lanes, F&& join) {
    auto from = [&](auto control) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xF, 0xF, true));
    };
    v = join(v, from(std::integral_constant<int, 0xB1>{}));       // quad_perm [1,0,3,2]
    v = join(v, from(std::integral_constant<int, 0x4E>{}));       // quad_perm [2,3,0,1]
    v = join(v, from(std::integral_constant<int, 0x141>{}));      // row_half_mirror
    if (lanes >= 16) v = join(v, from(std::integral_constant<int, 0x140>{}));      // row_mirror
    if (lanes >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if (lanes >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = join(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}

__device__ inline float largest_of_wave(float m) {
    return over_group(m, 64, [](float a, float b) { return fmaxf(a, b); });
}

// The factor in two halves: loads that go out before a kernel's others do, and the factor, the same in every lane, of what they bring.
// All lanes of the wavefront take part in both.
template <bool GATED>
class StoredFactor {
    static constexpr int kLoads = kMostLookers / 64;
    float scale = 1.0f, bias = 0.0f, dy[kLoads] = {}, both[GATED ? kLoads : 1] = {};

public:
    __device__ inline explicit StoredFactor(const GradientBounds& b) {
        if (b.lookers == 0) return;
        const int lane = threadIdx.x & 63;
        scale = b.parts[0];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) dy[i] = b.parts[2 + min(lane + 64 * i, b.lookers - 1)];
        if constexpr (GATED) {
            bias = b.parts[1];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) both[i] = b.parts[2 + b.lookers + min(lane + 64 * i, b.lookers - 1)];
        }
    }
    __device__ inline float operator()(int act) const {
        float most_dy = dy[0];
#pragma unroll
        for (int i = 1; i < kLoads; ++i) most_dy = fmaxf(most_dy, dy[i]);
        most_dy = largest_of_wave(most_dy);
        float bound = 1.2f * most_dy * scale;
        if constexpr (GATED) {
            float most = both[0];
#pragma unroll
            for (int i = 1; i < kLoads; ++i) most = fmaxf(most, both[i]);
            bound = 1.2f * (scale * largest_of_wave(most) + bias * most_dy);
            if (act == BNN_ACT_SIGMOID) bound = fmaxf(bound, most_dy);
            bound *= scale;
        }
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

// What a lane has of the magnitudes of a row that `lanes` neighbouring lanes (a power of two, 8 at least) take together: the largest, or the
// sum, of the finite ones.  Four groups of eight elements are on their way at once; load() and take() apart let two rows' be.
template <typename E, bool SUM>
struct RowMagnitude {
    const E* row;
    int groups, lane, lanes;
    E end;                     // an element past the last whole group
    float m = 0.0f;
    typename Vec8<E>::type v[4];
    __device__ inline RowMagnitude(const E* p, int cols, int l, int n) : row(p), groups(cols / 8), lane(l), lanes(n), end(E(0.0f)) {
        if (8 * groups + l < cols) end = p[8 * groups + l];
    }
    __device__ inline void load(int first) {           // groups from `first` on; those that are not there: the last one
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const typename Vec8<E>::any*>(row + 8 * int64_t(min(first + lane + i * lanes, groups - 1)));
    }
    __device__ inline void add(float magnitude) { m = SUM ? m + magnitude : fmaxf(m, magnitude); }
    __device__ inline void take(int first) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float of = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) of = SUM ? of + __builtin_fabsf(float(v[i][e])) : fmaxf(of, __builtin_fabsf(float(v[i][e])));
            if (!(of < __builtin_inff())) {             // an element is infinite or no number: without it
                of = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) of = SUM ? of + finite_magnitude(float(v[i][e])) : fmaxf(of, finite_magnitude(float(v[i][e])));
            }
            add(first + lane + i * lanes < groups ? of : 0.0f);
        }
    }
    __device__ inline float over_lanes() {
        add(finite_magnitude(float(end)));
        return over_group(m, lanes, [](float a, float b) { return SUM ? a + b : fmaxf(a, b); });
    }
};

template <typename E>
__device__ inline float largest_of_row(const E* p, int cols, int lane, int lanes) {
    RowMagnitude<E, false> r(p, cols, lane, lanes);
    for (int first = 0; first < r.groups; first += 4 * lanes) {
        r.load(first);
        r.take(first);
    }
    return r.over_lanes();
}

}  // namespace bnn
