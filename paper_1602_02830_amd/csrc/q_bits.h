// Products of quantised rows (quant_rows.h) with packed +-1 rows: operands of the matrix engine, epilogues, and the form for
// few rows.
//
// Weights move as bits and become operands in registers, a word of 32 weights at a time.  Both kinds of operand have a code whose sign bit
// alone tells it from its negative - 1.0 in 4-bit floats, 64 in whole numbers of 8 bits (0x40 and 0xC0) - so that a shift and one
// operation widen eight or four weights: 7 operations a word of 4-bit codes, 15 of 8-bit ones.  A sign is set where the bit is: operands are
// minus the weights, or minus 64 times them, and who reads the sums puts that right.  Sums of 8-bit codes are whole
// numbers of 32 bits, exact: 64 * 127 * K < 2^31 for K <= 2^18.  Products of 4-bit codes with +-1 are exact too, and the
// matrix engine applies the scales of the 32 elements of a lane to its sums in float32.
//
// (Floats of 8 bits would share the scaled instructions, but their products are added eight at a time aligned to the largest, with
// 11 bits below it: 128 + 0.0703125 gives 128.0625.  That is not a sum of 32 bits; whole numbers are, at the same rate.)
//
// The weights are the first operand, the activations the second: a lane has consecutive channels of one row of the result.
#pragma once

#include "gemm_staging.h"
#include "quant_rows.h"

namespace bnn {

typedef int v4i_t __attribute__((ext_vector_type(4)));
typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef int v16i_t __attribute__((ext_vector_type(16)));
typedef float v4f_t __attribute__((ext_vector_type(4)));

constexpr int64_t kMostI8 = int64_t(1) << 18;        // elements of the longest row of 8-bit codes

struct QProductArgs {
    const uint8_t* codes;      // [M][ld_c]
    const void* scales;        // float [M] or bytes [M][ld_s]
    const uint32_t* w;         // [rows of w][ld_w]
    const float* scale;        // [rows of w] or null
    const float* bias;
    const void* residual;      // linear: [M][ld_r] or null
    void* y;                   // [M][ld_y]; with out.codes null or h^
    QuantOut out;              // gated: codes of 4 bits of the result, or null
    int64_t ld_c, ld_s, ld_w, ld_r, ld_y;
    int M, N, K;               // N: columns of y
    int act, type;
    TileMap map;
};

enum QEpilogue { kQLinear, kQGated };
template <int EPI>
inline constexpr int kQHalves = EPI == kQGated ? 2 : 1;

// What the two kinds of rows differ in.
template <int ROWS>
struct RowsOf;

template <>
struct RowsOf<BNN_ROWS_MX4> {
    typedef float sum_t;
    static constexpr int kQuads = 1;                 // 16-byte pieces of 32 codes
    uint32_t signs = 0x88888888u, ones = 0x22222222u;
    // The constants in registers: with both in sight the compiler makes two operations with literals of the one.
    __device__ inline RowsOf() { asm("" : "+s"(signs), "+v"(ones)); }
    __device__ inline v4i_t operator()(uint32_t w) const {
        return v4i_t{int(((w << 3) & signs) | ones), int(((w << 2) & signs) | ones), int(((w << 1) & signs) | ones), int((w & signs) | ones)};
    }
    __device__ static inline float value(float sum, float) { return -sum; }
};

template <>
struct RowsOf<BNN_ROWS_I8> {
    typedef int sum_t;
    static constexpr int kQuads = 2;
    uint32_t signs = 0x80808080u, ones = 0x40404040u;
    __device__ inline RowsOf() { asm("" : "+s"(signs), "+v"(ones)); }
    // Words 4 * half to 4 * half + 3 of a block's eight.
    __device__ inline v4i_t operator()(uint32_t w, int half) const {
        v4i_t d;
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = int(((w << (7 - 4 * half - i)) & signs) | ones);
        return d;
    }
    __device__ static inline float value(int sum, float s) { return float(sum) * (-1.0f / 64) * s; }
};

__device__ inline v8i_t in_eight(v4i_t f) { return v8i_t{f[0], f[1], f[2], f[3], 0, 0, 0, 0}; }
__device__ inline v4i_t as_ints(uint4 v) { return v4i_t{int(v.x), int(v.y), int(v.z), int(v.w)}; }

constexpr int kFp4 = 4;                  // the matrix instructions' format of 4-bit floats
constexpr int kOne = 0x7F7F7F7F;         // scales of 1

// 16 channels x 16 rows x 128 elements; `scales` has four blocks', BLOCK is the one.
template <int BLOCK>
__device__ inline v4f_t mfma_mx4(v4i_t w, v4i_t x, v4f_t c, uint32_t scales) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, BLOCK, int(scales));
}

// The epilogue of W = 8 or 4 consecutive columns from n on of row m, from their sums (gated: of both halves): what is stored, in
// float32.
template <int EPI, int W, typename V>
__device__ inline void results(const QProductArgs& a, const float (&s)[kQHalves<EPI>][W], const V& scale, const V& bias, float (&v)[W]) {
    float z[W];
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] = fmaf(s[0][i], scale[0][i], bias[0][i]);
    if (a.type == BNN_F32) activate<false, W>(a.act, z, v);
    else activate<true, W>(a.act, z, v);
    if constexpr (EPI == kQGated) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= fmaf(s[1][i], scale[1][i], bias[1][i]);
    }
}

// `valid` of the columns exist.  PAST: stores go past the cache, which a large result does not fit (as are those of q_tiles.h:
// 4096 x 4096 -> 4096 of 8 bits 62 us against 65, 1000 x 784 -> 4096 in float32 12.0 against 13.7; BinaryFeedForward.forward, which reads them
// next, takes as long either way).
template <typename E, int EPI, int W, bool PAST>
__device__ inline void store_results(const QProductArgs& a, int m, int n, float (&v)[W], int64_t valid) {
    if constexpr (EPI == kQLinear) {
        if (a.residual) {
            float r[W];
            load_some<E, W>(static_cast<const E*>(a.residual) + int64_t(m) * a.ld_r + n, valid, r);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] += r[i];
        }
    }
    store_group<E, W, PAST>(static_cast<E*>(a.y) + int64_t(m) * a.ld_y + n, v, valid);
}

// All lanes of a quad that has a block of 32 columns come here together (W = 8).
template <int EPI, int W, bool PAST = false, typename V>
__device__ inline void finish_q(const QProductArgs& a, int m, int n, const float (&s)[kQHalves<EPI>][W], const V& scale, const V& bias) {
    if (m >= a.M) return;
    const int64_t valid = int64_t(a.N) - n;
    float v[W];
    if constexpr (EPI == kQGated && W == 8) {
        if (a.out.codes) {
            if ((n & ~31) >= a.N) return;
            results<EPI, W, V>(a, s, scale, bias, v);
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = i < valid ? v[i] : 0.0f;
            switch (a.type) {
                case BNN_BF16: return quantise_mx4<bf16_t>(a.out, m, n, v, a.N);
                case BNN_F16: return quantise_mx4<f16_t>(a.out, m, n, v, a.N);
                default: return quantise_mx4<float>(a.out, m, n, v, a.N);
            }
        }
    }
    if (valid <= 0) return;
    results<EPI, W, V>(a, s, scale, bias, v);
    switch (a.type) {
        case BNN_BF16: return store_results<bf16_t, EPI, W, PAST>(a, m, n, v, valid);
        case BNN_F16: return store_results<f16_t, EPI, W, PAST>(a, m, n, v, valid);
        default: return store_results<float, EPI, W, PAST>(a, m, n, v, valid);
    }
}

// Scale and bias of channel `row` of w, of a column that exists.
__device__ inline float scale_at(const QProductArgs& a, int64_t row, bool there) { return there && a.scale ? a.scale[row] : 1.0f; }
__device__ inline float bias_at(const QProductArgs& a, int64_t row, bool there) { return there && a.bias ? a.bias[row] : 0.0f; }

// ---- tiles of 16 rows ---------------------------------------------------------------------------------------------
// Every wavefront of a workgroup has the whole tile to itself and runs of 512 elements of K are dealt to them; a quarter of a wavefront
// has four blocks of 32 of a run: 16 bytes of each row of weights, 64 or 128 of each row of codes, all loaded before the first is
// needed.  The sums meet in LDS.

constexpr int kQRunK = 512, kQRows = 16, kQRunBlocks = kQRunK / 32;

// FN blocks of 16 channels (gated: of each half), one or two.
template <int ROWS, int EPI, int FN>
__global__ __launch_bounds__(512) void q_small_kernel(const QProductArgs a) {
    using R = RowsOf<ROWS>;
    using sum_t = typename R::sum_t;
    constexpr int HALVES = kQHalves<EPI>, BLOCKS = FN * HALVES;
    struct alignas(16) Four { sum_t v[4]; };
    extern __shared__ __attribute__((aligned(16))) char part_raw[];       // [wavefront][block][lane]
    Four* const part_s = reinterpret_cast<Four*>(part_raw);
    __shared__ float scale_s[BLOCKS * 16], bias_s[BLOCKS * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int r16 = lane & 15, quarter = lane >> 4, nb = (a.K + 31) >> 5;
    const int m0 = int(blockIdx.y) * kQRows, n0 = int(blockIdx.x) * (16 * FN);

    // Block b: columns n0 + 16 (b % FN) of half b / FN.
    for (int c = tid; c < BLOCKS * 16; c += blockDim.x) {
        const int b = c >> 4, col = n0 + (b % FN) * 16 + (c & 15);
        const int64_t at = int64_t(b / FN) * a.N + col;
        scale_s[c] = scale_at(a, at, col < a.N);
        bias_s[c] = bias_at(a, at, col < a.N);
    }
    const R minus_weights;
    const int64_t m = min(m0 + r16, a.M - 1);
    const uint8_t* const row = a.codes + m * a.ld_c;
    typedef sum_t acc_t __attribute__((ext_vector_type(4)));
    acc_t acc[BLOCKS] = {};
    for (int first = wave * kQRunBlocks; first < nb; first += waves * kQRunBlocks) {
        const int b0 = first + 4 * quarter;          // the lane's blocks: b0 to b0 + 3
        uint4 w[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const uint32_t* const wrow = a.w + (int64_t(b / FN) * a.N + min(n0 + (b % FN) * 16 + r16, a.N - 1)) * a.ld_w;
            if (b0 + 4 <= nb) w[b] = load_quad_any(wrow + b0);
            else w[b] = make_uint4(wrow[min(b0, nb - 1)], wrow[min(b0 + 1, nb - 1)], wrow[min(b0 + 2, nb - 1)], 0u);
        }
        uint4 x[4][R::kQuads];
        const uint4* const p = reinterpret_cast<const uint4*>(row) + int64_t(b0) * R::kQuads;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < R::kQuads; ++q) x[i][q] = b0 + i < nb ? p[i * R::kQuads + q] : make_uint4(0u, 0u, 0u, 0u);
        uint32_t powers = kOne;
        if constexpr (ROWS == BNN_ROWS_MX4) {
            // Bytes of blocks that are not there may be anything: a scale of 1 for their zeros.
            if (b0 < nb) powers = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.scales) + m * a.ld_s + b0);
            const int left = nb - b0;
            const uint32_t keep = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
            powers = (powers & keep) | (kOne & ~keep);
        }
        auto step = [&](auto which) {
            constexpr int i = decltype(which)::value;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const uint32_t word = i == 0 ? w[b].x : i == 1 ? w[b].y : i == 2 ? w[b].z : w[b].w;
                if constexpr (ROWS == BNN_ROWS_MX4) {
                    acc[b] = mfma_mx4<i>(minus_weights(word), as_ints(x[i][0]), acc[b], powers);
                } else {
                    acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(minus_weights(word, 0), as_ints(x[i][0]), acc[b], 0, 0, 0);
                    acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(minus_weights(word, 1), as_ints(x[i][1]), acc[b], 0, 0, 0);
                }
            }
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }
    // Lane: columns 4 quarter .. 4 quarter + 3 of row r16 of each block.
    if (m0 + r16 < a.M) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) part_s[(wave * BLOCKS + b) * 64 + lane] = Four{{acc[b][0], acc[b][1], acc[b][2], acc[b][3]}};
    }
    __syncthreads();
    if (wave != 0) return;
    // One block: a lane has four columns of a row, two: eight, and a quad 32 of them.
    constexpr int W = 4 * FN, PARTS = W / 4;
    const int mr = FN == 1 ? r16 : lane >> 2, c0 = FN == 1 ? 4 * quarter : 8 * (lane & 3);
    if (m0 + mr >= a.M) return;
    const float s_row = ROWS == BNN_ROWS_I8 && a.K > 0 ? static_cast<const float*>(a.scales)[m0 + mr] : 0.0f;
    float s[HALVES][W];
    const float *scale[HALVES], *bias[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        scale[h] = scale_s + h * FN * 16 + c0;
        bias[h] = bias_s + h * FN * 16 + c0;
        sum_t sum[W] = {};
        for (int v = 0; v < waves; ++v)
#pragma unroll
            for (int q = 0; q < PARTS; ++q) {
                const int c = c0 + 4 * q;
                const Four f = part_s[(v * BLOCKS + h * FN + (c >> 4)) * 64 + mr + 16 * ((c >> 2) & 3)];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[4 * q + e] += f.v[e];
            }
#pragma unroll
        for (int i = 0; i < W; ++i) s[h][i] = a.K > 0 ? R::value(sum[i], s_row) : 0.0f;
    }
    finish_q<EPI, W>(a, m0 + mr, n0 + c0, s, scale, bias);
}

template <int ROWS, int EPI, int FN>
int launch_q_small(QProductArgs a, hipStream_t s) {
    const int64_t blocks = ceil_div(a.N, 16 * FN), runs = ceil_div(a.K, kQRunK);
    const int waves = int(runs >= 8 ? 8 : runs < 1 ? 1 : runs);
    const size_t lds = size_t(waves) * FN * kQHalves<EPI> * 1024;
    // As many rows at a time as a grid has places for.
    const int64_t most = max_blocks(64 * waves) / blocks < 65535 ? max_blocks(64 * waves) / blocks : 65535, M = a.M;
    const int64_t size = type_bytes(a.type);
    if (most < 1) return BNN_ERR_UNSUPPORTED;
    for (int64_t first = 0; first < M; first += most * kQRows) {
        QProductArgs part = a;
        part.M = int(M - first < most * kQRows ? M - first : most * kQRows);
        if (first > 0) {
            auto move = [&](auto& p, int64_t bytes) {
                if (p) p = reinterpret_cast<std::decay_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + uintptr_t(first * bytes));
            };
            move(part.codes, a.ld_c);
            move(part.scales, ROWS == BNN_ROWS_I8 ? 4 : a.ld_s);
            move(part.residual, a.ld_r * size);
            move(part.y, a.ld_y * size);
            move(part.out.codes, a.out.ld_c);
            move(part.out.scales, a.out.ld_s);
            move(part.out.hat, a.out.ld_h * size);
        }
        q_small_kernel<ROWS, EPI, FN><<<dim3(uint32_t(blocks), uint32_t(ceil_div(part.M, kQRows))), dim3(64 * waves), lds, s>>>(part);
        const int st = check_launch();
        if (st != BNN_OK) return st;
    }
    return BNN_OK;
}

}  // namespace bnn
