// The product of real rows with packed +-1 rows, s[m][n] = sum_k x[m][k] w[n][k], as tiles of the matrix engine, and what
// its epilogues make of the sums while they are in registers.
//
// Each word of 32 weights becomes operands of 16-bit floats in registers (minus_weights in real_types.h), so weights move
// through memory and caches as bits and are never stored wider; the activations go through LDS, float32 ones as three
// bfloat16 terms whose sum they are, which makes the product as exact as a float32 one.  K is taken in steps of 64: the
// two halves of a wavefront take one word each of every weight row, and the activations' eight-element chunks in the same order.
//
// The MFMA's first operand are the weights, its second the activations: accumulator register i of lane l is column (m)
// l % 32 and, with the weight rows dealt to the lanes by consecutive_rows, output channel 16 (l / 32) + i of its block:
// a lane has 16 consecutive results of one row.
#pragma once

#include "gemm_staging.h"
#include "real_types.h"

namespace bnn {

struct ProductArgs {
    const void* x;             // [M][ld_x]
    const uint32_t* w;         // [rows of w][ld_w]
    const float* scale;        // [rows of w] or null
    const float* bias;
    const void* residual;      // linear: [M][ld_r] or null
    void* y;                   // [M][ld_y]
    const void* dy;            // backward: [M][ld_dy]
    float* part_scale;         // backward: sums over each tile's rows of dz * s and of dz, [tiles_m][channels], or null
    float* part_bias;
    int64_t ld_x, ld_w, ld_r, ld_y, ld_dy;
    int M, N, K;               // N: columns of y that exist (gated: F)
    int half;                  // gated backward: distance of the two halves' columns in y
    int channels;              // backward: rows of w
    int act;
    TileMap map;
};

enum Epilogue {
    kLinear,            // y = act(scale s + bias) + residual
    kGated,             // y = act(z gate) * z up
    kLinearBack,        // y = scale * dy * act'(z), and the partial sums
    kGatedBack          // the same for both halves
};

constexpr int kStepK = 64;          // elements of K a step

// TN wavefronts along the channels, TM along the rows, 32-row blocks FN x FM for each.
template <typename E, int EPI, int TM, int TN, int FM, int FN>
struct ProductTile {
    static constexpr bool kGatedForm = EPI == kGated || EPI == kGatedBack;
    static constexpr int kThreads = 64 * TM * TN;
    static constexpr int BM = 32 * TM * FM;
    static constexpr int CN = 32 * TN * FN;                       // channels: rows of w of a tile
    static constexpr int BN = kGatedForm ? CN / 2 : CN;           // columns of a tile of y
    static constexpr int kTerms = is_f32<E> ? 3 : 1;
    static constexpr int kChunks = BM * (kStepK / 8) / kThreads;  // chunks of eight elements that a thread stages
};

template <typename E, int EPI, int TM, int TN, int FM, int FN>
__global__ __launch_bounds__(64 * TM * TN) void bits_product_kernel(const ProductArgs a) {
    using S = ProductTile<E, EPI, TM, TN, FM, FN>;
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    constexpr bool FAST = !is_f32<E>;
    constexpr bool GATED = S::kGatedForm, BACK = EPI == kLinearBack || EPI == kGatedBack;
    __shared__ __attribute__((aligned(16))) O8 xs[2][S::kTerms][S::BM * 8];      // rows of 8 chunks, slot = chunk ^ row % 8
    __shared__ float scale_s[S::CN], bias_s[S::CN];
    __shared__ float sums_s[BACK ? 2 * TM * S::CN : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wn = wave % TN, wm = wave / TN, fr = lane & 31, fh = lane >> 5;
    int tm, tn;
    tile_of_block(blockIdx.x, a.map, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN;
    const int kw = (a.K + 31) >> 5;

    // Channel c of the tile (0 .. CN) is row channel_row(c) of w, or none.  A wavefront's blocks of the gated form are
    // FN / 2 of the gate's rows, then the same columns of the other half.
    auto block_col = [&](int f) { return n0 + (GATED ? wn * (16 * FN) + (f % (FN / 2 > 0 ? FN / 2 : 1)) * 32 : (wn * FN + f) * 32); };
    auto block_half = [&](int f) { return GATED && f >= FN / 2 ? 1 : 0; };

    for (int c = tid; c < S::CN; c += S::kThreads) {
        const int b = c >> 5, w_ = b / FN, f = b % FN;
        const int col = n0 + (GATED ? w_ * (16 * FN) + (f % (FN / 2 > 0 ? FN / 2 : 1)) * 32 : b * 32) + (c & 31);
        const int64_t row = int64_t(GATED && f >= FN / 2 ? a.N : 0) + col;
        const bool there = col < a.N;
        scale_s[c] = there && a.scale ? a.scale[row] : 1.0f;
        bias_s[c] = there && a.bias ? a.bias[row] : 0.0f;
    }

    const uint32_t* wrow[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f) {
        const int col = min(block_col(f) + consecutive_rows(fr), a.N - 1);          // a column that is not there: the last one
        wrow[f] = a.w + (int64_t(block_half(f)) * a.N + col) * a.ld_w;
    }

    const E* xrow[S::kChunks];
    bool row_there[S::kChunks];
#pragma unroll
    for (int i = 0; i < S::kChunks; ++i) {
        const int id = i * S::kThreads + tid, m = m0 + (id >> 3);
        row_there[i] = m < a.M;
        xrow[i] = static_cast<const E*>(a.x) + int64_t(min(m, a.M - 1)) * a.ld_x + (id & 7) * 8;
    }

    typename Vec8<E>::type stage[S::kChunks];
    uint32_t wnext[FN];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int c8 = ((i * S::kThreads + tid) & 7) * 8;
            stage[i] = load8<E>(xrow[i] + k0, row_there[i] ? int64_t(a.K) - k0 - c8 : 0);
        }
#pragma unroll
        for (int f = 0; f < FN; ++f) wnext[f] = wrow[f][min((k0 >> 5) + fh, kw - 1)];
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int id = i * S::kThreads + tid, row = id >> 3, slot = (id & 7) ^ (row & 7);
            if constexpr (is_f32<E>) {
                O8 t[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t part[3];
                    split3(stage[i][e], part);
                    t[0][e] = part[0];
                    t[1][e] = part[1];
                    t[2][e] = part[2];
                }
#pragma unroll
                for (int p = 0; p < 3; ++p) xs[buf][p][row * 8 + slot] = t[p];
            } else {
                xs[buf][0][row * 8 + slot] = stage[i];
            }
        }
    };

    v16f_t acc[FN][FM] = {};
    if (a.K > 0) {
        load(0);
        store(0);
    }
    for (int k0 = 0, buf = 0; k0 < a.K; k0 += kStepK, buf ^= 1) {
        uint32_t w[FN];
#pragma unroll
        for (int f = 0; f < FN; ++f) w[f] = wnext[f];
        __syncthreads();
        const bool more = k0 + kStepK < a.K;
        if (more) load(k0 + kStepK);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            O8 wf[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) wf[f] = minus_weights<O>(s < 2 ? spread_low(w[f]) : spread_high(w[f]), s & 1);
#pragma unroll
            for (int p = 0; p < S::kTerms; ++p)
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    const int row = (wm * FM + j) * 32 + fr;
                    const O8 xf = xs[buf][p][row * 8 + ((4 * fh + s) ^ (row & 7))];
#pragma unroll
                    for (int f = 0; f < FN; ++f) acc[f][j] = mfma16(wf[f], xf, acc[f][j]);
                }
        }
        if (more) store(buf ^ 1);
    }
    __syncthreads();

    // ---- epilogue: lane l has columns 16 fh .. 16 fh + 15 of row fr of each block ----
    E* const y = static_cast<E*>(a.y);
    if constexpr (EPI == kLinear) {
        const E* const residual = static_cast<const E*>(a.residual);
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            const int c0 = (wn * FN + f) * 32 + 16 * fh, n = block_col(f) + 16 * fh;
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = m0 + (wm * FM + j) * 32 + fr;
                if (m >= a.M || n >= a.N) continue;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int64_t valid = int64_t(a.N) - n - 8 * g;
                    typename Vec8<E>::type r = {};
                    if (residual) r = load8<E>(residual + int64_t(m) * a.ld_r + n + 8 * g, valid);
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = activate<FAST>(a.act, fmaf(-acc[f][j][8 * g + i], scale_s[c0 + 8 * g + i], bias_s[c0 + 8 * g + i])) + float(r[i]);
                    store8<E>(y + int64_t(m) * a.ld_y + n + 8 * g, v, valid);
                }
            }
        }
    } else if constexpr (EPI == kGated) {
#pragma unroll
        for (int f = 0; f < FN / 2; ++f) {
            const int cg = (wn * FN + f) * 32 + 16 * fh, cu = cg + 16 * FN, n = block_col(f) + 16 * fh;
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = m0 + (wm * FM + j) * 32 + fr;
                if (m >= a.M || n >= a.N) continue;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int e = 8 * g + i;
                        const float zg = fmaf(-acc[f][j][e], scale_s[cg + e], bias_s[cg + e]);
                        const float zu = fmaf(-acc[f + FN / 2][j][e], scale_s[cu + e], bias_s[cu + e]);
                        v[i] = activate<FAST>(a.act, zg) * zu;
                    }
                    store8<E>(y + int64_t(m) * a.ld_y + n + 8 * g, v, int64_t(a.N) - n - 8 * g);
                }
            }
        }
    } else {
        const E* const dy = static_cast<const E*>(a.dy);
        constexpr int HALVES = GATED ? 2 : 1, FY = FN / HALVES;
#pragma unroll
        for (int f = 0; f < FY; ++f) {
            const int c0 = (wn * FN + f) * 32 + 16 * fh, n = block_col(f) + 16 * fh;
            float sum_s[HALVES][16] = {}, sum_z[HALVES][16] = {};
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int m = m0 + (wm * FM + j) * 32 + fr;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int64_t valid = m < a.M ? int64_t(a.N) - n - 8 * g : 0;
                    const auto d = load8<E>(dy + int64_t(min(m, a.M - 1)) * a.ld_dy + n + 8 * g, valid);
                    float out[HALVES][8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int e = 8 * g + i;
                        const float s0 = -acc[f][j][e], z0 = fmaf(s0, scale_s[c0 + e], bias_s[c0 + e]);
                        float act, slope, dz[HALVES], s[HALVES];
                        activate_both<FAST>(a.act, z0, act, slope);
                        s[0] = s0;
                        if constexpr (GATED) {
                            const int cu = c0 + 16 * FN + e;
                            s[1] = -acc[f + FN / 2][j][e];
                            dz[0] = float(d[i]) * fmaf(s[1], scale_s[cu], bias_s[cu]) * slope;
                            dz[1] = float(d[i]) * act;
                        } else {
                            dz[0] = float(d[i]) * slope;
                        }
#pragma unroll
                        for (int h = 0; h < HALVES; ++h) {
                            // What is not there counts nothing, whatever its sums are.
                            dz[h] = i < valid ? dz[h] : 0.0f;
                            out[h][i] = i < valid ? dz[h] * scale_s[c0 + 16 * FN * h + e] : 0.0f;
                            sum_s[h][e] += i < valid ? dz[h] * s[h] : 0.0f;
                            sum_z[h][e] += dz[h];
                        }
                    }
                    if (m < a.M && n < a.half)         // columns from N up to `half` are written as zeros
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
                            store8<E>(y + int64_t(m) * a.ld_y + int64_t(h) * a.half + n + 8 * g, out[h], 8);
                }
            }
            // Over the 32 rows of the lanes of each half, then over the wavefronts of the same columns.
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float p = sum_s[h][e], q = sum_z[h][e];
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) {
                        p += __shfl_xor(p, off);
                        q += __shfl_xor(q, off);
                    }
                    if (fr == 0) {
                        const int c = c0 + 16 * FN * h + e;
                        sums_s[(wm * 2) * S::CN + c] = p;
                        sums_s[(wm * 2 + 1) * S::CN + c] = q;
                    }
                }
        }
        __syncthreads();
        for (int c = tid; c < S::CN; c += S::kThreads) {
            const int b = c >> 5, w_ = b / FN, f = b % FN;
            const int col = n0 + (GATED ? w_ * (16 * FN) + (f % FY) * 32 : b * 32) + (c & 31);
            if (col >= a.N) continue;
            float p = 0.0f, q = 0.0f;
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                p += sums_s[(t * 2) * S::CN + c];
                q += sums_s[(t * 2 + 1) * S::CN + c];
            }
            const int64_t at = int64_t(tm) * a.channels + (GATED && f >= FY ? a.N : 0) + col;
            if (a.part_scale) a.part_scale[at] = p;
            if (a.part_bias) a.part_bias[at] = q;
        }
    }
}

}  // namespace bnn
