// The product of real rows with packed +-1 rows, s[m][n] = sum_k x[m][k] w[n][k], as tiles of the matrix engine, and what
// its epilogues make of the sums while they are in registers.
//
// Each word of 32 weights becomes operands of 16-bit floats in registers (Widening in real_types.h), so weights move
// through memory and caches as bits and are never stored wider; the activations go through LDS, float32 ones as three
// bfloat16 terms whose sum they are, which makes the product as exact as a float32 one.  K is taken in steps of 64: the
// two halves of a wavefront take one word each of every weight row, and the activations' eight-element chunks in the same order.
//
// The MFMA's first operand are the weights, its second the activations: accumulator register i of lane l is column (m)
// l % 32 and, with the weight rows dealt to the lanes by consecutive_rows, output channel 16 (l / 32) + i of its block:
// a lane has 16 consecutive results of one row.
#pragma once

#include "gemm_staging.h"
#include "stored_gradient.h"

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

// What backward passes have besides, so that forward calls, which wait for their arguments too, have no more of them.
struct BackwardArgs : ProductArgs {
    GradientBounds bounds;     // float16: what ds is multiplied with follows from them
    float* units;              // [units_count] get one over that factor: the scale of the products that read ds
    int units_count;
};

enum Epilogue {
    kLinear,            // y = act(scale s + bias) + residual
    kGated,             // y = act(z gate) * z up
    kLinearBack,        // y = scale * dy * act'(z), and the partial sums
    kGatedBack          // the same for both halves
};

constexpr int kStepK = 64;          // elements of K a step

template <int EPI>
inline constexpr int kHalves = EPI == kGated || EPI == kGatedBack ? 2 : 1;
template <int EPI>
inline constexpr bool kBackward = EPI == kLinearBack || EPI == kGatedBack;

template <int EPI>
using ArgsOf = typename std::conditional<kBackward<EPI>, BackwardArgs, ProductArgs>::type;

// The epilogue of W = 8 (or 4) consecutive columns from n on of row m, from their sums (gated: of both halves).  scale, bias: of
// the columns of each half.  Backwards, ds is stored times `factor`, and sum_s and sum_z grow by dz * s and dz.
template <typename E, int EPI, int W>
__device__ inline void finish(const ProductArgs& a, int m, int n, const float (&s)[kHalves<EPI>][W], const float* const (&scale)[kHalves<EPI>],
                              const float* const (&bias)[kHalves<EPI>], float factor, float (&sum_s)[kHalves<EPI>][W], float (&sum_z)[kHalves<EPI>][W]) {
    constexpr bool FAST = !is_f32<E>;
    constexpr int HALVES = kHalves<EPI>;
    E* const y = static_cast<E*>(a.y) + int64_t(m) * a.ld_y + n;
    const int64_t valid = int64_t(a.N) - n;
    if (m >= a.M) return;
    if constexpr (EPI == kLinear) {
        if (valid <= 0) return;
        float r[W] = {}, z[W], v[W];
        if (a.residual) load_some<E, W>(static_cast<const E*>(a.residual) + int64_t(m) * a.ld_r + n, valid, r);
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] = fmaf(s[0][i], scale[0][i], bias[0][i]);
        activate<FAST, W>(a.act, z, v);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += r[i];
        store_group<E, W>(y, v, valid);
    } else if constexpr (EPI == kGated) {
        if (valid <= 0) return;
        float z[W], v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] = fmaf(s[0][i], scale[0][i], bias[0][i]);
        activate<FAST, W>(a.act, z, v);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= fmaf(s[1][i], scale[1][i], bias[1][i]);
        store_group<E, W>(y, v, valid);
    } else {
        if (n >= a.half) return;
        float d[W], z[W], f[W], slope[W], out[HALVES][W];
        load_some<E, W>(static_cast<const E*>(a.dy) + int64_t(m) * a.ld_dy + n, valid, d);
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] = fmaf(s[0][i], scale[0][i], bias[0][i]);
        activate_both<FAST, W>(a.act, z, f, slope);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float dz[HALVES];
            if constexpr (HALVES == 2) {
                dz[0] = d[i] * fmaf(s[1][i], scale[1][i], bias[1][i]) * slope[i];
                dz[1] = d[i] * f[i];
            } else {
                dz[0] = d[i] * slope[i];
            }
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                // A column that is not there counts nothing, whatever its sums are.
                out[h][i] = i < valid ? dz[h] * scale[h][i] * factor : 0.0f;
                sum_s[h][i] += i < valid ? dz[h] * s[h][i] : 0.0f;
                sum_z[h][i] += i < valid ? dz[h] : 0.0f;
            }
        }
        // Columns from N up to `half` are written as zeros.
#pragma unroll
        for (int h = 0; h < HALVES; ++h) store_group<E, W>(y + int64_t(h) * a.half, out[h], W);
    }
}

// The factor of stored gradients, in the two halves of StoredFactor; the workgroups leave one over it for the products that read them.
template <bool STORED, bool GATED>
struct Factor {
    StoredFactor<GATED> of;
    __device__ inline explicit Factor(const BackwardArgs& a) : of(a.bounds) {}
    __device__ inline float operator()(const BackwardArgs& a) const {
        const float factor = of(a.act);
        leave_units(a.units, a.units_count, factor);
        return factor;
    }
};
template <bool GATED>
struct Factor<false, GATED> {
    __device__ inline explicit Factor(const ProductArgs&) {}
    __device__ inline float operator()(const ProductArgs&) const { return 1.0f; }
};
template <typename E, int EPI>
using FactorOf = Factor<std::is_same<E, f16_t>::value && kBackward<EPI>, EPI == kGatedBack>;

// TN wavefronts along the channels, TM along the rows, 32-row blocks FN x FM for each.
template <typename E, int EPI, int TM, int TN, int FM, int FN>
struct ProductTile {
    static constexpr bool kGatedForm = EPI == kGated || EPI == kGatedBack;
    static constexpr int kThreads = 64 * TM * TN;
    static constexpr int BM = 32 * TM * FM;
    static constexpr int CN = 32 * TN * FN;                       // channels: rows of w of a tile
    static constexpr int BN = kGatedForm ? CN / 2 : CN;           // columns of a tile of y
    static constexpr int kTerms = is_f32<E> ? 3 : 1;
    // Three buffers let a wavefront run on from step to step, with the barrier in the middle; float32 rows have room for two.
    static constexpr int kBuffers = is_f32<E> && BM > 64 ? 2 : 3;
    static constexpr int HALVES = kHalves<EPI>, FY = FN / HALVES;
    struct Loop {
        typename Vec8<Operand<E>>::type x[kBuffers][kTerms][BM * 8];      // rows of 8 chunks, chunk c of a row at c ^ (row / 2) % 8
        uint4 w[2][4][CN];           // 512 elements of each weight row, 16 bytes of a row at a time
    };
    struct Sums {
        float4 block[TM * TN][HALVES][32 * 8];      // a wavefront's own: 32 rows of 32 columns, placed like x
    };
    union Shared {
        __device__ Shared() {}
        Loop loop;
        Sums sums;
    };
    static constexpr int kChunks = BM * (kStepK / 8) / kThreads;  // chunks of eight elements that a thread stages
};

template <typename E, int EPI, int TM, int TN, int FM, int FN, bool FAR = false>
__global__ __launch_bounds__(64 * TM * TN) void bits_product_kernel(const ArgsOf<EPI> a) {
    using S = ProductTile<E, EPI, TM, TN, FM, FN>;
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    constexpr bool GATED = S::kGatedForm, BACK = kBackward<EPI>;
    __shared__ typename S::Shared shared;
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

    constexpr int WQ = 4 * S::CN / S::kThreads;        // 16-byte pieces of weights that a thread stages
    const uint32_t* wrow[WQ];
#pragma unroll
    for (int i = 0; i < WQ; ++i) {
        const int c = (i * S::kThreads + tid) % S::CN, b = c >> 5, w_ = b / FN, f = b % FN;
        const int col = n0 + (GATED ? w_ * (16 * FN) + (f % (FN / 2 > 0 ? FN / 2 : 1)) * 32 : b * 32) + (c & 31);
        wrow[i] = a.w + (int64_t(GATED && f >= FN / 2 ? a.N : 0) + min(col, a.N - 1)) * a.ld_w;
    }
    uint4 wstage[WQ];
    auto load_w = [&](int word0) {
#pragma unroll
        for (int i = 0; i < WQ; ++i) {
            const int w0 = word0 + 4 * ((i * S::kThreads + tid) / S::CN);
            if (w0 + 4 <= kw) wstage[i] = load_quad_any(wrow[i] + w0);
            else wstage[i] = make_uint4(wrow[i][min(w0, kw - 1)], wrow[i][min(w0 + 1, kw - 1)], wrow[i][min(w0 + 2, kw - 1)], 0u);
        }
    };
    auto store_w = [&](int buf) {
#pragma unroll
        for (int i = 0; i < WQ; ++i) shared.loop.w[buf][(i * S::kThreads + tid) / S::CN][(i * S::kThreads + tid) % S::CN] = wstage[i];
    };
    auto read_w = [&](uint32_t (&w)[FN], int step) {
        const int word = 2 * (step & 7) + fh;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(&shared.loop.w[(step >> 3) & 1][word >> 2][(wn * FN) * 32 + consecutive_rows(fr)]) + (word & 3);
#pragma unroll
        for (int f = 0; f < FN; ++f) w[f] = p[f * 32 * 4];
    };

    // Activations: a uniform base that moves along K, and this thread's rows from there (rows that are not there: the last one).
    using Offset = typename std::conditional<FAR, int64_t, uint32_t>::type;
    const char* const xbase = static_cast<const char*>(a.x) + int64_t(m0) * a.ld_x * int64_t(sizeof(E));
    Offset xoff[S::kChunks];
#pragma unroll
    for (int i = 0; i < S::kChunks; ++i) {
        const int id = i * S::kThreads + tid;
        xoff[i] = (Offset(min(id >> 3, a.M - 1 - m0)) * Offset(a.ld_x) + Offset(id & 7) * 8) * Offset(sizeof(E));
    }
    typename Vec8<E>::type stage[S::kChunks];
    const int whole = a.K / kStepK;                  // steps that need no checks
    auto load = [&](int t) {
        const char* const p = xbase + int64_t(t) * (kStepK * int64_t(sizeof(E)));
        if (t < whole) {
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i) stage[i] = *reinterpret_cast<const typename Vec8<E>::any*>(p + xoff[i]);
        } else {
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i)
                stage[i] = load8<E>(reinterpret_cast<const E*>(p + xoff[i]), a.K - t * kStepK - ((i * S::kThreads + tid) & 7) * 8);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int id = i * S::kThreads + tid, row = id >> 3, slot = (id & 7) ^ ((row >> 1) & 7);
            O8 t[S::kTerms];
            terms_of<E>(stage[i], t);
#pragma unroll
            for (int p = 0; p < S::kTerms; ++p) shared.loop.x[buf][p][row * 8 + slot] = t[p];
        }
    };

    v16f_t acc[FN][FM] = {};
    // Operands of a quarter step: of activations straight from LDS, of weights widened from the step's words.
    auto read_x = [&](O8 (&xf)[S::kTerms][FM], int buf, int s) {
#pragma unroll
        for (int p = 0; p < S::kTerms; ++p)
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                const int row = (wm * FM + j) * 32 + fr;
                xf[p][j] = shared.loop.x[buf][p][row * 8 + ((4 * fh + s) ^ ((row >> 1) & 7))];
            }
    };
    const Widening<O> minus_weights;
    auto widen = [&](O8 (&wf)[FN], const uint32_t (&w)[FN], int s) {
#pragma unroll
        for (int f = 0; f < FN; ++f) wf[f] = minus_weights(s < 2 ? spread_low(w[f]) : spread_high(w[f]), s & 1);
    };
    const FactorOf<E, EPI> factor_parts(a);
    float factor = 1.0f;
    auto load_scales = [&]() {
        factor = factor_parts(a);
        for (int c = tid; c < S::CN; c += S::kThreads) {
            const int b = c >> 5, w_ = b / FN, f = b % FN;
            const int col = n0 + (GATED ? w_ * (16 * FN) + (f % (FN / 2 > 0 ? FN / 2 : 1)) * 32 : b * 32) + (c & 31);
            const int64_t row = int64_t(GATED && f >= FN / 2 ? a.N : 0) + col;
            const bool there = col < a.N;
            scale_s[c] = there && a.scale ? a.scale[row] : 1.0f;
            bias_s[c] = there && a.bias ? a.bias[row] : 0.0f;
        }
    };
    const int steps = (a.K + kStepK - 1) / kStepK;
    if (steps > 0) {
        uint32_t w[2][FN];                  // of this step and of the next
        O8 xf[2][S::kTerms][FM], wf[2][FN];
        load_w(0);
        load(0);
        load_scales();                      // while those are on their way
        store_w(0);
        store(0);
        if (steps > 1) load(1);
        __syncthreads();
        read_w(w[0], 0);
        read_x(xf[0], 0, 0);
        widen(wf[0], w[0], 0);
        int buf = 0;
        for (int t = 0; t < steps; ++t) {
            const int next = buf == S::kBuffers - 1 ? 0 : buf + 1;
            const bool more = t + 1 < steps;
            if constexpr (S::kBuffers == 3) {
                // Buffer `next` held step t - 2, which every wavefront has left behind since the barrier in step t - 1.
                if (more) store(next);
                if (t + 2 < steps) load(t + 2);
            }
            // The weights of the next 512 elements: the buffer that they take was last read in the step before the last.
            if ((t & 7) == 1 && t + 7 < steps) load_w((t + 7) * 2);
            if ((t & 7) == 5 && t + 3 < steps) store_w(((t + 3) >> 3) & 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (S::kBuffers == 3 && s == 2) {
                    __syncthreads();
                    read_w(w[1], t + 1);
                }
                if (s < 3) {
                    read_x(xf[(s + 1) & 1], buf, s + 1);
                    widen(wf[(s + 1) & 1], w[0], s + 1);
                } else if (S::kBuffers == 3) {
                    read_x(xf[0], next, 0);             // after the last step: read, not used
                    widen(wf[0], w[1], 0);
                }
#pragma unroll
                for (int p = 0; p < S::kTerms; ++p)
#pragma unroll
                    for (int j = 0; j < FM; ++j)
#pragma unroll
                        for (int f = 0; f < FN; ++f) acc[f][j] = mfma16(wf[s & 1][f], xf[s & 1][p][j], acc[f][j]);
                // Keeps the quarters apart: moved over their borders, reads lie in wait longer than they take.
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (S::kBuffers == 3) {
#pragma unroll
                for (int f = 0; f < FN; ++f) w[0][f] = w[1][f];
            } else if (more) {
                // Two buffers: `next` held step t - 1, which everyone had left before the barrier at this step's start.
                store(next);
                if (t + 2 < steps) load(t + 2);
                __syncthreads();
                read_w(w[0], t + 1);
                read_x(xf[0], next, 0);
                widen(wf[0], w[0], 0);
            }
            buf = next;
        }
    } else {
        load_scales();
    }
    __syncthreads();

    // ---- epilogue: a block at a time through a piece of LDS of the wavefront's own, so that four lanes have 32 consecutive columns of
    // a row between them: as the matrix engine leaves them, a store or a load of 1 KB would be 64 pieces of 64 cache lines.
    constexpr int HALVES = S::HALVES, FY = S::FY;
    auto& block = shared.sums.block[wave];
    const int rq = lane >> 2, cq = lane & 3;
#pragma unroll
    for (int f = 0; f < FY; ++f) {
        const int c0 = (wn * FN + f) * 32 + 8 * cq;          // its channel; the other half's is 16 FN further
        const float *scale[HALVES], *bias[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            scale[h] = scale_s + c0 + 16 * FN * h;
            bias[h] = bias_s + c0 + 16 * FN * h;
        }
        float sum_s[HALVES][8] = {}, sum_z[HALVES][8] = {};
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v16f_t& v = acc[f + FY * h][j];
                    block[h][fr * 8 + ((4 * fh + q) ^ ((fr >> 1) & 7))] = make_float4(-v[4 * q], -v[4 * q + 1], -v[4 * q + 2], -v[4 * q + 3]);
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int row = 16 * half + rq;
                float sums[HALVES][8];
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float4 v = block[h][row * 8 + ((2 * cq + q) ^ ((row >> 1) & 7))];
                        sums[h][4 * q] = v.x;
                        sums[h][4 * q + 1] = v.y;
                        sums[h][4 * q + 2] = v.z;
                        sums[h][4 * q + 3] = v.w;
                    }
                finish<E, EPI, 8>(a, m0 + (wm * FM + j) * 32 + row, block_col(f) + 8 * cq, sums, scale, bias, factor, sum_s, sum_z);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        if constexpr (BACK) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = sum_of_every_fourth(sum_s[h][i]), q = sum_of_every_fourth(sum_z[h][i]);
                    if (rq == 0) {
                        sums_s[(wm * 2) * S::CN + c0 + 16 * FN * h + i] = p;
                        sums_s[(wm * 2 + 1) * S::CN + c0 + 16 * FN * h + i] = q;
                    }
                }
        }
    }
    if constexpr (BACK) {
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
