// Products of quantised rows with packed weights in tiles of 64 to 256 rows and 256 channels through LDS.
//
// A step is 128 bytes of each row of codes: 256 elements of 4 bits or 128 of 8.  Its eight chunks of 16 bytes are taken four and
// four by the halves of a wavefront, chunk 4 h + s in quarter s of the step, so that the words of weights that a half needs (four of
// 4-bit steps, two of 8-bit ones) and its blocks' four scales lie together.  Each quarter is one matrix operation of 32 cycles a pair of
// blocks of 32 for either kind.  Weights and scales are staged 512 elements at a time.  Three buffers of codes let a wavefront run on
// from step to step, with the barrier in the middle of one; operands of the next quarter are read and widened under the products
// of this one.
#pragma once

#include "q_bits.h"

namespace bnn {

__device__ inline v16f_t mfma_q(v4i_t w, v4i_t x, v16f_t c, uint32_t scales, std::integral_constant<int, 0>) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, 0, int(scales));
}
__device__ inline v16f_t mfma_q(v4i_t w, v4i_t x, v16f_t c, uint32_t scales, std::integral_constant<int, 1>) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, 1, int(scales));
}
__device__ inline v16f_t mfma_q(v4i_t w, v4i_t x, v16f_t c, uint32_t scales, std::integral_constant<int, 2>) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, 2, int(scales));
}
__device__ inline v16f_t mfma_q(v4i_t w, v4i_t x, v16f_t c, uint32_t scales, std::integral_constant<int, 3>) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, 3, int(scales));
}
template <int S>
__device__ inline v16i_t mfma_q(v4i_t w, v4i_t x, v16i_t c, uint32_t, std::integral_constant<int, S>) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, c, 0, 0, 0);
}

// TM x TN wavefronts, of FM blocks of 32 rows and FN of 32 channels each.
template <int ROWS, int EPI, int TM, int TN, int FM, int FN>
struct QTile {
    static constexpr bool GATED = EPI == kQGated, MX4 = ROWS == BNN_ROWS_MX4;
    static constexpr int HALVES = kQHalves<EPI>, FY = FN / HALVES;
    static constexpr int kThreads = 64 * TM * TN, BM = 32 * TM * FM, CN = 32 * TN * FN, BN = CN / HALVES;
    static constexpr int kStepBlocks = MX4 ? 8 : 4;            // blocks of 32 elements a step
    static constexpr int kStageSteps = 16 / kStepBlocks;       // steps of a stage of weights
    static constexpr int kChunks = BM * 8 / kThreads;          // chunks that a thread stages
    static constexpr int kQuads = 4 * CN / kThreads;           // 16-byte pieces of weights
    static constexpr int kPowers = MX4 ? 4 * BM / kThreads : 1;        // four blocks' scales
    struct Loop {
        uint4 x[3][BM * 8];                  // chunk c of a row at c ^ (row / 2) % 8
        uint4 w[2][4][CN];                   // 512 elements of each row of weights, 16 bytes of a row at a time
        uint32_t powers[2][MX4 ? 4 : 1][MX4 ? BM : 1];
    };
    struct Sums {
        float4 block[TM * TN][FN][32 * 8];        // a wavefront's own: 32 rows of 32 columns each, placed like x
    };
    union Shared {
        __device__ Shared() {}
        Loop loop;
        Sums sums;
    };
};

template <int ROWS, int EPI, int TM, int TN, int FM, int FN>
__global__ __launch_bounds__(64 * TM * TN) void q_tile_kernel(const QProductArgs a) {
    using S = QTile<ROWS, EPI, TM, TN, FM, FN>;
    using R = RowsOf<ROWS>;
    using sum_t = typename R::sum_t;
    typedef sum_t acc_t __attribute__((ext_vector_type(16)));
    constexpr bool GATED = S::GATED, MX4 = S::MX4;
    constexpr int HALVES = S::HALVES, FY = S::FY;
    __shared__ typename S::Shared shared;
    __shared__ float scale_s[S::CN], bias_s[S::CN], row_s[MX4 ? 1 : S::BM];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wn = wave % TN, wm = wave / TN, fr = lane & 31, fh = lane >> 5;
    int tm, tn;
    tile_of_block(blockIdx.x, a.map, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN, nb = (a.K + 31) >> 5;

    // Channel c of the tile: a wavefront's blocks of the gated form are FY of the gate's rows, then the same columns of the other half.
    auto column = [&](int c) {
        const int b = c >> 5, f = b % FN;
        return n0 + (GATED ? b / FN * (32 * FY) + f % FY * 32 : b * 32) + (c & 31);
    };
    auto half_of = [&](int c) { return GATED && (c >> 5) % FN >= FY ? 1 : 0; };

    const uint32_t* wrow[S::kQuads];
#pragma unroll
    for (int i = 0; i < S::kQuads; ++i) {
        const int c = (i * S::kThreads + tid) % S::CN;
        wrow[i] = a.w + (int64_t(half_of(c)) * a.N + min(column(c), a.N - 1)) * a.ld_w;
    }
    uint4 wstage[S::kQuads];
    uint32_t pstage[S::kPowers];
    auto load_w = [&](int stage) {
#pragma unroll
        for (int i = 0; i < S::kQuads; ++i) {
            const int w0 = 16 * stage + 4 * ((i * S::kThreads + tid) / S::CN);
            if (w0 + 4 <= nb) wstage[i] = load_quad_any(wrow[i] + w0);
            else wstage[i] = make_uint4(wrow[i][min(w0, nb - 1)], wrow[i][min(w0 + 1, nb - 1)], wrow[i][min(w0 + 2, nb - 1)], 0u);
        }
        if constexpr (MX4) {
#pragma unroll
            for (int i = 0; i < S::kPowers; ++i) {
                const int id = i * S::kThreads + tid, b0 = 16 * stage + 4 * (id / S::BM);
                const int64_t m = min(m0 + id % S::BM, a.M - 1);
                // Bytes of blocks that are not there may be anything: a scale of 1 for their zeros.
                const uint32_t p = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.scales) + m * a.ld_s + min(b0, (nb - 1) & ~3));
                const int left = nb - b0;
                const uint32_t keep = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
                pstage[i] = (p & keep) | (kOne & ~keep);
            }
        }
    };
    auto store_w = [&](int stage) {
#pragma unroll
        for (int i = 0; i < S::kQuads; ++i) shared.loop.w[stage & 1][(i * S::kThreads + tid) / S::CN][(i * S::kThreads + tid) % S::CN] = wstage[i];
        if constexpr (MX4) {
#pragma unroll
            for (int i = 0; i < S::kPowers; ++i) shared.loop.powers[stage & 1][(i * S::kThreads + tid) / S::BM][(i * S::kThreads + tid) % S::BM] = pstage[i];
        }
    };
    // A step's words of this lane's half (of 8-bit steps two), and its blocks' scales.
    auto read_w = [&](uint4 (&w)[FN], uint32_t (&powers)[FM], int t) {
        const int stage = t / S::kStageSteps & 1, quad = MX4 ? 2 * (t & 1) + fh : t & 3;
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            const uint4* const p = &shared.loop.w[stage][quad][(wn * FN + f) * 32 + consecutive_rows(fr)];
            if constexpr (MX4) {
                w[f] = *p;
            } else {
                const uint2 two = reinterpret_cast<const uint2*>(p)[fh];
                w[f] = make_uint4(two.x, two.y, 0u, 0u);
            }
        }
        if constexpr (MX4) {
#pragma unroll
            for (int j = 0; j < FM; ++j) powers[j] = shared.loop.powers[stage][quad][(wm * FM + j) * 32 + fr];
        }
    };

    const uint8_t* const xbase = a.codes + int64_t(m0) * a.ld_c;
    int64_t xoff[S::kChunks];
#pragma unroll
    for (int i = 0; i < S::kChunks; ++i) {
        const int id = i * S::kThreads + tid;
        xoff[i] = int64_t(min(id >> 3, a.M - 1 - m0)) * a.ld_c + (id & 7) * 16;
    }
    uint4 stage[S::kChunks];
    const int whole = nb / S::kStepBlocks;
    auto load = [&](int t) {
        const uint8_t* const p = xbase + int64_t(t) * 128;
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            // The last step: chunks of blocks that are not there are zero.
            const int chunk = (i * S::kThreads + tid) & 7;
            if (t < whole || t * S::kStepBlocks + (MX4 ? chunk : chunk >> 1) < nb) stage[i] = *reinterpret_cast<const uint4*>(p + xoff[i]);
            else stage[i] = make_uint4(0u, 0u, 0u, 0u);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int id = i * S::kThreads + tid, row = id >> 3;
            shared.loop.x[buf][row * 8 + ((id & 7) ^ ((row >> 1) & 7))] = stage[i];
        }
    };

    acc_t acc[FN][FM] = {};
    auto read_x = [&](v4i_t (&xf)[FM], int buf, int s) {
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int row = (wm * FM + j) * 32 + fr;
            xf[j] = as_ints(shared.loop.x[buf][row * 8 + ((4 * fh + s) ^ ((row >> 1) & 7))]);
        }
    };
    const R minus_weights;
    auto widen = [&](v4i_t (&wf)[FN], const uint4 (&w)[FN], int s) {
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            if constexpr (MX4) wf[f] = minus_weights(s == 0 ? w[f].x : s == 1 ? w[f].y : s == 2 ? w[f].z : w[f].w);
            else wf[f] = minus_weights(s < 2 ? w[f].x : w[f].y, s & 1);
        }
    };
    auto load_scales = [&]() {
        for (int c = tid; c < S::CN; c += S::kThreads) {
            const int col = column(c);
            const int64_t row = int64_t(half_of(c)) * a.N + col;
            scale_s[c] = scale_at(a, row, col < a.N);
            bias_s[c] = bias_at(a, row, col < a.N);
        }
        if constexpr (!MX4) {
            for (int r = tid; r < S::BM; r += S::kThreads) row_s[r] = static_cast<const float*>(a.scales)[min(m0 + r, a.M - 1)];
        }
    };
    const int steps = (nb + S::kStepBlocks - 1) / S::kStepBlocks, stages = (nb + 15) / 16;
    {
        uint4 w[2][FN];                     // of this step and of the next
        uint32_t powers[2][FM];
        v4i_t xf[2][FM], wf[2][FN];
        load_w(0);
        load(0);
        load_scales();                      // while those are on their way
        store_w(0);
        store(0);
        if (steps > 1) load(1);
        __syncthreads();
        read_w(w[0], powers[0], 0);
        read_x(xf[0], 0, 0);
        widen(wf[0], w[0], 0);
        int buf = 0;
        for (int t = 0; t < steps; ++t) {
            const int next = buf == 2 ? 0 : buf + 1;
            // Buffer `next` held step t - 2, which every wavefront has left behind since the barrier in step t - 1.
            if (t + 1 < steps) store(next);
            if (t + 2 < steps) load(t + 2);
            // The next stage of weights: its place was last read in the stage before this one.
            const int in_stage = t % S::kStageSteps, after = t / S::kStageSteps + 1;
            if (in_stage == 0 && after < stages) load_w(after);
            if (in_stage == S::kStageSteps - 1 && after < stages) store_w(after);
            auto quarter = [&](auto which) {
                constexpr int s = decltype(which)::value;
                if (s == 2) {
                    __syncthreads();
                    read_w(w[1], powers[1], t + 1);          // after the last step: read, not used
                }
                if (s < 3) {
                    read_x(xf[(s + 1) & 1], buf, s + 1);
                    widen(wf[(s + 1) & 1], w[0], s + 1);
                } else {
                    read_x(xf[0], next, 0);
                    widen(wf[0], w[1], 0);
                }
#pragma unroll
                for (int j = 0; j < FM; ++j)
#pragma unroll
                    for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q(wf[s & 1][f], xf[s & 1][j], acc[f][j], powers[0][j], which);
                // Keeps the quarters apart: moved over their borders, reads lie in wait longer than they take.
                __builtin_amdgcn_sched_barrier(0);
            };
            quarter(std::integral_constant<int, 0>{});
            quarter(std::integral_constant<int, 1>{});
            quarter(std::integral_constant<int, 2>{});
            quarter(std::integral_constant<int, 3>{});
#pragma unroll
            for (int f = 0; f < FN; ++f) w[0][f] = w[1][f];
            if constexpr (MX4) {
#pragma unroll
                for (int j = 0; j < FM; ++j) powers[0][j] = powers[1][j];
            }
            buf = next;
        }
    }
    __syncthreads();

    // ---- epilogue: a row of blocks at a time through a piece of LDS of the wavefront's own, so that four lanes have 32 consecutive
    // columns of a row between them.  The loops run: what is done to the sums is there once, the accumulators' places are not to be
    // looked up.
    auto& block = shared.sums.block[wave];
    const int rq = lane >> 2, cq = lane & 3;
#pragma unroll 1
    for (int j = 0; j < FM; ++j) {
        const float s_of = MX4 ? 0.0f : row_s[(wm * FM + j) * 32 + fr];
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if (i != j) continue;
#pragma unroll
            for (int f = 0; f < FN; ++f)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const acc_t& v = acc[f][i];
                    block[f][fr * 8 + ((4 * fh + q) ^ ((fr >> 1) & 7))] =
                        make_float4(R::value(v[4 * q], s_of), R::value(v[4 * q + 1], s_of), R::value(v[4 * q + 2], s_of), R::value(v[4 * q + 3], s_of));
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
        for (int u = 0; u < 2 * FY; ++u) {
            const int f = u >> 1, row = 16 * (u & 1) + rq, c0 = (wn * FN + f) * 32 + 8 * cq;      // its channel; the other half's is 32 FY further
            const float *scale[HALVES], *bias[HALVES];
            float sums[HALVES][8];
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                scale[h] = scale_s + c0 + 32 * FY * h;
                bias[h] = bias_s + c0 + 32 * FY * h;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 v = block[f + FY * h][row * 8 + ((2 * cq + q) ^ ((row >> 1) & 7))];
                    sums[h][4 * q] = v.x;
                    sums[h][4 * q + 1] = v.y;
                    sums[h][4 * q + 2] = v.z;
                    sums[h][4 * q + 3] = v.w;
                }
            }
            finish_q<EPI, 8>(a, m0 + (wm * FM + j) * 32 + row, column(c0), sums, scale, bias);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// a.M, a.N, a.K > 0.
template <int ROWS, int EPI, int TM, int TN, int FM, int FN>
int launch_q_tile(QProductArgs a, hipStream_t s) {
    using S = QTile<ROWS, EPI, TM, TN, FM, FN>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    q_tile_kernel<ROWS, EPI, TM, TN, FM, FN><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

}  // namespace bnn
