// Products of quantised rows with packed weights in tiles of 128 or 64 rows and 256 channels: four wavefronts side by side, with 64
// channels each.  Two workgroups share a compute unit, so that one multiplies while the other finishes a tile or waits.
//
// A step is 64 bytes of each row of codes: 128 elements of 4 bits or 64 of 8.  Codes go from memory straight to LDS, several steps
// ahead, into a ring of buffers; weights and scales likewise, a stage of 512 elements ahead.  The count of loads on their way is known
// at every step, so a wavefront waits for those of the next step alone, and one barrier a step makes them everybody's.  The halves h of a
// wavefront take chunks 2 h and 2 h + 1 of 16 bytes of a step's rows, one for each of its two matrix operations a block, so that their
// words of weights and the scales of their blocks lie together.
//
// LDS has rows of 64 bytes, chunk c of row r at c ^ key(r): 16 lanes that read one chunk of their rows use all banks.
//
// Measured on the way, 8192 x 8192 x 8192 of 4 bits and 8192 x 8192 -> 4096 of 8, in us: through registers with one step of twice this size
// ahead, tiles of 256 rows by 8 wavefronts, 316 and 248; rows of weights and scales loaded by four lanes instead of one 298 and 249;
// straight to LDS, five steps ahead, 272 and 224; in tiles of 128 rows, two a unit, 269 and 226 (gated 8192 x 4096 -> 8192 of 4 bits, whose
// epilogue counts most, 281 instead of 302); a stage at a time without questions 253 and 213.  The same loop without its matrix
// operations takes 157 of the 253, the matrix engine alone 180 (6.1 PFLOP/s at the clock that its power leaves it; 3.4 and 164 of 8
// bits): the two overlap for the most part, at 2.1 GHz.  A library product of 8192^3 in int8 reaches 2.5 PFLOP/s, as this one.
#pragma once

#include "q_bits.h"

namespace bnn {

typedef __attribute__((address_space(3))) const void* lds_ptr_t;

// 16 bytes a lane from memory (4-byte aligned) to LDS: the wavefront's 1 KB from `at` on.  The compiler is not to know what these
// loads write: it would wait for all of them before each read of LDS.
__device__ inline void to_lds(const void* from, uint32_t at) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(__builtin_amdgcn_readfirstlane(at)) : "memory");
}

template <int N>
__device__ inline void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// What this wavefront's loads, for which it has waited, have brought is everybody's, as are its own writes.
__device__ inline void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

template <int S>
__device__ inline v16f_t mfma_q(v4i_t w, v4i_t x, v16f_t c, uint32_t scales) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(in_eight(w), in_eight(x), c, kFp4, kFp4, 0, kOne, S, int(scales));
}
template <int S>
__device__ inline v16i_t mfma_q(v4i_t w, v4i_t x, v16i_t c, uint32_t) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(w, x, c, 0, 0, 0);
}

// FM blocks of 32 rows.
template <int ROWS, int EPI, int FM>
struct QTile {
    static constexpr bool GATED = EPI == kQGated, MX4 = ROWS == BNN_ROWS_MX4;
    static constexpr int TN = 4, FN = 2, HALVES = kQHalves<EPI>, FY = FN / HALVES;
    static constexpr int kThreads = 64 * TN, BM = 32 * FM, CN = 32 * TN * FN, BN = CN / HALVES;
    static constexpr int kBuffers = 5, kAhead = kBuffers - 1;
    static constexpr int kStepBlocks = MX4 ? 4 : 2;                   // blocks of 32 elements a step
    static constexpr int kSteps = 16 / kStepBlocks;                   // steps of a stage
    static constexpr int kLoads = BM * 4 / kThreads;                  // of codes, a step and thread
    static constexpr int kStageLoads = CN * 4 / kThreads;             // of weights, a stage
    // Loads that may be on their way when a step begins, whose next step's codes have to be there: those of the steps after that, and
    // a stage's weights and scales, issued in its first step, while they are among them.  When a stage's last step begins, no more than those
    // issued after the next stage's weights.
    static constexpr int kStage = kStageLoads + (MX4 ? 1 : 0), kLeft = (kAhead - 2) * kLoads;
    static_assert(kSteps >= kAhead, "a stage's weights are older than the codes that a step leaves on their way");
    struct Loop {
        uint4 x[kBuffers][BM * 4];
        uint4 w[2][CN * 4];
        uint4 powers[2][MX4 ? BM : 1];       // of 4 bits: 16 blocks' scales of a row
    };
    union Shared {
        __device__ Shared() {}
        Loop loop;
        float4 block[TN][HALVES][32 * 8];    // the epilogue's, a wavefront's own: rows of 32 columns, chunk c of row r at c ^ (r / 2) % 8
    };
};

template <int ROWS, int EPI, int FM>
__global__ __launch_bounds__(256, 2) void q_tile_kernel(const QProductArgs a) {
    using S = QTile<ROWS, EPI, FM>;
    using R = RowsOf<ROWS>;
    using sum_t = typename R::sum_t;
    typedef sum_t acc_t __attribute__((ext_vector_type(16)));
    constexpr bool GATED = S::GATED, MX4 = S::MX4;
    constexpr int FN = S::FN, FY = S::FY, HALVES = S::HALVES;
    __shared__ typename S::Shared shared;
    __shared__ float scale_s[S::CN], bias_s[S::CN], row_s[MX4 ? 1 : S::BM];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, fh = lane >> 5;
    int tm, tn;
    tile_of_block(blockIdx.x, a.map, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN, nb = (a.K + 31) >> 5;
    const int steps = (nb + S::kStepBlocks - 1) / S::kStepBlocks, stages = (nb + 15) >> 4;

    // Channel c of the tile: a wavefront's blocks of the gated form are one of the gate's rows and the same columns of the other half.
    auto column = [&](int c) { return n0 + (GATED ? c >> 6 << 5 : c >> 5 << 5) + (c & 31); };
    auto half_of = [&](int c) { return GATED ? (c >> 5) & 1 : 0; };
    // Of rows of codes, which 16 lanes read in order, and of rows of weights, which they read in the order of consecutive_rows.
    auto x_key = [](int row) { return (row >> 2) & 3; };
    auto w_key = [](int row) { return ((row >> 2) & 1) | ((row >> 3) & 2); };

    // Lane l of load i: row (i * threads + tid) / 4 of a tile, its place tid % 4 there.
    const uint8_t* xrow[S::kLoads];
    const uint32_t* wrow[S::kStageLoads];
    const int xchunk = (tid & 3) ^ x_key(tid >> 2), wchunk = (tid & 3) ^ w_key(tid >> 2);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) xrow[i] = a.codes + int64_t(min(m0 + ((i * S::kThreads + tid) >> 2), a.M - 1)) * a.ld_c;
#pragma unroll
    for (int i = 0; i < S::kStageLoads; ++i) {
        const int c = (i * S::kThreads + tid) >> 2;
        wrow[i] = a.w + (int64_t(half_of(c)) * a.N + min(column(c), a.N - 1)) * a.ld_w;
    }
    const uint8_t* const prow = static_cast<const uint8_t*>(a.scales) + (MX4 ? int64_t(min(m0 + tid % S::BM, a.M - 1)) * a.ld_s : 0);
    const uint32_t x_at = uint32_t(uintptr_t(lds_ptr_t(&shared.loop.x[0][0]))), w_at = uint32_t(uintptr_t(lds_ptr_t(&shared.loop.w[0][0])));
    const uint32_t p_at = uint32_t(uintptr_t(lds_ptr_t(&shared.loop.powers[0][0])));
    // What lies past a row's end is loaded from its last bytes, and put right by mend_x and mend_w.
    auto load_x = [&](int t, int buf) {
        const uint32_t at = min(uint32_t(t) * 64 + xchunk * 16, uint32_t(nb) * (MX4 ? 16 : 32) - 16);
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) to_lds(xrow[i] + at, x_at + (buf * (S::BM * 4) + i * S::kThreads + wave * 64) * 16);
    };
    auto load_w = [&](int stage) {
        const uint32_t at = min(uint32_t(stage) * 64 + wchunk * 16, uint32_t(nb) * 4 - 16);
#pragma unroll
        for (int i = 0; i < S::kStageLoads; ++i)
            to_lds(reinterpret_cast<const char*>(wrow[i]) + at, w_at + ((stage & 1) * (S::CN * 4) + i * S::kThreads + wave * 64) * 16);
        // Twice the same where there are more threads than rows.
        if constexpr (MX4) to_lds(prow + 16 * min(stage, stages - 1), p_at + ((stage & 1) * S::BM + (wave * 64) % S::BM) * 16);
    };
    // A thread mends what it has loaded itself, when that is there and nobody has read it: chunks of blocks that are not there are zero
    // in the last step, ...
    auto mend_x = [&](int buf) {
        if (steps * S::kStepBlocks == nb) return;
        if ((steps - 1) * S::kStepBlocks + (MX4 ? xchunk : xchunk >> 1) < nb) return;
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) shared.loop.x[buf][i * S::kThreads + tid] = make_uint4(0u, 0u, 0u, 0u);
    };
    // ... words of the last stage in their places (a piece that is not whole has the row's last four), and scales of blocks that are not
    // there, whose bytes may be anything, 1.
    auto mend_w = [&]() {
        const int stage = stages - 1, left = nb - 16 * stage - 4 * wchunk;       // words of the piece that are there
        if (left > 0 && left < 4) {
#pragma unroll
            for (int i = 0; i < S::kStageLoads; ++i) {
                uint4& v = shared.loop.w[stage & 1][i * S::kThreads + tid];
                v = left == 3 ? make_uint4(v.y, v.z, v.w, 0u) : left == 2 ? make_uint4(v.z, v.w, 0u, 0u) : make_uint4(v.w, 0u, 0u, 0u);
            }
        }
        if constexpr (MX4) {
            uint32_t* const p = reinterpret_cast<uint32_t*>(&shared.loop.powers[stage & 1][tid % S::BM]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int there = nb - 16 * stage - 4 * i;
                const uint32_t keep = there >= 4 ? ~0u : there > 0 ? (1u << (8 * there)) - 1 : 0u;
                p[i] = (p[i] & keep) | (kOne & ~keep);
            }
        }
    };

    acc_t acc[FN][FM] = {};
    auto read_x = [&](v4i_t (&xf)[FM], int buf, int s) {
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int row = 32 * j + fr;
            xf[j] = as_ints(shared.loop.x[buf][row * 4 + ((2 * fh + s) ^ x_key(row))]);
        }
    };
    // Words of step t: of this half two of 4-bit steps, one of 8-bit ones; and its two blocks' scales.
    auto read_words = [&](uint2 (&w)[FN], int t, int in_stage) {
        const int stage = t / S::kSteps & 1;
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            const int row = (wave * FN + f) * 32 + consecutive_rows(fr);
            const uint4* const p = &shared.loop.w[stage][row * 4 + ((MX4 ? in_stage : in_stage >> 1) ^ w_key(row))];
            if constexpr (MX4) w[f] = reinterpret_cast<const uint2*>(p)[fh];
            else w[f].x = reinterpret_cast<const uint32_t*>(p)[2 * (in_stage & 1) + fh];
        }
    };
    auto read_w = [&](uint2 (&w)[FN], uint32_t (&powers)[FM], int t, int in_stage) {
        const int stage = t / S::kSteps & 1;
        read_words(w, t, in_stage);
        if constexpr (MX4) {
#pragma unroll
            for (int j = 0; j < FM; ++j)
                powers[j] = reinterpret_cast<const uint32_t*>(&shared.loop.powers[stage][32 * j + fr])[in_stage] >> (16 * fh);
        }
    };
    const R minus_weights;
    auto widen = [&](v4i_t (&wf)[FN], const uint2 (&w)[FN], int s) {
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            if constexpr (MX4) wf[f] = minus_weights(s == 0 ? w[f].x : w[f].y);
            else wf[f] = minus_weights(w[f].x, s);
        }
    };

    load_w(0);
#pragma unroll
    for (int t = 0; t < S::kAhead; ++t) load_x(min(t, steps - 1), t);
    for (int c = tid; c < S::CN; c += S::kThreads) {
        const int col = column(c);
        const int64_t row = int64_t(half_of(c)) * a.N + col;
        scale_s[c] = scale_at(a, row, col < a.N);
        bias_s[c] = bias_at(a, row, col < a.N);
    }
    if constexpr (!MX4) {
        for (int r = tid; r < S::BM; r += S::kThreads) row_s[r] = static_cast<const float*>(a.scales)[min(m0 + r, a.M - 1)];
    }
    {
        uint2 w[2][FN];                      // of this step and of the next
        uint32_t powers[2][FM];
        v4i_t xf[2][FM], wf[2][FN];
        wait_loads<(S::kAhead - 1) * S::kLoads>();
        if (stages == 1) mend_w();
        if (steps == 1) mend_x(0);
        meet();
        read_w(w[0], powers[0], 0, 0);
        read_x(xf[0], 0, 0);
        widen(wf[0], w[0], 0);
        int buf = 0, last = S::kAhead, in_stage = 0, t = 0;           // buffer of this step, and of the one that is loaded in it
        {
            // Stages with nothing to ask: what a step is to its stage is known, and a row's scales of a stage are loaded at once.
            uint4 stage_powers[MX4 ? FM : 1];
            auto read_powers = [&](int stage) {
                if constexpr (MX4) {
#pragma unroll
                    for (int j = 0; j < FM; ++j) stage_powers[j] = shared.loop.powers[stage & 1][32 * j + fr];
                }
            };
            auto step = [&](auto which) {
                constexpr int in = decltype(which)::value, now = in & 1, then = now ^ 1, after = (in + 1) % S::kSteps;
                const int next = buf == S::kAhead ? 0 : buf + 1;
                wait_loads<in >= 1 && in <= S::kAhead - 1 && in < S::kSteps - 1 ? S::kLeft + S::kStage : S::kLeft>();
                meet();
                load_x(t + in + S::kAhead, last);
                if (in == 0) load_w(t / S::kSteps + 1);
                read_words(w[then], t + in + 1, after);
                if constexpr (MX4) {
                    if (after == 0) read_powers(t / S::kSteps + 1);
#pragma unroll
                    for (int j = 0; j < FM; ++j) {
                        const uint4& p = stage_powers[j];
                        powers[then][j] = (after == 0 ? p.x : after == 1 ? p.y : after == 2 ? p.z : p.w) >> (16 * fh);
                    }
                }
                read_x(xf[1], buf, 1);
                widen(wf[1], w[now], 1);
#pragma unroll
                for (int j = 0; j < FM; ++j)
#pragma unroll
                    for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q<0>(wf[0][f], xf[0][j], acc[f][j], powers[now][j]);
                // Keeps the halves of a step apart: moved over their borders, reads lie in wait longer than they take.
                __builtin_amdgcn_sched_barrier(0);
                read_x(xf[0], next, 0);
                widen(wf[0], w[then], 0);
#pragma unroll
                for (int j = 0; j < FM; ++j)
#pragma unroll
                    for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q<1>(wf[1][f], xf[1][j], acc[f][j], powers[now][j]);
                __builtin_amdgcn_sched_barrier(0);
                last = buf;
                buf = next;
            };
            if (2 * S::kSteps < steps) read_powers(0);
            for (; t + 2 * S::kSteps < steps; t += S::kSteps) {
                step(std::integral_constant<int, 0>{});
                step(std::integral_constant<int, 1>{});
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
                if constexpr (S::kSteps == 8) {
                    step(std::integral_constant<int, 4>{});
                    step(std::integral_constant<int, 5>{});
                    step(std::integral_constant<int, 6>{});
                    step(std::integral_constant<int, 7>{});
                }
            }
        }
        for (; t < steps; ++t) {
            const int next = buf == S::kAhead ? 0 : buf + 1;
            // Everybody is done with step t - 1 at the barrier, whose buffer the loads of this step take.
            if (t + S::kAhead < steps) {
                if (in_stage >= 1 && in_stage <= S::kAhead - 1 && in_stage < S::kSteps - 1) wait_loads<S::kLeft + S::kStage>();
                else wait_loads<S::kLeft>();
            } else if (t + 3 < steps) {
                wait_loads<2 * S::kLoads>();                          // codes that were asked for after the next step's
            } else {
                if (t + 3 == steps) wait_loads<S::kLoads>();
                else wait_loads<0>();
                if (t + 2 == steps) mend_x(next);
            }
            if (in_stage == S::kSteps - 1 && t / S::kSteps == stages - 2) mend_w();
            meet();
            if (t + S::kAhead < steps) load_x(t + S::kAhead, last);
            if (in_stage == 0) load_w(t / S::kSteps + 1);             // after the last stage: loaded, not used
            in_stage = in_stage == S::kSteps - 1 ? 0 : in_stage + 1;
            read_w(w[1], powers[1], t + 1, in_stage);                 // after the last step: read, not used
            read_x(xf[1], buf, 1);
            widen(wf[1], w[0], 1);
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q<0>(wf[0][f], xf[0][j], acc[f][j], powers[0][j]);
            // Keeps the halves of a step apart: moved over their borders, reads lie in wait longer than they take.
            __builtin_amdgcn_sched_barrier(0);
            read_x(xf[0], next, 0);
            widen(wf[0], w[1], 0);
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q<1>(wf[1][f], xf[1][j], acc[f][j], powers[0][j]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int f = 0; f < FN; ++f) w[0][f] = w[1][f];
            if constexpr (MX4) {
#pragma unroll
                for (int j = 0; j < FM; ++j) powers[0][j] = powers[1][j];
            }
            last = buf;
            buf = next;
        }
    }
    wait_loads<0>();                         // none may still write what the epilogue's pieces take
    __syncthreads();

    // ---- epilogue: a block at a time through a piece of LDS of the wavefront's own, so that four lanes have 32 consecutive columns of
    // a row between them.  The loops over rows run: what is done to the sums is there once.
    auto& block = shared.block[wave];
    const int rq = lane >> 2, cq = lane & 3;
#pragma unroll
    for (int f = 0; f < FY; ++f) {
        const int c0 = (wave * FN + f) * 32 + 8 * cq;                 // the lane's first channel; the other half's is 32 further
        float scale[HALVES][8], bias[HALVES][8];
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                scale[h][i] = scale_s[c0 + 32 * h + i];
                bias[h][i] = bias_s[c0 + 32 * h + i];
            }
#pragma unroll 1
        for (int j = 0; j < FM; ++j) {
            const float s_of = MX4 ? 0.0f : row_s[32 * j + fr];
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if (i != j) continue;
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const acc_t& v = acc[f + h][i];
                        block[h][fr * 8 + ((4 * fh + q) ^ ((fr >> 1) & 7))] =
                            make_float4(R::value(v[4 * q], s_of), R::value(v[4 * q + 1], s_of), R::value(v[4 * q + 2], s_of), R::value(v[4 * q + 3], s_of));
                    }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
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
                finish_q<EPI, 8, true>(a, m0 + 32 * j + row, column(c0), sums, scale, bias);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

constexpr int64_t kLeastTileK = 97;          // rows of weights have four words to load at a time

// a.M, a.N > 0, a.K >= kLeastTileK.
template <int ROWS, int EPI, int FM>
int launch_q_tile(QProductArgs a, hipStream_t s) {
    using S = QTile<ROWS, EPI, FM>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    q_tile_kernel<ROWS, EPI, FM><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

}  // namespace bnn
