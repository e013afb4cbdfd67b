// Products of quantised rows with packed weights where tiles through LDS (q_tiles.h) do not fill the chip: every wavefront of a workgroup
// has the whole tile of 32 or 64 rows and 64 channels to itself and runs of K are dealt to them, so that no wavefront waits for
// another until the sums meet in LDS.  A wavefront loads its operands as the matrix engine wants them, a run at a time, and the next run's in
// the place of what it has just multiplied.
#pragma once

#include "q_tiles.h"

namespace bnn {

constexpr int kQWavesRunK = 256;          // elements of K a wavefront takes at a time: half of it has four blocks of 32

// FM blocks of 32 rows, two of 32 channels (gated: one of each half).
template <int ROWS, int EPI, int FM>
__global__ __launch_bounds__(512) void q_waves_kernel(const QProductArgs a) {
    using R = RowsOf<ROWS>;
    using sum_t = typename R::sum_t;
    typedef sum_t acc_t __attribute__((ext_vector_type(16)));
    constexpr bool MX4 = ROWS == BNN_ROWS_MX4;
    constexpr int FN = 2, HALVES = kQHalves<EPI>, FY = FN / HALVES, CN = 32 * FN, BN = CN / HALVES, CHUNKS = 4 * R::kQuads;
    struct alignas(16) Four { sum_t v[4]; };
    extern __shared__ __attribute__((aligned(16))) char part_raw[];       // the sums, [wavefront][row block][block][register / 4][lane]
    Four* const part_s = reinterpret_cast<Four*>(part_raw);
    __shared__ float scale_s[CN], bias_s[CN];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int fr = lane & 31, fh = lane >> 5;
    int tm, tn;
    tile_of_block(blockIdx.x, a.map, tm, tn);
    const int m0 = tm * (32 * FM), n0 = tn * BN, nb = (a.K + 31) >> 5;

    // Block f of the tile: columns n0 + 32 (f % FY) of half f / FY.
    const uint32_t* wrow[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f)
        wrow[f] = a.w + (int64_t(f / FY) * a.N + min(n0 + (f % FY) * 32 + consecutive_rows(fr), a.N - 1)) * a.ld_w;
    const uint8_t *xrow[FM], *prow[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int64_t m = min(m0 + 32 * j + fr, a.M - 1);
        xrow[j] = a.codes + m * a.ld_c;
        prow[j] = static_cast<const uint8_t*>(a.scales) + m * a.ld_s;
    }
    uint4 w[FN], x[FM][CHUNKS];
    uint32_t powers[FM];
    auto load_w = [&](int b0) {              // b0: the half's first block
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            if (b0 + 4 <= nb) w[f] = load_quad_any(wrow[f] + b0);
            else w[f] = make_uint4(wrow[f][min(b0, nb - 1)], wrow[f][min(b0 + 1, nb - 1)], wrow[f][min(b0 + 2, nb - 1)], 0u);
        }
        if constexpr (MX4) {
            // Bytes of blocks that are not there may be anything: a scale of 1 for their zeros.
            const int left = nb - b0;
            const uint32_t keep = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
#pragma unroll
            for (int j = 0; j < FM; ++j) powers[j] = (*reinterpret_cast<const uint32_t*>(prow[j] + min(b0, (nb - 1) & ~3)) & keep) | (kOne & ~keep);
        }
    };
    auto load_x = [&](int b0, int c) {
        const bool there = b0 + c / R::kQuads < nb;
#pragma unroll
        for (int j = 0; j < FM; ++j)
            x[j][c] = there ? *(reinterpret_cast<const uint4*>(xrow[j]) + int64_t(b0) * R::kQuads + c) : make_uint4(0u, 0u, 0u, 0u);
    };
    const R minus_weights;
    acc_t acc[FN][FM] = {};
    const int step = 8 * waves;
    int first = 8 * wave;
    if (first < nb) {
        load_w(first + 4 * fh);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) load_x(first + 4 * fh, c);
    }
    for (int c = tid; c < CN; c += blockDim.x) {
        const int f = c >> 5, col = n0 + (f % FY) * 32 + (c & 31);
        const int64_t row = int64_t(f / FY) * a.N + col;
        scale_s[c] = scale_at(a, row, col < a.N);
        bias_s[c] = bias_at(a, row, col < a.N);
    }
    for (; first < nb; first += step) {
        uint4 wc[FN];
        uint32_t pc[FM];
#pragma unroll
        for (int f = 0; f < FN; ++f) wc[f] = w[f];
#pragma unroll
        for (int j = 0; j < FM; ++j) pc[j] = MX4 ? powers[j] : 0u;
        const int next = first + step + 4 * fh;
        const bool more = first + step < nb;
        if (more) load_w(next);
        auto chunk = [&](auto which) {
            constexpr int c = decltype(which)::value, i = c / R::kQuads;
            v4i_t wf[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                const uint32_t word = i == 0 ? wc[f].x : i == 1 ? wc[f].y : i == 2 ? wc[f].z : wc[f].w;
                if constexpr (MX4) wf[f] = minus_weights(word);
                else wf[f] = minus_weights(word, c & 1);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int f = 0; f < FN; ++f) acc[f][j] = mfma_q<i>(wf[f], as_ints(x[j][c]), acc[f][j], pc[j]);
            if (more) load_x(next, c);
        };
        chunk(std::integral_constant<int, 0>{});
        chunk(std::integral_constant<int, 1>{});
        chunk(std::integral_constant<int, 2>{});
        chunk(std::integral_constant<int, 3>{});
        if constexpr (!MX4) {
            chunk(std::integral_constant<int, 4>{});
            chunk(std::integral_constant<int, 5>{});
            chunk(std::integral_constant<int, 6>{});
            chunk(std::integral_constant<int, 7>{});
        }
    }
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part_s[((wave * FM + j) * FN + f) * 256 + q * 64 + lane] =
                    Four{{acc[f][j][4 * q], acc[f][j][4 * q + 1], acc[f][j][4 * q + 2], acc[f][j][4 * q + 3]}};
    __syncthreads();
    // A lane has eight columns of a row, a quad 32: column c of row r is register c % 16 of lane r + 32 (c / 16).
    const int rq = lane >> 2, cq = lane & 3;
    for (int unit = wave; unit < 2 * FM * FY; unit += waves) {
        const int f = unit % FY, j = unit / (2 * FY), row = 16 * (unit / FY & 1) + rq, m = m0 + 32 * j + row, c0 = f * 32 + 8 * cq;
        if (m >= a.M) continue;
        const float s_row = MX4 ? 0.0f : static_cast<const float*>(a.scales)[m];
        float s[HALVES][8];
        const float *scale[HALVES], *bias[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            scale[h] = scale_s + c0 + 32 * FY * h;
            bias[h] = bias_s + c0 + 32 * FY * h;
            sum_t sum[8] = {};
            for (int v = 0; v < waves; ++v)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const Four p = part_s[((v * FM + j) * FN + h * FY + f) * 256 + (2 * (cq & 1) + q) * 64 + row + 32 * (cq >> 1)];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[4 * q + e] += p.v[e];
                }
#pragma unroll
            for (int i = 0; i < 8; ++i) s[h][i] = R::value(sum[i], s_row);
        }
        finish_q<EPI, 8>(a, m, n0 + c0, s, scale, bias);
    }
}

// a.M, a.N, a.K > 0.
template <int ROWS, int EPI, int FM>
int launch_q_waves(QProductArgs a, hipStream_t s) {
    constexpr int BN = 64 / kQHalves<EPI>;
    const int64_t tiles_m = ceil_div(a.M, 32 * FM), tiles_n = ceil_div(a.N, BN), runs = ceil_div(a.K, kQWavesRunK);
    const int most = FM == 1 ? 8 : 4, waves = int(runs < most ? runs : most);
    if (tiles_m * tiles_n > max_blocks(64 * waves)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    q_waves_kernel<ROWS, EPI, FM><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(64 * waves), size_t(waves) * FM * 8192, s>>>(a);
    return check_launch();
}

}  // namespace bnn
