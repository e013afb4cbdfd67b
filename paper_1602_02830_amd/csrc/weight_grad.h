// The gradient of the weights as if they were real, dw[n][k] = scale[n] * sum_m g[m][n] x[m][k]: a product of two real
// matrices over their rows.
//
// Both operands lie with the summed index as their slow one, so a tile is staged as it lies in memory and the 16-bit types
// are turned on their way to registers by the transposing LDS read (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 elements
// and get 4 rows' elements of one column each); float32 goes through the matrix engine's float32 form, which takes one
// element a lane and needs no turning.
#pragma once

#include "gemm_staging.h"
#include "real_types.h"

namespace bnn {

struct WeightGradArgs {
    const void* g;             // [M][ld_g]
    const void* x;             // [M][ld_x]
    void* dw;                  // [F or 2 F][ld_dw], or null: only the sums are wanted
    const float* row_scale;    // [F] or null
    const uint32_t* w;         // the weights' bits [F][ld_w] for dscale, or null
    float* part;               // [tiles_k][F]: sum over the tile's k of dw / row_scale * w
    int64_t ld_g, ld_x, ld_dw, ld_w;
    int M, K;                  // rows; columns of x
    int cols;                  // columns of g
    int half, F;               // columns half .. 2 half of g are the second F rows of dw; columns F .. half of a half are none
    TileMap map;
};

constexpr int kGradTile = 128;

template <typename E>
__global__ __launch_bounds__(256) void weight_grad_kernel(const WeightGradArgs a) {
    constexpr int STEP = 32, PITCH = kGradTile + 32;          // a row's start moves on by half of the banks or a quarter
    using E8 = typename Vec8<E>::type;
    __shared__ __attribute__((aligned(32))) E gs[2][STEP * PITCH], xs[2][STEP * PITCH];
    __shared__ float sums_s[2][kGradTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wk = wave & 1, wn = wave >> 1, fr = lane & 31, fh = lane >> 5;
    int tn, tk;
    tile_of_block(blockIdx.x, a.map, tn, tk);
    const int n0 = tn * kGradTile, k0 = tk * kGradTile;

    E8 gv[2], xv[2];
    auto load = [&](int m0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = i * 256 + tid, m = m0 + (id >> 4), c = (id & 15) * 8;
            const int64_t row = min(m, a.M - 1);
            gv[i] = load8<E>(static_cast<const E*>(a.g) + row * a.ld_g + n0 + c, m < a.M ? a.cols - n0 - c : 0);
            xv[i] = load8<E>(static_cast<const E*>(a.x) + row * a.ld_x + k0 + c, m < a.M ? a.K - k0 - c : 0);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = i * 256 + tid, at = (id >> 4) * PITCH + (id & 15) * 8;
            *reinterpret_cast<E8*>(&gs[buf][at]) = gv[i];
            *reinterpret_cast<E8*>(&xs[buf][at]) = xv[i];
        }
    };

    v16f_t acc[2][2] = {};         // [block of k][block of n]
    if (a.M > 0) {
        load(0);
        store(0);
    }
    for (int m0 = 0, buf = 0; m0 < a.M; m0 += STEP, buf ^= 1) {
        __syncthreads();
        const bool more = m0 + STEP < a.M;
        if (more) load(m0 + STEP);
        if constexpr (is_f32<E>) {
#pragma unroll 4
            for (int t = 0; t < STEP / 2; ++t) {
                float xk[2], gn[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xk[i] = xs[buf][(2 * t + fh) * PITCH + wk * 64 + i * 32 + consecutive_rows(fr)];
                    gn[i] = gs[buf][(2 * t + fh) * PITCH + wn * 64 + i * 32 + fr];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(xk[i], gn[j], acc[i][j], 0, 0, 0);
            }
        } else {
            typedef short v4s_t __attribute__((ext_vector_type(4)));
            typedef short v8s_t __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
            // Lane i of a group of 16 reads row i / 4, four columns; the group's lanes get 16 columns in the order of
            // their source lanes, so the columns of x can come as consecutive_rows wants them.
            const int i = lane & 15, b = (lane >> 4) & 1, t = i & 3, row = 8 * fh + (i >> 2);
            const int col_k = 16 * (t & 1) + 8 * b + 4 * (t >> 1), col_n = 16 * b + 4 * t;
            auto read = [&](E* tile, int s, int col) {
                E* p = tile + (16 * s + row) * PITCH + col;
                const v4s_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)p);
                const v4s_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p + 4 * PITCH));
                return __builtin_bit_cast(E8, v8s_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            };
#pragma unroll
            for (int s = 0; s < STEP / 16; ++s) {
                E8 xk[2], gn[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    xk[q] = read(xs[buf], s, wk * 64 + q * 32 + col_k);
                    gn[q] = read(gs[buf], s, wn * 64 + q * 32 + col_n);
                }
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[q][j] = mfma16(xk[q], gn[j], acc[q][j]);
            }
        }
        if (more) store(buf ^ 1);
    }

    // Lane l has k = 16 fh .. 16 fh + 15 of column n = fr of each block.
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = n0 + wn * 64 + j * 32 + fr, second = c >= a.half ? 1 : 0, f = c - second * a.half;
        const bool there = c < a.cols && f < a.F;
        const int64_t n = int64_t(second) * a.F + f;
        const float scale = there && a.row_scale ? a.row_scale[n] : 1.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = k0 + wk * 64 + i * 32 + 16 * fh;
            if (!there || k >= a.K) continue;
            if (a.dw) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[i][j][8 * g + e] * scale;
                    store8<E>(static_cast<E*>(a.dw) + n * a.ld_dw + k + 8 * g, v, int64_t(a.K) - k - 8 * g);
                }
            }
            if (a.w) {
                const uint32_t bits = a.w[n * a.ld_w + (k >> 5)] >> (16 * fh);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k + e < a.K) sum += (bits >> e) & 1u ? acc[i][j][e] : -acc[i][j][e];
            }
        }
        sum += __shfl_xor(sum, 32);
        if (a.w && fh == 0) sums_s[wk][wn * 64 + j * 32 + fr] = sum;
    }
    if (!a.w) return;
    __syncthreads();
    if (tid < kGradTile && n0 + tid < a.F) a.part[int64_t(tk) * a.F + n0 + tid] = sums_s[0][tid] + sums_s[1][tid];
}

}  // namespace bnn
