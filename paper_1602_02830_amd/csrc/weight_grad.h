// The gradient of the weights as if they were real, dw[n][k] = scale[n] * sum_m g[m][n] x[m][k]: a product of two real
// matrices over their rows.
//
// Both operands lie with the summed index as their slow one, so a tile is staged as it lies in memory and turned on its way
// to registers by the transposing LDS read (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 elements and get 4 rows' elements
// of one column each).  A tile's rows lie 64 bytes past a multiple of the 256 bytes of all banks apart, so that the four rows
// of 64 bytes that 32 lanes read are the 64 banks.  float32 operands are staged as three bfloat16 terms each, of whose nine products
// all but the smallest are made: what is left out is below 2^-28 of a product.  An infinity times another operand's
// term of zero is a NaN where float32 has an infinity: a tile with a NaN is summed up once more from terms that are not zero.  Made for
// every tile, those cost a third of the kernel's time (4096 x 2048 x 2048: 351 us against 250); looking for a NaN costs 1 - 4 % (253 us).
#pragma once

#include "gemm_staging.h"
#include "real_types.h"

namespace bnn {

struct WeightGradArgs {
    const void* g;             // [M][ld_g]
    const void* x;             // [M][ld_x]
    void* dw;                  // [F or 2 F][ld_dw], or null: only the sums are wanted
    const float* row_scale;    // [F or 2 F] or null
    const uint32_t* w;         // the weights' bits [F][ld_w] for dscale, or null
    float* part;               // [tiles_k][F]: sum over the tile's k of dw / row_scale * w
    float* pieces;             // [splits][F or 2 F][K]: float32 sums over a part of the rows each, instead of dw and part
    int64_t ld_g, ld_x, ld_dw, ld_w;
    int M, K;                  // rows; columns of x
    int cols;                  // columns of g
    int half, F;               // columns half .. 2 half of g are the second F rows of dw; columns F .. half of a half are none
    int channels;              // rows of dw
    int splits, split_rows;    // rows of M that a workgroup sums: a multiple of kGradStep
    TileMap map;
};

constexpr int kGradStep = 32;          // rows a step

// TK wavefronts along k, TN along n, 32-column blocks FK x FN for each.
template <typename E, int TK, int TN, int FK, int FN>
struct GradTile {
    static constexpr int kThreads = 64 * TK * TN, BK = 32 * TK * FK, BN = 32 * TN * FN;
    static constexpr int kTerms = is_f32<E> ? 3 : 1;
    static constexpr int kBuffers = is_f32<E> ? 2 : 3;
    static constexpr int kPitchK = BK + 32, kPitchN = BN + 32;
    static constexpr int kChunksK = kGradStep * BK / 8 / kThreads, kChunksN = kGradStep * BN / 8 / kThreads;
};

// GENERAL: fewer than eight columns on a side.
template <typename E, int TK, int TN, int FK, int FN, bool GENERAL>
__global__ __launch_bounds__(64 * TK * TN) void weight_grad_kernel(const WeightGradArgs a) {
    using S = GradTile<E, TK, TN, FK, FN>;
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    using E8 = typename Vec8<E>::type;
    __shared__ __attribute__((aligned(16))) O gs[S::kBuffers][S::kTerms][kGradStep * S::kPitchN];
    __shared__ __attribute__((aligned(16))) O xs[S::kBuffers][S::kTerms][kGradStep * S::kPitchK];
    __shared__ float sums_s[TK][S::BN];
    __shared__ int none_s[TK * TN];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wk = wave % TK, wn = wave / TK, fr = lane & 31, fh = lane >> 5;
    int tile = blockIdx.x, split = 0, tn, tk;
    if (a.splits > 1) {
        split = tile % a.splits;
        tile /= a.splits;
    }
    tile_of_block(tile, a.map, tn, tk);
    const int n0 = tn * S::BN, k0 = tk * S::BK;
    const int64_t m_first = int64_t(split) * a.split_rows;
    const int rows = int(min(int64_t(a.M) - m_first, int64_t(a.split_rows)));          // > 0 unless M is 0

    // Chunk i of a thread: a row of the step and eight columns.  Loads ask no questions: what lies past a row's end is loaded from its
    // last eight elements instead, rows that are not there from the last one, and both are put right on the way to LDS.
    const char* const g_first = static_cast<const char*>(a.g) + (m_first * a.ld_g + n0) * int64_t(sizeof(E));
    const char* const x_first = static_cast<const char*>(a.x) + (m_first * a.ld_x + k0) * int64_t(sizeof(E));
    const char *gp = g_first, *xp = x_first;
    E8 gv[S::kChunksN], xv[S::kChunksK];
    const int left_n = a.cols - n0, left_k = a.K - k0;
    const bool inside = left_n >= S::BN && left_k >= S::BK;
    auto load = [&](int t) {
        const int left = rows - t * kGradStep;               // rows from this step on
#pragma unroll
        for (int i = 0; i < S::kChunksN; ++i) {
            const int id = i * S::kThreads + tid, r = id / (S::BN / 8), c = id % (S::BN / 8) * 8;
            if constexpr (GENERAL) gv[i] = load8<E>(reinterpret_cast<const E*>(gp) + int64_t(min(r, left - 1)) * a.ld_g + c, left_n - c);
            else gv[i] = *reinterpret_cast<const typename Vec8<E>::any*>(gp + (int64_t(min(r, left - 1)) * a.ld_g + min(c, left_n - 8)) * int64_t(sizeof(E)));
        }
#pragma unroll
        for (int i = 0; i < S::kChunksK; ++i) {
            const int id = i * S::kThreads + tid, r = id / (S::BK / 8), c = id % (S::BK / 8) * 8;
            if constexpr (GENERAL) xv[i] = load8<E>(reinterpret_cast<const E*>(xp) + int64_t(min(r, left - 1)) * a.ld_x + c, left_k - c);
            else xv[i] = *reinterpret_cast<const typename Vec8<E>::any*>(xp + (int64_t(min(r, left - 1)) * a.ld_x + min(c, left_k - 8)) * int64_t(sizeof(E)));
        }
        gp += kGradStep * a.ld_g * int64_t(sizeof(E));
        xp += kGradStep * a.ld_x * int64_t(sizeof(E));
    };
    auto store = [&](int t, int buf, auto nonzero) {
        const int left = rows - t * kGradStep;
        if (left < kGradStep || (!GENERAL && !inside)) {
#pragma unroll
            for (int i = 0; i < S::kChunksN; ++i) {
                const int id = i * S::kThreads + tid, r = id / (S::BN / 8), c = id % (S::BN / 8) * 8;
                gv[i] = row_end<E>(gv[i], r >= left ? 0 : GENERAL ? 8 : left_n - c);
            }
#pragma unroll
            for (int i = 0; i < S::kChunksK; ++i) {
                const int id = i * S::kThreads + tid, r = id / (S::BK / 8), c = id % (S::BK / 8) * 8;
                xv[i] = row_end<E>(xv[i], r >= left ? 0 : GENERAL ? 8 : left_k - c);
            }
        }
        auto write = [&](auto* dst, int at, const E8& v) {       // dst: the buffer's terms
            O8 t[S::kTerms];
            terms_of<E, decltype(nonzero)::value>(v, t);
#pragma unroll
            for (int p = 0; p < S::kTerms; ++p) *reinterpret_cast<O8*>(&dst[p][at]) = t[p];
        };
#pragma unroll
        for (int i = 0; i < S::kChunksN; ++i) {
            const int id = i * S::kThreads + tid;
            write(gs[buf], id / (S::BN / 8) * S::kPitchN + id % (S::BN / 8) * 8, gv[i]);
        }
#pragma unroll
        for (int i = 0; i < S::kChunksK; ++i) {
            const int id = i * S::kThreads + tid;
            write(xs[buf], id / (S::BK / 8) * S::kPitchK + id % (S::BK / 8) * 8, xv[i]);
        }
    };

    // Lane i of a group of 16 reads row i / 4, four columns; the group's lanes get 16 columns in the order of their source
    // lanes, so the columns of x can come as consecutive_rows wants them.
    typedef short v4s_t __attribute__((ext_vector_type(4)));
    typedef short v8s_t __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
    const int i16 = lane & 15, b16 = (lane >> 4) & 1, t4 = i16 & 3, row = 8 * fh + (i16 >> 2);
    const int at_k = row * S::kPitchK + wk * FK * 32 + 16 * (t4 & 1) + 8 * b16 + 4 * (t4 >> 1);
    const int at_n = row * S::kPitchN + wn * FN * 32 + 16 * b16 + 4 * t4;
    auto turned = [&](O* p, int four_rows) {
        const v4s_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)p);
        const v4s_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(p + four_rows));
        return __builtin_bit_cast(O8, v8s_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    };
    v16f_t acc[FK][FN] = {};
    O8 xf[2][S::kTerms][FK], gf[2][S::kTerms][FN];
    auto read = [&](int to, int buf, int s) {
#pragma unroll
        for (int p = 0; p < S::kTerms; ++p) {
#pragma unroll
            for (int i = 0; i < FK; ++i) xf[to][p][i] = turned(&xs[buf][p][at_k + 16 * s * S::kPitchK + 32 * i], 4 * S::kPitchK);
#pragma unroll
            for (int j = 0; j < FN; ++j) gf[to][p][j] = turned(&gs[buf][p][at_n + 16 * s * S::kPitchN + 32 * j], 4 * S::kPitchN);
        }
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int p = 0; p < S::kTerms; ++p)
#pragma unroll
            for (int q = 0; q < S::kTerms && q + p < 4; ++q)          // all but the product of the two smallest
#pragma unroll
                for (int i = 0; i < FK; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = mfma16(xf[from][p][i], gf[from][q][j], acc[i][j]);
    };
    static_assert(kGradStep == 32, "two products of 16 rows a step");
    const int steps = (rows + kGradStep - 1) / kGradStep;
    auto sum_up = [&](auto nonzero) {
        if (steps <= 0) return;
        load(0);
        store(0, 0, nonzero);
        if (steps > 1) load(1);
        __syncthreads();
        read(0, 0, 0);
        int buf = 0;
        for (int t = 0; t < steps; ++t) {
            const int next = buf == S::kBuffers - 1 ? 0 : buf + 1;
            const bool more = t + 1 < steps;
            // Three buffers: `next` held step t - 2, which every wavefront has left behind since the barrier in step t - 1.
            if constexpr (S::kBuffers == 3) {
                if (more) store(t + 1, next, nonzero);
            }
            if (S::kBuffers == 3 ? t + 2 < steps : t > 0 && more) load(S::kBuffers == 3 ? t + 2 : t + 1);
            read(1, buf, 1);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (S::kBuffers == 3) {
                __syncthreads();
                read(0, next, 0);              // after the last step: read, not used
            }
            multiply(1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (S::kBuffers == 2) {
                // Two buffers: `next` held step t - 1, which everyone had left before the barrier at this step's start.
                if (more) {
                    store(t + 1, next, nonzero);
                    __syncthreads();
                    read(0, next, 0);
                }
            }
            buf = next;
        }
    };
    sum_up(std::false_type{});
    if constexpr (is_f32<E>) {
        float all = 0.0f;                      // no number if one of them is none
#pragma unroll
        for (int i = 0; i < FK; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) all += acc[i][j][e];
        const bool in_wave = __ballot(all != all) != 0;
        if (lane == 0) none_s[wave] = in_wave;
        __syncthreads();
        int any = 0;
#pragma unroll
        for (int w = 0; w < TK * TN; ++w) any |= none_s[w];
        if (any) {
#pragma unroll
            for (int i = 0; i < FK; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = v16f_t{};
            gp = g_first;
            xp = x_first;
            sum_up(std::true_type{});
        }
    }

    // Lane l has k = 16 fh .. 16 fh + 15 of column n = fr of each block.
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int c = n0 + (wn * FN + j) * 32 + fr, second = c >= a.half ? 1 : 0, f = c - second * a.half;
        const bool there = c < a.cols && f < a.F;
        const int64_t n = int64_t(second) * a.F + f;
        const float scale = there && a.row_scale ? a.row_scale[n] : 1.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < FK; ++i) {
            const int k = k0 + (wk * FK + i) * 32 + 16 * fh;
            if (!there || k >= a.K) continue;
            if (a.pieces) {
                float* const out = a.pieces + (int64_t(split) * a.channels + n) * a.K + k;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[i][j][8 * g + e];
                    store8<float>(out + 8 * g, v, int64_t(a.K) - k - 8 * g);
                }
                continue;
            }
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
        if (a.w && fh == 0) sums_s[wk][(wn * FN + j) * 32 + fr] = sum;
    }
    if (!a.w || a.pieces) return;
    __syncthreads();
    for (int c = tid; c < S::BN; c += S::kThreads) {
        if (n0 + c >= a.F) continue;
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < TK; ++t) sum += sums_s[t][c];
        a.part[int64_t(tk) * a.F + n0 + c] = sum;
    }
}

// What the parts of the rows have, joined: dw and dscale of one row of dw a workgroup.
template <typename E>
__global__ __launch_bounds__(256) void join_pieces_kernel(const WeightGradArgs a, float* dscale) {
    __shared__ float sums_s[4];
    const int64_t n = blockIdx.x;
    const float scale = a.row_scale ? a.row_scale[n] : 1.0f;
    float sum = 0.0f;
    for (int64_t k = int64_t(threadIdx.x) * 8; k < a.K; k += 256 * 8) {
        float v[8] = {};
        for (int s = 0; s < a.splits; ++s) {
            const auto p = load8<float>(a.pieces + (int64_t(s) * a.channels + n) * a.K + k, a.K - k);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += p[e];
        }
        if (a.w) {
            const uint32_t bits = a.w[n * a.ld_w + (k >> 5)] >> (k & 31);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k + e < a.K) sum += (bits >> e) & 1u ? v[e] : -v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        if (a.dw) store8<E>(static_cast<E*>(a.dw) + n * a.ld_dw + k, v, a.K - k);
    }
    if (!a.w) return;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if ((threadIdx.x & 63) == 0) sums_s[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) dscale[n] = (sums_s[0] + sums_s[1]) + (sums_s[2] + sums_s[3]);
}

}  // namespace bnn
