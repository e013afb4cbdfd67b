// The same product and epilogues for problems that do not fill the chip with large tiles: every wavefront of a workgroup has
// the whole tile to itself and runs of K are dealt to them, so that no wavefront waits for another until the sums meet in LDS.
//
// What bounds small products is not arithmetic but waiting: a call is a few trips to memory, and shared through LDS, a step of 16
// matrix operations (512 cycles of them) took 1600 - 2000 cycles of barriers and LDS reads on tiles of 64 - 128 rows.  Here a
// wavefront loads its operands as the matrix engine wants them, a run of K at a time, and the next run's in the place of
// what it has just multiplied.  The price is the cache's: it looks up one line a cycle for four neighbouring lanes, which
// here are four rows, so a load of 1 KB takes 64 cycles of it.  Through a piece of LDS of each wavefront's own, filled in
// whole lines, larger products were faster (64 x 4096 x 8192: 15.7 us against 20.5), but those that are left to this kernel slower
// (333 x 2 x 2047 x 1000: 11.2 us against 9.4).
#pragma once

#include "bits_product.h"

namespace bnn {

constexpr int kRunK = 256;          // elements of K a wavefront takes at a time: half of it has 128, four words of a row of weights

// Tiles of 32 FM rows and 32 FN channels.
template <typename E, int EPI, int FM, int FN>
struct WavesTile {
    static constexpr int HALVES = kHalves<EPI>, FY = FN / HALVES;
    static constexpr int BM = 32 * FM, CN = 32 * FN, BN = CN / HALVES;
    static size_t lds_bytes(int waves) { return size_t(waves) * FM * FN * 4096; }
};

// The word of a row of weights that 32 elements from 32 i on are in.
__device__ inline uint32_t word_of(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }

// Rows of 16-bit elements that do not begin with a 32-bit word: a 16-byte load from the middle of a word takes the cache more than
// twice as long (93 x 295 x 4979 float16: 29.3 us, K = 4978 11.9).  So (ODD) a lane loads whole words from the one on that its
// first element is in, one more than its elements fill, and shifts them together where its row needs that (12.7 us).  Every word
// has an element of the row in it.  The row's last, partial run is loaded as it lies.
struct WholeWords {
    uint32_t by;                         // bits
    template <typename E>
    __device__ inline explicit WholeWords(const E* row) : by(8 * (uint32_t(reinterpret_cast<uintptr_t>(row)) & 3u)) {}
    // Eight elements, of which `after` holds the last one.
    template <typename V>
    __device__ inline V operator()(const V& v, uint32_t after) const {
        const v4u_t q = __builtin_bit_cast(v4u_t, v);
        return __builtin_bit_cast(V, v4u_t{__builtin_amdgcn_alignbit(q[1], q[0], by), __builtin_amdgcn_alignbit(q[2], q[1], by),
                                           __builtin_amdgcn_alignbit(q[3], q[2], by), __builtin_amdgcn_alignbit(after, q[3], by)});
    }
};
template <typename V>
__device__ inline uint32_t first_word(const V& v) {
    return __builtin_bit_cast(v4u_t, v)[0];
}
template <typename E>
__device__ inline const E* word_begin(const E* p) {
    return reinterpret_cast<const E*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
}
// Some rows begin inside a word, and are longer than `longer`: below that the partial run is most of the row.
template <typename E>
inline bool odd_rows(const ProductArgs& a, int longer) {
    return !is_f32<E> && a.K > longer && (!aligned_to(a.x, 4) || a.ld_x % 2 != 0);
}

template <typename E, int EPI, int FM, int FN, bool ODD>
__global__ __launch_bounds__(512) void bits_waves_kernel(const ArgsOf<EPI> a) {
    using S = WavesTile<E, EPI, FM, FN>;
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    using E8 = typename Vec8<E>::type;
    constexpr int HALVES = S::HALVES, FY = S::FY, TERMS = kTermsOf<E>;
    constexpr bool BACK = kBackward<EPI>;
    extern __shared__ __attribute__((aligned(16))) float4 part_s[];       // the sums, [wavefront][row block][block][register / 4][lane]
    __shared__ float scale_s[S::CN], bias_s[S::CN];
    __shared__ float sums_s[BACK ? FM * 2 * S::CN : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int fr = lane & 31, fh = lane >> 5;
    int tm, tn;
    tile_of_block(blockIdx.x, a.map, tm, tn);
    const int m0 = tm * S::BM, n0 = tn * S::BN, kw = (a.K + 31) >> 5;

    const FactorOf<E, EPI> factor_parts(a);
    // Block f of the tile: columns n0 + 32 (f % FY) of half f / FY.
    for (int c = tid; c < S::CN; c += blockDim.x) {
        const int f = c >> 5, col = n0 + (f % FY) * 32 + (c & 31);
        const int64_t row = int64_t(f / FY) * a.N + col;
        const bool there = col < a.N;
        scale_s[c] = there && a.scale ? a.scale[row] : 1.0f;
        bias_s[c] = there && a.bias ? a.bias[row] : 0.0f;
    }
    const uint32_t* wrow[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f)
        wrow[f] = a.w + (int64_t(f / FY) * a.N + min(n0 + (f % FY) * 32 + consecutive_rows(fr), a.N - 1)) * a.ld_w;
    const E* xrow[FM];
#pragma unroll
    for (int j = 0; j < FM; ++j) xrow[j] = static_cast<const E*>(a.x) + int64_t(min(m0 + 32 * j + fr, a.M - 1)) * a.ld_x;

    uint4 wv[FN];
    auto load_w = [&](int r) {
        const int w0 = 8 * r + 4 * fh;
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            if (w0 + 4 <= kw) wv[f] = load_quad_any(wrow[f] + w0);
            else wv[f] = make_uint4(wrow[f][min(w0, kw - 1)], wrow[f][min(w0 + 1, kw - 1)], wrow[f][min(w0 + 2, kw - 1)], 0u);
        }
    };
    E8 xv[4][FM][4];                     // [quarter of a run][block][group of eight elements]
    uint32_t after[FM];                  // the word past a run
    auto load_x = [&](int r, int i) {
        const int64_t k = int64_t(r) * kRunK + 128 * fh + 32 * i;
        if ((r + 1) * int64_t(kRunK) <= a.K) {
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    xv[i][j][s] = *reinterpret_cast<const typename Vec8<E>::any*>((ODD ? word_begin(xrow[j]) : xrow[j]) + k + 8 * s);
            if constexpr (ODD) {
                // Also where the row begins with a word: what follows it is then not looked at, and need not be there.
                if (i == 3) {
#pragma unroll
                    for (int j = 0; j < FM; ++j) after[j] = *reinterpret_cast<const uint32_t*>(word_begin(xrow[j] + k + 31));
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int s = 0; s < 4; ++s) xv[i][j][s] = load8<E>(xrow[j] + k + 8 * s, a.K - k - 8 * s);
        }
    };
    const Widening<O> minus_weights;
    v16f_t acc[FN][FM] = {};
    const int runs = (a.K + kRunK - 1) / kRunK;
    if (wave < runs) {
        load_w(wave);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_x(wave, i);
    }
    const float factor = factor_parts(a);                  // while those are on their way
    for (int r = wave; r < runs; r += waves) {
        uint4 wc[FN];
#pragma unroll
        for (int f = 0; f < FN; ++f) wc[f] = wv[f];
        const bool more = r + waves < runs;
        if (more) load_w(r + waves);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (int64_t(r) * kRunK + 32 * i >= a.K) break;                 // nothing left for either half
            if constexpr (ODD) {
                if ((r + 1) * int64_t(kRunK) <= a.K) {
#pragma unroll
                    for (int j = 0; j < FM; ++j) {
                        const WholeWords whole(xrow[j]);
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            xv[i][j][s] = whole(xv[i][j][s], s < 3 ? first_word(xv[i][j][s + 1]) : i < 3 ? first_word(xv[i + 1][j][0]) : after[j]);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                O8 wf[FN];
#pragma unroll
                for (int f = 0; f < FN; ++f) {
                    const uint32_t word = word_of(wc[f], i);
                    wf[f] = minus_weights(s < 2 ? spread_low(word) : spread_high(word), s & 1);
                }
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    O8 term[TERMS];
                    terms_of<E>(xv[i][j][s], term);
#pragma unroll
                    for (int p = 0; p < TERMS; ++p)
#pragma unroll
                        for (int f = 0; f < FN; ++f) acc[f][j] = mfma16(wf[f], term[p], acc[f][j]);
                }
            }
            if (more) load_x(r + waves, i);
        }
    }

    // The sums; then a lane has eight columns of a row.
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part_s[((wave * FM + j) * FN + f) * 256 + q * 64 + lane] =
                    make_float4(acc[f][j][4 * q], acc[f][j][4 * q + 1], acc[f][j][4 * q + 2], acc[f][j][4 * q + 3]);
    __syncthreads();
    for (int unit = wave; unit < 2 * FM * FY; unit += waves) {
        const int g = unit & 1, f = (unit >> 1) % FY, j = (unit >> 1) / FY;
        float sums[HALVES][8] = {}, sum_s[HALVES][8] = {}, sum_z[HALVES][8] = {};
        for (int v = 0; v < waves; ++v)
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 p = part_s[((v * FM + j) * FN + h * FY + f) * 256 + (2 * g + q) * 64 + lane];
                    sums[h][4 * q] -= p.x;
                    sums[h][4 * q + 1] -= p.y;
                    sums[h][4 * q + 2] -= p.z;
                    sums[h][4 * q + 3] -= p.w;
                }
        const int c0 = f * 32 + 16 * fh + 8 * g;
        const float *scale[HALVES], *bias[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            scale[h] = scale_s + c0 + 32 * FY * h;
            bias[h] = bias_s + c0 + 32 * FY * h;
        }
        finish<E, EPI, 8>(a, m0 + j * 32 + fr, n0 + c0, sums, scale, bias, factor, sum_s, sum_z);
        if constexpr (BACK) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = sum_of_32(sum_s[h][i]), q = sum_of_32(sum_z[h][i]);
                    if (fr == 0) {
                        sums_s[(j * 2) * S::CN + c0 + 32 * FY * h + i] = p;
                        sums_s[(j * 2 + 1) * S::CN + c0 + 32 * FY * h + i] = q;
                    }
                }
        }
    }
    if constexpr (BACK) {
        __syncthreads();
        for (int c = tid; c < S::CN; c += blockDim.x) {
            const int f = c >> 5, col = n0 + (f % FY) * 32 + (c & 31);
            if (col >= a.N) continue;
            float p = 0.0f, q = 0.0f;
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                p += sums_s[(j * 2) * S::CN + c];
                q += sums_s[(j * 2 + 1) * S::CN + c];
            }
            const int64_t at = int64_t(tm) * a.channels + int64_t(f / FY) * a.N + col;
            if (a.part_scale) a.part_scale[at] = p;
            if (a.part_bias) a.part_bias[at] = q;
        }
    }
}

// ---- tiles of 16 rows ---------------------------------------------------------------------------------------------
// Blocks of 16 channels, so that narrow layers still have a workgroup for every compute unit, and runs of 512 elements of K, of
// which a quarter of a wavefront has 128: one 16-byte load of each row of weights.  All of a run's loads are on their way before
// the first arrives, so a call takes one trip to memory for each run that a wavefront has, and the widening of the weights.
// Beyond 16 rows these tiles are twice as many as those above, with half as much of x to look up for each: faster as long as two rounds
// of the chip hold them (64 x 8192 -> 512, 128 of them: 10.3 us against 19.5; 128 x 4096 -> 1024, 512: 10.4 against 11.7;
// 256 x 4096 -> 1024, 1024: 17.8 against 11.9).

constexpr int kSmallRunK = 512, kSmallRows = 16;

// FN blocks of 16 channels (gated: of each half).
template <typename E, int EPI, int FN, bool ODD>
__global__ __launch_bounds__(512) void bits_small_kernel(const ArgsOf<EPI> a) {
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    constexpr int HALVES = kHalves<EPI>, BLOCKS = FN * HALVES, TERMS = kTermsOf<E>;
    constexpr bool BACK = kBackward<EPI>;
    extern __shared__ __attribute__((aligned(16))) float4 part_s[];       // [wavefront][block][lane]
    __shared__ float scale_s[BLOCKS * 16], bias_s[BLOCKS * 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int r16 = lane & 15, quarter = lane >> 4, kw = (a.K + 31) >> 5;
    const int tm = int(blockIdx.y), n0 = int(blockIdx.x) * (16 * FN), m = tm * kSmallRows + r16;

    const FactorOf<E, EPI> factor_parts(a);
    // Block b: columns n0 + 16 (b % FN) of half b / FN.
    for (int c = tid; c < BLOCKS * 16; c += blockDim.x) {
        const int b = c >> 4, col = n0 + (b % FN) * 16 + (c & 15);
        const int64_t at = int64_t(b / FN) * a.N + col;
        scale_s[c] = col < a.N && a.scale ? a.scale[at] : 1.0f;
        bias_s[c] = col < a.N && a.bias ? a.bias[at] : 0.0f;
    }
    const Widening<O> minus_weights;
    const E* const xrow = static_cast<const E*>(a.x) + int64_t(min(m, a.M - 1)) * a.ld_x;
    v4f_t acc[BLOCKS] = {};
    for (int64_t k0 = int64_t(wave) * kSmallRunK; k0 < a.K; k0 += int64_t(waves) * kSmallRunK) {
        const int64_t k = k0 + 128 * quarter;
        const int w0 = int(k >> 5);
        uint4 w[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const uint32_t* const row = a.w + (int64_t(b / FN) * a.N + min(n0 + (b % FN) * 16 + r16, a.N - 1)) * a.ld_w;
            if (w0 + 4 <= kw) w[b] = load_quad_any(row + w0);
            else w[b] = make_uint4(row[min(w0, kw - 1)], row[min(w0 + 1, kw - 1)], row[min(w0 + 2, kw - 1)], 0u);
        }
        typename Vec8<E>::type xv[16];
        if (k0 + kSmallRunK <= a.K) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                xv[i] = *reinterpret_cast<const typename Vec8<E>::any*>((ODD ? word_begin(xrow) : xrow) + k + 8 * i);
            if constexpr (ODD) {
                const uint32_t after = *reinterpret_cast<const uint32_t*>(word_begin(xrow + k + 127));
                const WholeWords whole(xrow);
#pragma unroll
                for (int i = 0; i < 16; ++i) xv[i] = whole(xv[i], i < 15 ? first_word(xv[i + 1]) : after);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) xv[i] = load8<E>(xrow + k + 8 * i, a.K - k - 8 * i);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            O8 term[TERMS];
            terms_of<E>(xv[i], term);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const uint32_t word = word_of(w[b], i >> 2);
                const O8 wf = minus_weights((i & 2) ? spread_high(word) : spread_low(word), i & 1);
#pragma unroll
                for (int p = 0; p < TERMS; ++p) acc[b] = mfma32(wf, term[p], acc[b]);
            }
        }
    }
    const float factor = factor_parts(a);
    // Lane: columns 4 quarter .. 4 quarter + 3 of row m of each block.
    if (m < a.M) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) part_s[(wave * BLOCKS + b) * 64 + lane] = make_float4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
    }
    __syncthreads();
    for (int f = wave; f < FN; f += waves) {
        if (!BACK && m >= a.M) continue;           // backwards all lanes are in the sums, those of no row with nothing
        float s[HALVES][4] = {}, sum_s[HALVES][4] = {}, sum_z[HALVES][4] = {};
        const float *scale[HALVES], *bias[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            scale[h] = scale_s + (h * FN + f) * 16 + 4 * quarter;
            bias[h] = bias_s + (h * FN + f) * 16 + 4 * quarter;
            for (int v = 0; v < waves; ++v) {
                const float4 p = part_s[(v * BLOCKS + h * FN + f) * 64 + lane];
                s[h][0] -= p.x;
                s[h][1] -= p.y;
                s[h][2] -= p.z;
                s[h][3] -= p.w;
            }
        }
        finish<E, EPI, 4>(a, m, n0 + f * 16 + 4 * quarter, s, scale, bias, factor, sum_s, sum_z);
        if constexpr (BACK) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int off = 8; off > 0; off >>= 1) {
                        sum_s[h][i] += __shfl_xor(sum_s[h][i], off);
                        sum_z[h][i] += __shfl_xor(sum_z[h][i], off);
                    }
                    const int col = n0 + f * 16 + 4 * quarter + i;
                    if (r16 != 0 || col >= a.N) continue;
                    const int64_t at = int64_t(tm) * a.channels + int64_t(h) * a.N + col;
                    if (a.part_scale) a.part_scale[at] = sum_s[h][i];
                    if (a.part_bias) a.part_bias[at] = sum_z[h][i];
                }
        }
    }
}

template <typename E, int EPI, int FN>
int launch_small(const ArgsOf<EPI>& a, int waves, hipStream_t s) {
    const int64_t blocks = ceil_div(kBackward<EPI> ? a.half : a.N, 16 * FN), tiles_m = ceil_div(a.M, kSmallRows);
    if (blocks * tiles_m > max_blocks(64 * waves) || tiles_m > 65535) return BNN_ERR_UNSUPPORTED;
    const dim3 grid{uint32_t(blocks), uint32_t(tiles_m)}, block{uint32_t(64 * waves)};
    const size_t lds = size_t(waves) * FN * kHalves<EPI> * 1024;
    if constexpr (!is_f32<E>) {
        // Up to four rows are few lines, and the extra word costs more (1 x 4095 -> 4096: 4.4 us against 4.9).
        if (a.M > 4 && odd_rows<E>(a, 2 * kSmallRunK)) {
            bits_small_kernel<E, EPI, FN, true><<<grid, block, lds, s>>>(a);
            return check_launch();
        }
    }
    bits_small_kernel<E, EPI, FN, false><<<grid, block, lds, s>>>(a);
    return check_launch();
}

template <typename E, int EPI, int FM, int FN>
int launch_waves(ArgsOf<EPI> a, int waves, hipStream_t s) {
    using S = WavesTile<E, EPI, FM, FN>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(kBackward<EPI> ? a.half : a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(64 * waves)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    const dim3 grid(uint32_t(tiles_m * tiles_n)), block(64 * waves);
    if constexpr (!is_f32<E>) {
        if (odd_rows<E>(a, kRunK)) {
            bits_waves_kernel<E, EPI, FM, FN, true><<<grid, block, S::lds_bytes(waves), s>>>(a);
            return check_launch();
        }
    }
    bits_waves_kernel<E, EPI, FM, FN, false><<<grid, block, S::lds_bytes(waves), s>>>(a);
    return check_launch();
}

}  // namespace bnn
