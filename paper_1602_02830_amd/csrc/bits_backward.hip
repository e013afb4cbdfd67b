// Backward passes of the products with packed weights: bnn_linear_bits_backward and bnn_gated_bits_backward.
//
//   1. the gradient before the scale, ds = dz * scale, in the activations' type.  With an activation (or a gate) the product
//      of the forward pass is made again and its epilogue turns the sums into ds and the column sums for dscale and dbias
//      while they are in registers; without one, dz is dy: a pass over dy makes ds and dbias (nothing at all without a scale).
//      Rounding ds to 16 bits is what lets the next two products run on 16-bit matrix instructions, and halves its way through
//      memory; their sums, and the column sums, which are taken before it, have 32 bits.  float16 gradients are stored times a power
//      of two (stored_gradient.h) whose bounds are looked up first, in the launch that transposes the weights.
//   2. dx = ds w: the same tile product as forwards, on the weights' bits transposed (a 16th or a 32nd of an operand's bytes).
//   3. dw = ds^T x.  Without an activation it is made of dy itself, the scale put on the sums, and
//      dscale[n] = sum_k w[n][k] sum_m dy[m][n] x[m][k] comes out of the same sums.
//   4. column sums of the tiles joined, in a fixed order.
#include "bit_transpose.h"
#include "bits_launch.h"
#include "join_sums.h"
#include "weight_grad.h"

namespace bnn {

namespace {

// ---- transposed weights ------------------------------------------------------------------------------------------
// out[k] bit n of a row of `half` columns a half: w[n][k] and, from column `half` on, w[F + n][k]; 0 for rows that are not there.
// A workgroup turns 256 rows x 128 columns: each half wavefront blocks of 32 x 32 in registers, LDS puts words of a row together.
constexpr int kTurnWords = 8, kTurnK = 128;

struct TurnArgs {
    const uint32_t* w;
    uint32_t* out;
    int64_t ld_w, ld_out;
    int F, half, halves, K, blocks_k;
    int blocks;                // workgroups that transpose; 0: none is wanted
};

__device__ inline void transpose_weights(const TurnArgs& a) {
    __shared__ uint32_t turned[kTurnK][kTurnWords + 1];
    const int tid = threadIdx.x, half_wave = tid >> 5, l = tid & 31;
    const int bn = blockIdx.x / uint32_t(a.blocks_k), bk = int(blockIdx.x) - bn * a.blocks_k;
    const int word0 = bn * kTurnWords, k0 = bk * kTurnK, words = a.half * a.halves / 32, kw = (a.K + 31) >> 5;
#pragma unroll
    for (int i = 0; i < kTurnWords * 4 / 8; ++i) {
        const int b = i * 8 + half_wave, wn = b >> 2, q = b & 3;
        const int c = (word0 + wn) * 32 + l, second = c >= a.half ? 1 : 0, f = c - second * a.half;
        const int kword = (k0 >> 5) + q;
        uint32_t v = 0;
        if (word0 + wn < words && f < a.F && kword < kw) v = a.w[(int64_t(second) * a.F + f) * a.ld_w + kword];
        turned[q * 32 + l][wn] = transpose_bits_32_lanes(v);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurnK * kTurnWords / 256; ++i) {
        const int id = i * 256 + tid, row = id / kTurnWords, wn = id % kTurnWords;
        if (k0 + row < a.K && word0 + wn < words) a.out[int64_t(k0 + row) * a.ld_out + word0 + wn] = turned[row][wn];
    }
}

// ---- bounds of float16 gradients (stored_gradient.h) ---------------------------------------------------------------

struct BoundArgs {
    const f16_t *dy, *x;       // x: null where the bound does not need it
    const float *scale, *bias;
    float* parts;              // as GradientBounds has them
    int64_t ld_dy, ld_x, M;
    int cols, K, channels;
    int lanes;                 // of a wavefront that take a row together: a power of two, 8 at least
    int lookers;
    int blocks;                // workgroups: one at the scale, one at the bias, and the lookers; 0: none
};

__device__ inline void look_for_bounds(const BoundArgs& a, int block) {
    __shared__ float2 wave_s[4];
    const int tid = threadIdx.x;
    float most = 0.0f, both = 0.0f;
    if (block < 2) {
        const float* const v = block == 0 ? a.scale : a.bias;
        if (v) most = largest_of_row(v + int64_t(tid >> 6) * (a.channels / 4), tid < 192 ? a.channels / 4 : a.channels - 3 * (a.channels / 4), tid & 63, 64);
        else most = block == 0 ? 1.0f : 0.0f;
    } else {
        const int per_block = 256 / a.lanes, lane = tid & (a.lanes - 1);
        for (int64_t m = int64_t(block - 2) * per_block + tid / a.lanes; m < a.M; m += int64_t(a.lookers) * per_block) {
            if (!a.x) {
                most = fmaxf(most, largest_of_row(a.dy + m * a.ld_dy, a.cols, lane, a.lanes));
                continue;
            }
            RowMagnitude<f16_t, false> dy(a.dy + m * a.ld_dy, a.cols, lane, a.lanes);
            RowMagnitude<f16_t, true> x(a.x + m * a.ld_x, a.K, lane, a.lanes);
            for (int first = 0; first < max(dy.groups, x.groups); first += 4 * a.lanes) {
                if (first < dy.groups) dy.load(first);
                if (first < x.groups) x.load(first);
                if (first < dy.groups) dy.take(first);
                if (first < x.groups) x.take(first);
            }
            const float largest = dy.over_lanes();
            most = fmaxf(most, largest);
            both = fmaxf(both, largest * x.over_lanes());
        }
    }
    most = largest_of_wave(most);
    both = largest_of_wave(both);
    if ((tid & 63) == 0) wave_s[tid >> 6] = make_float2(most, both);
    __syncthreads();
    if (tid != 0) return;
    a.parts[block] = fmaxf(fmaxf(wave_s[0].x, wave_s[1].x), fmaxf(wave_s[2].x, wave_s[3].x));
    if (block >= 2) a.parts[block + a.lookers] = fmaxf(fmaxf(wave_s[0].y, wave_s[1].y), fmaxf(wave_s[2].y, wave_s[3].y));
}

// What the products need and what does not wait for them, in one launch: workgroups that transpose, then those that look.  LOOK: there
// are some, whose loads in flight take registers: 4 wavefronts a SIMD instead of 8.
template <bool LOOK>
__global__ __launch_bounds__(256) void prepare_kernel(const TurnArgs t, const BoundArgs b) {
    if (!LOOK || int(blockIdx.x) < t.blocks) transpose_weights(t);
    else look_for_bounds(b, int(blockIdx.x) - t.blocks);
}

// ---- dy * scale and the column sums of dy ------------------------------------------------------------------------
// A workgroup takes `strip` rows x 512 columns, a thread eight columns of every fourth row.
template <typename E>
__global__ __launch_bounds__(256) void scale_and_sum_kernel(const E* dy, int64_t ld_dy, const float* scale, E* ds, int64_t ld_ds,
                                                            float* part, int M, int N, int strip, int blocks_n,
                                                            const GradientBounds bounds, float* units, int units_count) {
    __shared__ float sums_s[4][512];
    const float factor = StoredFactor<false>(bounds)(BNN_ACT_NONE);
    leave_units(units, units_count, factor);
    const int tid = threadIdx.x, c = tid & 63, r = tid >> 6;
    const int bm = blockIdx.x / uint32_t(blocks_n), bn = int(blockIdx.x) - bm * blocks_n;
    const int n = bn * 512 + c * 8;
    const int64_t first = int64_t(bm) * strip, last = min(first + strip, int64_t(M));
    float sc[8], sum[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) sc[i] = scale && n + i < N ? scale[n + i] : 1.0f;
    for (int64_t m = first + r; m < last; m += 4) {
        const auto v = load8<E>(dy + m * ld_dy + n, int64_t(N) - n);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum[i] += float(v[i]);
            o[i] = float(v[i]) * sc[i] * factor;
        }
        if (ds && n < ld_ds) store8<E>(ds + m * ld_ds + n, o, 8);
    }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums_s[r][c * 8 + i] = sum[i];
    __syncthreads();
    for (int i = tid; i < 512; i += 256)
        if (bn * 512 + i < N) part[int64_t(bm) * N + bn * 512 + i] = sums_s[0][i] + sums_s[1][i] + sums_s[2][i] + sums_s[3][i];
}

// ---- the plan ----------------------------------------------------------------------------------------------------

constexpr int kStrips = 256;       // strips of rows for the column sums without a product

inline int64_t round_up(int64_t v, int64_t to) { return ceil_div(v, to) * to; }

// How dw is made: tiles of 256, 128 or 64 rows and columns, and over how many parts of the rows, whose sums are then joined.
//
// By an estimate in microseconds: a round of the chip - so many workgroups as are on it together - takes a start and so much for
// each step of 32 rows, half a round of tiles of 128 less; parts cost a launch and their way through memory.  It takes what is, or is
// within 6 % of, the fastest of all that were tried at 23 sizes (a whole backward pass, us): 4096 x 4096 x 4096 bfloat16 with tiles of
// 256 in one part 280, in two 334, tiles of 128 319; 16384 x 1024 x 1024 with tiles of 128 in four parts 120, of 64 in two 155;
// 15213 x 5896 x 385 float32 128 in four 1218, in one 1330, 64 in one 1638; 1000 x 1024 x 1024 bfloat16 64 in one 31, in two 35.
// One size misses it by 12 % (3488 x 712 x 3968: 106, with two parts 94).
struct GradPlan {
    int tile = 64, splits = 1, split_rows;
    bool general;
    GradPlan(bool f32, int64_t M, int64_t cols, int64_t channels, int64_t K) : split_rows(int(M)), general(cols < 8 || K < 8) {
        struct Kind {
            int tile, together;
            float step, start;
        };
        static constexpr Kind kKinds[2][3] = {{{256, 256, 0.98f, 8.0f}, {128, 512, 0.60f, 5.0f}, {64, 512, 0.35f, 1.0f}},
                                              {{128, 256, 2.0f, 8.0f}, {64, 512, 1.2f, 3.0f}, {0, 0, 0.0f, 0.0f}}};
        const float piece_us = float(channels) * float(K) * (8.0f / 4.7e6f);
        float least = 0.0f;
        for (const Kind& kind : kKinds[f32 ? 1 : 0]) {
            if (kind.tile == 0 || (general && kind.tile != 64)) continue;
            const int64_t tiles = ceil_div(cols, kind.tile) * ceil_div(K, kind.tile);
            for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
                if (parts > 1 && parts * int64_t(8 * kGradStep) > M) break;
                const int64_t groups = tiles * parts, rest = groups % kind.together;
                const float rounds = float(groups / kind.together) +
                                     (rest == 0 ? 0.0f : kind.tile == 128 && 2 * rest <= kind.together && !f32 ? 0.6f : 1.0f);
                const float us = rounds * (float(ceil_div(ceil_div(M, parts), kGradStep)) * kind.step + kind.start) +
                                 (parts > 1 ? 3.0f + float(parts) * piece_us : 0.0f);
                if (least == 0.0f || us < least) {
                    least = us;
                    tile = kind.tile;
                    splits = parts;
                }
            }
        }
        if (splits > 1) {
            split_rows = int(round_up(ceil_div(M, splits), kGradStep));
            splits = int(ceil_div(M, split_rows));
        }
    }
};

// Everything a call puts into its workspace, by sizes alone.  cols: columns of dy (gated: F).
struct Plan {
    int64_t half, halves, ds_cols, wt_ld, strip, part_rows;
    int64_t ds_at, wt_at, scale_at, bias_at, pieces_at, bounds_at, units_at, bytes;
    Form form;
    bool recompute;
    GradPlan grad;
    Plan(int type, int64_t M, int64_t cols, int64_t K, int act, bool gated)
        : recompute(gated || act != BNN_ACT_NONE), grad(type == BNN_F32, M, recompute ? round_up(cols, 64) * (gated ? 2 : 1) : cols, gated ? 2 * cols : cols, K) {
        const int64_t size = type_bytes(type);
        halves = gated ? 2 : 1;
        half = round_up(cols, 64);
        ds_cols = half * halves;
        wt_ld = round_up(ds_cols / 32, 4);
        const int64_t channels = halves * cols;
        form = product_form(type == BNN_F32, M, cols, int(halves));
        strip = round_up(ceil_div(M > 0 ? M : 1, kStrips), 4);
        // Tiles of a form with 64-bit offsets have 128 rows: never more of them than of the smaller of the two.
        const int64_t rows = rows_of_form(form);
        part_rows = ceil_div(M, recompute ? (rows < 128 ? rows : 128) : strip);
        const int64_t scale_rows = recompute ? part_rows : ceil_div(K, 64);
        auto take = [&](int64_t b) {
            const int64_t at = bytes;
            bytes += round_up(b, 256);
            return at;
        };
        bytes = 0;
        ds_at = take(M * ds_cols * size);
        wt_at = take(K * wt_ld * 4);
        scale_at = take(scale_rows * channels * 4);
        bias_at = take(part_rows * channels * 4);
        pieces_at = take(grad.splits > 1 ? grad.splits * channels * K * 4 : 0);
        bounds_at = take(type == BNN_F16 ? kMostBoundParts * int64_t(sizeof(float)) : 0);
        units_at = take(type == BNN_F16 ? (K > channels ? K : channels) * 4 : 0);
    }
};

template <typename E, int TK, int TN, int FK, int FN, bool GENERAL = false>
int launch_grad(WeightGradArgs a, hipStream_t s) {
    using S = GradTile<E, TK, TN, FK, FN>;
    const int64_t tiles_n = ceil_div(a.cols, S::BN), tiles_k = ceil_div(a.K, S::BK);
    if (tiles_n * tiles_k * a.splits > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_n, tiles_k);
    weight_grad_kernel<E, TK, TN, FK, FN, GENERAL><<<dim3(uint32_t(tiles_n * tiles_k * a.splits)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

// dw and, where a.w is given, dscale, or its parts (in `part`), which are then among what is to be joined.
template <typename E>
int weight_gradient(const GradPlan& g, WeightGradArgs a, float* pieces, float* part, float* dscale, JoinArgs& join, hipStream_t s) {
    a.splits = g.splits;
    a.split_rows = g.split_rows;
    a.pieces = g.splits > 1 ? pieces : nullptr;
    a.part = part;
    int st;
    if (g.general) st = launch_grad<E, 2, 2, 1, 1, true>(a, s);
    else if (g.tile == 64) st = launch_grad<E, 2, 2, 1, 1>(a, s);
    else if (is_f32<E> || g.tile == 128) st = launch_grad<E, 2, 4, 2, 1>(a, s);
    else if constexpr (!is_f32<E>) st = launch_grad<E, 4, 2, 2, 4>(a, s);
    if (st != BNN_OK) return st;
    if (g.splits > 1) {
        join_pieces_kernel<E><<<dim3(uint32_t(a.channels)), dim3(256), 0, s>>>(a, dscale);
        return check_launch();
    }
    if (a.w) join.add(part, ceil_div(a.K, g.tile), dscale);
    return BNN_OK;
}

template <typename E>
int backward(const Plan& p, bool gated, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w,
             const float* scale, const float* bias, int act, void* dx, int64_t ld_dx, void* dw, int64_t ld_dw, float* dscale,
             float* dbias, int64_t M, int64_t cols, int64_t K, char* ws, hipStream_t s) {
    E* const ds = reinterpret_cast<E*>(ws + p.ds_at);
    uint32_t* const wt = reinterpret_cast<uint32_t*>(ws + p.wt_at);
    float* const part_scale = reinterpret_cast<float*>(ws + p.scale_at);
    float* const part_bias = reinterpret_cast<float*>(ws + p.bias_at);
    const int64_t channels = p.halves * cols;
    int st = BNN_OK;
    JoinArgs join{};
    join.N = int(channels);
    const void* g = ds;                // what dx is made of
    int64_t ld_g = p.ds_cols, cols_g = p.ds_cols, part_rows = p.part_rows;
    const bool make_ds = p.recompute || (scale && dx);
    TurnArgs turn{};
    if (dx && M > 0 && K > 0 && cols > 0) {
        const int64_t blocks_n = ceil_div(p.ds_cols / 32, kTurnWords), blocks_k = ceil_div(K, kTurnK);
        if (blocks_n * blocks_k > max_blocks(256) - kMostBoundParts) return BNN_ERR_UNSUPPORTED;
        turn = TurnArgs{w, wt, ld_w, p.wt_ld, int(cols), int(p.half), int(p.halves), int(K), int(blocks_k), int(blocks_n * blocks_k)};
    }
    GradientBounds bounds{};
    float* units = nullptr;            // one over what ds is multiplied with, where it is, for each channel of dx and dw
    int units_count = 0;
    BoundArgs look{};
    if constexpr (std::is_same<E, f16_t>::value) {
        if (make_ds && (dx || dw) && M > 0 && K > 0 && cols > 0) {
            float* const parts = reinterpret_cast<float*>(ws + p.bounds_at);
            // A wavefront a row while there is one for each; then as few lanes as load a row in one go, four groups of eight elements each.
            const int64_t longest = gated && K > cols ? K : cols;
            int lanes = 64;
            while (M > 4 * kMostLookers && lanes > 8 && longest <= (lanes / 2) * 32) lanes /= 2;
            const int64_t wanted = ceil_div(M * lanes, 256);
            bounds = GradientBounds{parts, int(wanted < kMostLookers ? wanted : kMostLookers)};
            units = reinterpret_cast<float*>(ws + p.units_at);
            units_count = int(K > channels ? K : channels);
            look = BoundArgs{static_cast<const E*>(dy), gated ? static_cast<const E*>(x) : nullptr, scale, bias, parts, ld_dy, ld_x, M,
                             int(cols), int(K), int(channels), lanes, bounds.lookers, 2 + bounds.lookers};
        }
    }
    if (turn.blocks + look.blocks > 0) {
        const dim3 grid(uint32_t(turn.blocks + look.blocks)), block(256);
        if (look.blocks > 0) prepare_kernel<true><<<grid, block, 0, s>>>(turn, look);
        else prepare_kernel<false><<<grid, block, 0, s>>>(turn, look);
        if ((st = check_launch()) != BNN_OK) return st;
    }
    if (p.recompute && M > 0 && cols > 0) {
        BackwardArgs a{};
        a.x = x; a.ld_x = ld_x; a.w = w; a.ld_w = ld_w; a.scale = scale; a.bias = bias; a.act = act;
        a.dy = dy; a.ld_dy = ld_dy; a.y = ds; a.ld_y = p.ds_cols; a.half = int(p.half); a.channels = int(channels);
        a.part_scale = dscale ? part_scale : nullptr;
        a.part_bias = dbias ? part_bias : nullptr;
        a.bounds = bounds; a.units = units; a.units_count = units_count;
        a.M = int(M); a.N = int(cols); a.K = int(K);
        part_rows = ceil_div(M, rows_of_tile<E>(p.form, ld_x));
        st = gated ? launch_form<E, kGatedBack>(a, p.form, s) : launch_form<E, kLinearBack>(a, p.form, s);
    } else if (!p.recompute) {
        if (!make_ds) {
            g = dy;
            ld_g = ld_dy;
            cols_g = cols;
        }
        if (M > 0 && cols > 0 && (make_ds || dbias)) {
            const int64_t blocks_n = ceil_div(p.half, 512);
            if (p.part_rows * blocks_n > max_blocks(256)) return BNN_ERR_UNSUPPORTED;
            scale_and_sum_kernel<E><<<dim3(uint32_t(p.part_rows * blocks_n)), dim3(256), 0, s>>>(
                static_cast<const E*>(dy), ld_dy, scale, make_ds ? ds : nullptr, p.ds_cols, dbias ? part_bias : nullptr, int(M),
                int(cols), int(p.strip), int(blocks_n), bounds, units, units_count);
            st = check_launch();
        }
    }
    if (st != BNN_OK) return st;
    if (dx && M > 0 && K > 0) {
        ProductArgs a{};
        a.x = g; a.ld_x = ld_g; a.w = wt; a.ld_w = p.wt_ld; a.y = dx; a.ld_y = ld_dx; a.scale = units;
        a.M = int(M); a.N = int(K); a.K = int(cols > 0 ? cols_g : 0);
        if ((st = launch_form<E, kLinear>(a, product_form(is_f32<E>, M, K, 1), s)) != BNN_OK) return st;
    }
    const bool scale_by_k = dscale && !p.recompute;
    if ((dw || scale_by_k) && cols > 0 && K > 0) {
        WeightGradArgs a{};
        a.g = p.recompute ? ds : dy; a.ld_g = p.recompute ? p.ds_cols : ld_dy;
        a.x = x; a.ld_x = ld_x; a.dw = dw; a.ld_dw = ld_dw;
        a.row_scale = p.recompute ? units : scale;
        a.w = scale_by_k ? w : nullptr; a.ld_w = ld_w;
        a.M = int(M); a.K = int(K); a.cols = int(p.recompute ? p.ds_cols : cols); a.half = int(p.half); a.F = int(cols);
        a.channels = int(channels);
        if ((st = weight_gradient<E>(p.grad, a, reinterpret_cast<float*>(ws + p.pieces_at), part_scale, dscale, join, s)) != BNN_OK)
            return st;
    }
    if (dscale && (p.recompute || K == 0)) join.add(part_scale, p.recompute ? part_rows : 0, dscale);
    if (dbias) join.add(part_bias, part_rows, dbias);
    return join_sums<E>(join, s);
}

// Sizes that a call takes; BNN_OK or what it answers.
int check_sizes(int type, int64_t M, int64_t cols, int64_t K, int act, bool gated) {
    if (cols < 0 || cols > kMaxDim / 2) return BNN_ERR_INVALID_ARG;
    const int st = check_product(type, nullptr, K, nullptr, ceil_div(K, 32), nullptr, nullptr, act, 0, gated ? 2 * cols : cols, K);
    if (st != BNN_OK) return st;
    if (M < 0 || M > kMaxDim) return BNN_ERR_INVALID_ARG;
    // Both products have K and the channels as columns and as what is summed over; the tiles' ends stay below 2^31.
    if (M > kMaxDim - 512 || K > kMaxDim - 512 || cols > kMaxDim / 2 - 512) return BNN_ERR_UNSUPPORTED;
    return BNN_OK;
}

int check_backward(int type, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w,
                   const float* scale, const float* bias, int act, const void* dx, int64_t ld_dx, const void* dw, int64_t ld_dw,
                   const float* dscale, const float* dbias, int64_t M, int64_t cols, int64_t K, bool gated, const void* ws,
                   int64_t ws_bytes) {
    int st = check_sizes(type, M, cols, K, act, gated);
    if (st != BNN_OK) return st;
    st = check_product(type, x, ld_x, w, ld_w, scale, bias, act, M, gated ? 2 * cols : cols, K);
    if (st != BNN_OK) return st;
    const int64_t size = type_bytes(type);
    if (ld_dy < cols || ld_dy > kMaxDim || (dx && (ld_dx < K || ld_dx > kMaxDim)) || (dw && (ld_dw < K || ld_dw > kMaxDim)))
        return BNN_ERR_INVALID_ARG;
    if (M > 0 && cols > 0 && !dy) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(dy, size) || !aligned_to(dx, size) || !aligned_to(dw, size) || !aligned_to(dscale, 4) || !aligned_to(dbias, 4) ||
        !aligned_to(ws, 16))
        return BNN_ERR_ALIGNMENT;
    const int64_t need = Plan(type, M, cols, K, act, gated).bytes;
    if (ws_bytes < need || (need > 0 && !ws)) return BNN_ERR_INVALID_ARG;
    return BNN_OK;
}

int run_backward(int type, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w,
                 const float* scale, const float* bias, int act, void* dx, int64_t ld_dx, void* dw, int64_t ld_dw, float* dscale,
                 float* dbias, int64_t M, int64_t cols, int64_t K, bool gated, void* ws, int64_t ws_bytes, void* stream) {
    int st = check_backward(type, dy, ld_dy, x, ld_x, w, ld_w, scale, bias, act, dx, ld_dx, dw, ld_dw, dscale, dbias, M, cols, K,
                            gated, ws, ws_bytes);
    if (st != BNN_OK) return st;
    const Plan p(type, M, cols, K, act, gated);
    with_type(type, [&](auto e) {
        st = backward<decltype(e)>(p, gated, dy, ld_dy, x, ld_x, w, ld_w, scale, bias, act, dx, ld_dx, dw, ld_dw, dscale, dbias, M,
                                   cols, K, static_cast<char*>(ws), static_cast<hipStream_t>(stream));
    });
    return st;
}

}  // namespace
}  // namespace bnn

extern "C" int64_t bnn_linear_bits_backward_workspace(int type, int64_t M, int64_t N, int64_t K, int act) {
    using namespace bnn;
    return check_sizes(type, M, N, K, act, false) == BNN_OK ? Plan(type, M, N, K, act, false).bytes : -1;
}

extern "C" int64_t bnn_gated_bits_backward_workspace(int type, int64_t M, int64_t F, int64_t K, int act) {
    using namespace bnn;
    return check_sizes(type, M, F, K, act, true) == BNN_OK ? Plan(type, M, F, K, act, true).bytes : -1;
}

extern "C" int bnn_linear_bits_backward(int type, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const uint32_t* w,
                                        int64_t ld_w, const float* scale, const float* bias, int act, void* dx, int64_t ld_dx,
                                        void* dw, int64_t ld_dw, float* dscale, float* dbias, int64_t M, int64_t N, int64_t K,
                                        void* workspace, int64_t workspace_bytes, void* stream) {
    return bnn::run_backward(type, dy, ld_dy, x, ld_x, w, ld_w, scale, bias, act, dx, ld_dx, dw, ld_dw, dscale, dbias, M, N, K, false,
                             workspace, workspace_bytes, stream);
}

extern "C" int bnn_gated_bits_backward(int type, const void* dh, int64_t ld_dh, const void* x, int64_t ld_x, const uint32_t* w,
                                       int64_t ld_w, const float* scale, const float* bias, int act, void* dx, int64_t ld_dx,
                                       void* dw, int64_t ld_dw, float* dscale, float* dbias, int64_t M, int64_t F, int64_t K,
                                       void* workspace, int64_t workspace_bytes, void* stream) {
    return bnn::run_backward(type, dh, ld_dh, x, ld_x, w, ld_w, scale, bias, act, dx, ld_dx, dw, ld_dw, dscale, dbias, M, F, K, true,
                             workspace, workspace_bytes, stream);
}
