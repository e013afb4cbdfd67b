// Products of quantised rows with packed weights and their epilogues in one launch: bnn_linear_q_bits and bnn_gated_q_bits.
#include "q_waves.h"

namespace bnn {

namespace {

// The form of a product, by an estimate of its time in us from sizes alone.  What it rests on (8-bit codes, then 4-bit ones), with results of
// 16 bits; those of float32 take longer from several rounds of tiles on (4096 x 784 -> 4096 45 and 42 us, of 16 bits 24 and 20).
//   tiles of 128 or 64 rows, two a compute unit: a start of a call, and for each round of the chip a start and its steps.
//     1024 x 4096 -> 4096  64 rows 23 and 16, 128 rows 31 and 23, wavefronts 51 and 30
//     4096 x 4096 -> 4096  64 rows 68 and 45, 128 rows 63 and 41
//     2048 x 512 -> 8192   64 rows 21 and 18, 128 rows 18 and 16, wavefronts 27 and 22
//   wavefronts on tiles of 32 rows (of 64 too for 4-bit codes): their tiles' elements, or the runs that one has to go through.
//     256 x 4096 -> 4096   32 rows 15.8 and 9.7, tiles of 64 rows 20 and 14, of 16 rows 25 and 15
//     512 x 4096 -> 4096   32 rows 28 and 17, 64 rows 36 and 15.4, tiles of 64 rows 20 and 14.5
//   tiles of 16 rows: likewise.
//     64 x 4096 -> 4096    16 rows 8.7 and 5.7, 32 rows 8.4 and 6.5
//     300 x 8192 -> 512    16 rows 12.2 and 8.7, 32 rows 12.5 and 9.4, 64 rows 21.7 and 14.8
enum QForm { kQSmall, kQWaves32, kQWaves64, kQTile64, kQTile128 };

struct Round { double start, step; };        // of one tile a unit, of two

inline double tiles_time(int64_t tiles, double steps, Round one, Round two) {
    const int64_t units = 256, rest = tiles % (2 * units);
    const double a = one.start + steps * one.step, b = two.start + steps * two.step;
    return 3 + double(tiles / (2 * units)) * b + (rest == 0 ? 0 : rest <= units ? a : b);
}

// channels: rows of w.
inline QForm q_form(bool i8, int64_t M, int64_t channels, int64_t K) {
    const double k = double(K);
    auto tiles = [&](int64_t rows, int64_t cols) { return ceil_div(M, rows) * ceil_div(channels, cols); };
    auto apart = [&](int64_t t, double start, double element, double tile, int64_t run, double wait) {
        const double work = double(t) * (k * element + tile), line = double(ceil_div(K, run)) * wait;
        return start + (work > line ? work : line);
    };
    QForm best = kQSmall;
    double least = apart(tiles(16, 32), i8 ? 3.3 : 2.8, i8 ? 2.5e-6 : 1.5e-6, 0, 4096, 0.9);
    auto consider = [&](QForm form, double time) {
        if (time < least) {
            least = time;
            best = form;
        }
    };
    if (K > 0) consider(kQWaves32, apart(tiles(32, 64), i8 ? 4 : 3.5, i8 ? 5.6e-6 : 2.9e-6, i8 ? 1e-4 : 8e-4, 2048, 1.3));
    if (K > 0 && !i8) consider(kQWaves64, apart(tiles(64, 64), 3.5, 4.7e-6, 4e-3, 1024, 1.4));
    if (K >= kLeastTileK) {
        const double steps = k / (i8 ? 64 : 128);
        consider(kQTile64, i8 ? tiles_time(tiles(64, 256), steps, {5.5, 0.22}, {7, 0.41}) : tiles_time(tiles(64, 256), steps, {5, 0.22}, {7, 0.45}));
        consider(kQTile128, i8 ? tiles_time(tiles(128, 256), steps, {9, 0.33}, {11, 0.75}) : tiles_time(tiles(128, 256), steps, {9, 0.35}, {11, 0.83}));
    }
    return best;
}

template <int ROWS, int EPI>
int forward(const QProductArgs& a, hipStream_t s) {
    constexpr bool I8 = ROWS == BNN_ROWS_I8;
    switch (q_form(I8, a.M, int64_t(a.N) * kQHalves<EPI>, a.K)) {
        case kQTile128: return launch_q_tile<ROWS, EPI, 4>(a, s);
        case kQTile64: return launch_q_tile<ROWS, EPI, 2>(a, s);
        case kQWaves64:
            if constexpr (!I8) return launch_q_waves<ROWS, EPI, 2>(a, s);
            [[fallthrough]];
        case kQWaves32: return launch_q_waves<ROWS, EPI, 1>(a, s);
        default: break;
    }
    // One block of 16 columns a workgroup where rows or tiles are few (8 x 8192 -> 4096: 5.1 and 4.3 us against 5.8 and 5.0 with two;
    // 16 rows of 8-bit codes 7.4 against 7.1, gated 16 x 4096 -> 8192 8.1 and 5.8 against 6.7 and 5.4).  Codes of the result are made of
    // 32 columns at a time.
    if (!a.out.codes && (a.M <= 8 || ceil_div(a.M, kQRows) * ceil_div(a.N, 16) <= (I8 ? 128 : 256))) return launch_q_small<ROWS, EPI, 1>(a, s);
    return launch_q_small<ROWS, EPI, 2>(a, s);
}

// channels: rows of w.
int check_q_product(int rows, const uint8_t* codes, int64_t ld_c, const void* scales, int64_t ld_s, const uint32_t* w, int64_t ld_w,
                    const float* scale, const float* bias, int act, int type, int64_t M, int64_t channels, int64_t K) {
    if (M < 0 || channels < 0 || K < 0 || M > kMaxDim || channels > kMaxDim || K > kMaxK) return BNN_ERR_INVALID_ARG;
    if (type_bytes(type) == 0 || act < BNN_ACT_NONE || act > BNN_ACT_SIGMOID) return BNN_ERR_INVALID_ARG;
    const bool any = M > 0 && channels > 0 && K > 0;
    const int st = check_rows(rows, codes, ld_c, scales, ld_s, any ? M : 0, K);
    if (st != BNN_OK) return st;
    if (ld_w < ceil_div(K, 32) || ld_w > kMaxDim || (any && !w)) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(w, 4) || !aligned_to(scale, 4) || !aligned_to(bias, 4)) return BNN_ERR_ALIGNMENT;
    if (M > kMaxDim - 512 || channels > kMaxDim - 512 || K > kMaxDim - 1024) return BNN_ERR_UNSUPPORTED;      // within a tile of 2^31
    return rows == BNN_ROWS_I8 && K > kMostI8 ? BNN_ERR_UNSUPPORTED : BNN_OK;
}

}  // namespace
}  // namespace bnn

extern "C" int bnn_linear_q_bits(int rows, const uint8_t* codes, int64_t ld_c, const void* scales, int64_t ld_s, const uint32_t* w,
                                 int64_t ld_w, const float* scale, const float* bias, int act, int type, const void* residual,
                                 int64_t ld_r, void* y, int64_t ld_y, int64_t M, int64_t N, int64_t K, void* stream) {
    using namespace bnn;
    const int st = check_q_product(rows, codes, ld_c, scales, ld_s, w, ld_w, scale, bias, act, type, M, N, K);
    if (st != BNN_OK) return st;
    if (ld_y < N || ld_y > kMaxDim || (residual && (ld_r < N || ld_r > kMaxDim))) return BNN_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return BNN_OK;
    if (!y) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(y, type_bytes(type)) || !aligned_to(residual, type_bytes(type))) return BNN_ERR_ALIGNMENT;
    QProductArgs a{};
    a.codes = codes; a.ld_c = ld_c; a.scales = scales; a.ld_s = ld_s; a.w = w; a.ld_w = ld_w; a.scale = scale; a.bias = bias; a.act = act;
    a.type = type; a.residual = residual; a.ld_r = ld_r; a.y = y; a.ld_y = ld_y;
    a.M = int(M); a.N = int(N); a.K = int(K);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return rows == BNN_ROWS_I8 ? forward<BNN_ROWS_I8, kQLinear>(a, s) : forward<BNN_ROWS_MX4, kQLinear>(a, s);
}

extern "C" int bnn_gated_q_bits(int rows, const uint8_t* codes, int64_t ld_c, const void* scales, int64_t ld_s, const uint32_t* w,
                                int64_t ld_w, const float* scale, const float* bias, int act, int type, void* h, int64_t ld_h,
                                uint8_t* out_codes, int64_t ld_oc, uint8_t* out_scales, int64_t ld_os, int64_t M, int64_t F, int64_t K,
                                void* stream) {
    using namespace bnn;
    if (F < 0 || F > kMaxDim / 2) return BNN_ERR_INVALID_ARG;
    int st = check_q_product(rows, codes, ld_c, scales, ld_s, w, ld_w, scale, bias, act, type, M, 2 * F, K);
    if (st != BNN_OK) return st;
    if (h && (ld_h < F || ld_h > kMaxDim)) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(h, type_bytes(type))) return BNN_ERR_ALIGNMENT;
    if ((out_codes != nullptr) != (out_scales != nullptr)) return BNN_ERR_INVALID_ARG;
    if (out_codes && (st = check_rows(BNN_ROWS_MX4, out_codes, ld_oc, out_scales, ld_os, M, F)) != BNN_OK) return st;
    if (M == 0 || F == 0) return BNN_OK;
    if (!h && !out_codes) return BNN_ERR_INVALID_ARG;
    QProductArgs a{};
    a.codes = codes; a.ld_c = ld_c; a.scales = scales; a.ld_s = ld_s; a.w = w; a.ld_w = ld_w; a.scale = scale; a.bias = bias; a.act = act;
    a.type = type; a.y = h; a.ld_y = ld_h;
    a.out = QuantOut{out_codes, out_scales, h, ld_oc, ld_os, ld_h};
    a.M = int(M); a.N = int(F); a.K = int(K);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return rows == BNN_ROWS_I8 ? forward<BNN_ROWS_I8, kQGated>(a, s) : forward<BNN_ROWS_MX4, kQGated>(a, s);
}
