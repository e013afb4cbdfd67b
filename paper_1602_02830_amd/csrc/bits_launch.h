// Which kernel a product on real activations takes, and its launch; the checks that the entry points share.
#pragma once

#include "bits_waves.h"

namespace bnn {

int check_product(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale, const float* bias,
                  int act, int64_t M, int64_t channels, int64_t K);

// a.M, a.N > 0.
template <typename E, int EPI, int TM, int TN, int FM, int FN, bool FAR = false>
int launch_product(ArgsOf<EPI> a, hipStream_t s) {
    using S = ProductTile<E, EPI, TM, TN, FM, FN>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(kBackward<EPI> ? a.half : a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    bits_product_kernel<E, EPI, TM, TN, FM, FN, FAR><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

// The form of a product, by its sizes alone: tiles of 16 rows by a wavefront each where there are few of them (their file has the
// figures), then the following.
//
// Tiles have 256 channels and 256, 128 or 64 rows, and the time of one is a start of 7 - 10 us and a step of 64 elements of K,
// measured in us: 1.6 (256 rows, one a compute unit), 0.75 - 1.0 (128 rows, one) and 0.55 (64 rows, one a compute unit; 1.14 with
// two).  The fewest rounds of the chip win: 4000 x 4096 x 1000 takes 36.6 / 39.7 / 42.9 us, 3000 x 8192 x 4096 226 / 193 / 219,
// 1500 x 8192 x 2048 67.4 / 67.7 / 60.4.  Where tiles of 64 rows do not fill the chip, wavefronts that share nothing are faster
// (500 x 3062 x 784: 8.3 us against 12.1; 256 x 4096 x 4096: 15.5 against 38; 1000 x 4096 x 784, 256 tiles: 16.8 against 14.1).
// float32 has three times the products a step: 64 rows, or 128 from two rounds of them on (4000 x 4096 x 1000: 103 us against 98);
// 1000 x 4096 x 784 takes 26 us against 38 of wavefronts, 500 x 3062 x 784 (96 tiles) 20.6 against 18.3.
enum Form { kSmallForm, kWavesForm, kTile64, kTile128, kTile256 };

inline int64_t rows_of_form(Form f) { return f == kTile256 ? 256 : f == kTile128 ? 128 : f == kTile64 ? 64 : f == kWavesForm ? 32 : 16; }

// N columns of `halves` rows of weights each.
inline Form product_form(bool f32, int64_t M, int64_t N, int halves) {
    constexpr int64_t kUnits = 256;
    if (M <= kSmallRows || ceil_div(M, kSmallRows) * ceil_div(N, 16) <= 2 * kUnits) return kSmallForm;
    const int64_t channels = halves * N;
    const int64_t across = ceil_div(channels, 256), t64 = ceil_div(M, 64) * across, t128 = ceil_div(M, 128) * across, t256 = ceil_div(M, 256) * across;
    if (t64 < (f32 ? 128 : 224)) return kWavesForm;
    if (f32) return t128 >= 2 * kUnits ? kTile128 : kTile64;
    // Hundredths of a step's time.
    const int64_t c256 = 160 * ceil_div(t256, kUnits), c128 = 100 * ceil_div(t128, kUnits);
    const int64_t rest = t64 % (2 * kUnits), c64 = 114 * (t64 / (2 * kUnits)) + (rest == 0 ? 0 : rest <= kUnits ? 58 : 114);
    return c256 <= c128 && c256 <= c64 ? kTile256 : c128 <= c64 ? kTile128 : kTile64;
}

// Rows so far apart that 32 bits do not hold a tile's offsets take tiles of 128 rows with 64-bit ones.
template <typename E>
inline bool far_rows(int64_t ld_x) {
    return ld_x > (int64_t(1) << 32) / (256 * int64_t(sizeof(E))) - kStepK;
}

// Rows of a tile of the form that launch_form takes: what backward sums are counted in.
template <typename E>
inline int64_t rows_of_tile(Form form, int64_t ld_x) {
    return form >= kTile64 && far_rows<E>(ld_x) ? 128 : rows_of_form(form);
}

template <typename E, int EPI>
int launch_form(const ArgsOf<EPI>& a, Form form, hipStream_t s) {
    constexpr int HALVES = kHalves<EPI>;
    if (form == kSmallForm) {
        const int waves = int(a.K >= 8 * kSmallRunK ? 8 : a.K <= kSmallRunK ? 1 : ceil_div(a.K, kSmallRunK));
        // Rows are read again for every 16 channels: two blocks a workgroup where there are enough for that (16 rows of
        // 2 x 8192 x 4096: 8.5 us against 11.2; one row 6.7 against 6.7, and 4096 x 8192 with one block 5.1 against 6.7).
        if (a.M > 4 && a.N >= 256 * 32) return launch_small<E, EPI, 2>(a, waves, s);
        return launch_small<E, EPI, 1>(a, waves, s);
    }
    if (form == kWavesForm) {
        const int waves = int(a.K >= 4 * kRunK ? 4 : a.K <= kRunK ? 1 : ceil_div(a.K, kRunK));
        // 128 channels a tile where there are more tiles of 64 than compute units and a run for every wavefront (154 x 4942 ->
        // 5199: 16.5 us against 21.7; 64 x 4096 -> 8192, 256 tiles of 64: 14.5 against 12.1; 500 x 784 -> 3062: 8.8 against 7.9).
        if constexpr (!is_f32<E>) {
            if (a.K >= 4 * kRunK && ceil_div(a.M, 32) * ceil_div(int64_t(a.N) * HALVES, 64) > 256)
                return launch_waves<E, EPI, 1, 4>(a, waves, s);
        }
        return launch_waves<E, EPI, 1, 2>(a, waves, s);
    }
    if (far_rows<E>(a.ld_x)) return launch_product<E, EPI, 2, 2, 2, 2, true>(a, s);
    if constexpr (!is_f32<E>) {
        if (form == kTile256) return launch_product<E, EPI, 2, 4, 4, 2>(a, s);
    }
    if (form == kTile64) return launch_product<E, EPI, 2, 4, 1, 2>(a, s);
    return launch_product<E, EPI, 2, 4, 2, 2>(a, s);
}

}  // namespace bnn
