// Launches of the tile products on real activations, and the checks that their entry points share.
#pragma once

#include "bits_product.h"

namespace bnn {

int check_product(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale, const float* bias,
                  int act, int64_t M, int64_t channels, int64_t K);

// a.M, a.N > 0.
template <typename E, int EPI, int TM, int TN, int FM, int FN, bool FAR = false>
int launch_product(ProductArgs a, hipStream_t s) {
    using S = ProductTile<E, EPI, TM, TN, FM, FN>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(EPI == kLinearBack || EPI == kGatedBack ? a.half : a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    bits_product_kernel<E, EPI, TM, TN, FM, FN, FAR><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

// The tile that a product takes, by its sizes: rows of a tile (256, 128), or kFarRows.
constexpr int kFarRows = -1;

template <typename E>
int product_rows(int64_t M, int64_t channels, int64_t ld_x) {
    // Rows so far apart that 32 bits do not hold a tile's offsets: 64-bit ones, in one form.
    if (ld_x > ((int64_t(1) << 32) / (256 * int64_t(sizeof(E))))) return kFarRows;
    if (is_f32<E>) return 128;
    return ceil_div(M, 256) * ceil_div(channels, 256) >= 200 ? 256 : 128;
}

inline int64_t rows_of_tile(int form) { return form == kFarRows ? 128 : form; }

template <typename E, int EPI>
int launch_tiles(const ProductArgs& a, int form, hipStream_t s) {
    if (form == kFarRows) return launch_product<E, EPI, 2, 2, 2, 2, true>(a, s);
    if constexpr (!is_f32<E>) {
        if (form == 256) return launch_product<E, EPI, 2, 4, 4, 2>(a, s);
    }
    return launch_product<E, EPI, 2, 4, 2, 2>(a, s);
}

}  // namespace bnn
