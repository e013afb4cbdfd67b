// Launches of the tile products on real activations, and the checks that their entry points share.
#pragma once

#include "bits_product.h"

namespace bnn {

int check_product(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale, const float* bias,
                  int act, int64_t M, int64_t channels, int64_t K);

// a.M, a.N > 0.
template <typename E, int EPI, int TM, int TN, int FM, int FN>
int launch_product(ProductArgs a, hipStream_t s) {
    using S = ProductTile<E, EPI, TM, TN, FM, FN>;
    const int64_t tiles_m = ceil_div(a.M, S::BM), tiles_n = ceil_div(EPI == kLinearBack || EPI == kGatedBack ? a.half : a.N, S::BN);
    if (tiles_m * tiles_n > max_blocks(S::kThreads)) return BNN_ERR_UNSUPPORTED;
    a.map = tile_map(tiles_m, tiles_n);
    bits_product_kernel<E, EPI, TM, TN, FM, FN><<<dim3(uint32_t(tiles_m * tiles_n)), dim3(S::kThreads), 0, s>>>(a);
    return check_launch();
}

}  // namespace bnn
