// Products of real rows with packed weights and their epilogues in one launch: bnn_linear_bits (bias, activation,
// residual) and bnn_gated_bits (both projections of a gated feed-forward, the activation and their product).
#include "bits_launch.h"

namespace bnn {

// What the entry points of the products check alike.  channels: rows of w.
int check_product(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale, const float* bias,
                  int act, int64_t M, int64_t channels, int64_t K) {
    if (M < 0 || channels < 0 || K < 0 || M > kMaxDim || channels > kMaxDim || K > kMaxK) return BNN_ERR_INVALID_ARG;
    const int64_t size = type_bytes(type);
    if (size == 0 || act < BNN_ACT_NONE || act > BNN_ACT_SIGMOID) return BNN_ERR_INVALID_ARG;
    if (ld_x < K || ld_w < ceil_div(K, 32) || ld_x > kMaxDim || ld_w > kMaxDim) return BNN_ERR_INVALID_ARG;
    if (M > 0 && channels > 0 && K > 0 && (!x || !w)) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(x, size) || !aligned_to(w, 4) || !aligned_to(scale, 4) || !aligned_to(bias, 4)) return BNN_ERR_ALIGNMENT;
    if (M > kMaxDim - 512 || channels > kMaxDim - 512 || K > kMaxDim - 512) return BNN_ERR_UNSUPPORTED;      // within a tile of 2^31
    return BNN_OK;
}

namespace {

template <int EPI>
int forward(int type, const ProductArgs& a, void* stream) {
    int status = BNN_ERR_INVALID_ARG;
    const Form form = product_form(type == BNN_F32, a.M, a.N, kHalves<EPI>);
    with_type(type, [&](auto e) { status = launch_form<decltype(e), EPI>(a, form, static_cast<hipStream_t>(stream)); });
    return status;
}

}  // namespace
}  // namespace bnn

extern "C" int bnn_linear_bits(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale,
                               const float* bias, int act, const void* residual, int64_t ld_r, void* y, int64_t ld_y,
                               int64_t M, int64_t N, int64_t K, void* stream) {
    using namespace bnn;
    const int st = check_product(type, x, ld_x, w, ld_w, scale, bias, act, M, N, K);
    if (st != BNN_OK) return st;
    if (ld_y < N || ld_y > kMaxDim || (residual && (ld_r < N || ld_r > kMaxDim))) return BNN_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return BNN_OK;
    if (!y) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(y, type_bytes(type)) || !aligned_to(residual, type_bytes(type))) return BNN_ERR_ALIGNMENT;
    ProductArgs a{};
    a.x = x; a.ld_x = ld_x; a.w = w; a.ld_w = ld_w; a.scale = scale; a.bias = bias; a.act = act;
    a.residual = residual; a.ld_r = ld_r; a.y = y; a.ld_y = ld_y;
    a.M = int(M); a.N = int(N); a.K = int(K);
    return forward<kLinear>(type, a, stream);
}

extern "C" int bnn_gated_bits(int type, const void* x, int64_t ld_x, const uint32_t* w, int64_t ld_w, const float* scale,
                              const float* bias, int act, void* h, int64_t ld_h, int64_t M, int64_t F, int64_t K, void* stream) {
    using namespace bnn;
    if (F < 0 || F > kMaxDim / 2) return BNN_ERR_INVALID_ARG;
    const int st = check_product(type, x, ld_x, w, ld_w, scale, bias, act, M, 2 * F, K);
    if (st != BNN_OK) return st;
    if (ld_h < F || ld_h > kMaxDim) return BNN_ERR_INVALID_ARG;
    if (M == 0 || F == 0) return BNN_OK;
    if (!h) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(h, type_bytes(type))) return BNN_ERR_ALIGNMENT;
    ProductArgs a{};
    a.x = x; a.ld_x = ld_x; a.w = w; a.ld_w = ld_w; a.scale = scale; a.bias = bias; a.act = act;
    a.y = h; a.ld_y = ld_h;
    a.M = int(M); a.N = int(F); a.K = int(K);
    return forward<kGated>(type, a, stream);
}
