// Products of quantised rows with packed weights and their epilogues in one launch: bnn_linear_q_bits and bnn_gated_q_bits.
#include "q_tiles.h"

namespace bnn {

namespace {

template <int ROWS, int EPI>
int forward(const QProductArgs& a, hipStream_t s) {
    if (a.M > 64 && a.K > 0) return launch_q_tile<ROWS, EPI, 2, 4, 4, 2>(a, s);
    // Codes of the result are made of 32 columns at a time.
    if (a.out.codes) return launch_q_small<ROWS, EPI, 2>(a, s);
    return launch_q_small<ROWS, EPI, 1>(a, s);
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
