// Products of real rows with packed weights and their epilogues in one launch: bnn_linear_bits (bias, activation,
// residual) and bnn_gated_bits (both projections of a gated feed-forward, the activation and their product).
#include "bits_launch.h"

namespace bnn {

namespace {

// ---- few rows --------------------------------------------------------------------------------------------------
// Up to 32 rows of x fill one block of the matrix engine, and what bounds the call is how fast the weights arrive and are
// widened.  A workgroup takes 32 columns of y; its wavefronts share K, 128 elements at a time each, and their sums meet in LDS.

template <typename E, int EPI>
__global__ __launch_bounds__(1024) void bits_rows_kernel(const ProductArgs a) {
    constexpr bool GATED = EPI == kGated, FAST = !is_f32<E>;
    constexpr int FN = GATED ? 2 : 1, TERMS = is_f32<E> ? 3 : 1;
    using O = Operand<E>;
    using O8 = typename Vec8<O>::type;
    extern __shared__ float part_s[];                     // [wavefront][block][register][lane]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int fr = lane & 31, fh = lane >> 5;
    const int n0 = int(blockIdx.x) * 32;
    const int kw = (a.K + 31) >> 5;

    const int col = min(n0 + consecutive_rows(fr), a.N - 1);
    const uint32_t* wrow[FN];
#pragma unroll
    for (int f = 0; f < FN; ++f) wrow[f] = a.w + (int64_t(f) * a.N + col) * a.ld_w;
    const E* const xrow = static_cast<const E*>(a.x) + int64_t(min(fr, a.M - 1)) * a.ld_x;

    const Widening<O> minus_weights;
    v16f_t acc[FN] = {};
    for (int64_t k0 = int64_t(wave) * 128; k0 < a.K; k0 += int64_t(waves) * 128) {
        const int kl = int(k0) + 64 * fh, word = kl >> 5;
        uint32_t w[FN][2];
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            w[f][0] = wrow[f][min(word, kw - 1)];
            w[f][1] = wrow[f][min(word + 1, kw - 1)];
        }
        typename Vec8<E>::type xv[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) xv[s] = load8<E>(xrow + kl + 8 * s, int64_t(a.K) - kl - 8 * s);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            O8 t[TERMS];
            if constexpr (is_f32<E>) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16_t part[3];
                    split3(xv[s][e], part);
                    t[0][e] = part[0];
                    t[1][e] = part[1];
                    t[2][e] = part[2];
                }
            } else {
                t[0] = xv[s];
            }
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                const uint32_t word_s = w[f][s >> 2];
                const O8 wf = minus_weights((s & 2) ? spread_high(word_s) : spread_low(word_s), s & 1);
#pragma unroll
                for (int p = 0; p < TERMS; ++p) acc[f] = mfma16(wf, t[p], acc[f]);
            }
        }
    }
    if (fr < a.M) {
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) part_s[((wave * FN + f) * 16 + i) * 64 + lane] = acc[f][i];
    }
    __syncthreads();
    // Eight columns of a row for each thread.
    for (int slot = tid; slot < 128; slot += blockDim.x) {
        const int l = slot & 63, g = slot >> 6, m = l & 31, n = n0 + 16 * (l >> 5) + 8 * g;
        if (m >= a.M || n >= a.N) continue;
        float s[FN][8] = {};
        for (int w_ = 0; w_ < waves; ++w_)
#pragma unroll
            for (int f = 0; f < FN; ++f)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[f][i] += part_s[((w_ * FN + f) * 16 + 8 * g + i) * 64 + l];
        const int64_t valid = int64_t(a.N) - n;
        typename Vec8<E>::type r = {};
        if (!GATED && a.residual) r = load8<E>(static_cast<const E*>(a.residual) + int64_t(m) * a.ld_r + n, valid);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float z[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                const int64_t c = int64_t(f) * a.N + min(n + i, a.N - 1);
                z[f] = fmaf(-s[f][i], a.scale ? a.scale[c] : 1.0f, a.bias ? a.bias[c] : 0.0f);
            }
            if constexpr (GATED) v[i] = activate<FAST>(a.act, z[0]) * z[1];
            else v[i] = activate<FAST>(a.act, z[0]) + float(r[i]);
        }
        store8<E>(static_cast<E*>(a.y) + int64_t(m) * a.ld_y + n, v, valid);
    }
}

template <typename E, int EPI>
int launch_rows(const ProductArgs& a, hipStream_t s) {
    constexpr int FN = EPI == kGated ? 2 : 1;
    const int waves = int(a.K >= 16 * 128 ? 16 : a.K <= 128 ? 1 : ceil_div(a.K, 128));
    bits_rows_kernel<E, EPI><<<dim3(uint32_t(ceil_div(a.N, 32))), dim3(64 * waves), size_t(waves) * FN * 16 * 64 * 4, s>>>(a);
    return check_launch();
}

template <typename E, int EPI>
int launch_forward(const ProductArgs& a, hipStream_t s) {
    if (a.M <= 32) return launch_rows<E, EPI>(a, s);
    return launch_tiles<E, EPI>(a, product_rows<E>(a.M, int64_t(a.N) * (EPI == kGated ? 2 : 1), a.ld_x), s);
}

}  // namespace

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
    with_type(type, [&](auto e) { status = launch_forward<decltype(e), EPI>(a, static_cast<hipStream_t>(stream)); });
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
