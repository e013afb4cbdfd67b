// Rows of reals to codes of 8 or 4 bits with scales, and back (bnn_quantize_rows, bnn_dequantize_rows): bound by memory.
#include "quant_rows.h"
#include "row_layout.h"

namespace bnn {

namespace {

struct QuantiseArgs {
    const void* x;
    QuantOut out;
    int64_t ld_x;
    int M, K;
    FastDiv by_row;          // 4 bits: by the groups of eight elements of a row
};

// Wavefronts of a compute unit that walk over rows: 16384 x 4096 bfloat16 45 us without x^ (4.5 TB/s; with 16 wavefronts 52, with 32 47), 56 with
// it (6.0 TB/s; 58 and 61), on the same matrix again and again; 16384 x 8192 with it, on another each time, 124 (5.4 TB/s).  4-bit codes, whose
// rows need no second look, 24 and 43.
constexpr int kQuantiseWaves = 24;

// A row in the registers of its workgroup: its largest magnitude, then its codes.  Workgroups walk over rows, the next row's loads
// on their way while one is worked on.
template <typename E, typename L>
__global__ __launch_bounds__(64 * L::WAVES) void quantise_i8_kernel(const QuantiseArgs a) {
    __shared__ uint32_t largest_s[2 * L::WAVES];
    Largest<L::WAVES> largest(largest_s);
    const int K = a.K;
    Row<E, L> x;
    int64_t m = blockIdx.x;
    x.load(a.x, m, a.ld_x, K);
    for (; m < a.M; m += gridDim.x) {
        Values<L> v;
        x.widened(K, v);
        x.load(a.x, min(m + int64_t(gridDim.x), int64_t(a.M) - 1), a.ld_x, K);      // the next row, or the last one again
        store_row_i8<E, L>(a.out, m, K, v, largest);
    }
}

// Rows of any length, read twice, the second time from the cache where that holds what is on its way: 4096 x 20000 bfloat16 93 us, 2.6 TB/s, with
// x^ 105; 1000 x 65536 71.
template <typename E>
__global__ __launch_bounds__(1024) void quantise_i8_long_kernel(const QuantiseArgs a) {
    __shared__ uint32_t largest_s[2 * 16];
    Largest<16> largest(largest_s);
    const int64_t K = a.K;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
        const E* const row = static_cast<const E*>(a.x) + m * a.ld_x;
        uint32_t most = 0;
        float v[8];
        for (int64_t c = threadIdx.x * 8; c < K; c += 8192) {
            load_some<E, 8>(row + c, K - c, v);
            most = max(most, largest_of_8(v));
        }
        const float s = i8_scale(largest(most));
        if (threadIdx.x == 0) static_cast<float*>(a.out.scales)[m] = s;
        for (int64_t c = threadIdx.x * 8; (c & ~int64_t(31)) < K; c += 8192) {
            load_some<E, 8>(row + c, K - c, v);
            quantise_i8<E>(a.out, m, c, v, s, K);
        }
    }
}

constexpr int kGroups = 2;          // groups of eight elements a thread

// The groups of a launch's rows numbered through, four lanes to a block.
template <typename F>
__device__ inline void each_group(const FastDiv& by_row, int groups_a_row, int M, F&& f) {
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
        const int64_t id = (int64_t(blockIdx.x) * kGroups + u) * 256 + threadIdx.x;
        if (id >= int64_t(M) * groups_a_row) continue;
        const int row = by_row(int(id));
        f(row, int64_t(int(id) - row * groups_a_row) * 8);
    }
}

template <typename E>
__global__ __launch_bounds__(256) void quantise_mx4_kernel(const QuantiseArgs a) {
    each_group(a.by_row, 4 * ((a.K + 31) >> 5), a.M, [&](int64_t m, int64_t c) {
        float v[8];
        load_some<E, 8>(static_cast<const E*>(a.x) + m * a.ld_x + c, a.K - c, v);
        quantise_mx4<E>(a.out, m, c, v, a.K);
    });
}

// 16384 x 4096 to bfloat16 42 us from 8 bits (4.9 TB/s), 40 from 4; to float32 78 and 79.
template <typename E, int ROWS>
__global__ __launch_bounds__(256) void dequantise_kernel(const QuantiseArgs a) {
    each_group(a.by_row, 4 * ((a.K + 31) >> 5), a.M, [&](int64_t m, int64_t c) {
        float v[8];
        if constexpr (ROWS == BNN_ROWS_I8) {
            const uint2 words = *reinterpret_cast<const uint2*>(a.out.codes + m * a.out.ld_c + c);
            i8_values(i8_turn_back(words), static_cast<const float*>(a.out.scales)[m], v);
        } else {
            const uint32_t word = *reinterpret_cast<const uint32_t*>(a.out.codes + m * a.out.ld_c + (c >> 1));
            mx4_values(mx4_turn(word), static_cast<const uint8_t*>(a.out.scales)[m * a.out.ld_s + (c >> 5)], v);
        }
        if (c < a.K) store_group<E, 8>(static_cast<E*>(a.out.hat) + m * a.out.ld_h + c, v, a.K - c);
    });
}

// Launches for as many rows at a time as have fewer than 2^31 groups.
template <typename F>
int each_part(QuantiseArgs a, int64_t size, int64_t K, int64_t M, F&& launch) {
    const int64_t groups = 4 * ceil_div(K, 32), most = groups > 0 ? (kMaxDim - 1024) / groups : M;
    a.by_row = fast_div(groups);
    for (int64_t first = 0; first < M; first += most) {
        const int64_t rows = M - first < most ? M - first : most;
        QuantiseArgs part = a;
        part.M = int(rows);
        part.x = static_cast<const char*>(a.x) + first * a.ld_x * size;
        part.out.codes += first * a.out.ld_c;
        part.out.scales = static_cast<char*>(a.out.scales) + first * (a.out.ld_s > 0 ? a.out.ld_s : 4);
        if (a.out.hat) part.out.hat = static_cast<char*>(a.out.hat) + first * a.out.ld_h * size;
        launch(part, dim3(uint32_t(ceil_div(rows * groups, 256 * kGroups))));
        const int st = check_launch();
        if (st != BNN_OK) return st;
    }
    return BNN_OK;
}

int check_reals(int type, const void* x, int64_t ld, int64_t M, int64_t K) {
    if (M < 0 || K < 0 || M > kMaxDim || K > kMaxK || type_bytes(type) == 0 || ld < K || ld > kMaxDim) return BNN_ERR_INVALID_ARG;
    if (!aligned_to(x, type_bytes(type))) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}

}  // namespace
}  // namespace bnn

extern "C" int bnn_quantize_rows(int rows, int type, const void* x, int64_t ld_x, uint8_t* codes, int64_t ld_c, void* scales,
                                 int64_t ld_s, void* hat, int64_t ld_h, int64_t M, int64_t K, void* stream) {
    using namespace bnn;
    int st = check_reals(type, x, ld_x, M, K);
    if (st == BNN_OK && hat) st = check_reals(type, hat, ld_h, M, K);
    if (st == BNN_OK) st = check_rows(rows, codes, ld_c, scales, ld_s, M, K);
    if (st != BNN_OK) return st;
    if (K > kMaxK - 16384) return BNN_ERR_UNSUPPORTED;
    if (M == 0) return BNN_OK;
    if (K > 0 && !x) return BNN_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    QuantiseArgs a{x, {codes, scales, hat, ld_c, rows == BNN_ROWS_I8 ? 0 : ld_s, ld_h}, ld_x, int(M), int(K), {}};
    with_type(type, [&](auto e) {
        using E = decltype(e);
        if (rows == BNN_ROWS_MX4) {
            if (K > 0) st = each_part(a, type_bytes(type), K, M, [&](const QuantiseArgs& part, dim3 grid) { quantise_mx4_kernel<E><<<grid, 256, 0, s>>>(part); });
        } else if (K == 0 || K > kMaxRowHeld) {
            quantise_i8_long_kernel<E><<<dim3(uint32_t(M < 512 ? M : 512)), 1024, 0, s>>>(a);
            st = check_launch();
        } else {
            with_row(K, [&](auto layout) {
                using L = decltype(layout);
                const int threads = L::threads(K);
                const int64_t together = 256 * (64 * kQuantiseWaves / threads);
                quantise_i8_kernel<E, L><<<dim3(uint32_t(M < together ? M : together)), dim3(uint32_t(threads)), 0, s>>>(a);
            });
            st = check_launch();
        }
    });
    return st;
}

extern "C" int bnn_dequantize_rows(int rows, int type, const uint8_t* codes, int64_t ld_c, const void* scales, int64_t ld_s, void* x,
                                   int64_t ld_x, int64_t M, int64_t K, void* stream) {
    using namespace bnn;
    int st = check_reals(type, x, ld_x, M, K);
    if (st == BNN_OK) st = check_rows(rows, codes, ld_c, scales, ld_s, M, K);
    if (st != BNN_OK) return st;
    if (K > kMaxK - 16384) return BNN_ERR_UNSUPPORTED;
    if (M == 0 || K == 0) return BNN_OK;
    if (!x) return BNN_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    QuantiseArgs a{nullptr, {const_cast<uint8_t*>(codes), const_cast<void*>(scales), x, ld_c, rows == BNN_ROWS_I8 ? 0 : ld_s, ld_x}, 0, int(M), int(K), {}};
    with_type(type, [&](auto e) {
        using E = decltype(e);
        st = each_part(a, type_bytes(type), K, M, [&](const QuantiseArgs& part, dim3 grid) {
            if (rows == BNN_ROWS_I8) dequantise_kernel<E, BNN_ROWS_I8><<<grid, 256, 0, s>>>(part);
            else dequantise_kernel<E, BNN_ROWS_MX4><<<grid, 256, 0, s>>>(part);
        });
    });
    return st;
}
