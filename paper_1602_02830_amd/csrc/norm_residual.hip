// What stands between two blocks, forwards and backwards: the norm after a block, its gate and residual scale, the sum with
// the stream and the norm before the next block (bnn_norm_residual, bnn_norm_residual_backward).
//
// Both are bound by memory: every matrix is read or written once.  A workgroup holds a whole row in registers (8 or 16
// elements a thread, 64 to 1024 threads by the row's length), so that the statistics of y, the new stream r and the
// statistics of r need nothing but two to four sums over the workgroup.  Variances are sums of squared distances from the
// mean, taken after it.  Workgroups walk over rows, the next row's loads on their way while one is worked on, with the gammas and
// betas in registers: read for every row, these 32-bit vectors were as much traffic to the caches as a row of 16-bit elements.
// Backwards a workgroup walks a strip of rows and keeps the sums over rows (of the gammas, betas and the gate) in registers;
// strips' sums are joined by a second launch in a fixed order.
#include "join_sums.h"

namespace bnn {

namespace {

constexpr int64_t kMaxNormRow = 16384;       // elements of the longest row that a workgroup holds in registers
constexpr int kNormWaves = 16;               // wavefronts of a compute unit that walk over rows forwards

__device__ inline float sum_of_wave(float v) {
    v = sum_of_32(v);
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

template <int WAVES>
struct Sums {
    float* lds;              // [2][WAVES][2]
    int turn;
    // Sums of a and of b over the workgroup, the same in every thread.  Two buffers in turn: a thread writes one again
    // only after the barrier of the sum between, by which everyone has read it.
    __device__ inline float2 operator()(float a, float b) {
        a = sum_of_wave(a);
        b = sum_of_wave(b);
        if constexpr (WAVES > 1) {
            float* p = lds + turn * 2 * WAVES;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) {
                p[2 * (threadIdx.x >> 6)] = a;
                p[2 * (threadIdx.x >> 6) + 1] = b;
            }
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                a += p[2 * w];
                b += p[2 * w + 1];
            }
        }
        return make_float2(a, b);
    }
};

// Columns of chunk `i` of a thread.
template <int WAVES>
__device__ inline int first_col(int i) {
    return (i * 64 * WAVES + int(threadIdx.x)) * 8;
}

// A row's part of this thread, as it lies in memory: element e of chunk i is column first_col(i) + e.  Loads ask no questions, so
// that the compiler knows how many are on their way: what lies past the row's end is loaded from its last eight elements (SHORT: rows
// of fewer than eight, an element at a time), and put right by `widened`.
template <typename E, int WAVES, int CH>
struct Row {
    typename Vec8<E>::type v[CH];
    template <bool SHORT>
    __device__ inline void load(const void* matrix, int64_t m, int64_t ld, int D) {
        const E* const row = static_cast<const E*>(matrix) + m * ld;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = first_col<WAVES>(i);
            if constexpr (SHORT) v[i] = load8<E>(row + c, D - c);
            else v[i] = *reinterpret_cast<const typename Vec8<E>::any*>(row + min(c, D - 8));
        }
    }
    // As floats, zero past the row's end.
    template <bool SHORT>
    __device__ inline void widened(int D, float (&to)[CH][8]) const {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = first_col<WAVES>(i);
            typename Vec8<E>::type q = v[i];
            // The wavefront's last chunk lies past the row's end: some of them have to be moved.
            if (!SHORT && __builtin_amdgcn_readfirstlane(c) + 512 > D) q = row_end<E>(q, D - c);
#pragma unroll
            for (int e = 0; e < 8; ++e) to[i][e] = float(q[e]);
        }
    }
};

template <int WAVES, int CH, bool SHORT>
__device__ inline void load_vector(const float* p, int D, float otherwise, float (&v)[CH][8]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = otherwise;
        return;
    }
    Row<float, WAVES, CH> row;
    row.template load<SHORT>(p, 0, 0, D);
    row.template widened<SHORT>(D, v);
}

template <typename E, int WAVES, int CH>
__device__ inline void store_row(E* row, int D, const float (&v)[CH][8]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = first_col<WAVES>(i);
        if (c < D) store8<E>(row + c, v[i], D - c);
    }
}

template <int CH, typename F>
__device__ inline void each(F&& f) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) f(i, e);
}

// v -> (v - mean) / sqrt(var + eps), or v / sqrt(mean(v^2) + eps); returns the factor.  Elements past the row's end stay zero.
template <int WAVES, int CH>
__device__ inline float normalise(int kind, float (&v)[CH][8], int D, float eps, Sums<WAVES>& sums) {
    if (kind == BNN_NORM_LAYER) {
        float s = 0.0f;
        each<CH>([&](int i, int e) { s += v[i][e]; });
        const float mean = sums(s, 0.0f).x / float(D);
        each<CH>([&](int i, int e) { v[i][e] = first_col<WAVES>(i) + e < D ? v[i][e] - mean : 0.0f; });
    }
    float s = 0.0f;
    each<CH>([&](int i, int e) { s = fmaf(v[i][e], v[i][e], s); });
    const float inv = 1.0f / sqrtf(sums(s, 0.0f).x / float(D) + eps);
    each<CH>([&](int i, int e) { v[i][e] *= inv; });
    return inv;
}

struct NormArgs {
    const void *y, *x, *gate;
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta;
    void *r, *n;
    int64_t ld_y, ld_x, ld_gate, ld_r, ld_n, rows_per_gate;
    float res_scale, eps;
    int post, pre, M, D;
};

// BETAS: a norm has one.
template <typename E, int WAVES, int CH, bool BETAS, bool SHORT>
__global__ __launch_bounds__(64 * WAVES) void norm_residual_kernel(const NormArgs a) {
    __shared__ float sums_s[4 * WAVES];
    Sums<WAVES> sums{sums_s, 0};
    const int D = a.D;
    float post_g[CH][8], pre_g[CH][8], post_b[BETAS ? CH : 1][8], pre_b[BETAS ? CH : 1][8];
    Row<E, WAVES, CH> y, x, gate;
    int64_t m = blockIdx.x, gate_row = m / a.rows_per_gate;
    y.template load<SHORT>(a.y, m, a.ld_y, D);
    if (a.x) x.template load<SHORT>(a.x, m, a.ld_x, D);
    if (a.gate) gate.template load<SHORT>(a.gate, gate_row, a.ld_gate, D);
    load_vector<WAVES, CH, SHORT>(a.post_gamma, D, 1.0f, post_g);
    load_vector<WAVES, CH, SHORT>(a.pre_gamma, D, 1.0f, pre_g);
    if constexpr (BETAS) {
        load_vector<WAVES, CH, SHORT>(a.post_beta, D, 0.0f, post_b);
        load_vector<WAVES, CH, SHORT>(a.pre_beta, D, 0.0f, pre_b);
    }
    for (; m < a.M; m += gridDim.x) {
        float v[CH][8], xv[CH][8], g[CH][8];
        y.template widened<SHORT>(D, v);
        if (a.x) x.template widened<SHORT>(D, xv);
        if (a.gate) gate.template widened<SHORT>(D, g);
        // The next row, or the last one again.
        const int64_t next = min(m + int64_t(gridDim.x), int64_t(a.M) - 1);
        y.template load<SHORT>(a.y, next, a.ld_y, D);
        if (a.x) x.template load<SHORT>(a.x, next, a.ld_x, D);
        if (a.gate && (gate_row + 1) * a.rows_per_gate <= next) {
            gate_row = next / a.rows_per_gate;
            gate.template load<SHORT>(a.gate, gate_row, a.ld_gate, D);
        }
        if (a.post != BNN_NORM_NONE) {
            normalise<WAVES, CH>(a.post, v, D, a.eps, sums);
            each<CH>([&](int i, int e) { v[i][e] *= post_g[i][e]; });
            if constexpr (BETAS) each<CH>([&](int i, int e) { v[i][e] += post_b[i][e]; });
        }
        each<CH>([&](int i, int e) {
            float t = v[i][e] * a.res_scale;
            if (a.gate) t *= g[i][e];
            v[i][e] = a.x ? xv[i][e] + t : t;
            // 0 * inf of a scale that is none must not reach the sums from columns that are not there.
            if (first_col<WAVES>(i) + e >= D) v[i][e] = 0.0f;
        });
        if (a.r) store_row<E, WAVES, CH>(static_cast<E*>(a.r) + m * a.ld_r, D, v);
        if (a.pre != BNN_NORM_NONE) {
            normalise<WAVES, CH>(a.pre, v, D, a.eps, sums);
            each<CH>([&](int i, int e) { v[i][e] *= pre_g[i][e]; });
            if constexpr (BETAS) each<CH>([&](int i, int e) { v[i][e] += pre_b[i][e]; });
            store_row<E, WAVES, CH>(static_cast<E*>(a.n) + m * a.ld_n, D, v);
        }
    }
}

// ---- backwards ---------------------------------------------------------------------------------------------------

// Strips of rows, one a workgroup.  per_gate > 0: a gate's rows are per_gate strips, whose sums of dgate are joined;
// per_gate == 0: a strip is whole gates (or there is no dgate) and its workgroup writes their gradients itself.
struct Strips {
    int64_t rows, per_gate, count;
};

inline int64_t strip_target(int64_t D) { return D <= 512 ? 4096 : D <= 1024 ? 2048 : D <= 2048 ? 1024 : D <= 4096 ? 512 : 256; }

inline Strips strips_of(int64_t M, int64_t D, int64_t rows_per_gate, bool dgate) {
    const int64_t rows = ceil_div(M > 0 ? M : 1, strip_target(D));
    if (!dgate) return Strips{rows, 0, ceil_div(M, rows)};
    const int64_t R = rows_per_gate < M ? rows_per_gate : (M > 0 ? M : 1);
    if (R <= rows) return Strips{rows / R * R, 0, ceil_div(M, rows / R * R)};
    const int64_t per = ceil_div(R, rows);
    return Strips{ceil_div(R, per), per, ceil_div(M, R) * per};
}

struct NormBackArgs {
    const void *dr, *dn, *y, *r, *gate;
    const float *post_gamma, *post_beta, *pre_gamma;
    void *dx, *dy, *dgate;
    float* part;             // [sums wanted][strips][D]
    int64_t ld_dr, ld_dn, ld_y, ld_r, ld_gate, ld_dx, ld_dy, ld_dgate, rows_per_gate;
    int64_t part_step;       // strips * D
    float res_scale, eps;
    int at_gate, at_post_gamma, at_post_beta, at_pre_gamma, at_pre_beta;      // which of part's sums, -1: not wanted
    int post, pre, M, D;
    Strips strips;
};

// From d, the gradient of a norm's result times gamma, and the normalised row to the gradient of its input.
template <int WAVES, int CH>
__device__ inline void norm_gradient(int kind, float (&d)[CH][8], const float (&hat)[CH][8], float inv, int D, Sums<WAVES>& sums) {
    float s1 = 0.0f, s2 = 0.0f;
    each<CH>([&](int i, int e) {
        s1 += d[i][e];
        s2 = fmaf(d[i][e], hat[i][e], s2);
    });
    const float2 s = sums(s1, s2);
    const float m1 = kind == BNN_NORM_LAYER ? s.x / float(D) : 0.0f, m2 = s.y / float(D);
    each<CH>([&](int i, int e) { d[i][e] = inv * (d[i][e] - m1 - hat[i][e] * m2); });
}

// Wavefronts a SIMD: with 16-bit rows of up to 4096 elements a few spilled registers are cheaper than a second workgroup that does
// not fit (16384 x 4096 bfloat16: 197 us against 233), with float32 rows they are not (329 us against 422).
template <typename E, int WAVES, int CH>
inline constexpr int kBackwardWaves = CH == 1 && !is_f32<E> ? 4 : WAVES == 16 ? 4 : 2;

template <typename E, int WAVES, int CH, bool BETAS, bool SHORT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(kBackwardWaves<E, WAVES, CH>))) void norm_residual_backward_kernel(const NormBackArgs a) {
    __shared__ float sums_s[4 * WAVES];
    Sums<WAVES> sums{sums_s, 0};
    const int D = a.D;
    const int64_t strip = blockIdx.x, R = a.rows_per_gate;
    int64_t first, last;
    if (a.strips.per_gate > 0) {
        const int64_t g = strip / a.strips.per_gate, part = strip - g * a.strips.per_gate;
        first = g * R + part * a.strips.rows;
        last = min(min(first + a.strips.rows, (g + 1) * R), int64_t(a.M));
    } else {
        first = strip * a.strips.rows;
        last = min(first + a.strips.rows, int64_t(a.M));
    }
    const bool norm = a.pre != BNN_NORM_NONE;
    float sum_gate[CH][8] = {}, sum_pre[CH][8] = {}, sum_post[CH][8] = {};
    float sum_pre_b[BETAS ? CH : 1][8] = {}, sum_post_b[BETAS ? CH : 1][8] = {};
    float post_g[CH][8], pre_g[CH][8];
    Row<E, WAVES, CH> y, r, dn, dr, gate;
    int64_t gate_row = 0, gate_end = 0;
    auto load = [&](int64_t m) {
        y.template load<SHORT>(a.y, m, a.ld_y, D);
        if (norm) {
            dn.template load<SHORT>(a.dn, m, a.ld_dn, D);
            r.template load<SHORT>(a.r, m, a.ld_r, D);
        }
    };
    if (first < last) {
        load(first);
        load_vector<WAVES, CH, SHORT>(a.post_gamma, D, 1.0f, post_g);
        load_vector<WAVES, CH, SHORT>(a.pre_gamma, D, 1.0f, pre_g);
    }
    for (int64_t m = first; m < last; ++m) {
        float d[CH][8], v[CH][8];
        // Of this row, needed after the first sums.
        if (a.dr) dr.template load<SHORT>(a.dr, m, a.ld_dr, D);
        if (a.gate && m >= gate_end) {
            gate_row = m / R;
            gate_end = (gate_row + 1) * R;
            gate.template load<SHORT>(a.gate, gate_row, a.ld_gate, D);
        }
        y.template widened<SHORT>(D, v);
        float hat[CH][8];
        if (norm) {
            dn.template widened<SHORT>(D, d);
            r.template widened<SHORT>(D, hat);
        }
        load(min(m + 1, last - 1));                 // the next row, or the last one again
        if (norm) {
            const float inv = normalise<WAVES, CH>(a.pre, hat, D, a.eps, sums);
            each<CH>([&](int i, int e) {
                sum_pre[i][e] = fmaf(d[i][e], hat[i][e], sum_pre[i][e]);
                if constexpr (BETAS) sum_pre_b[i][e] += d[i][e];
                d[i][e] *= pre_g[i][e];
            });
            norm_gradient<WAVES, CH>(a.pre, d, hat, inv, D, sums);
        } else {
            each<CH>([&](int i, int e) { d[i][e] = 0.0f; });
        }
        if (a.dr) {
            dr.template widened<SHORT>(D, hat);
            each<CH>([&](int i, int e) { d[i][e] += hat[i][e]; });
        }
        if (a.dx) store_row<E, WAVES, CH>(static_cast<E*>(a.dx) + m * a.ld_dx, D, d);

        float inv = 1.0f;
        if (a.post != BNN_NORM_NONE) inv = normalise<WAVES, CH>(a.post, v, D, a.eps, sums);
        each<CH>([&](int i, int e) { d[i][e] = first_col<WAVES>(i) + e < D ? d[i][e] * a.res_scale : 0.0f; });
        if (a.dgate) {
            // t = gamma * hat + beta
            each<CH>([&](int i, int e) { sum_gate[i][e] = fmaf(d[i][e], v[i][e] * post_g[i][e], sum_gate[i][e]); });
            if (a.post_beta) {
                float beta[CH][8];
                load_vector<WAVES, CH, SHORT>(a.post_beta, D, 0.0f, beta);
                each<CH>([&](int i, int e) { sum_gate[i][e] = fmaf(d[i][e], beta[i][e], sum_gate[i][e]); });
            }
            if (a.strips.per_gate == 0 && (m + 1 == last || m + 1 == gate_end)) {
                store_row<E, WAVES, CH>(static_cast<E*>(a.dgate) + gate_row * a.ld_dgate, D, sum_gate);
                each<CH>([&](int i, int e) { sum_gate[i][e] = 0.0f; });
            }
        }
        if (a.gate) {
            gate.template widened<SHORT>(D, hat);
            each<CH>([&](int i, int e) { d[i][e] *= hat[i][e]; });
        }
        if (a.post != BNN_NORM_NONE) {
            each<CH>([&](int i, int e) {
                sum_post[i][e] = fmaf(d[i][e], v[i][e], sum_post[i][e]);
                if constexpr (BETAS) sum_post_b[i][e] += d[i][e];
                d[i][e] *= post_g[i][e];
            });
            if (a.dy) norm_gradient<WAVES, CH>(a.post, d, v, inv, D, sums);
        }
        if (a.dy) store_row<E, WAVES, CH>(static_cast<E*>(a.dy) + m * a.ld_dy, D, d);
    }
    float* const part = a.part + strip * D;
    if (a.at_gate >= 0) store_row<float, WAVES, CH>(part + a.at_gate * a.part_step, D, sum_gate);
    if (a.at_pre_gamma >= 0) store_row<float, WAVES, CH>(part + a.at_pre_gamma * a.part_step, D, sum_pre);
    if (a.at_post_gamma >= 0) store_row<float, WAVES, CH>(part + a.at_post_gamma * a.part_step, D, sum_post);
    if constexpr (BETAS) {
        if (a.at_pre_beta >= 0) store_row<float, WAVES, CH>(part + a.at_pre_beta * a.part_step, D, sum_pre_b);
        if (a.at_post_beta >= 0) store_row<float, WAVES, CH>(part + a.at_post_beta * a.part_step, D, sum_post_b);
    }
}

// Calls f<WAVES, CH, SHORT>() for rows of D elements.  Forwards 16 elements a thread, for fewer wavefronts at the barriers;
// backwards, with the sums over rows beside them, 8 where the row is short enough.
template <bool FORWARD, typename F>
inline void with_row(int64_t D, F&& f) {
    using std::false_type;
    using std::integral_constant;
    using std::true_type;
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    if (D < 8) f(One{}, One{}, true_type{});
    else if (D <= 512) f(One{}, One{}, false_type{});
    else if constexpr (FORWARD) {
        if (D <= 1024) f(One{}, Two{}, false_type{});
        else if (D <= 2048) f(Two{}, Two{}, false_type{});
        else if (D <= 3072) f(integral_constant<int, 3>{}, Two{}, false_type{});
        else if (D <= 4096) f(integral_constant<int, 4>{}, Two{}, false_type{});
        else if (D <= 6144) f(integral_constant<int, 6>{}, Two{}, false_type{});
        else if (D <= 8192) f(integral_constant<int, 8>{}, Two{}, false_type{});
        else f(integral_constant<int, 16>{}, Two{}, false_type{});
    } else {
        if (D <= 1024) f(Two{}, One{}, false_type{});
        else if (D <= 2048) f(integral_constant<int, 4>{}, One{}, false_type{});
        else if (D <= 3072) f(integral_constant<int, 6>{}, One{}, false_type{});
        else if (D <= 4096) f(integral_constant<int, 8>{}, One{}, false_type{});
        else if (D <= 6144) f(integral_constant<int, 6>{}, Two{}, false_type{});
        else if (D <= 8192) f(integral_constant<int, 8>{}, Two{}, false_type{});
        else f(integral_constant<int, 16>{}, Two{}, false_type{});
    }
}

bool norm_kind(int kind) { return kind == BNN_NORM_NONE || kind == BNN_NORM_RMS || kind == BNN_NORM_LAYER; }

int check_norm_sizes(int64_t M, int64_t D, int64_t rows_per_gate) {
    if (M < 0 || D < 0 || rows_per_gate < 1 || M > kMaxDim || D > kMaxDim || rows_per_gate > kMaxDim) return BNN_ERR_INVALID_ARG;
    return D > kMaxNormRow ? BNN_ERR_UNSUPPORTED : BNN_OK;
}

// A matrix of the call: there or not wanted, with rows of D.
struct Operand2 {
    const void* p;
    int64_t ld;
};

}  // namespace
}  // namespace bnn

extern "C" int bnn_norm_residual(int type, const void* y, int64_t ld_y, const void* x, int64_t ld_x, const void* gate,
                                 int64_t ld_gate, int64_t rows_per_gate, float res_scale, int post, const float* post_gamma,
                                 const float* post_beta, int pre, const float* pre_gamma, const float* pre_beta, float eps, void* r,
                                 int64_t ld_r, void* n, int64_t ld_n, int64_t M, int64_t D, void* stream) {
    using namespace bnn;
    const int64_t size = type_bytes(type);
    if (size == 0 || !norm_kind(post) || !norm_kind(pre)) return BNN_ERR_INVALID_ARG;
    const int st = check_norm_sizes(M, D, rows_per_gate);
    if (st != BNN_OK) return st;
    if ((post != BNN_NORM_LAYER && post_beta) || (post == BNN_NORM_NONE && post_gamma) || (pre != BNN_NORM_LAYER && pre_beta) ||
        (pre == BNN_NORM_NONE && pre_gamma))
        return BNN_ERR_INVALID_ARG;
    for (const Operand2& o : {Operand2{y, ld_y}, Operand2{x, ld_x}, Operand2{gate, ld_gate}, Operand2{r, ld_r}, Operand2{n, ld_n}}) {
        if (o.p && (o.ld < D || o.ld > kMaxDim)) return BNN_ERR_INVALID_ARG;
        if (!aligned_to(o.p, size)) return BNN_ERR_ALIGNMENT;
    }
    for (const float* p : {post_gamma, post_beta, pre_gamma, pre_beta})
        if (!aligned_to(p, 4)) return BNN_ERR_ALIGNMENT;
    if (M == 0 || D == 0) return BNN_OK;
    if (!y || (n != nullptr) != (pre != BNN_NORM_NONE) || (!r && !n)) return BNN_ERR_INVALID_ARG;
    NormArgs a{y, x, gate, post_gamma, post_beta, pre_gamma, pre_beta, r, n, ld_y, ld_x, ld_gate, ld_r, ld_n, rows_per_gate,
               res_scale, eps, post, pre, int(M), int(D)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool betas = post_beta || pre_beta;
    with_type(type, [&](auto e) {
        with_row<true>(D, [&](auto waves, auto ch, auto is_short) {
            // As many workgroups as are on the chip together, each walking over rows.
            const int64_t together = 256 * (kNormWaves / waves);
            const dim3 grid(uint32_t(M < together ? M : together)), block(64 * waves);
            if (betas) norm_residual_kernel<decltype(e), waves, ch, true, is_short><<<grid, block, 0, s>>>(a);
            else norm_residual_kernel<decltype(e), waves, ch, false, is_short><<<grid, block, 0, s>>>(a);
        });
    });
    return check_launch();
}

extern "C" int64_t bnn_norm_residual_backward_workspace(int64_t M, int64_t D, int64_t rows_per_gate) {
    using namespace bnn;
    if (check_norm_sizes(M, D, rows_per_gate) != BNN_OK) return -1;
    const int64_t with = strips_of(M, D, rows_per_gate, true).count, without = strips_of(M, D, rows_per_gate, false).count;
    return 5 * (with > without ? with : without) * D * 4;
}

extern "C" int bnn_norm_residual_backward(int type, const void* dr, int64_t ld_dr, const void* dn, int64_t ld_dn, const void* y,
                                          int64_t ld_y, const void* r, int64_t ld_r, const void* gate, int64_t ld_gate,
                                          int64_t rows_per_gate, float res_scale, int post, const float* post_gamma,
                                          const float* post_beta, int pre, const float* pre_gamma, float eps, void* dx,
                                          int64_t ld_dx, void* dy, int64_t ld_dy, void* dgate, int64_t ld_dgate,
                                          float* dpost_gamma, float* dpost_beta, float* dpre_gamma, float* dpre_beta, int64_t M,
                                          int64_t D, void* workspace, int64_t workspace_bytes, void* stream) {
    using namespace bnn;
    const int64_t size = type_bytes(type);
    if (size == 0 || !norm_kind(post) || !norm_kind(pre)) return BNN_ERR_INVALID_ARG;
    int st = check_norm_sizes(M, D, rows_per_gate);
    if (st != BNN_OK) return st;
    if ((post != BNN_NORM_LAYER && (post_beta || dpost_beta)) || (post == BNN_NORM_NONE && (post_gamma || dpost_gamma)) ||
        (pre != BNN_NORM_LAYER && dpre_beta) || (pre == BNN_NORM_NONE && (pre_gamma || dpre_gamma)) || (dgate && !gate))
        return BNN_ERR_INVALID_ARG;
    for (const Operand2& o : {Operand2{dr, ld_dr}, Operand2{dn, ld_dn}, Operand2{y, ld_y}, Operand2{r, ld_r}, Operand2{gate, ld_gate},
                              Operand2{dx, ld_dx}, Operand2{dy, ld_dy}, Operand2{dgate, ld_dgate}}) {
        if (o.p && (o.ld < D || o.ld > kMaxDim)) return BNN_ERR_INVALID_ARG;
        if (!aligned_to(o.p, size)) return BNN_ERR_ALIGNMENT;
    }
    for (const float* p : {post_gamma, post_beta, pre_gamma, static_cast<const float*>(dpost_gamma), static_cast<const float*>(dpost_beta),
                           static_cast<const float*>(dpre_gamma), static_cast<const float*>(dpre_beta)})
        if (!aligned_to(p, 4)) return BNN_ERR_ALIGNMENT;
    if (!aligned_to(workspace, 16)) return BNN_ERR_ALIGNMENT;
    if (D == 0) return BNN_OK;
    const bool norm = pre != BNN_NORM_NONE;
    if (M > 0 && (!y || (dn != nullptr) != norm || (norm && !r))) return BNN_ERR_INVALID_ARG;
    const int64_t need = bnn_norm_residual_backward_workspace(M, D, rows_per_gate);
    if (workspace_bytes < need || (need > 0 && !workspace)) return BNN_ERR_INVALID_ARG;

    hipStream_t s = static_cast<hipStream_t>(stream);
    NormBackArgs a{};
    a.strips = strips_of(M, D, rows_per_gate, dgate != nullptr);
    if (a.strips.count > max_blocks(1024)) return BNN_ERR_UNSUPPORTED;
    a.dr = dr; a.dn = dn; a.y = y; a.r = r; a.gate = gate; a.post_gamma = post_gamma; a.post_beta = post_beta; a.pre_gamma = pre_gamma;
    a.dx = dx; a.dy = dy; a.dgate = dgate; a.part = static_cast<float*>(workspace);
    a.ld_dr = ld_dr; a.ld_dn = ld_dn; a.ld_y = ld_y; a.ld_r = ld_r; a.ld_gate = ld_gate; a.ld_dx = ld_dx; a.ld_dy = ld_dy;
    a.ld_dgate = ld_dgate;
    // With one gate for all rows its rows are the matrix's.
    a.rows_per_gate = rows_per_gate < M ? rows_per_gate : (M > 0 ? M : 1);
    a.part_step = a.strips.count * D;
    a.res_scale = res_scale; a.eps = eps; a.post = post; a.pre = pre; a.M = int(M); a.D = int(D);
    JoinArgs join{};
    int vectors = 0;
    auto want = [&](float* out) {
        if (!out) return -1;
        join.out[vectors] = out;
        return vectors++;
    };
    a.at_post_gamma = want(dpost_gamma);
    a.at_post_beta = want(dpost_beta);
    a.at_pre_gamma = want(dpre_gamma);
    a.at_pre_beta = want(dpre_beta);
    a.at_gate = dgate && a.strips.per_gate > 0 ? vectors : -1;
    if (M > 0) {
        const bool betas = dpost_beta || dpre_beta;
        with_type(type, [&](auto e) {
            with_row<false>(D, [&](auto waves, auto ch, auto is_short) {
                const dim3 grid(uint32_t(a.strips.count)), block(64 * waves);
                if (betas) norm_residual_backward_kernel<decltype(e), waves, ch, true, is_short><<<grid, block, 0, s>>>(a);
                else norm_residual_backward_kernel<decltype(e), waves, ch, false, is_short><<<grid, block, 0, s>>>(a);
            });
        });
        if ((st = check_launch()) != BNN_OK) return st;
    }
    join.part = a.part;
    join.part_step = a.part_step;
    join.per_group = int(a.strips.count);
    join.N = int(D);
    if (vectors > 0 && (st = join_sums<float>(join, 1, vectors, s)) != BNN_OK) return st;
    if (a.at_gate >= 0 && M > 0) {
        join.part = a.part + a.at_gate * a.part_step;
        join.per_group = int(a.strips.per_gate);
        join.out[0] = dgate;
        join.ld_out = ld_dgate;
        with_type(type, [&](auto e) { st = join_sums<decltype(e)>(join, ceil_div(M, a.rows_per_gate), 1, s); });
        return st;
    }
    return BNN_OK;
}
