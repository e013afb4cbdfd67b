// What stands between two blocks, forwards and backwards: the norm after a block, its gate and residual scale, the sum with
// the stream and the norm before the next block (bnn_norm_residual, bnn_norm_residual_backward).
//
// Both are bound by memory: every matrix is read or written once.  A workgroup holds a whole row in registers (16 elements a
// thread), so that the statistics of y, the new stream r and the statistics of r need nothing but two to four sums over the
// workgroup.  Variances are sums of squared distances from the mean, taken after it.  Workgroups walk over rows, the next row's loads
// on their way while one is worked on.  With 8 elements a thread and twice the wavefronts at each barrier the same rows took longer
// (10000 x 2049 float32 backwards, root-mean-square norms: 155 us against 125, and 116 without a gate), with 4 longer still.
//
// Forwards the gammas and betas stay in registers: read for every row, these 32-bit vectors were as much traffic to the caches as
// a row of 16-bit elements.  16384 x 4096 bfloat16, root-mean-square norms and a gate: 114 us, 4.7 TB/s, as fast as a large copy.
//
// Backwards y and r are both at hand from the start, and their norms share their sums; then follow one pair of sums for the
// gradient of each norm.  A workgroup walks a strip of rows and keeps the sums over rows (of the gammas, betas and the gate) in
// registers, the gammas and the beta in LDS; strips' sums are joined by a second launch in a fixed order.  16384 x 4096 bfloat16:
// 176 us, 4.6 TB/s; 10000 x 2049 float32 with layer norms, a gate and all their gradients 179 us, 2.8 TB/s: five sums over rows instead of
// two, for which 256 registers are 36 bytes a lane too few, in three wavefronts of whose places a third are empty.  Rows past 8192
// elements do not fit the registers: 324 - 596 bytes a lane go to scratch memory (4000 x 16000 bfloat16: 555 us, 1.4 TB/s), forwards
// 28 - 316 (118 us).
#include "join_sums.h"
#include "row_layout.h"

namespace bnn {

namespace {

constexpr int kNormWaves = 16;               // wavefronts of a compute unit that walk over rows forwards

template <typename L>
__device__ inline void take_off(float mean, Values<L>& v, int D) {
    each<L>([&](int i, int e) { v[i][e] -= mean; });
    trim<L>(v, D);
}

__device__ inline float one_over_root(float squares, int D, float eps) { return 1.0f / sqrtf(squares / float(D) + eps); }

// v -> (v - mean) / sqrt(var + eps), or v / sqrt(mean(v^2) + eps).
template <typename L>
__device__ inline void normalise(int kind, Values<L>& v, int D, float eps, Sums<L::WAVES>& sums) {
    if (kind == BNN_NORM_LAYER) take_off<L>(sums(sum_of<L>(v), 0.0f).x / float(D), v, D);
    const float inv = one_over_root(sums(sum_of_squares<L>(v), 0.0f).x, D, eps);
    each<L>([&](int i, int e) { v[i][e] *= inv; });
}

// Two rows at once, for as many sums as one of them takes (kind BNN_NORM_NONE: left as it is); returns the factors.
template <typename L>
__device__ inline float2 normalise_both(int kind_a, Values<L>& a, int kind_b, Values<L>& b, int D, float eps, Sums<L::WAVES>& sums) {
    float2 inv = make_float2(1.0f, 1.0f);
    if (kind_a == BNN_NORM_LAYER || kind_b == BNN_NORM_LAYER) {
        const float2 s = sums(sum_of<L>(a), sum_of<L>(b));
        if (kind_a == BNN_NORM_LAYER) take_off<L>(s.x / float(D), a, D);
        if (kind_b == BNN_NORM_LAYER) take_off<L>(s.y / float(D), b, D);
    }
    if (kind_a != BNN_NORM_NONE || kind_b != BNN_NORM_NONE) {
        const float2 s = sums(sum_of_squares<L>(a), sum_of_squares<L>(b));
        if (kind_a != BNN_NORM_NONE) {
            inv.x = one_over_root(s.x, D, eps);
            each<L>([&](int i, int e) { a[i][e] *= inv.x; });
        }
        if (kind_b != BNN_NORM_NONE) {
            inv.y = one_over_root(s.y, D, eps);
            each<L>([&](int i, int e) { b[i][e] *= inv.y; });
        }
    }
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

// With codes of n (bnn_rows) in the place of n: calls without them have no more arguments than they had.
struct NormRowsArgs : NormArgs {
    QuantOut out;
};

constexpr int kReals = -1;                   // in the place of a bnn_rows: n as it is

// Wavefronts of a compute unit that walk over rows and give codes: as many as are there together, so that no workgroup begins when others
// end.  16384 x 4096 bfloat16, root-mean-square norms, with codes of 8 bits and n^, on the same matrices again and again: 100 us,
// 6.0 TB/s (on others each time 123, 4.9 TB/s), with 16 wavefronts 116, with 8 116; of 4 bits 93, without n^
// 89 and 76 (on others each time 103 and 89).  Rows of one group a lane take fewer registers: 100000 x 300 with 16 85, with 12 93.  A third sum over the
// workgroup for the scale is what 8 bits cost more; in registers for 16 wavefronts (128 of them) the kernels spill 60 bytes (143 for then 125 us).
//
// r, codes and n^ are stored past the cache: 100 us are 125 otherwise, for 1000 rows 9.0 are 11.2.  Not in float32 with n^, whose lanes have two
// pieces of 16 bytes side by side, so that no store fills a line: 16384 x 4096 235 us instead of 169, without n^ 116 instead of 121.
template <typename L>
constexpr int kNormRowsWaves = L::CH == 1 ? 16 : 12;

// BETAS: a norm has one.
template <typename E, typename L, bool BETAS, int ROWS = kReals>
__global__ __launch_bounds__(64 * L::WAVES) void norm_residual_kernel(const typename std::conditional<ROWS == kReals, NormArgs, NormRowsArgs>::type a) {
    __shared__ float2 sums_s[2 * L::WAVES];
    Sums<L::WAVES> sums(sums_s);
    __shared__ uint32_t largest_s[ROWS == BNN_ROWS_I8 ? 2 * L::WAVES : 1];
    Largest<ROWS == BNN_ROWS_I8 ? L::WAVES : 1> largest(largest_s);
    const int D = a.D;
    Values<L> post_g, pre_g, post_b, pre_b;
    Row<E, L> y, x, gate;
    int64_t m = blockIdx.x, gate_row = m / a.rows_per_gate;
    y.load(a.y, m, a.ld_y, D);
    if (a.x) x.load(a.x, m, a.ld_x, D);
    if (a.gate) gate.load(a.gate, gate_row, a.ld_gate, D);
    // 4000 x 16000 bfloat16 with betas 188 us as rows, 226 otherwise; without betas 300 x 16384 float32 42 and 49, one row of 16000 float32
    // 14.0 and 16.1, of bfloat16 6.7 and 7.0.
    constexpr bool AS_ROW = L::WAVES == 16 && (BETAS || ROWS == kReals);
    load_vector<L, AS_ROW>(a.post_gamma, D, 1.0f, post_g);
    load_vector<L, AS_ROW>(a.pre_gamma, D, 1.0f, pre_g);
    if constexpr (BETAS) {
        load_vector<L, AS_ROW>(a.post_beta, D, 0.0f, post_b);
        load_vector<L, AS_ROW>(a.pre_beta, D, 0.0f, pre_b);
    }
    for (; m < a.M; m += gridDim.x) {
        Values<L> v, xv, g;
        y.widened(D, v);
        if (a.x) x.widened(D, xv);
        if (a.gate) gate.widened(D, g);
        // The next row, or the last one again.
        const int64_t next = min(m + int64_t(gridDim.x), int64_t(a.M) - 1);
        y.load(a.y, next, a.ld_y, D);
        if (a.x) x.load(a.x, next, a.ld_x, D);
        if (a.gate && (gate_row + 1) * a.rows_per_gate <= next) {
            gate_row = next / a.rows_per_gate;
            gate.load(a.gate, gate_row, a.ld_gate, D);
        }
        if (a.post != BNN_NORM_NONE) {
            normalise<L>(a.post, v, D, a.eps, sums);
            each<L>([&](int i, int e) { v[i][e] *= post_g[i][e]; });
            if constexpr (BETAS) each<L>([&](int i, int e) { v[i][e] += post_b[i][e]; });
        }
        each<L>([&](int i, int e) {
            float t = v[i][e] * a.res_scale;
            if (a.gate) t *= g[i][e];
            v[i][e] = a.x ? xv[i][e] + t : t;
        });
        trim<L>(v, D);           // 0 * inf of a scale that is none must not reach the sums from columns that are not there
        if (a.r) {
            E* const r = static_cast<E*>(a.r) + m * a.ld_r;
            bool past = ROWS != kReals;
            if constexpr (ROWS != kReals && is_f32<E>) past = !a.out.hat;
            if (past) store_row<E, L, ROWS != kReals>(r, D, v);
            else store_row<E, L>(r, D, v);
        }
        if (a.pre != BNN_NORM_NONE) {
            normalise<L>(a.pre, v, D, a.eps, sums);
            each<L>([&](int i, int e) { v[i][e] *= pre_g[i][e]; });
            if constexpr (BETAS) each<L>([&](int i, int e) { v[i][e] += pre_b[i][e]; });
            if constexpr (ROWS == kReals) store_row<E, L>(static_cast<E*>(a.n) + m * a.ld_n, D, v);
        }
        if constexpr (ROWS == BNN_ROWS_I8) store_row_i8<E, L, !is_f32<E>>(a.out, m, D, v, largest);
        if constexpr (ROWS == BNN_ROWS_MX4) store_row_mx4<E, L, !is_f32<E>>(a.out, m, D, v);
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
template <typename L>
__device__ inline void norm_gradient(int kind, Values<L>& d, const Values<L>& hat, float inv, int D, Sums<L::WAVES>& sums) {
    float s1 = 0.0f, s2 = 0.0f;
    each<L>([&](int i, int e) {
        s1 += d[i][e];
        s2 = fmaf(d[i][e], hat[i][e], s2);
    });
    const float2 s = sums(s1, s2);
    const float m1 = kind == BNN_NORM_LAYER ? s.x / float(D) : 0.0f, m2 = s.y / float(D);
    each<L>([&](int i, int e) { d[i][e] = inv * (d[i][e] - m1 - hat[i][e] * m2); });
}

// Vectors of a row's layout, in LDS: each thread reads what it has written.
template <typename L>
struct Kept {
    static constexpr int kQuads = L::CH * L::G / 4;
    static constexpr bool kThree = kQuads * 64 * L::WAVES * 16 * 3 < 160 * 1024;      // what fits: two or three
    float4* lds;             // [vector][quad][thread]
    __device__ inline void put(int which, const Values<L>& v) {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            const float* const p = &v[q * 4 / L::G][q * 4 % L::G];
            lds[(which * kQuads + q) * (64 * L::WAVES) + threadIdx.x] = make_float4(p[0], p[1], p[2], p[3]);
        }
    }
    __device__ inline void get(int which, Values<L>& v) const {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            float* const p = &v[q * 4 / L::G][q * 4 % L::G];
            const float4 f = lds[(which * kQuads + q) * (64 * L::WAVES) + threadIdx.x];
            p[0] = f.x;
            p[1] = f.y;
            p[2] = f.z;
            p[3] = f.w;
        }
    }
};

// Wavefronts a SIMD: what leaves registers for the row and its sums.
template <typename E, typename L>
inline constexpr int kBackwardWaves = L::WAVES == 16 ? 4 : L::CH == 2 || is_f32<E> ? 2 : 4;

// BETAS: a norm has one, or its gradient is wanted.
template <typename E, typename L, bool BETAS>
__global__ __launch_bounds__(64 * L::WAVES) __attribute__((amdgpu_waves_per_eu((kBackwardWaves<E, L>)))) void norm_residual_backward_kernel(const NormBackArgs a) {
    __shared__ float2 sums_s[2 * L::WAVES];
    Sums<L::WAVES> sums(sums_s);
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
    Values<L> sum_gate = {}, sum_pre = {}, sum_post = {}, sum_pre_b = {}, sum_post_b = {};
    __shared__ float4 kept_s[(BETAS && Kept<L>::kThree ? 3 : 2) * Kept<L>::kQuads * 64 * L::WAVES];
    Kept<L> kept{kept_s};
    enum { kPostGamma, kPreGamma, kPostBeta };
    Row<E, L> y, r, dn, dr, gate;
    int64_t gate_row = 0, gate_end = 0;
    auto load = [&](int64_t m) {
        y.load(a.y, m, a.ld_y, D);
        if (norm) {
            dn.load(a.dn, m, a.ld_dn, D);
            r.load(a.r, m, a.ld_r, D);
        }
    };
    if (first < last) {
        load(first);
        Values<L> v;
        // 1000 x 16000 bfloat16 147 us as rows, 156 otherwise; with betas 100 x 9001 85 and 78.
        constexpr bool AS_ROW = L::WAVES == 16 && !BETAS;
        load_vector<L, AS_ROW>(a.post_gamma, D, 1.0f, v);
        kept.put(kPostGamma, v);
        load_vector<L, AS_ROW>(a.pre_gamma, D, 1.0f, v);
        kept.put(kPreGamma, v);
        if constexpr (BETAS && Kept<L>::kThree) {
            load_vector<L>(a.post_beta, D, 0.0f, v);
            kept.put(kPostBeta, v);
        }
    }
    for (int64_t m = first; m < last; ++m) {
        Values<L> d, v, hat;
        // Of this row, needed after the first sums.
        if (a.dr) dr.load(a.dr, m, a.ld_dr, D);
        if (a.gate && m >= gate_end) {
            gate_row = m / R;
            gate_end = (gate_row + 1) * R;
            gate.load(a.gate, gate_row, a.ld_gate, D);
        }
        y.widened(D, v);
        if (norm) {
            dn.widened(D, d);
            r.widened(D, hat);
        }
        load(min(m + 1, last - 1));                 // the next row, or the last one again
        if (!norm) each<L>([&](int i, int e) { hat[i][e] = 0.0f; });
        const float2 inv = normalise_both<L>(a.pre, hat, a.post, v, D, a.eps, sums);
        Values<L> gamma;
        if (norm) {
            kept.get(kPreGamma, gamma);
            each<L>([&](int i, int e) {
                sum_pre[i][e] = fmaf(d[i][e], hat[i][e], sum_pre[i][e]);
                if constexpr (BETAS) sum_pre_b[i][e] += d[i][e];
                d[i][e] *= gamma[i][e];
            });
            norm_gradient<L>(a.pre, d, hat, inv.x, D, sums);
        } else {
            each<L>([&](int i, int e) { d[i][e] = 0.0f; });
        }
        if (a.dr) {
            dr.widened(D, hat);
            each<L>([&](int i, int e) { d[i][e] += hat[i][e]; });
        }
        if (a.dx) store_row<E, L>(static_cast<E*>(a.dx) + m * a.ld_dx, D, d);

        each<L>([&](int i, int e) { d[i][e] = L::first_col(i) + e < D ? d[i][e] * a.res_scale : 0.0f; });
        kept.get(kPostGamma, gamma);
        if (a.dgate) {
            // t = gamma * hat + beta
            each<L>([&](int i, int e) { sum_gate[i][e] = fmaf(d[i][e], v[i][e] * gamma[i][e], sum_gate[i][e]); });
            if constexpr (BETAS) {
                Values<L> beta;
                if constexpr (Kept<L>::kThree) kept.get(kPostBeta, beta);
                else load_vector<L, is_f32<E>>(a.post_beta, D, 0.0f, beta);      // 4000 x 9001 float32 1239 us as rows, 1279 otherwise
                each<L>([&](int i, int e) { sum_gate[i][e] = fmaf(d[i][e], beta[i][e], sum_gate[i][e]); });
            }
            if (a.strips.per_gate == 0 && (m + 1 == last || m + 1 == gate_end)) {
                store_row<E, L>(static_cast<E*>(a.dgate) + gate_row * a.ld_dgate, D, sum_gate);
                each<L>([&](int i, int e) { sum_gate[i][e] = 0.0f; });
            }
        }
        if (a.gate) {
            gate.widened(D, hat);
            each<L>([&](int i, int e) { d[i][e] *= hat[i][e]; });
        }
        if (a.post != BNN_NORM_NONE) {
            each<L>([&](int i, int e) {
                sum_post[i][e] = fmaf(d[i][e], v[i][e], sum_post[i][e]);
                if constexpr (BETAS) sum_post_b[i][e] += d[i][e];
                d[i][e] *= gamma[i][e];
            });
            if (a.dy) norm_gradient<L>(a.post, d, v, inv.y, D, sums);
        }
        if (a.dy) store_row<E, L>(static_cast<E*>(a.dy) + m * a.ld_dy, D, d);
    }
    float* const part = a.part + strip * D;
    if (a.at_gate >= 0) store_row<float, L>(part + a.at_gate * a.part_step, D, sum_gate);
    if (a.at_pre_gamma >= 0) store_row<float, L>(part + a.at_pre_gamma * a.part_step, D, sum_pre);
    if (a.at_post_gamma >= 0) store_row<float, L>(part + a.at_post_gamma * a.part_step, D, sum_post);
    if constexpr (BETAS) {
        if (a.at_pre_beta >= 0) store_row<float, L>(part + a.at_pre_beta * a.part_step, D, sum_pre_b);
        if (a.at_post_beta >= 0) store_row<float, L>(part + a.at_post_beta * a.part_step, D, sum_post_b);
    }
}

bool norm_kind(int kind) { return kind == BNN_NORM_NONE || kind == BNN_NORM_RMS || kind == BNN_NORM_LAYER; }

int check_norm_sizes(int64_t M, int64_t D, int64_t rows_per_gate) {
    if (M < 0 || D < 0 || rows_per_gate < 1 || M > kMaxDim || D > kMaxDim || rows_per_gate > kMaxDim) return BNN_ERR_INVALID_ARG;
    return D > kMaxRowHeld ? BNN_ERR_UNSUPPORTED : BNN_OK;
}

// A matrix of the call: there or not wanted, with rows of D.
struct Operand2 {
    const void* p;
    int64_t ld;
};

// What both entry points check; a.n: n, or the place of n^.
int check_norm(int type, const NormArgs& a, int64_t M, int64_t D) {
    const int64_t size = type_bytes(type);
    if (size == 0 || !norm_kind(a.post) || !norm_kind(a.pre)) return BNN_ERR_INVALID_ARG;
    const int st = check_norm_sizes(M, D, a.rows_per_gate);
    if (st != BNN_OK) return st;
    if ((a.post != BNN_NORM_LAYER && a.post_beta) || (a.post == BNN_NORM_NONE && a.post_gamma) || (a.pre != BNN_NORM_LAYER && a.pre_beta) ||
        (a.pre == BNN_NORM_NONE && a.pre_gamma))
        return BNN_ERR_INVALID_ARG;
    for (const Operand2& o : {Operand2{a.y, a.ld_y}, Operand2{a.x, a.ld_x}, Operand2{a.gate, a.ld_gate}, Operand2{a.r, a.ld_r}, Operand2{a.n, a.ld_n}}) {
        if (o.p && (o.ld < D || o.ld > kMaxDim)) return BNN_ERR_INVALID_ARG;
        if (!aligned_to(o.p, size)) return BNN_ERR_ALIGNMENT;
    }
    for (const float* p : {a.post_gamma, a.post_beta, a.pre_gamma, a.pre_beta})
        if (!aligned_to(p, 4)) return BNN_ERR_ALIGNMENT;
    return BNN_OK;
}

template <int ROWS, typename A>
int launch_norm(int type, A a, int64_t M, int64_t D, void* stream) {
    a.M = int(M);
    a.D = int(D);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool betas = a.post_beta || a.pre_beta;
    with_type(type, [&](auto e) {
        with_row(D, [&](auto layout) {
            using L = decltype(layout);
            // As many workgroups as are on the chip together, each walking over rows.
            const int threads = L::threads(D);
            constexpr int WAVES = ROWS == kReals ? kNormWaves : kNormRowsWaves<L>;
            const int64_t together = 256 * (64 * WAVES / threads > 0 ? 64 * WAVES / threads : 1);
            const dim3 grid(uint32_t(M < together ? M : together)), block(uint32_t(threads), 1, 1);
            if (betas) norm_residual_kernel<decltype(e), L, true, ROWS><<<grid, block, 0, s>>>(a);
            else norm_residual_kernel<decltype(e), L, false, ROWS><<<grid, block, 0, s>>>(a);
        });
    });
    return check_launch();
}

}  // namespace
}  // namespace bnn

extern "C" int bnn_norm_residual(int type, const void* y, int64_t ld_y, const void* x, int64_t ld_x, const void* gate,
                                 int64_t ld_gate, int64_t rows_per_gate, float res_scale, int post, const float* post_gamma,
                                 const float* post_beta, int pre, const float* pre_gamma, const float* pre_beta, float eps, void* r,
                                 int64_t ld_r, void* n, int64_t ld_n, int64_t M, int64_t D, void* stream) {
    using namespace bnn;
    const NormArgs a{y, x, gate, post_gamma, post_beta, pre_gamma, pre_beta, r, n, ld_y, ld_x, ld_gate, ld_r, ld_n, rows_per_gate,
                     res_scale, eps, post, pre, 0, 0};
    const int st = check_norm(type, a, M, D);
    if (st != BNN_OK || M == 0 || D == 0) return st;
    if (!y || (n != nullptr) != (pre != BNN_NORM_NONE) || (!r && !n)) return BNN_ERR_INVALID_ARG;
    return launch_norm<kReals>(type, a, M, D, stream);
}

extern "C" int bnn_norm_residual_q(int type, const void* y, int64_t ld_y, const void* x, int64_t ld_x, const void* gate,
                                   int64_t ld_gate, int64_t rows_per_gate, float res_scale, int post, const float* post_gamma,
                                   const float* post_beta, int pre, const float* pre_gamma, const float* pre_beta, float eps, void* r,
                                   int64_t ld_r, int rows, uint8_t* codes, int64_t ld_c, void* scales, int64_t ld_s, void* hat,
                                   int64_t ld_h, int64_t M, int64_t D, void* stream) {
    using namespace bnn;
    NormRowsArgs a{};
    static_cast<NormArgs&>(a) = NormArgs{y, x, gate, post_gamma, post_beta, pre_gamma, pre_beta, r, hat, ld_y, ld_x, ld_gate, ld_r, ld_h, rows_per_gate,
                                         res_scale, eps, post, pre, 0, 0};
    int st = check_norm(type, a, M, D);
    if (st == BNN_OK) st = check_rows(rows, codes, ld_c, scales, ld_s, M, D);
    if (st != BNN_OK || M == 0) return st;
    if (D == 0) return bnn_quantize_rows(rows, type, nullptr, 0, codes, ld_c, scales, ld_s, nullptr, 0, M, 0, stream);      // scales of rows of nothing
    if (!y) return BNN_ERR_INVALID_ARG;
    a.out = QuantOut{codes, scales, hat, ld_c, ld_s, ld_h};
    return rows == BNN_ROWS_I8 ? launch_norm<BNN_ROWS_I8>(type, a, M, D, stream) : launch_norm<BNN_ROWS_MX4>(type, a, M, D, stream);
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
    join.N = int(D);
    auto want = [&](float* out) {
        if (!out) return -1;
        join.add(a.part + join.vectors * a.part_step, a.strips.count, out);
        return join.vectors - 1;
    };
    a.at_post_gamma = want(dpost_gamma);
    a.at_post_beta = want(dpost_beta);
    a.at_pre_gamma = want(dpre_gamma);
    a.at_pre_beta = want(dpre_beta);
    a.at_gate = dgate && a.strips.per_gate > 0 ? join.vectors : -1;
    if (M > 0) {
        const bool betas = post_beta || dpost_beta || dpre_beta;
        with_type(type, [&](auto e) {
            with_row(D, [&](auto layout) {
                using L = decltype(layout);
                const dim3 grid(uint32_t(a.strips.count)), block(uint32_t(L::threads(D)));
                if (betas) norm_residual_backward_kernel<decltype(e), L, true><<<grid, block, 0, s>>>(a);
                else norm_residual_backward_kernel<decltype(e), L, false><<<grid, block, 0, s>>>(a);
            });
        });
        if ((st = check_launch()) != BNN_OK) return st;
    }
    if (a.at_gate >= 0 && M > 0) {
        join.group_part = a.part + a.at_gate * a.part_step;
        join.groups = int(ceil_div(M, a.rows_per_gate));
        join.per_group = int(a.strips.per_gate);
        join.out_groups = dgate;
        join.ld_out = ld_dgate;
    }
    with_type(type, [&](auto e) { st = join_sums<decltype(e)>(join, s); });
    return st;
}
