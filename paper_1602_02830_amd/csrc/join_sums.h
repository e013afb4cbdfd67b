// The second half of a sum over rows: what workgroups have summed over their rows each, joined in a fixed order.
//
// A vector is the sum of its `parts` sums of N columns; beside vectors there may be one matrix, whose row g is the sum of its
// parts g * per_group to (g + 1) * per_group.  One launch for all of them.  A workgroup of 1024 threads takes `cols` columns of a
// vector or of a row, and each thread of a column its share of the parts, eight loads at a time: with four threads a column and one
// load at a time, joining 512 parts of 4096 columns took longer than what they came from.
#pragma once

#include "real_types.h"

namespace bnn {

constexpr int kMostJoined = 4;          // vectors of one launch
constexpr int kJoinThreads = 1024;

struct JoinArgs {
    const float* part[kMostJoined];     // [parts][N]
    float* out[kMostJoined];
    int parts[kMostJoined];
    const float* group_part;            // [groups][per_group][N]
    void* out_groups;                   // [groups][ld_out]
    int64_t ld_out;
    int vectors, groups, per_group, N, cols, group_cols;      // cols: powers of two
    inline void add(const float* sums, int64_t count, float* to) {
        part[vectors] = sums;
        parts[vectors] = int(count);
        out[vectors++] = to;
    }
};

template <typename E>
__global__ __launch_bounds__(kJoinThreads) void join_sums_kernel(const JoinArgs a) {
    __shared__ float sums_s[kJoinThreads];
    const int of_vectors = a.vectors * ((a.N + a.cols - 1) / a.cols);
    const bool matrix = int(blockIdx.x) >= of_vectors;
    const int cols = matrix ? a.group_cols : a.cols, blocks_n = (a.N + cols - 1) / cols, step = kJoinThreads / cols;
    const int block = int(blockIdx.x) - (matrix ? of_vectors : 0), row = block / blocks_n;
    const int c = threadIdx.x & (cols - 1), n = (block - row * blocks_n) * cols + c;
    const int parts = matrix ? a.per_group : a.parts[row];
    const float* const part = (matrix ? a.group_part + int64_t(row) * parts * a.N : a.part[row]) + min(n, a.N - 1);
    float s = 0.0f;
    int t = threadIdx.x / uint32_t(cols);
    for (; t + 7 * step < parts; t += 8 * step) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = part[int64_t(t + step * i) * a.N];
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; t < parts; t += step) s += part[int64_t(t) * a.N];
    // The threads of a column in a wavefront, then its wavefronts.
    for (int off = 32; off >= cols; off >>= 1) s += __shfl_xor(s, off);
    const int lanes = min(cols, 64);
    if ((threadIdx.x & 63) < lanes) sums_s[(threadIdx.x >> 6) * lanes + (threadIdx.x & 63)] = s;
    __syncthreads();
    if (threadIdx.x >= cols || n >= a.N) return;
    s = 0.0f;
    for (int w = c; w < kJoinThreads / 64 * lanes; w += cols) s += sums_s[w];
    if (matrix) static_cast<E*>(a.out_groups)[row * a.ld_out + n] = E(s);
    else a.out[row][n] = s;
}

// E: the type of out_groups.
template <typename E>
inline int join_sums(JoinArgs a, hipStream_t s) {
    if (a.N == 0) return BNN_OK;
    // 32 columns a workgroup, fewer where that leaves most of the chip idle (three vectors of 300 columns, 3750 parts each: 30
    // workgroups 11.7 us, 114 of them 5.5), more where a column has only a few parts.
    a.cols = (a.vectors + a.groups) * ceil_div(a.N, 32) >= 128 ? 32 : 8;
    a.group_cols = a.per_group <= 32 ? 256 : a.cols;
    const int64_t blocks = a.vectors * ceil_div(a.N, a.cols) + a.groups * ceil_div(a.N, a.group_cols);
    if (blocks > max_blocks(kJoinThreads)) return BNN_ERR_UNSUPPORTED;
    if (blocks == 0) return BNN_OK;
    join_sums_kernel<E><<<dim3(uint32_t(blocks)), dim3(kJoinThreads), 0, s>>>(a);
    return check_launch();
}

}  // namespace bnn
