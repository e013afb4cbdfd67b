// The second half of a sum over rows: what workgroups have summed over their rows each, joined in a fixed order.
//
// parts of N sums each; out[g][n] = sum over the parts g * per_group .. of part[n].  A workgroup takes 32 columns, with 32 threads
// for each, every one of them 1/32 of the parts, eight loads at a time: with four threads a column, one load at a time, joining
// 512 parts of 4096 columns took longer than what they came from.
#pragma once

#include "real_types.h"

namespace bnn {

constexpr int kMostJoined = 4;          // vectors of one launch

struct JoinArgs {
    const float* part;
    int64_t part_step;                  // from the first vector's parts to the next one's
    int64_t ld_out;                     // from group to group
    void* out[kMostJoined];
    int per_group, N, blocks_n;
};

template <typename E>
__global__ __launch_bounds__(1024) void join_sums_kernel(const JoinArgs a) {
    __shared__ float sums_s[32][33];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    const int64_t group = blockIdx.x / uint32_t(a.blocks_n);
    const int n = (int(blockIdx.x) - int(group) * a.blocks_n) * 32 + c;
    const float* const part = a.part + blockIdx.y * a.part_step + group * a.per_group * a.N + min(n, a.N - 1);
    float s = 0.0f;
    int t = q;
    for (; t + 7 * 32 < a.per_group; t += 8 * 32) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = part[int64_t(t + 32 * i) * a.N];
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; t < a.per_group; t += 32) s += part[int64_t(t) * a.N];
    sums_s[q][c] = s;
    __syncthreads();
    // Each half wavefront joins one column.
    s = sums_s[c][q];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor(s, off);
    const int m = (int(blockIdx.x) - int(group) * a.blocks_n) * 32 + q;
    if (c == 0 && m < a.N) static_cast<E*>(a.out[blockIdx.y])[group * a.ld_out + m] = E(s);
}

// groups * per_group parts; `vectors` of them, each with parts of its own.
template <typename E>
inline int join_sums(JoinArgs a, int64_t groups, int vectors, hipStream_t s) {
    a.blocks_n = int(ceil_div(a.N, 32));
    if (groups * a.blocks_n > max_blocks(1024)) return BNN_ERR_UNSUPPORTED;
    join_sums_kernel<E><<<dim3(uint32_t(groups * a.blocks_n), uint32_t(vectors)), dim3(1024), 0, s>>>(a);
    return check_launch();
}

}  // namespace bnn
