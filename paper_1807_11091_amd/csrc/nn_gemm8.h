// The 8-bit matrix products of the feed-forward operators (nn_gemm8.hip):
//   z[m][n] = sum over blocks b of 128 k of sx[m][b] sw[n / 128][b] sum over k in b of x[m][k] w[n][k]
// for e4m3 codes x and w with binary32 scales sx and sw, and an epilogue.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nn_gemm.h"
#include "structadmm.h"

namespace sa {

struct Gemm8 {
    int64_t M, N, K;
    int type;          // SA_BF16 or SA_F16: the 16-bit results' type
    int gated;         // two products, with w[0] and w[1]; result act(first) * second
    sa_matrix8 x;      // [M, K], row blocks
    sa_matrix8 w[2];   // [N, K], square blocks, one pitch and one pair of scale strides
    Epilogue e;        // Y may be NULL
    sa_matrix8 q;      // the result in 8 bits, row blocks; codes NULL: none
    int exact;         // whole products whatever the results
};

size_t gemm8_workspace(const Gemm8 &g);
int gemm8(const Gemm8 &g, void *ws, hipStream_t stream);

}  // namespace sa
