// The matrix products of the feed-forward operators (nn_gemm.hip):
//   C[m][n] = sum over parts p and k < K of Mside_p(m, k) * Nside_p(n, k)
// for 16-bit operands, binary32 sums on the matrix cores, and an epilogue.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "structadmm.h"

namespace sa {

// An operand: element (r, k) stands at p[r * ld + k], or at p[k * ld + r] when
// `across` is set (its rows run across the sum).
struct Operand {
    const void *p;
    int64_t ld;
    int across;
};

// What becomes of the sums.
struct Epilogue {
    int act;              // sa_act
    int out_f32;          // Y and R are binary32 (else the operands' type)
    const float *bias;    // [N] or NULL; with `gated`, of the gate
    const float *bias2;   // gated: of the other projection
    const void *R;        // or NULL
    int64_t ldr;
    void *Y;
    int64_t ldy;
    void *Z, *Z2;         // pre-activations or NULL (Z2: gated)
    int64_t ldz;
    int past = 0;         // 16-bit results go past the caches, in kernels that can
};

struct Gemm {
    int64_t M, N, K;
    int type;             // SA_BF16 or SA_F16
    // gated: two products of the M side with n[0] and n[1], Y = act(first) * second
    int gated;
    // parts = 2: the sum runs over m[0] n[0] and then m[1] n[1]
    int parts;
    // batch = 2: two products, m[0] n[0] to e.Y and m[1] n[0] to y1
    int batch;
    Operand m[2], n[2];
    Epilogue e;
    void *y1;
};

// Workspace of a product: of its pointers only the operands' alignment matters.
size_t gemm_workspace(const Gemm &g);

constexpr int kMaxProducts = 2;

// Launches n <= kMaxProducts products that do not read each other's results, each with a
// workspace of its own; the operands that they need copied are copied by one launch before
// them.  The small products of a gradient (dX first) share a launch.
int gemm(const Gemm *const *g, void *const *ws, int n, hipStream_t stream);

}  // namespace sa
