// Matrix products of the feed-forward operators on the gfx950 matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nn_gemm.h"
#include "nn_types.h"
#include "sa_host.h"

namespace sa {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ inline f32x4 mfma(Vec8<__bf16>::type a, Vec8<__bf16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(Vec8<_Float16>::type a, Vec8<_Float16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// One output from its sum(s): bias, activation, product or residual.
template <typename T>
__device__ inline void finish(const Epilogue &e, bool gated, void *Y, int64_t m, int64_t n, float s, float s2) {
    float z = e.bias ? s + e.bias[n] : s;
    if (e.Z) reinterpret_cast<T *>(e.Z)[m * e.ldz + n] = (T)z;
    float y = act_value(e.act, z);
    if (gated) {
        const float u = e.bias2 ? s2 + e.bias2[n] : s2;
        if (e.Z2) reinterpret_cast<T *>(e.Z2)[m * e.ldz + n] = (T)u;
        y *= u;
    }
    if (e.out_f32) {
        if (e.R) y += reinterpret_cast<const float *>(e.R)[m * e.ldr + n];
        reinterpret_cast<float *>(Y)[m * e.ldy + n] = y;
    } else {
        if (e.R) y += (float)reinterpret_cast<const T *>(e.R)[m * e.ldr + n];
        reinterpret_cast<T *>(Y)[m * e.ldy + n] = (T)y;
    }
}

// 64 x 64 outputs per workgroup of four wavefronts, slices of 32 k through LDS,
// any layout of the operands, element by element.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_gemm_any(Gemm g) {
    constexpr int BT = 64, BK = 32, P = BK + 8;
    typedef typename Vec8<T>::type vec;
    __shared__ __attribute__((aligned(16))) T sm[BT * P], sn[GATED ? 2 : 1][BT * P];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t mtiles = (g.M + BT - 1) / BT;
    const int64_t m0 = blockIdx.x % mtiles * BT, n0 = blockIdx.x / mtiles * BT;
    const int z = blockIdx.z;
    const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
    f32x4 acc[GATED ? 2 : 1][2][2] = {};
    auto fill = [&](T *dst, const Operand &o, int64_t r0, int64_t rows, int64_t k0) {
        const T *p = reinterpret_cast<const T *>(o.p);
        for (int i = tid; i < BT * BK; i += 256) {
            const int r = o.across ? i % BT : i / BK, k = o.across ? i / BT : i % BK;
            const bool in = r0 + r < rows && k0 + k < g.K;
            dst[r * P + k] = in ? p[o.across ? (k0 + k) * o.ld + r0 + r : (r0 + r) * o.ld + k0 + k] : (T)0.0f;
        }
    };
    for (int part = 0; part < g.parts; ++part)
        for (int64_t k0 = 0; k0 < g.K; k0 += BK) {
            fill(sm, g.m[g.batch > 1 ? z : part], m0, g.M, k0);
            fill(sn[0], g.n[part], n0, g.N, k0);
            if constexpr (GATED) fill(sn[1], g.n[1], n0, g.N, k0);
            __syncthreads();
            const int fo = (lane & 15) * P + (lane >> 4) * 8;
#pragma unroll
            for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[h][i][j] = mfma(*reinterpret_cast<const vec *>(&sn[h][(wn + i * 16) * P + fo]),
                                            *reinterpret_cast<const vec *>(&sm[(wm + j * 16) * P + fo]), acc[h][i][j]);
            __syncthreads();
        }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + wn + i * 16 + (lane >> 4) * 4 + r, m = m0 + wm + j * 16 + (lane & 15);
                if (m < g.M && n < g.N)
                    finish<T>(g.e, GATED, z ? g.y1 : g.e.Y, m, n, acc[0][i][j][r], GATED ? acc[GATED][i][j][r] : 0.0f);
            }
}

template <typename T>
int run(const Gemm &g, hipStream_t stream) {
    const int64_t tiles = ((g.M + 63) / 64) * ((g.N + 63) / 64);
    if (tiles >= (int64_t(1) << 31)) return fail(SA_E_UNSUPPORTED, "matrix product of more than 2^31 tiles");
    const dim3 grid((unsigned)tiles, 1, g.batch);
    if (g.gated) hipLaunchKernelGGL((k_gemm_any<T, true>), grid, dim3(256), 0, stream, g);
    else hipLaunchKernelGGL((k_gemm_any<T, false>), grid, dim3(256), 0, stream, g);
    return check_hip(hipGetLastError(), "k_gemm_any");
}

}  // namespace

size_t gemm_workspace(const Gemm &) { return 0; }

int gemm(const Gemm &g, void *, hipStream_t stream) {
    if (g.M == 0 || g.N == 0) return SA_OK;
    return g.type == SA_BF16 ? run<__bf16>(g, stream) : run<_Float16>(g, stream);
}

}  // namespace sa
