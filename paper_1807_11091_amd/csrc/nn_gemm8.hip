// 8-bit matrix products with block scales on the gfx950 matrix cores, and the entry points
// of the operators made of them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nn_epilogue.h"
#include "nn_gemm8.h"
#include "nn_quant.h"
#include "nn_tile.h"
#include "nn_types.h"
#include "sa_host.h"

namespace sa {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight codes as bfloat16, which holds every e4m3 value.
__device__ inline Vec8<__bf16>::type widen(int lo, int hi) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const pair c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return Vec8<__bf16>::type{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A block's products of 16 rows with 16, a lane's 32 codes of each in a and b.  How k is
// spread over lanes and bytes does not matter as long as both operands agree.
//
// The codes are widened for the bfloat16 instructions, whose binary32 sums are good to
// 1e-8 here.  The 8-bit ones (all that take e4m3, of 32 or 128 k) cut the products of a
// group of k 14 bits below its largest: sums of 128 are off by 1.3e-5 of their size.
__device__ inline f32x4 block_products(i32x8 a, i32x8 b) {
    f32x4 c = {};
#pragma unroll
    for (int q = 0; q < 4; ++q)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a[2 * q], a[2 * q + 1]), widen(b[2 * q], b[2 * q + 1]), c, 0, 0, 0);
    return c;
}

__device__ inline void add_scaled(f32x4 &acc, f32x4 part, float scale) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(part[e], scale, acc[e]);
}

// Binary32 sums of a product in memory, before its epilogue: [split][gated ? 2 : 1][M][pitch].
struct Partial8 {
    float *p;
    int64_t pitch;  // N rounded up to 8
    int split;      // parts of k
    int keep;       // the sums go to p (always with split > 1)
};

__device__ inline float *partial_at(const Partial8 &q, const Gemm8 &g, int chunk, int half, int64_t m, int64_t n) {
    const int64_t plane = (int64_t)chunk * (g.gated ? 2 : 1) + half;
    return q.p + (plane * g.M + m) * q.pitch + n;
}

// Adds the parts in their order and finishes 8 outputs per thread, sixteen threads a block
// of 128 outputs.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_join8(Gemm8 g, Partial8 q, int64_t first) {
    const uint32_t chunks = (uint32_t)(((g.N + kBlock - 1) / kBlock) * 16);
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    // the long division only where the short one does not do
    const int64_t m = i >> 32 ? i / chunks : (uint32_t)i / chunks, n = (i - m * chunks) * 8;
    if (m >= g.M) return;  // whole blocks
    const int cnt = (int)max((int64_t)0, min((int64_t)8, g.N - n));
    float s[8] = {}, u[8] = {}, t[8];
    if (cnt > 0) {
        for (int c = 0; c < q.split; ++c) {
            load_vec<float, 8>(partial_at(q, g, c, 0, m, n), t);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += t[e];
            if constexpr (GATED) {
                load_vec<float, 8>(partial_at(q, g, c, 1, m, n), t);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] += t[e];
            }
        }
        Addends<T, 8> with;
        with.has_r = false;
        with.load_bias(g.e, n, cnt);
        finish_values<T, GATED, 8>(g.e, m, n, cnt, s, u, with);
        if (g.e.Y) put_values<T, 8>(g.e, g.e.Y, m, n, cnt, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = e < cnt ? s[e] : 0.0f;
    }
    if (g.q.codes)
        quantise_row(s, cnt, g.q.codes + m * g.q.ld + n, g.q.scales + m * g.q.scale_row + n / kBlock * g.q.scale_col);
}

// ------------------------------------------------------------- few rows of M
// k_rows8: products with few rows of M, bound by reading the weights once and by latency.
// A workgroup of 8 wavefronts takes NF * 16 of their rows and MF * 16 of M; its wavefronts
// take the blocks of k in turn, U at a time, and feed the matrix cores straight from
// memory.  Their sums are joined through LDS in a fixed order.  Rows past M or N read the
// last row and are not stored.
template <typename T, bool GATED, int NF, int MF, int U>
__global__ __launch_bounds__(512) void k_rows8(Gemm8 g, Partial8 q) {
    constexpr int NW = 8, H = GATED ? 2 : 1;
    __shared__ float sums[NW][NF * H * MF][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, kg = (lane >> 4) * 16;
    const int64_t n0 = (int64_t)blockIdx.x * NF * 16, m0 = (int64_t)blockIdx.z * MF * 16;
    const int K = (int)g.K;
    // blocks of k of this workgroup
    const int blocks = (K + kBlock - 1) / kBlock;
    const int b0 = (int)((int64_t)blocks * blockIdx.y / q.split), b1 = (int)((int64_t)blocks * (blockIdx.y + 1) / q.split);

    const uint8_t *wp[H * NF], *xp[MF];
    const float *sx[MF], *sw[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int f = 0; f < NF; ++f) wp[h * NF + f] = g.w[h].codes + min(n0 + f * 16 + r, g.N - 1) * g.w[h].ld + kg;
        sw[h] = g.w[h].scales + n0 / kBlock * g.w[h].scale_row;  // NF * 16 divides 128: one block row
    }
#pragma unroll
    for (int j = 0; j < MF; ++j) {
        const int64_t m = min(m0 + j * 16 + r, g.M - 1);
        xp[j] = g.x.codes + m * g.x.ld + kg;
        sx[j] = g.x.scales + m * g.x.scale_row;
    }

    f32x4 acc[H * NF][MF] = {};
    for (int b = b0 + wave * U; b < b1; b += NW * U) {
        i32x8 w[U][H * NF], x[U][MF];
        float cx[U][MF], cw[U][H];
        // this lane's bytes of a block: chunks of 16 at kg and kg + 64, zeros past K
        auto load = [&](const uint8_t *p, int k) {
            union {
                i32x4 h[2];
                i32x8 v;
            } o;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int n = K - k - i * 64 - kg;
                o.h[i] = i32x4{};
                if (n > 0) o.h[i] = *reinterpret_cast<const i32x4 *>(p + k + i * 64);
                if (n < 16)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int have = n - e * 4;
                        if (have < 4) o.h[i][e] = have <= 0 ? 0 : o.h[i][e] & ((1 << have * 8) - 1);
                    }
            }
            return o.v;
        };
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int at = min(b + s, b1 - 1), k = b + s < b1 ? at * kBlock : K;
#pragma unroll
            for (int f = 0; f < H * NF; ++f) w[s][f] = load(wp[f], k);
#pragma unroll
            for (int j = 0; j < MF; ++j) {
                x[s][j] = load(xp[j], k);
                cx[s][j] = b + s < b1 ? sx[j][at * g.x.scale_col] : 0.0f;
            }
#pragma unroll
            for (int h = 0; h < H; ++h) cw[s][h] = b + s < b1 ? sw[h][at * g.w[h].scale_col] : 0.0f;
        }
#pragma unroll
        for (int s = 0; s < U; ++s)
#pragma unroll
            for (int f = 0; f < H * NF; ++f)
#pragma unroll
                for (int j = 0; j < MF; ++j) add_scaled(acc[f][j], block_products(w[s][f], x[s][j]), cx[s][j] * cw[s][f / NF]);
    }
#pragma unroll
    for (int f = 0; f < H * NF; ++f)
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wave][f * MF + j][r * 16 + (lane >> 4) * 4 + e] = acc[f][j][e];
    __syncthreads();
    // one output per thread: row m of M, 16 consecutive n
    for (int i = threadIdx.x; i < NF * MF * 256; i += 512) {
        const int f = i / (MF * 256), j = i / 256 % MF, at = i & 255;
        const int64_t m = m0 + j * 16 + (at >> 4), n = n0 + f * 16 + (at & 15);
        if (m >= g.M || n >= g.N) continue;
        float z[1] = {0.0f}, u[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            z[0] += sums[w][f * MF + j][at];
            if constexpr (GATED) u[0] += sums[w][(NF + f) * MF + j][at];
        }
        if (q.keep) {
            *partial_at(q, g, blockIdx.y, 0, m, n) = z[0];
            if constexpr (GATED) *partial_at(q, g, blockIdx.y, 1, m, n) = u[0];
        } else {
            finish<T, GATED, 1>(g.e, g.e.Y, m, n, 1, z, u);
        }
    }
}

// ---------------------------------------------------------------- host side
struct Plan8 {
    int split;
    int keep;  // the epilogue runs in k_join8
};

Plan8 plan_of(const Gemm8 &g) { return Plan8{1, g.q.codes != nullptr}; }

size_t partial_bytes(const Gemm8 &g, const Plan8 &p) {
    return p.keep ? (size_t)p.split * (g.gated ? 2 : 1) * g.M * round_up(g.N, 8) * sizeof(float) : 0;
}

template <typename T, bool GATED>
int join(const Gemm8 &g, const Partial8 &q, hipStream_t stream) {
    const int64_t blocks = (g.M * round_up(g.N, kBlock) / 8 + 255) / 256;
    constexpr int64_t most = int64_t(1) << 20;  // HIP counts a launch's threads along x in 32 bits
    for (int64_t at = 0; at < blocks; at += most) {
        hipLaunchKernelGGL((k_join8<T, GATED>), dim3((unsigned)std::min(most, blocks - at)), dim3(256), 0, stream, g, q, at);
        if (int rc = check_hip(hipGetLastError(), "k_join8")) return rc;
    }
    return SA_OK;
}

template <typename T, bool GATED>
int run(const Gemm8 &g, const Plan8 &p, const Partial8 &q, hipStream_t stream) {
    constexpr int NF = 1, MF = 4;
    hipLaunchKernelGGL((k_rows8<T, GATED, NF, MF, 1>), dim3((unsigned)((g.N + NF * 16 - 1) / (NF * 16)), q.split,
                       (unsigned)((g.M + MF * 16 - 1) / (MF * 16))), dim3(512), 0, stream, g, q);
    if (int rc = check_hip(hipGetLastError(), "k_rows8")) return rc;
    return q.keep ? join<T, GATED>(g, q, stream) : SA_OK;
}

Gemm8 product(const sa_linear8_desc &d) {
    return Gemm8{d.M, d.N, d.K, d.type, 0, d.X, {d.W, sa_matrix8{}},
                 Epilogue{d.act, d.out_type == SA_F32, d.bias, nullptr, d.R, d.ldr, d.Y, d.ldy, d.Z, nullptr, d.ldz}, d.Q};
}

Gemm8 product(const sa_glu8_desc &d) {
    return Gemm8{d.M, d.N, d.K, d.type, 1, d.X, {d.Wg, d.Wu},
                 Epilogue{d.act, 0, d.bg, d.bu, nullptr, 0, d.H, d.ldh, d.G, d.U, d.ldgu}, d.Q};
}

// A query that comes before the outputs is for all of them.
template <typename D>
size_t workspace(const D &d, const void *y) {
    Gemm8 g = product(d);
    if (!y && !g.q.codes) g.q.codes = reinterpret_cast<uint8_t *>(16);
    return gemm8_workspace(g);
}

}  // namespace

size_t gemm8_workspace(const Gemm8 &g) {
    if (g.M == 0 || g.N == 0) return 0;
    return partial_bytes(g, plan_of(g));
}

int gemm8(const Gemm8 &g, void *ws, hipStream_t stream) {
    if (g.M == 0 || g.N == 0) return SA_OK;
    const Plan8 p = plan_of(g);
    const Partial8 q{static_cast<float *>(ws), round_up(g.N, 8), p.split, p.keep};
    if (g.type == SA_BF16) return g.gated ? run<__bf16, true>(g, p, q, stream) : run<__bf16, false>(g, p, q, stream);
    return g.gated ? run<_Float16, true>(g, p, q, stream) : run<_Float16, false>(g, p, q, stream);
}

}  // namespace sa

using namespace sa;

extern "C" size_t structadmm_linear8_workspace(const sa_linear8_desc *desc) {
    if (!desc || validate_linear8_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc, desc->Y);
}

extern "C" int structadmm_linear8_fwd(const sa_linear8_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "linear8_fwd: desc is required");
    if (int rc = validate_linear8(*desc)) return rc;
    const Gemm8 g = product(*desc);
    if (int rc = check_workspace("linear8_fwd", desc->ws, desc->ws_bytes, gemm8_workspace(g))) return rc;
    return gemm8(g, desc->ws, stream);
}

extern "C" size_t structadmm_glu8_workspace(const sa_glu8_desc *desc) {
    if (!desc || validate_glu8_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc, desc->H);
}

extern "C" int structadmm_glu8_fwd(const sa_glu8_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "glu8_fwd: desc is required");
    if (int rc = validate_glu8(*desc)) return rc;
    const Gemm8 g = product(*desc);
    if (int rc = check_workspace("glu8_fwd", desc->ws, desc->ws_bytes, gemm8_workspace(g))) return rc;
    return gemm8(g, desc->ws, stream);
}
