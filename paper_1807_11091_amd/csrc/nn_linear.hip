// Entry points of the linear layer and of the gated pair of projections, and the
// element-wise part of their gradients.
//
//   linear    dz = dy act'(z);  dx = dz W, dW = dz^T x, dbias = sum over rows of dz
//   gated     dg = dh u act'(g), du = dh act(g);  dx = dg Wg + du Wu,
//             dWg = dg^T x, dWu = du^T x, dbg and dbu their column sums
//
// dz (dg and du) go to the workspace in the operands' type, as the matrix cores
// read them; the bias gradients are summed from the binary32 values.  That rounding is
// the price of the 16-bit products: binary32 values would have to go in as sums of two
// 16-bit ones, for twice the products.  Against binary64 it takes the error of dX and
// dW from 2.1e-4 to 2.9e-4 of their size in binary16 and from 1.7e-3 to 2.3e-3 in
// bfloat16, whatever dW's type; without an activation dz is dY itself and nothing is
// rounded.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nn_columns.h"
#include "nn_gemm.h"
#include "nn_types.h"
#include "sa_host.h"

namespace sa {
namespace {

constexpr int kV = 8;
constexpr int kRowGroups = 8;   // groups of 32 threads of a workgroup, each a row at a time
constexpr int kStripes = 256;   // row stripes whose column sums are joined, at most

struct SlopeArgs {
    int64_t M, ldd, ldz, ldu, ldo;
    int N, act;
    int64_t stripe;             // rows of one workgroup
    const void *dY, *Z, *U;
    void *o0, *o1;              // dz, or dg and du; NULL: sums only
    float *part;                // [stripes][2][N] column sums of dz, or of dg and du; or NULL
};

// Workgroup (x, y): 256 columns of the rows [y, y + 1) * stripe.  Bound by memory; rows
// in groups of 32 threads, not wavefronts, since 64 threads a row took 193 us where this
// takes 156.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_slope(SlopeArgs a) {
    constexpr int H = GATED ? 2 : 1;
    __shared__ float join[kRowGroups][256];
    const int t = threadIdx.x & 31, rg = threadIdx.x >> 5;
    const int c = blockIdx.x * 256 + t * kV, n = min(kV, a.N - c);
    const int64_t r0 = blockIdx.y * a.stripe, r1 = min(a.M, r0 + a.stripe);
    float s[H][kV] = {};
    auto load = [&](const void *p, int64_t at, float (&v)[kV]) {
        if (n == kV) load_vec<T, kV>(reinterpret_cast<const T *>(p) + at, v);
        else load_part<T, kV>(reinterpret_cast<const T *>(p) + at, n, v);
    };
    auto store = [&](void *p, int64_t at, const float (&v)[kV]) {
        if (n == kV) store_vec<T, kV>(reinterpret_cast<T *>(p) + at, v);
        else store_part<T, kV>(reinterpret_cast<T *>(p) + at, n, v);
    };
    if (n > 0)
        for (int64_t r = r0 + rg; r < r1; r += kRowGroups) {
            float d[kV], z[kV], u[kV];
            load(a.dY, r * a.ldd + c, d);
            if (a.Z) load(a.Z, r * a.ldz + c, z);
            if constexpr (GATED) load(a.U, r * a.ldu + c, u);
            float v[kV], slope[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) v[i] = slope[i] = 1.0f;
            if (a.Z) activate<true, kV>(a.act, z, v, slope);
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                if constexpr (GATED) {
                    z[i] = d[i] * v[i];             // du
                    d[i] = d[i] * u[i] * slope[i];  // dg
                    s[GATED][i] += z[i];
                } else {
                    d[i] *= slope[i];
                }
                s[0][i] += d[i];
            }
            if (a.o0) store(a.o0, r * a.ldo + c, d);
            if constexpr (GATED)
                if (a.o1) store(a.o1, r * a.ldo + c, z);
        }
    if (!a.part) return;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kV; ++i) join[rg][t * kV + i] = s[h][i];
        __syncthreads();
        const int col = blockIdx.x * 256 + threadIdx.x;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowGroups; ++w) v += join[w][threadIdx.x];
        if (col < a.N) a.part[((int64_t)blockIdx.y * 2 + h) * a.N + col] = v;
    }
}

// Short stripes, since nothing but many workgroups hides the latency of the loads:
// gated, 8192 x 9830 bfloat16 took 222 us in 64 stripes and takes 156 us in 256, 5.2
// TB/s; 256 x 1024 float16 took 12 us in stripes of 32 rows and takes 4.4 us in stripes
// of 8, a row per group.
int64_t stripe_rows(int64_t M) { return round_up(std::max<int64_t>((M + kStripes - 1) / kStripes, 1), kRowGroups); }
int stripes_of(int64_t M) { return (int)((M + stripe_rows(M) - 1) / stripe_rows(M)); }

int slope(const SlopeArgs &s, int type, bool gated, float *b0, float *b1, hipStream_t stream) {
    SlopeArgs a = s;
    a.stripe = stripe_rows(a.M);
    const int stripes = stripes_of(a.M);
    if (a.N > 0 && stripes > 0) {
        const dim3 grid((a.N + 255) / 256, stripes);
        if (type == SA_BF16) {
            if (gated) hipLaunchKernelGGL((k_slope<__bf16, true>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((k_slope<__bf16, false>), grid, dim3(256), 0, stream, a);
        } else {
            if (gated) hipLaunchKernelGGL((k_slope<_Float16, true>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((k_slope<_Float16, false>), grid, dim3(256), 0, stream, a);
        }
        if (int rc = check_hip(hipGetLastError(), "k_slope")) return rc;
    }
    return a.N > 0 && (b0 || b1) ? join_columns(a.part, stripes, a.N, b0, b1, stream) : SA_OK;
}

// Takes `bytes` of the workspace, 256-byte aligned.
struct Arena {
    uint8_t *base;
    size_t used;
    void *take(size_t bytes) {
        void *p = base ? base + used : nullptr;
        used += (size_t)round_up((int64_t)bytes, 256);
        return p;
    }
};

// The steps of a backward pass, laid out over a workspace at `ws` (NULL to size it).
struct BwdPlan {
    SlopeArgs slope;
    bool gated, need_slope, need_sums;
    Gemm dx, dw;
    void *ws_dx, *ws_dw;
    size_t bytes;
};

BwdPlan plan_bwd(int64_t M, int64_t N, int64_t K, int type, int dw_type, int act, bool gated, const void *dY, int64_t lddy,
                 const void *Z, const void *U, int64_t ldz, const void *X, int64_t ldx, const void *W0, const void *W1,
                 int64_t ldw, void *dX, int64_t lddx, void *dW0, void *dW1, int64_t lddw, bool bias, void *ws) {
    BwdPlan p{};
    Arena arena{static_cast<uint8_t *>(ws), 0};
    const int64_t ldo = round_up(N, 64);
    const bool rewrite = gated || act != SA_ACT_NONE;  // dz is not dY itself
    p.gated = gated;
    p.need_sums = bias;
    p.need_slope = bias || (rewrite && (dX || dW0));
    p.slope = SlopeArgs{M, lddy, ldz, ldz, ldo, (int)N, act, 0, dY, rewrite ? Z : nullptr, U, nullptr, nullptr, nullptr};
    Operand d0{dY, lddy, 0}, d1{nullptr, 0, 0};
    if (rewrite && (dX || dW0)) {
        p.slope.o0 = arena.take((size_t)M * ldo * 2);
        d0 = Operand{p.slope.o0, ldo, 0};
        if (gated) {
            p.slope.o1 = arena.take((size_t)M * ldo * 2);
            d1 = Operand{p.slope.o1, ldo, 0};
        }
    }
    if (bias) p.slope.part = static_cast<float *>(arena.take((size_t)2 * stripes_of(M) * N * sizeof(float)));
    Operand t0 = d0, t1 = d1;
    t0.across = t1.across = 1;
    // dX[m][k] = sum over n of dz[m][n] W[n][k]
    p.dx = Gemm{M, K, N, type, 0, gated ? 2 : 1, 1, {d0, d1}, {Operand{W0, ldw, 1}, Operand{W1, ldw, 1}}, Epilogue{}, nullptr};
    p.dx.e.Y = dX;
    p.dx.e.ldy = lddx;
    // dW[n][k] = sum over m of dz[m][n] X[m][k]
    p.dw = Gemm{N, K, M, type, 0, 1, gated ? 2 : 1, {t0, t1}, {Operand{X, ldx, 1}, Operand{}}, Epilogue{}, dW1};
    p.dw.e.Y = dW0;
    p.dw.e.ldy = lddw;
    p.dw.e.out_f32 = dw_type == SA_F32;
    p.ws_dx = arena.take(dX ? gemm_workspace(p.dx) : 0);
    p.ws_dw = arena.take(dW0 ? gemm_workspace(p.dw) : 0);
    p.bytes = arena.used;
    return p;
}

int run_bwd(const BwdPlan &p, int type, float *b0, float *b1, hipStream_t stream) {
    if (p.need_slope)
        if (int rc = slope(p.slope, type, p.gated, b0, b1, stream)) return rc;
    const Gemm *g[2];
    void *ws[2];
    int n = 0;
    if (p.dx.e.Y) g[n] = &p.dx, ws[n++] = p.ws_dx;
    if (p.dw.e.Y) g[n] = &p.dw, ws[n++] = p.ws_dw;
    return gemm(g, ws, n, stream);
}

BwdPlan plan(const sa_linear_bwd_desc &d, void *ws) {
    return plan_bwd(d.M, d.N, d.K, d.type, d.dw_type, d.act, false, d.dY, d.lddy, d.Z, nullptr, d.ldz, d.X, d.ldx, d.W,
                    nullptr, d.ldw, d.dX, d.lddx, d.dW, nullptr, d.lddw, d.dbias != nullptr, ws);
}

BwdPlan plan(const sa_glu_bwd_desc &d, void *ws) {
    return plan_bwd(d.M, d.N, d.K, d.type, d.dw_type, d.act, true, d.dH, d.lddh, d.G, d.U, d.ldgu, d.X, d.ldx, d.Wg, d.Wu,
                    d.ldw, d.dX, d.lddx, d.dWg, d.dWu, d.lddw, d.dbg || d.dbu, ws);
}

Gemm product(const sa_linear_desc &d) {
    return Gemm{d.M, d.N, d.K, d.type, 0, 1, 1, {Operand{d.X, d.ldx, 0}, Operand{}}, {Operand{d.W, d.ldw, 0}, Operand{}},
                Epilogue{d.act, d.out_type == SA_F32, d.bias, nullptr, d.R, d.ldr, d.Y, d.ldy, d.Z, nullptr, d.ldz}, nullptr};
}

Gemm product(const sa_glu_desc &d) {
    return Gemm{d.M, d.N, d.K, d.type, 1, 1, 1, {Operand{d.X, d.ldx, 0}, Operand{}},
                {Operand{d.Wg, d.ldw, 0}, Operand{d.Wu, d.ldw, 0}},
                Epilogue{d.act, 0, d.bg, d.bu, nullptr, 0, d.H, d.ldh, d.G, d.U, d.ldgu}, nullptr};
}

// A size query may come before the buffers.  An operand that is NULL then counts as one
// whose rows start anywhere, and a backward descriptor without its first matrix as one of
// every output, so that the size covers each call that may follow.
template <typename P>
void assume(P *&p) {
    if (!p) p = reinterpret_cast<P *>(alignof(uint16_t));
}

size_t workspace(sa_linear_desc d) {
    assume(d.X);
    assume(d.W);
    return gemm_workspace(product(d));
}

size_t workspace(sa_glu_desc d) {
    assume(d.X);
    assume(d.Wg);
    assume(d.Wu);
    return gemm_workspace(product(d));
}

size_t workspace(sa_linear_bwd_desc d) {
    if (!d.dY && d.M > 0 && d.N > 0) {
        assume(d.dY);
        assume(d.dX);
        assume(d.dW);
        assume(d.dbias);
    }
    assume(d.X);
    assume(d.W);
    return plan(d, nullptr).bytes;
}

size_t workspace(sa_glu_bwd_desc d) {
    if (!d.dH && d.M > 0 && d.N > 0) {
        assume(d.dH);
        assume(d.dX);
        assume(d.dWg);
        assume(d.dWu);
        assume(d.dbg);
        assume(d.dbu);
    }
    assume(d.X);
    assume(d.Wg);
    assume(d.Wu);
    return plan(d, nullptr).bytes;
}

}  // namespace
}  // namespace sa

using namespace sa;

extern "C" size_t structadmm_linear_workspace(const sa_linear_desc *desc) {
    if (!desc || validate_linear_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc);
}

extern "C" int structadmm_linear_fwd(const sa_linear_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "linear_fwd: desc is required");
    if (int rc = validate_linear(*desc)) return rc;
    const Gemm g = product(*desc);
    if (int rc = check_workspace("linear_fwd", desc->ws, desc->ws_bytes, gemm_workspace(g))) return rc;
    const Gemm *one = &g;
    return gemm(&one, &desc->ws, 1, stream);
}

extern "C" size_t structadmm_linear_bwd_workspace(const sa_linear_bwd_desc *desc) {
    if (!desc || validate_linear_bwd_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc);
}

extern "C" int structadmm_linear_bwd(const sa_linear_bwd_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "linear_bwd: desc is required");
    if (int rc = validate_linear_bwd(*desc)) return rc;
    const BwdPlan p = plan(*desc, desc->ws);
    if (int rc = check_workspace("linear_bwd", desc->ws, desc->ws_bytes, p.bytes)) return rc;
    return run_bwd(p, desc->type, desc->dbias, nullptr, stream);
}

extern "C" size_t structadmm_glu_workspace(const sa_glu_desc *desc) {
    if (!desc || validate_glu_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc);
}

extern "C" int structadmm_glu_fwd(const sa_glu_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "glu_fwd: desc is required");
    if (int rc = validate_glu(*desc)) return rc;
    const Gemm g = product(*desc);
    if (int rc = check_workspace("glu_fwd", desc->ws, desc->ws_bytes, gemm_workspace(g))) return rc;
    const Gemm *one = &g;
    return gemm(&one, &desc->ws, 1, stream);
}

extern "C" size_t structadmm_glu_bwd_workspace(const sa_glu_bwd_desc *desc) {
    if (!desc || validate_glu_bwd_sizes(*desc) != SA_OK) return 0;
    return workspace(*desc);
}

extern "C" int structadmm_glu_bwd(const sa_glu_bwd_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "glu_bwd: desc is required");
    if (int rc = validate_glu_bwd(*desc)) return rc;
    const BwdPlan p = plan(*desc, desc->ws);
    if (int rc = check_workspace("glu_bwd", desc->ws, desc->ws_bytes, p.bytes)) return rc;
    return run_bwd(p, desc->type, desc->dbg, desc->dbu, stream);
}
