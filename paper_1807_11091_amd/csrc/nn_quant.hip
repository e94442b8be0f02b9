// Quantisation of a matrix to 8 bits, as it stands and transposed.
//
// Both kernels are bound by memory: X is read once, a byte a code written.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nn_quant.h"
#include "nn_types.h"
#include "sa_conv_device.h"
#include "sa_host.h"

namespace sa {
namespace {

struct QuantArgs {
    int64_t rows, ldx;
    int cols;
    const void *X;
    sa_matrix8 Q, QT;
};

template <typename T>
__device__ inline void load8(const T *row, int n, float (&v)[8]) {
    if (n >= 8) load_vec<T, 8>(row, v);
    else load_part<T, 8>(row, n, v);
}

// Row blocks, not transposed.  Workgroup (x, y): 16 rows, a block of 128 columns; sixteen
// threads a row, so that the rows' scales go out side by side.  8192 x 9830 bfloat16 takes 50
// us (4.85 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void k_quant_rows(QuantArgs a, int64_t row0) {
    const int64_t row = row0 + (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int c = blockIdx.y * kBlock + (threadIdx.x & 15) * 8;
    const int n = row < a.rows ? a.cols - c : 0;
    float v[8];
    load8<T>(reinterpret_cast<const T *>(a.X) + (n > 0 ? row * a.ldx + c : 0), n, v);
    quantise_row(v, n, a.Q.codes + row * a.Q.ld + c, a.Q.scales + row * a.Q.scale_row + blockIdx.y * a.Q.scale_col);
}

// A tile of 128 x 128; workgroups walk bands of four tile rows.  Thread t holds 8 x 8 values,
// rows t / 16 * 8 and columns t % 16 * 8 on; the transposed codes go through LDS, so that both
// results leave in whole lines, past the caches.  8192 x 9830 bfloat16 both ways round takes
// 84 us (3.9 TB/s; 89 us with ordinary stores), 8192 x 4096 binary32 38 us (5.4; 46 us, and 54
// in columns of tiles).
template <typename T, bool SQUARE>
__global__ __launch_bounds__(256) void k_quant_tile(QuantArgs a, int64_t tile0, int tiles) {
    __shared__ float part[4][kBlock];
    // the tile's transposed codes, eight rows a word; a column's words XOR-swizzled, so that
    // the columns of a store fall on distinct banks
    __shared__ uint2 turned[kBlock][kBlock / 8];
    constexpr int BAND = 4;
    const int across = (a.cols + kBlock - 1) / kBlock;
    const int band = blockIdx.x / (BAND * across), in = blockIdx.x - band * BAND * across, h = min(BAND, tiles - band * BAND);
    const int64_t tr = tile0 + band * BAND + in % h;
    const int cb = in / h;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int rr = (t >> 4) * 8, cc = (t & 15) * 8;
    const int64_t r0 = tr * kBlock + rr;
    const int c0 = cb * kBlock + cc;
    const int nc = min(a.cols - c0, 8), nr = (int)max((int64_t)0, min(a.rows - r0, (int64_t)8));
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool in = i < nr && nc > 0;
        load8<T>(reinterpret_cast<const T *>(a.X) + (in ? (r0 + i) * a.ldx + c0 : 0), in ? nc : 0, v[i]);
    }
    float col[8];  // largest of this thread's 8 rows in each of its columns
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        col[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) col[j] = fmaxf(col[j], fabsf(v[i][j]));
    }
    float s = 0.0f, inv = 0.0f;
    if constexpr (SQUARE) {
        const float w = lanes_max<1, 64>(largest(col));
        if (lane == 0) part[wave][0] = w;
        __syncthreads();
        s = block_scale(fmaxf(fmaxf(part[0][0], part[1][0]), fmaxf(part[2][0], part[3][0])));
        inv = block_inverse(s);
        if (t == 0) {
            if (a.Q.codes) a.Q.scales[tr * a.Q.scale_row + cb * a.Q.scale_col] = s;
            if (a.QT.codes) a.QT.scales[cb * a.QT.scale_row + tr * a.QT.scale_col] = s;
        }
    }
    if (a.Q.codes)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint8_t *codes = a.Q.codes + (r0 + i) * a.Q.ld + c0;
            const int n = i < nr ? nc : 0;
            if constexpr (SQUARE) {
                if (n > 0) store_codes(codes, n, codes8(v[i], inv));
            } else {
                quantise_row(v[i], n, codes, a.Q.scales + (r0 + i) * a.Q.scale_row + cb * a.Q.scale_col);
            }
        }
    if (!a.QT.codes) return;
    float down[8];
    if constexpr (!SQUARE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) col[j] = lanes_max<16, 64>(col[j]);
        if (lane < 16)
#pragma unroll
            for (int j = 0; j < 8; ++j) part[wave][cc + j] = col[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float all = fmaxf(fmaxf(part[0][cc + j], part[1][cc + j]), fmaxf(part[2][cc + j], part[3][cc + j]));
            const float sc = block_scale(all);
            down[j] = block_inverse(sc);
            if (rr == 0 && j < nc) a.QT.scales[(c0 + j) * a.QT.scale_row + tr * a.QT.scale_col] = sc;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = v[i][j];
        turned[cc + j][(rr >> 3) ^ (cc >> 3)] = codes8(w, SQUARE ? inv : down[j]);
    }
    __syncthreads();
    // eight columns' rows at a time, 16 codes a thread
    const int at = (t & 7) * 16;
    const int n = (int)min(a.rows - (tr * kBlock + at), (int64_t)16);
#pragma unroll
    for (int j = 0; j < kBlock / 32; ++j) {
        const int c = j * 32 + (t >> 3);
        const int col0 = cb * kBlock + c;
        if (col0 >= a.cols || n <= 0) continue;
        const uint2 lo = turned[c][(at >> 3) ^ (c >> 3)], hi = turned[c][(at >> 3 | 1) ^ (c >> 3)];
        uint8_t *p = a.QT.codes + col0 * a.QT.ld + tr * kBlock + at;
        if (n == 16) {
            nt_store16(p, make_uint4(lo.x, lo.y, hi.x, hi.y));
        } else {
            store_codes(p, n, lo);
            if (n > 8) store_codes(p + 8, n - 8, hi);
        }
    }
}

// f(at, n): the launches over `count` workgroups along x, of at most 2^20 each (HIP counts
// a launch's threads along x in 32 bits)
template <typename F>
int in_launches(const char *who, int64_t count, int64_t most, F &&f) {
    for (int64_t at = 0; at < count; at += most) {
        f(at, (unsigned)std::min(most, count - at));
        if (int rc = check_hip(hipGetLastError(), who)) return rc;
    }
    return SA_OK;
}

template <typename T>
int quantise(const QuantArgs &a, bool square, hipStream_t stream) {
    const unsigned across = (unsigned)((a.cols + kBlock - 1) / kBlock);
    if (!square && !a.QT.codes)
        return in_launches("k_quant_rows", (a.rows + 15) / 16, int64_t(1) << 20, [&](int64_t at, unsigned n) {
            hipLaunchKernelGGL(k_quant_rows<T>, dim3(n, across), dim3(256), 0, stream, a, at * 16);
        });
    return in_launches("k_quant_tile", (a.rows + kBlock - 1) / kBlock, std::max<int64_t>((int64_t(1) << 20) / across, 1), [&](int64_t at, unsigned n) {
        if (square) hipLaunchKernelGGL((k_quant_tile<T, true>), dim3(n * across), dim3(256), 0, stream, a, at, (int)n);
        else hipLaunchKernelGGL((k_quant_tile<T, false>), dim3(n * across), dim3(256), 0, stream, a, at, (int)n);
    });
}

}  // namespace
}  // namespace sa

using namespace sa;

extern "C" int structadmm_quantize8(const sa_quantize8_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "quantize8: desc is required");
    const sa_quantize8_desc &d = *desc;
    if (int rc = validate_quantize8(d)) return rc;
    if (d.rows == 0 || d.cols == 0) return SA_OK;
    const QuantArgs a{d.rows, d.ldx, (int)d.cols, d.X, d.Q, d.QT};
    const bool square = d.block_rows == SA_BLOCK;
    if (d.type == SA_BF16) return quantise<__bf16>(a, square, stream);
    if (d.type == SA_F16) return quantise<_Float16>(a, square, stream);
    return quantise<float>(a, square, stream);
}
