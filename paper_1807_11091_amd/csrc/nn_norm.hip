// Layer norm over the rows of a matrix and its gradient.
//
//   forward   mean = sum x / n, rstd = (sum (x - mean)^2 / n + eps)^-1/2,
//             y = (x - mean) rstd gamma + beta
//   backward  with xn = (x - mean) rstd and t = dy gamma:
//             dx = rstd (t - sum t / n - xn sum(t xn) / n) + dr,
//             dgamma = sum over rows of dy xn, dbeta = sum over rows of dy
//
// Both are bound by HBM: the forward pass reads x and writes y, the backward pass
// reads dy, x (and dr) and writes dx, each once.
//
// TPR threads hold one row in registers (CH vectors of 8 elements each), so the
// row is read once and the variance is summed over x - mean, not as a difference
// of two large sums.  The mean's own rounding is taken out by the sum of x - mean.  Sums run in binary32 over at most 32 elements a thread and
// then over the threads in a fixed tree.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "nn_columns.h"
#include "nn_types.h"
#include "sa_host.h"

namespace sa {
namespace {

constexpr int kV = 8;  // elements per vector

// Rows of TPR threads each that a workgroup of the register kernels takes at a time.
// WIDE: four of 192 threads instead of two, for the backward kernel of 16-bit types: a
// CU holds one workgroup of it, which needs that many loads in flight (16384 x 2560
// bfloat16 66.7 us with two, 54.8 with four).  Rows of 384 threads, one a
// workgroup, were not tried in pairs.
template <int TPR, bool WIDE = false>
struct Rows {
    static constexpr int per_group =
        TPR <= 64 ? 8 : TPR <= 128 ? 4 : TPR <= 192 && WIDE ? 4 : TPR <= 256 ? 2 : 1;
    static constexpr int threads = TPR * per_group;
};

// Two sums over the TPR threads of a row, in a fixed order; every thread of the row
// receives them.  A row of several wavefronts needs a barrier, which every thread of
// the workgroup calls; tmp holds two sets, used in turn (turn = 0, 1, 0, ..), so that
// one barrier per call is enough.
template <int TPR, int NT>
__device__ inline void row_sums(float &a, float &b, float2 (*tmp)[NT / 64], int turn) {
    a = wave_sum_f32(a);
    b = wave_sum_f32(b);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6, first = threadIdx.x / TPR * (TPR / 64);
        if ((threadIdx.x & 63) == 0) tmp[turn & 1][wave] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) {
            const float2 t = tmp[turn & 1][first + w];
            a += t.x;
            b += t.y;
        }
    }
}

// A chunk as it is stored, in words, so that it takes no more registers than that.
template <typename T>
struct Raw {
    static constexpr int kWords = kV * sizeof(T) / 4, kPer = 4 / sizeof(T);
    unsigned w[kWords];

    // The chunk at c of a row.  One load for every thread and no branch, so that nothing
    // waits for it here: where the row ends inside the chunk or before it, the row's last
    // kV values, which place() moves.  SHORT: rows of fewer than kV columns, by value.
    template <bool SHORT>
    __device__ void load(const T *row, int c, int cols) {
        if constexpr (!SHORT) {
            __builtin_memcpy(w, row + (unsigned)min(c, cols - kV), sizeof w);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
            for (int i = 0; i < kV - 1; ++i)
                if (i < cols) {
                    unsigned bits = 0;
                    __builtin_memcpy(&bits, row + i, sizeof(T));
                    w[i / kPer] |= bits << (i % kPer * 16);
                }
        }
    }

    // The loaded values to their places, zeros from column end on.
    template <bool SHORT>
    __device__ void place(int c, int cols, int end) {
        const int by = SHORT ? 0 : c + kV - cols;
        if (by > 0 && by < kV) {
#pragma unroll
            for (int step = kWords / 2; step > 0; step /= 2)
                if (by / kPer & step)
#pragma unroll
                    for (int i = 0; i < kWords; ++i) w[i] = i + step < kWords ? w[i + step] : 0;
            if (by % kPer)
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = w[i] >> 16 | (i + 1 < kWords ? w[i + 1] << 16 : 0);
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = c < end ? w[i] : 0;
    }

    __device__ float operator[](int i) const {
        T v;
        const unsigned x = w[i / kPer] >> i % kPer * 16;
        __builtin_memcpy(&v, &x, sizeof v);
        return (float)v;
    }

    // Keeps the compiler from carrying what it computed from the values in registers.
    __device__ void renew() {
#pragma unroll
        for (unsigned &x : w) asm volatile("" : "+v"(x));
    }
};

template <typename T>
__device__ inline void load_chunk(const T *row, int c, int cols, float (&v)[kV]) {
    if (c + kV <= cols) load_vec<T, kV>(row + c, v);
    else load_part<T, kV>(row + c, cols - c, v);
}

template <typename T>
__device__ inline void store_chunk(T *row, int c, int cols, const float (&v)[kV]) {
    if (c + kV <= cols) store_vec<T, kV>(row + c, v);
    else store_part<T, kV>(row + c, cols - c, v);
}

// gamma or beta of a chunk (`other` where the pointer is NULL or past the row)
__device__ inline void load_param(const float *p, int c, int cols, float other, float (&v)[kV]) {
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] = other;
    if (p && c < cols) load_chunk<float>(p, c, cols, v);
}

// The sum of up to this many equal values is exact: nothing to take out of their mean.
template <typename T>
constexpr int64_t kExactSum = int64_t(1) << (24 - (sizeof(T) == 4 ? 24 : std::is_same_v<T, _Float16> ? 11 : 8));

// The statistics of a row from s = sum d^2 and q = sum d over d = x - m, m the rounded mean:
// returns rstd and takes the mean's own rounding, `off`, out of m.  A row of equal values
// has d = off exactly, that is x - mean = 0.  In a batch of 16384 x 4096 bfloat16, whose
// means need none of this, it would take 50.5 us instead of 46.4.
__device__ inline float row_stats(float s, float q, float n, float eps, bool exact, float &m, float &off) {
    float var = s / n;
    off = 0.0f;
    if (!exact) {
        const float mean_d = q / n;
        if (fabsf(mean_d) < __builtin_inff()) off = mean_d;  // an infinite or NaN row stays one
        m += off;
        var -= off * off;
        if (var < 0.0f) var = 0.0f;
    }
    return 1.0f / sqrtf(var + eps);
}

struct FwdArgs {
    int64_t rows, ldx, ldy;
    int cols;
    float eps;
    const void *X;
    const float *gamma, *beta;
    void *Y;
    float *mean, *rstd;
};

template <typename T, int TPR, int CH, bool SHORT>
__global__ __launch_bounds__(Rows<TPR>::threads) void k_ln_fwd(FwdArgs a) {
    constexpr int NT = Rows<TPR>::threads, RPB = Rows<TPR>::per_group;
    constexpr bool kExact = (int64_t)TPR * CH * kV <= kExactSum<T>;
    __shared__ float2 tmp[2][NT / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const bool in = row < a.rows;  // threads of a row past the last one only keep the barriers
    const T *x = reinterpret_cast<const T *>(a.X) + (in ? row : 0) * a.ldx;
    const float n = (float)a.cols;
    Raw<T> raw[CH];
    float v[CH][kV];
    float s = 0.0f, q = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) raw[k].template load<SHORT>(x, (k * TPR + t) * kV, a.cols);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        raw[k].template place<SHORT>((k * TPR + t) * kV, a.cols, a.cols);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            v[k][i] = raw[k][i];
            s += v[k][i];
        }
    }
    row_sums<TPR, NT>(s, q, tmp, 0);
    float mean = s / n, off;
    s = q = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float d = (k * TPR + t) * kV + i < a.cols ? v[k][i] - mean : 0.0f;
            v[k][i] = d;
            s = fmaf(d, d, s);
            if (!kExact) q += d;
        }
    row_sums<TPR, NT>(s, q, tmp, 1);
    if (!in) return;
    const float rstd = row_stats(s, q, n, a.eps, kExact, mean, off);
    if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = reinterpret_cast<T *>(a.Y) + row * a.ldy;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * TPR + t) * kV;
        if (c >= a.cols) continue;
        float g[kV], b[kV];
        load_param(a.gamma, c, a.cols, 1.0f, g);
        load_param(a.beta, c, a.cols, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kV; ++i) g[i] = fmaf((v[k][i] - off) * rstd, g[i], b[i]);
        store_chunk<T>(y, c, a.cols, g);
    }
}

// Rows longer than the registers hold: the row is read three times.
template <typename T>
__global__ __launch_bounds__(1024) void k_ln_fwd_long(FwdArgs a) {
    constexpr int NT = 1024;
    __shared__ float2 tmp[2][NT / 64];
    const int64_t row = blockIdx.x;
    const T *x = reinterpret_cast<const T *>(a.X) + row * a.ldx;
    T *y = reinterpret_cast<T *>(a.Y) + row * a.ldy;
    const float n = (float)a.cols;
    float s = 0.0f, q = 0.0f, v[kV];
    for (int c = threadIdx.x * kV; c < a.cols; c += NT * kV) {
        load_chunk<T>(x, c, a.cols, v);
#pragma unroll
        for (int i = 0; i < kV; ++i) s += v[i];
    }
    row_sums<NT, NT>(s, q, tmp, 0);
    const float first = s / n;
    float mean = first, off;
    s = q = 0.0f;
    for (int c = threadIdx.x * kV; c < a.cols; c += NT * kV) {
        load_chunk<T>(x, c, a.cols, v);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float d = c + i < a.cols ? v[i] - first : 0.0f;
            s = fmaf(d, d, s);
            q += d;
        }
    }
    row_sums<NT, NT>(s, q, tmp, 1);
    const float rstd = row_stats(s, q, n, a.eps, a.cols <= kExactSum<T>, mean, off);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = threadIdx.x * kV; c < a.cols; c += NT * kV) {
        float g[kV], b[kV];
        load_chunk<T>(x, c, a.cols, v);
        load_param(a.gamma, c, a.cols, 1.0f, g);
        load_param(a.beta, c, a.cols, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kV; ++i) g[i] = fmaf((v[i] - first - off) * rstd, g[i], b[i]);
        store_chunk<T>(y, c, a.cols, g);
    }
}

struct BwdArgs {
    int64_t rows, lddy, ldx, lddr, lddx;
    int cols;
    const void *dY, *X;
    const float *mean, *rstd, *gamma;
    const void *dR;
    void *dX;
    float *part;  // [workgroups][2][cols]: sums of dy xn and of dy, or NULL
};

// Workgroup b takes the rows b * RPB + i, then those gridDim.x * RPB further on, and
// keeps its columns' sums of dy xn and dy in registers.  A CU holds one workgroup, so
// what hides the memory's latency is the next row's x and dy, read while this row is
// worked on: into a second set of registers, the loop unrolled by two, since a copy
// from one set to the other would wait for them.  Bound by memory: 16384 x 4096
// bfloat16 in 104 us with the joining of the sums, 5.2 TB/s over x, dy, dr and dx (209 us
// without the next row, 134 us when copies waited for it).
template <typename T, int TPR, int CH, bool SHORT>
__global__ __launch_bounds__((Rows<TPR, sizeof(T) == 2>::threads), (Rows<TPR, sizeof(T) == 2>::threads > 512 ? 3 : 2)) void k_ln_bwd(BwdArgs a) {
    constexpr int NT = Rows<TPR, sizeof(T) == 2>::threads, RPB = Rows<TPR, sizeof(T) == 2>::per_group;
    constexpr bool kAhead = CH <= 2;  // more would not fit the registers
    __shared__ float2 tmp[2][NT / 64];
    __shared__ float join[RPB > 1 ? RPB * TPR * kV : 1];
    const int t = threadIdx.x % TPR, rg = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const float n = (float)a.cols;
    float gamma[CH][kV], sg[CH][kV], sb[CH][kV];
    auto weigh = [&](int k) { load_param(a.gamma, (k * TPR + t) * kV, a.cols, 1.0f, gamma[k]); };
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        if constexpr (kAhead) weigh(k);
#pragma unroll
        for (int i = 0; i < kV; ++i) sg[k][i] = sb[k][i] = 0.0f;
    }
    struct Row {
        Raw<T> x[CH], y[CH];
        float mean, rstd;
    };
    auto fetch = [&](Row &w, int64_t row) {
        row = min(row, a.rows - 1);
        const T *x = reinterpret_cast<const T *>(a.X) + row * a.ldx;
        const T *dy = reinterpret_cast<const T *>(a.dY) + row * a.lddy;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * TPR + t) * kV;
            w.x[k].template load<SHORT>(x, c, a.cols);
            w.y[k].template load<SHORT>(dy, c, a.cols);
        }
        w.mean = a.mean[row];
        w.rstd = a.rstd[row];
    };
    // Works on the row in w while next is read, after this row's dR.
    auto work = [&](Row &w, int64_t row, Row &next, int64_t next_row, int turn) {
        Raw<T> r[CH];
        if (a.dR) {
            const T *dr = reinterpret_cast<const T *>(a.dR) + min(row, a.rows - 1) * a.lddr;
#pragma unroll
            for (int k = 0; k < CH; ++k) r[k].template load<SHORT>(dr, (k * TPR + t) * kV, a.cols);
        }
        if constexpr (kAhead) fetch(next, next_row);
        const int end = row < a.rows ? a.cols : 0;  // 0: a row past the last one
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * TPR + t) * kV;
            w.x[k].template place<SHORT>(c, a.cols, end);
            w.y[k].template place<SHORT>(c, a.cols, end);
            if constexpr (!kAhead) weigh(k);
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const float dy = w.y[k][i], d = dy * gamma[k][i];
                const float xn = c + i < end ? (w.x[k][i] - w.mean) * w.rstd : 0.0f;
                sg[k][i] = fmaf(dy, xn, sg[k][i]);
                sb[k][i] += dy;
                s1 += d;
                s2 = fmaf(d, xn, s2);
            }
        }
        if (!a.dX) return;  // the same for every thread
        row_sums<TPR, NT>(s1, s2, tmp, turn);
        s1 /= n;
        s2 /= n;
        T *dx = reinterpret_cast<T *>(a.dX) + row * a.lddx;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * TPR + t) * kV;
            if (c >= end) continue;
            w.x[k].renew();
            w.y[k].renew();
            if constexpr (!kAhead) weigh(k);
            float o[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const float xn = (w.x[k][i] - w.mean) * w.rstd;
                o[i] = w.rstd * (w.y[k][i] * gamma[k][i] - s1 - xn * s2);
            }
            if (a.dR) {
                r[k].template place<SHORT>(c, a.cols, a.cols);
#pragma unroll
                for (int i = 0; i < kV; ++i) o[i] += r[k][i];
            }
            store_chunk<T>(dx, c, a.cols, o);
        }
    };
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + rg;
    Row one, two;
    if constexpr (!kAhead) {
        int turn = 0;
        for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += step, row += step, turn ^= 1) {
            fetch(one, row);
            work(one, row, two, 0, turn);
        }
    } else {
        fetch(one, row);
        for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += 2 * step, row += 2 * step) {
            work(one, row, two, row + step, 0);
            if (base + step >= a.rows) break;
            work(two, row + step, one, row + 2 * step, 1);
        }
    }
    if (!a.part) return;
    float *pg = a.part + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            float v[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) v[i] = half ? sb[k][i] : sg[k][i];
            if constexpr (RPB > 1) {  // the row groups of the workgroup, in their order
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kV; ++i) join[(rg * kV + i) * TPR + t] = v[i];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    v[i] = 0.0f;
                    for (int w = 0; w < RPB; ++w) v[i] += join[(w * kV + i) * TPR + t];
                }
            }
            const int c = (k * TPR + t) * kV;
            if (rg == 0 && c < a.cols) store_chunk<float>(pg + half * a.cols, c, a.cols, v);
        }
}

// Rows longer than the registers hold: dX in three reads of the row.
template <typename T>
__global__ __launch_bounds__(1024) void k_ln_bwd_long(BwdArgs a) {
    constexpr int NT = 1024;
    __shared__ float2 tmp[2][NT / 64];
    const float n = (float)a.cols;
    const int64_t row = blockIdx.x;
    const T *x = reinterpret_cast<const T *>(a.X) + row * a.ldx;
    const T *dy = reinterpret_cast<const T *>(a.dY) + row * a.lddy;
    const T *dr = a.dR ? reinterpret_cast<const T *>(a.dR) + row * a.lddr : nullptr;
    T *dx = reinterpret_cast<T *>(a.dX) + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f, v[kV], d[kV], g[kV], r[kV];
    for (int c = threadIdx.x * kV; c < a.cols; c += NT * kV) {
        load_chunk<T>(x, c, a.cols, v);
        load_chunk<T>(dy, c, a.cols, d);
        load_param(a.gamma, c, a.cols, 1.0f, g);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float xn = c + i < a.cols ? (v[i] - mean) * rstd : 0.0f;
            s1 += d[i] * g[i];
            s2 = fmaf(d[i] * g[i], xn, s2);
        }
    }
    row_sums<NT, NT>(s1, s2, tmp, 0);
    s1 /= n;
    s2 /= n;
    for (int c = threadIdx.x * kV; c < a.cols; c += NT * kV) {
        load_chunk<T>(x, c, a.cols, v);
        load_chunk<T>(dy, c, a.cols, d);
        load_param(a.gamma, c, a.cols, 1.0f, g);
#pragma unroll
        for (int i = 0; i < kV; ++i) r[i] = 0.0f;
        if (dr) load_chunk<T>(dr, c, a.cols, r);
#pragma unroll
        for (int i = 0; i < kV; ++i) r[i] += rstd * (d[i] * g[i] - s1 - (v[i] - mean) * rstd * s2);
        store_chunk<T>(dx, c, a.cols, r);
    }
}

// Their column sums: workgroup (x, y) takes 64 columns and every gridDim.y-th row.
template <typename T>
__global__ __launch_bounds__(64) void k_ln_params_long(BwdArgs a) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= a.cols) return;
    float g = 0.0f, b = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float x = (float)reinterpret_cast<const T *>(a.X)[row * a.ldx + c];
        const float dy = (float)reinterpret_cast<const T *>(a.dY)[row * a.lddy + c];
        g = fmaf(dy, (x - a.mean[row]) * a.rstd[row], g);
        b += dy;
    }
    float *p = a.part + (int64_t)blockIdx.y * 2 * a.cols;
    p[c] = g;
    p[a.cols + c] = b;
}

constexpr int kMaxRegCols = 512 * 4 * kV;  // the longest row held in registers

// Calls f<TPR, CH, SHORT>() for the narrowest shape that holds a row.
template <typename F>
void by_width(int64_t cols, F &&f) {
    const int64_t v = (cols + kV - 1) / kV;
    if (cols < kV) f.template operator()<64, 1, true>();
    else if (v <= 64) f.template operator()<64, 1, false>();
    else if (v <= 128) f.template operator()<128, 1, false>();
    else if (v <= 256) f.template operator()<128, 2, false>();
    else if (v <= 384) f.template operator()<192, 2, false>();
    else if (v <= 512) f.template operator()<256, 2, false>();
    else if (v <= 768) f.template operator()<384, 2, false>();
    else if (v <= 1024) f.template operator()<512, 2, false>();
    else f.template operator()<512, 4, false>();
}

// HIP counts a launch's threads along x in 32 bits: calls f(at, n) for rows [at, at + n)
// of at most kLaunchThreads / (threads a row) rows, a launch each.  2^28 threads keep the
// GPU busy for 100 us and more, so that the launches follow each other without a gap.
constexpr int64_t kLaunchThreads = int64_t(1) << 28;
template <typename F>
int by_rows(const char *who, int64_t rows, int threads, F &&f) {
    const int64_t most = kLaunchThreads / threads;
    for (int64_t at = 0; at < rows; at += most) {
        f(at, std::min(most, rows - at));
        if (int rc = check_hip(hipGetLastError(), who)) return rc;
    }
    return SA_OK;
}

// The n rows of a call from row `at` on.
template <typename T, typename P>
void skip_rows(P *&p, int64_t at, int64_t ld) {
    using E = std::conditional_t<std::is_const_v<P>, const T, T>;
    if (p) p = static_cast<E *>(p) + at * ld;
}
template <typename T>
FwdArgs rows_from(FwdArgs a, int64_t at, int64_t n) {
    a.rows = n;
    skip_rows<T>(a.X, at, a.ldx);
    skip_rows<T>(a.Y, at, a.ldy);
    skip_rows<float>(a.mean, at, 1);
    skip_rows<float>(a.rstd, at, 1);
    return a;
}
template <typename T>
BwdArgs rows_from(BwdArgs a, int64_t at, int64_t n) {
    a.rows = n;
    skip_rows<T>(a.dY, at, a.lddy);
    skip_rows<T>(a.X, at, a.ldx);
    skip_rows<T>(a.dR, at, a.lddr);
    skip_rows<T>(a.dX, at, a.lddx);
    skip_rows<float>(a.mean, at, 1);
    skip_rows<float>(a.rstd, at, 1);
    return a;
}

template <typename T>
struct LaunchFwd {
    const FwdArgs &a;
    hipStream_t stream;
    int rc;
    template <int TPR, int CH, bool SHORT>
    void operator()() {
        rc = by_rows("k_ln_fwd", a.rows, TPR, [&](int64_t at, int64_t n) {
            constexpr int RPB = Rows<TPR>::per_group;
            hipLaunchKernelGGL((k_ln_fwd<T, TPR, CH, SHORT>), dim3((unsigned)((n + RPB - 1) / RPB)), dim3(Rows<TPR>::threads), 0,
                               stream, rows_from<T>(a, at, n));
        });
    }
};

template <typename T>
struct LaunchBwd {
    const BwdArgs &a;
    int groups;
    hipStream_t stream;
    template <int TPR, int CH, bool SHORT>
    void operator()() {
        hipLaunchKernelGGL((k_ln_bwd<T, TPR, CH, SHORT>), dim3(groups), dim3(Rows<TPR, sizeof(T) == 2>::threads), 0, stream, a);
    }
};

// Rows that one workgroup of the backward kernel holds at a time.
struct RowsAtATime {
    bool wide;
    int rows;
    template <int TPR, int CH, bool SHORT>
    void operator()() {
        rows = wide ? Rows<TPR, true>::per_group : Rows<TPR>::per_group;
    }
};

// Workgroups of the backward pass (0: no rows): as many as the CUs hold at a time, so
// that each runs once.  Rows of up to 1024 columns take half the registers: there two
// fit a CU (65536 x 1024 bfloat16 114 us with 256 workgroups, 89 with 512); longer ones
// lose by it (32768 x 2048 86 and 92 us).
int bwd_groups(int64_t rows, int64_t cols, int type) {
    RowsAtATime r{type != SA_F32, 1};
    if (cols <= kMaxRegCols) by_width(cols, r);
    return (int)std::min<int64_t>((rows + r.rows - 1) / r.rows, cols <= 1024 ? 512 : 256);
}

template <typename T>
int fwd(const FwdArgs &a, hipStream_t stream) {
    if (a.cols <= kMaxRegCols) {
        LaunchFwd<T> launch{a, stream, SA_OK};
        by_width(a.cols, launch);
        return launch.rc;
    }
    return by_rows("k_ln_fwd_long", a.rows, 1024, [&](int64_t at, int64_t n) {
        hipLaunchKernelGGL(k_ln_fwd_long<T>, dim3((unsigned)n), dim3(1024), 0, stream, rows_from<T>(a, at, n));
    });
}

template <typename T>
int bwd(const BwdArgs &a, int groups, hipStream_t stream) {
    if (a.cols <= kMaxRegCols) {
        by_width(a.cols, LaunchBwd<T>{a, groups, stream});
        return check_hip(hipGetLastError(), "k_ln_bwd");
    }
    if (a.part) {  // first: dX may overwrite dY
        hipLaunchKernelGGL(k_ln_params_long<T>, dim3((a.cols + 63) / 64, groups), dim3(64), 0, stream, a);
        if (int rc = check_hip(hipGetLastError(), "k_ln_params_long")) return rc;
    }
    if (!a.dX) return SA_OK;
    return by_rows("k_ln_bwd_long", a.rows, 1024, [&](int64_t at, int64_t n) {
        hipLaunchKernelGGL(k_ln_bwd_long<T>, dim3((unsigned)n), dim3(1024), 0, stream, rows_from<T>(a, at, n));
    });
}

}  // namespace
}  // namespace sa

using namespace sa;

extern "C" int structadmm_layer_norm_fwd(const sa_layer_norm_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "layer_norm_fwd: desc is required");
    const sa_layer_norm_desc &d = *desc;
    if (int rc = validate_layer_norm(d)) return rc;
    if (d.rows == 0) return SA_OK;
    const FwdArgs a{d.rows, d.ldx, d.ldy, (int)d.cols, d.eps, d.X, d.gamma, d.beta, d.Y, d.mean, d.rstd};
    if (d.type == SA_BF16) return fwd<__bf16>(a, stream);
    if (d.type == SA_F16) return fwd<_Float16>(a, stream);
    return fwd<float>(a, stream);
}

static size_t ln_bwd_bytes(const sa_layer_norm_bwd_desc &d) {
    return d.dgamma || d.dbeta ? (size_t)bwd_groups(d.rows, d.cols, d.type) * 2 * d.cols * sizeof(float) : 0;
}

extern "C" size_t structadmm_layer_norm_bwd_workspace(const sa_layer_norm_bwd_desc *desc) {
    if (!desc || validate_layer_norm_bwd_sizes(*desc) != SA_OK) return 0;
    sa_layer_norm_bwd_desc d = *desc;
    float any;
    if (!d.dY && d.rows > 0) d.dgamma = &any;  // before the buffers: as for every output
    return ln_bwd_bytes(d);
}

extern "C" int structadmm_layer_norm_bwd(const sa_layer_norm_bwd_desc *desc, hipStream_t stream) {
    clear_error();
    if (!desc) return fail(SA_E_ARG, "layer_norm_bwd: desc is required");
    const sa_layer_norm_bwd_desc &d = *desc;
    if (int rc = validate_layer_norm_bwd(d)) return rc;
    const size_t need = ln_bwd_bytes(d);
    if (int rc = check_workspace("layer_norm_bwd", d.ws, d.ws_bytes, need)) return rc;
    const int groups = bwd_groups(d.rows, d.cols, d.type);
    BwdArgs a{d.rows, d.lddy, d.ldx, d.lddr, d.lddx, (int)d.cols, d.dY, d.X, d.mean, d.rstd, d.gamma, d.dR, d.dX,
              d.dgamma || d.dbeta ? static_cast<float *>(d.ws) : nullptr};
    if (groups > 0) {
        int rc;
        if (d.type == SA_BF16) rc = bwd<__bf16>(a, groups, stream);
        else if (d.type == SA_F16) rc = bwd<_Float16>(a, groups, stream);
        else rc = bwd<float>(a, groups, stream);
        if (rc) return rc;
    }
    if (d.dgamma || d.dbeta)
        return join_columns(static_cast<const float *>(d.ws), groups, (int)d.cols, d.dgamma, d.dbeta, stream);
    return SA_OK;
}
