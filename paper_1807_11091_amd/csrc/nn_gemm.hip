// Matrix products of the feed-forward operators on the gfx950 matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <map>
#include <mutex>
#include <type_traits>
#include <utility>

#include "nn_gemm.h"
#include "nn_types.h"
#include "sa_conv_device.h"
#include "sa_host.h"

namespace sa {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ inline f32x4 mfma(Vec8<__bf16>::type a, Vec8<__bf16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(Vec8<_Float16>::type a, Vec8<_Float16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ inline f32x16 mfma(Vec8<__bf16>::type a, Vec8<__bf16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma(Vec8<_Float16>::type a, Vec8<_Float16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// What the outputs' sums are joined with, loaded ahead of them.
template <typename T, int V>
struct Addends {
    typedef T vec __attribute__((ext_vector_type(V)));
    float bias[V], bias2[V];  // if the epilogue has them
    vec r;                    // if has_r (whole vectors of the operands' type only)
    bool has_r;

    __device__ void load_bias(const Epilogue &e, int64_t n, int cnt) {
        if (e.bias) {
            if (cnt == V) load_vec<float, V>(e.bias + n, bias);
            else load_part<float, V>(e.bias + n, cnt, bias);
        }
        if (e.bias2) {
            if (cnt == V) load_vec<float, V>(e.bias2 + n, bias2);
            else load_part<float, V>(e.bias2 + n, cnt, bias2);
        }
    }
};

// V (cnt < V at a row's end) consecutive outputs from their sums z (and u).
template <typename T, bool GATED, int V>
__device__ inline void finish(const Epilogue &e, void *Y, int64_t m, int64_t n, int cnt, float (&z)[V], float (&u)[V],
                              const Addends<T, V> &with) {
    auto put = [&](auto *p, const float (&v)[V]) {
        using E = typename std::remove_reference<decltype(*p)>::type;
        if (cnt == V) store_vec<E, V>(p, v);
        else store_part<E, V>(p, cnt, v);
    };
    auto add = [&](const auto *p) {
        using E = typename std::remove_cv<typename std::remove_reference<decltype(*p)>::type>::type;
        float t[V];
        if (cnt == V) load_vec<E, V>(p, t);
        else load_part<E, V>(p, cnt, t);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] += t[i];
    };
    if (e.bias)
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] += with.bias[i];
    if (e.Z) put(reinterpret_cast<T *>(e.Z) + m * e.ldz + n, z);
    if (e.act != SA_ACT_NONE) activate<false, V>(e.act, z, z, z);
    if constexpr (GATED) {
        if (e.bias2)
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] += with.bias2[i];
        if (e.Z2) put(reinterpret_cast<T *>(e.Z2) + m * e.ldz + n, u);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] *= u[i];
    }
    if (with.has_r)
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] += (float)with.r[i];
    else if (e.R) {
        if (e.out_f32) add(reinterpret_cast<const float *>(e.R) + m * e.ldr + n);
        else add(reinterpret_cast<const T *>(e.R) + m * e.ldr + n);
    }
    if (e.out_f32) put(reinterpret_cast<float *>(Y) + m * e.ldy + n, z);
    else put(reinterpret_cast<T *>(Y) + m * e.ldy + n, z);
}

template <typename T, bool GATED, int V>
__device__ inline void finish(const Epilogue &e, void *Y, int64_t m, int64_t n, int cnt, float (&z)[V], float (&u)[V]) {
    Addends<T, V> with;
    with.has_r = false;
    with.load_bias(e, n, cnt);
    finish<T, GATED, V>(e, Y, m, n, cnt, z, u, with);
}

// Where binary32 partial sums of a product go when k is split over workgroups:
// [split][batch][gated ? 2 : 1][M][pitch].
struct Partial {
    float *p;
    int64_t pitch;  // N rounded up to 8
    int split;      // 1: none
};

__device__ inline float *partial_at(const Partial &q, const Gemm &g, int chunk, int z, int half, int64_t m, int64_t n) {
    const int64_t plane = ((int64_t)chunk * g.batch + z) * (g.gated ? 2 : 1) + half;
    return q.p + (plane * g.M + m) * q.pitch + n;
}

// Adds the chunks in their order and finishes 8 outputs per thread.
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void k_join(Gemm g, Partial q) {
    const int64_t chunks = q.pitch / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= g.M * chunks) return;
    // the long division only where the short one does not do
    const int64_t m = i >> 32 ? i / chunks : (uint32_t)i / (uint32_t)chunks, n = (i - m * chunks) * 8;
    const int z = blockIdx.y;
    float s[8] = {}, u[8] = {}, t[8];
    for (int c = 0; c < q.split; ++c) {
        load_vec<float, 8>(partial_at(q, g, c, z, 0, m, n), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += t[e];
        if constexpr (GATED) {
            load_vec<float, 8>(partial_at(q, g, c, z, 1, m, n), t);
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] += t[e];
        }
    }
    finish<T, GATED, 8>(g.e, z ? g.y1 : g.e.Y, m, n, (int)min((int64_t)8, g.N - n), s, u);
}

// ------------------------------------------------------------- few rows of M
// k_rows: products with few rows of M (single tokens, small batches), bound by
// reading the N side's matrices once and by latency.  A workgroup of 8 wavefronts
// takes NF * 16 of their rows and MF * 16 of M; its wavefronts take k in turn, in
// blocks of U * 32, and feed the MFMAs straight from memory (the weights are used
// once or a few times: LDS would only add a copy, and barriers).  Their sums are
// joined through LDS in a fixed order.  Rows past M or N read the last row and are
// not stored.  1 x 4096 x 9830 bfloat16 takes 15.6 us (5.2 TB/s of weights), gated
// 16 x 9830 x 4096 37.4 us (4.3 TB/s; 68 us in tiles).
template <typename T, bool GATED, int NF, int MF, int U>
__global__ __launch_bounds__(512) void k_rows(Gemm g, Partial q) {
    typedef typename Vec8<T>::type vec;
    constexpr int NW = 8, H = GATED ? 2 : 1, STEP = 32 * U;
    __shared__ float sums[NW][NF * H * MF][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, kg = (lane >> 4) * 8;
    const int64_t n0 = (int64_t)blockIdx.x * NF * 16, m0 = (int64_t)blockIdx.z * MF * 16;
    const int K = (int)g.K;
    // chunk of k of this workgroup, in whole blocks of all its wavefronts
    const int blocks = (K + STEP - 1) / STEP;
    const int b0 = (int)((int64_t)blocks * blockIdx.y / q.split), b1 = (int)((int64_t)blocks * (blockIdx.y + 1) / q.split);

    const T *wp[H * NF], *xp[MF];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int f = 0; f < NF; ++f)
            wp[h * NF + f] = reinterpret_cast<const T *>(g.n[h].p) + min(n0 + f * 16 + r, g.N - 1) * g.n[h].ld + kg;
#pragma unroll
    for (int j = 0; j < MF; ++j) xp[j] = reinterpret_cast<const T *>(g.m[0].p) + min(m0 + j * 16 + r, g.M - 1) * g.m[0].ld + kg;

    f32x4 acc[H * NF][MF] = {};
    for (int b = b0 + wave; b < b1; b += NW) {
        const int k = b * STEP;
        if (k + STEP <= K) {
            vec w[U][H * NF], x[U][MF];
#pragma unroll
            for (int s = 0; s < U; ++s) {
#pragma unroll
                for (int f = 0; f < H * NF; ++f) __builtin_memcpy(&w[s][f], wp[f] + k + s * 32, 16);
#pragma unroll
                for (int j = 0; j < MF; ++j) __builtin_memcpy(&x[s][j], xp[j] + k + s * 32, 16);
            }
            __builtin_amdgcn_sched_barrier(0);  // every load of the block goes out before the first product
#pragma unroll
            for (int s = 0; s < U; ++s)
#pragma unroll
                for (int f = 0; f < H * NF; ++f)
#pragma unroll
                    for (int j = 0; j < MF; ++j) acc[f][j] = mfma(w[s][f], x[s][j], acc[f][j]);
        } else {  // the last block: zeros past K
            auto part = [&](const T *p, int at) {
                vec v = {};
                const int n = K - at - kg;
                if (n >= 8) __builtin_memcpy(&v, p + at, 16);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < n) v[e] = p[at + e];
                return v;
            };
#pragma unroll 1
            for (int at = k; at < K; at += 32) {
                vec x[MF];
#pragma unroll
                for (int j = 0; j < MF; ++j) x[j] = part(xp[j], at);
#pragma unroll
                for (int f = 0; f < H * NF; ++f) {
                    const vec w = part(wp[f], at);
#pragma unroll
                    for (int j = 0; j < MF; ++j) acc[f][j] = mfma(w, x[j], acc[f][j]);
                }
            }
        }
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
        if (q.split > 1) {
            *partial_at(q, g, blockIdx.y, 0, 0, m, n) = z[0];
            if constexpr (GATED) *partial_at(q, g, blockIdx.y, 0, 1, m, n) = u[0];
        } else {
            finish<T, GATED, 1>(g.e, g.e.Y, m, n, 1, z, u);
        }
    }
}

// ------------------------------------------------------------ tiled product
// k_gemm: BN x BM outputs (N side by M side) per workgroup of WN x WM wavefronts.
// Operands travel in stages of BK k through a ring of S LDS buffers, written by
// buffer_load ... lds (16 bytes per lane, S - 1 stages ahead).  The N side is the
// row operand of the MFMAs, so a lane's four sums are consecutive in n.
//
// LDS layouts (64 banks of 4 bytes, 256 bytes per clock):
//   - an operand whose rows run along k: [row][BK], the 16-byte chunks of a row
//     XOR-swizzled so that the rows of a fragment read hit distinct banks;
//   - an operand whose rows run across k: [k][rows], read by ds_read_b64_tr_b16,
//     which hands each lane 4 consecutive k of its row (16 lanes transpose a block
//     of 4 k by 16 rows); its units of 2 MI bytes are XOR-swizzled by k, so that 32
//     lanes hit distinct banks (8 k of 16 rows, or 4 k of 32).
// The swizzle is applied to the source address (the DMA writes lanes in order).
//
// The products of a large one are bound by power, not by issue: at full load the clock
// falls to 1.7 .. 2.0 GHz, and fewer cycles lower it further.  8192 x 4096 x 4096 takes
// 205 us (1.34 PFLOP/s) in 256 x 256 tiles with 16x16x32 MFMAs and 217 .. 230 us with
// 32x32x16 ones, which need fewer cycles and more power; a 128 x 128 tile, bound by the
// latency of its stages, takes 32 us for 64 of them with the latter and 45 with the
// former.  A third stage in flight gained nothing in the largest tile (its loads land in
// time) and nothing further in the smallest.

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxLds = 160 * 1024;

__device__ inline int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a raw buffer of `bytes` at base, both wavefront-uniform
__device__ inline i32x4 buffer_at(uint64_t base, uint32_t bytes) {
    return i32x4{uni((int)(uint32_t)base), uni((int)((uint32_t)(base >> 32) & 0xffffu)), uni((int)bytes), kRsrcWord3};
}

// 16 bytes per lane straight from memory to LDS: lane i's land at lds + AT + 16 * i.
// Inline asm: after the compiler's own LDS-DMA builtin every LDS read waits for
// all loads in flight.  The statement has no outputs; the waits are wait_vm().
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int AT>
__device__ inline void dma16(i32x4 r, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voff),
                 "s"(r), "s"(soff), "n"(AT)
                 : "memory", "scc", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ inline void wait_vm() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// this wavefront's LDS accesses done, then the workgroup's barrier
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One operand's part of a stage: B rows by BK k, NW wavefronts.
template <typename T, bool ACROSS, int B, int BK, int NW, int MI>
struct Side {
    typedef typename Vec8<T>::type vec;
    static constexpr int bytes = B * BK * 2;
    static constexpr int loads = bytes / 1024 / NW;  // per wavefront
    static constexpr int pitch = ACROSS ? B * 2 : BK * 2;
    static constexpr int cpr = pitch / 16;           // 16-byte chunks of an LDS row
    static_assert(bytes % (1024 * NW) == 0, "whole loads per wavefront");

    // swizzle of row r (rows along k) or of k (rows across)
    __device__ static int swz(int r) {
        if constexpr (ACROSS) return (MI == 16 ? (r & 3) | ((r >> 3) & 1) << 2 : r & 3) & (B / MI - 1);
        else if constexpr (BK == 64) return (r >> 1) & 7;
        else return (((r >> 2) ^ (r >> 3)) & 1) << 1 | ((r >> 3) & 1);
    }
    // LDS row and source chunk of this lane's part of load i.  Where rows run along
    // k the loads lie a multiple of the swizzle's period apart: one chunk for all.
    static_assert(ACROSS || NW * 64 / cpr % 16 == 0 || loads == 1, "one chunk per lane");
    __device__ static void place(int i, int wave, int lane, int &row, int &chunk) {
        const int at = (i * NW + wave) * 64 + lane;
        row = at / cpr;
        const int c = at % cpr;
        chunk = ACROSS ? c ^ swz(row) * (MI / 8) : c ^ swz(row);
    }

    uint32_t off[loads];  // byte offset of each load from the tile's origin
    int kc;               // first k of this lane's chunks (rows along k)

    __device__ void setup(int64_t ld, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < loads; ++i) {
            int row, chunk;
            place(i, wave, lane, row, chunk);
            off[i] = (uint32_t)row * (uint32_t)ld * 2u + chunk * 16u;
            if (i == 0) kc = chunk * 8;
        }
    }

    // Where the next stage's loads read: BK k of the rows at the buffer's base.  Rows
    // past the matrix and k past K read as 0; a chunk that K cuts is completed by
    // mend().  The buffer's range is rounded up to whole chunks: the bytes past the
    // matrix's end lie in the aligned 16 bytes that hold its last element, and never
    // reach a result.
    struct Cursor {
        i32x4 rs;
        uint32_t so;
    };
    // at k0 of the rows at p (the tile's first row; `rows` of them in the matrix)
    __device__ static Cursor open(const T *p, int64_t ld, int rows, int K, int k0) {
        Cursor c;
        const int r = min(rows, B);
        if constexpr (ACROSS) {
            const int n = min(K - k0, BK);
            const uint32_t range = (((uint32_t)(n - 1) * (uint32_t)ld + r) * 2u + 15u) & ~15u;
            c.rs = buffer_at(reinterpret_cast<uint64_t>(p) + (uint64_t)k0 * (uint64_t)ld * 2u, range);
            c.so = 0;
        } else {
            const uint32_t range = (((uint32_t)(r - 1) * (uint32_t)ld + (uint32_t)K) * 2u + 15u) & ~15u;
            c.rs = buffer_at(reinterpret_cast<uint64_t>(p), range);
            c.so = uni(k0 * 2);
        }
        return c;
    }
    // to the stage that follows; step = BK * ld * 2 (ACROSS)
    __device__ static void advance(Cursor &c, uint32_t step) {
        if constexpr (ACROSS) {
            const uint64_t base = ((uint64_t)(uint32_t)c.rs[1] << 32 | (uint32_t)c.rs[0]) + step;
            c.rs[0] = uni((int)(uint32_t)base);
            c.rs[1] = uni((int)(uint32_t)(base >> 32));
        } else {
            c.so = uni(c.so + BK * 2);
        }
    }
    // Lanes whose chunk begins at `k` or past it read zeros from here on (rows along k;
    // offsets are below 2^31, one with the top bit set lies past every range).
    __device__ void limit(int k) {
        if constexpr (!ACROSS)
#pragma unroll
            for (int i = 0; i < loads; ++i) off[i] = kc < k ? off[i] & ~kInvalidOffset : off[i] | kInvalidOffset;
    }
    // load I of a stage
    template <int I>
    __device__ void load(const Cursor &c, uint32_t lds) const {
        dma16<I * NW * 1024>(c.rs, off[I], c.so, lds);
    }

    // The chunk that holds k = K - 1, in LDS: its elements past K become +0 (after this
    // wavefront's loads have landed); n: k of K's last stage.
    __device__ void mend(uint8_t *lds, int n, int wave, int lane) const {
        if constexpr (!ACROSS) {
            if (kc != (n & ~7)) return;
#pragma unroll
            for (int i = 0; i < loads; ++i) {
                vec *q = reinterpret_cast<vec *>(lds + (i * NW + wave) * 1024 + lane * 16);
                vec v = *q;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= (n & 7)) v[e] = (T)0.0f;
                *q = v;
            }
        }
    }

    // Lane offsets of fragment reads: fragment f holds rows MI f + (0 .. MI - 1), step q
    // KQ k, 8 of them in each lane.
    static constexpr int KQ = 512 / MI;
    static constexpr int nfo = ACROSS ? 1 : BK / KQ;
    uint32_t fo[nfo];

    __device__ void setup_reads(int lane) {
        const int g = lane / MI;  // the lane's 8 k
        if constexpr (ACROSS) {
            const int k = g * 8 + ((lane & 15) >> 2);
            fo[0] = k * pitch + swz(k) * (MI * 2) + (lane & (MI - 16)) * 2 + (lane & 3) * 8;
        } else {
            const int r = lane & (MI - 1);
#pragma unroll
            for (int q = 0; q < nfo; ++q) fo[q] = r * pitch + (((q * (KQ / 8) + g) ^ swz(r)) << 4);
        }
    }

    // fragment f (rows from row0, a multiple of MI) of step q
    __device__ vec read(const uint8_t *lds, int row0, int f, int q) const {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) s16x4 *ptr;
            const uint8_t *p = lds + (fo[0] ^ (uint32_t)((row0 + MI * f) * 2)) + q * KQ * pitch;
            union {
                s16x4 h[2];
                vec v;
            } x;
            x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p));
            x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p + 4 * pitch));
            return x.v;
        } else {
            return *reinterpret_cast<const vec *>(lds + fo[q] + (row0 + MI * f) * pitch);
        }
    }
};

template <int BN, int BM, int WN, int WM, int BK, int S, int MI>
struct TileCfg {
    static constexpr int NW = WN * WM, NT = NW * 64;
    static constexpr int TN = BN / WN / MI, TM = BM / WM / MI;  // fragments of a wavefront
    static constexpr int stage = (BN + BM) * BK * 2;
    static constexpr int lds = S * stage;
    static_assert(lds <= kMaxLds, "LDS");
};

// f(j) with j, below N, as a constant: registers cannot be indexed
template <int N, typename F>
__device__ inline void pick(int j, F &&f) {
    if constexpr (N > 0) {
        if (j == N - 1) f(std::integral_constant<int, N - 1>{});
        else pick<N - 1>(j, f);
    }
}

// f(0), .. f(N - 1) with constants
template <int N, int I = 0, typename F>
__device__ inline void each(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

struct TileArgs {
    Gemm g;
    Partial part;
    int mtiles, ntiles, tiles, groups;  // tiles: of all batches and chunks; groups: workgroups
};

// Workgroup `block` of a.groups.
template <typename T, bool NA, bool MA, bool GATED, int BN, int BM, int WN, int WM, int BK, int S, int MI>
__device__ __forceinline__ void tile_product(const TileArgs &a, int block) {
    using Cfg = TileCfg<BN, BM, WN, WM, BK, S, MI>;
    constexpr int NROWS = GATED ? BN / 2 : BN;  // n of a tile; gated: one half of the N side per projection
    using NSide = Side<T, NA, NROWS, BK, Cfg::NW, MI>;
    using MSide = Side<T, MA, BM, BK, Cfg::NW, MI>;
    typedef typename Vec8<T>::type vec;
    constexpr int TN = Cfg::TN, TM = Cfg::TM, KS = BK / NSide::KQ, TNG = GATED ? TN / 2 : TN;
    constexpr int NL = NSide::loads * (GATED ? 2 : 1), L = NL + MSide::loads;  // loads of a stage
    constexpr int RATE = (L + 2 * TN - 1) / (2 * TN);                  // loads that go out with a fragment row
    constexpr int L0 = TN * RATE < L ? TN * RATE : L;                  // loads of a stage in the step that begins it
    static_assert(BK == 64 && TNG > 0 && L * (S - 1) < 64, "shape");
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];

    const Gemm &g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int wn = wave % WN, wm = wave / WN;

    // Workgroup b runs on XCD b mod 8, which walks one contiguous range of tiles
    // (its own L2); its workgroups take the range's tiles in turn.
    const int xcd = block & 7, local = block >> 3;
    const int per = a.tiles >> 3, extra = a.tiles & 7;
    const int first = uni(xcd * per + min(xcd, extra) + local);
    const int end = uni((xcd + 1) * per + min(xcd + 1, extra));
    const int stride = uni((a.groups >> 3) + (xcd < (a.groups & 7) ? 1 : 0));
    if (first >= end) return;
    const int mine = (end - first + stride - 1) / stride;  // tiles of this workgroup

    const int K = uni((int)g.K);  // a sum over rows may have 2^31 - 1 terms: nothing is added to K
    const int sp = K / BK + (K % BK != 0), ns = NA && !MA ? sp * uni(g.parts) : sp;  // stages of a part, of a tile
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
    const int64_t nld = g.n[0].ld, mld = g.m[0].ld;  // parts and batches share their pitch

    // A tile: bands of 8 M tiles, down each band first, so that neighbours share operands
    struct Tile {
        int64_t m0, n0;
        int z, chunk;
        int s0, s1;  // its stages
    };
    auto tile_at = [&](int i) {
        int t = first + i * stride;
        const int one = a.mtiles * a.ntiles;
        Tile q;
        q.chunk = t / (one * g.batch);
        t -= q.chunk * one * g.batch;
        q.z = t / one;
        t -= q.z * one;
        q.s0 = uni(ns * q.chunk / a.part.split);
        q.s1 = uni(ns * (q.chunk + 1) / a.part.split);
        const int band = t / (8 * a.ntiles), in = t - band * 8 * a.ntiles;
        const int h = min(8, a.mtiles - band * 8);
        q.m0 = (int64_t)(band * 8 + in % h) * BM;
        q.n0 = (int64_t)(in / h) * NROWS;
        return q;
    };

    NSide nside;
    MSide mside;
    nside.setup(nld, wave, lane);
    mside.setup(mld, wave, lane);
    nside.setup_reads(lane);
    mside.setup_reads(lane);

    // The loads run over the stages of all tiles without a break, S stages ahead of
    // the products: the next tile's first stages arrive while this one's results go
    // out.  A run of stages below K differs from stage to stage by one addition per
    // operand; what else there is to work out (60 and more scalar instructions, which
    // a wavefront's products do not hide) is done between runs.
    constexpr bool TWO = NA && !MA;  // the sum may have two parts (MA: there may be two batches)
    typename NSide::Cursor nc, nc1;
    typename MSide::Cursor mc;
    uint32_t lat = lds0 + wave * 1024, nstep = uni((int)(BK * nld * 2)), mstep = uni((int)(BK * mld * 2));
    int run = 0, lstage = 0, lend = 0, ltile = -1, lslot = 0;
    int cuts = 0;  // slots that hold, or will, a chunk which K cuts
    auto next_run = [&]() {
        if (lstage == lend) ++ltile;
        if (ltile >= mine) {  // past the last stage: the loads write zeros that are not used
            nc.rs[2] = nc1.rs[2] = mc.rs[2] = 0;
            nc.so = nc1.so = mc.so = 0;
            run = 1;
            return;
        }
        const Tile q = tile_at(ltile);
        if (lstage == lend) {
            lstage = q.s0;
            lend = q.s1;
        }
        const int64_t no = NA ? q.n0 : q.n0 * nld, mo = MA ? q.m0 : q.m0 * mld;
        const int nrows = uni((int)min(g.N - q.n0, (int64_t)NROWS)), mrows = uni((int)min(g.M - q.m0, (int64_t)BM));
        const bool second = TWO && lstage >= sp;
        const int st = second ? lstage - sp : lstage, k0 = st * BK;
        nc = NSide::open(reinterpret_cast<const T *>(second ? g.n[1].p : g.n[0].p) + no, nld, nrows, K, k0);
        if constexpr (GATED) nc1 = NSide::open(reinterpret_cast<const T *>(g.n[1].p) + no, nld, nrows, K, k0);
        mc = MSide::open(reinterpret_cast<const T *>(second || (MA && q.z) ? g.m[1].p : g.m[0].p) + mo, mld, mrows, K, k0);
        nside.limit(K - k0);
        mside.limit(K - k0);
        if (BK > K - k0 && (K & 7) != 0) cuts |= 1 << lslot;
        run = uni(BK <= K - k0 ? min(K / BK - st, lend - lstage) : 1);
        lstage += run;
    };
    // The stage that is loaded next: begin, its loads 0 .. L - 1, end.
    const int tail = K & (BK - 1);
    auto begin_stage = [&]() {
        if (run == 0) next_run();
        --run;
    };
    auto load = [&](auto which) {
        constexpr int i = decltype(which)::value;
        if constexpr (i < NSide::loads) nside.template load<i>(nc, lat);
        else if constexpr (i < NL) nside.template load<i - NSide::loads>(nc1, lat + NSide::bytes);
        else if constexpr (i < L) mside.template load<i - NL>(mc, lat + BN * BK * 2);
    };
    auto end_stage = [&]() {
        NSide::advance(nc, nstep);
        if constexpr (GATED) NSide::advance(nc1, nstep);
        MSide::advance(mc, mstep);
        lslot = lslot + 1 == S ? 0 : lslot + 1;
        lat = lslot == 0 ? lds0 + wave * 1024 : lat + Cfg::stage;
    };
    // zeros past K in the stage that has landed in `slot`
    auto mend = [&](int slot) {
        if (uni(cuts >> slot & 1) == 0) return;
        asm volatile("" ::: "memory");  // a branch of its own: nothing below is done without it
        cuts &= ~(1 << slot);
        uint8_t *at = smem + slot * Cfg::stage;
        nside.mend(at, tail, wave, lane);
        if constexpr (GATED) nside.mend(at + NSide::bytes, tail, wave, lane);
        mside.mend(at + BN * BK * 2, tail, wave, lane);
    };

    using Acc = typename std::conditional<MI == 16, f32x4, f32x16>::type;
    Acc acc[TN][TM];
    vec fa[TN], fb[2][TM];
    const int nrow = wn * (NROWS / WN), mrow = wm * (BM / WM);
    auto readn = [&](const uint8_t *st, int i, int q) {
        if constexpr (GATED) return nside.read(st + (i >= TNG ? NSide::bytes : 0), nrow, i % TNG, q);
        else return nside.read(st, nrow, i, q);
    };
    auto readm = [&](const uint8_t *st, int j, int q) { return mside.read(st + BN * BK * 2, mrow, j, q); };

    int slot = 0;
    if (ns > 0) {
        for (int s = 0; s + 1 < S; ++s) {
            begin_stage();
            each<L>(load);
            end_stage();
        }
        begin_stage();
        each<L0>(load);  // the others go out with the first products
        wait_vm<L *(S - 2) + L0>();
        mend(0);
        lds_barrier();
    }

    // A stage is multiplied, a fragment row at a time; each row's N fragment is
    // replaced by the next step's as soon as the row has been issued.  In the last
    // step the next stage's fragments are read, and the loads of the stage S ahead,
    // into this one's buffer, begin; they end in the first step of the next stage.
    auto multiply = [&]() {
        const uint8_t *cur = smem + slot * Cfg::stage;
        slot = slot + 1 == S ? 0 : slot + 1;
        const uint8_t *nxt = smem + slot * Cfg::stage;
#pragma unroll
        for (int q = 0; q < KS; ++q) {
            const bool last = q == KS - 1;
            const uint8_t *from = last ? nxt : cur;
            const int fq = last ? 0 : q + 1;
#pragma unroll
            for (int i = 0; i < TN; ++i) {
#pragma unroll
                for (int j = 0; j < TM; ++j) acc[i][j] = mfma(fa[i], fb[q & 1][j], acc[i][j]);
                if (i == 0 && last) {
                    // the next stage has landed, this one has been read by all
                    wait_vm<L *(S - 2)>();
                    mend(slot);
                    lds_barrier();
                    begin_stage();
                }
                if (i == 0) {
#pragma unroll
                    for (int j = 0; j < TM; ++j) fb[(q + 1) & 1][j] = readm(from, j, fq);
                }
                fa[i] = readn(from, i, fq);
                if (last || q == 0) {
                    pick<TN>(i, [&](auto ic) {
                        constexpr int at = decltype(ic)::value * RATE;
                        if (last) each<RATE>([&](auto e) { load(std::integral_constant<int, at + decltype(e)::value>{}); });
                        else each<RATE>([&](auto e) { load(std::integral_constant<int, TN * RATE + at + decltype(e)::value>{}); });
                    });
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (q == 0) end_stage();
        }
    };

#pragma unroll 1
    for (int ti = 0; ti < mine; ++ti) {
        const Tile q = tile_at(ti);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = Acc{};
        if (ns > 0) {
#pragma unroll
            for (int j = 0; j < TM; ++j) fb[0][j] = readm(smem + slot * Cfg::stage, j, 0);
#pragma unroll
            for (int i = 0; i < TN; ++i) fa[i] = readn(smem + slot * Cfg::stage, i, 0);
#pragma unroll 1
            for (int s = q.s0; s < q.s1; ++s) multiply();
        }

        // Results straight from the registers.  A lane holds 4 consecutive n of every 16
        // (MI = 16) or 8; exchanging the odd rows of 16 lanes, or the upper half, of one
        // such group with the even ones, or the lower half, of the next leaves 8
        // consecutive n in each lane, for 16-byte stores.
        void *Y = q.z ? g.y1 : g.e.Y;
        constexpr int H = GATED ? 2 : 1, F = MI == 16 ? 2 : 1;  // fragments of a projection taken together
        static_assert(TNG % F == 0, "pairs of fragments");
        const int nl = MI == 16 ? ((lane >> 4) & 1) * 16 + (lane >> 5) * 8 : (lane >> 5) * 8;
        // A row of fragments shares its bias; where there is an R, it is read before the
        // first of them is stored, so that there is one wait for memory and not one for
        // each (8192 x 4096 x 9830 bfloat16 545 and 520 us).  Without one that would cost
        // instructions for nothing: 6144 x 11264 x 512 108 and 118 us.
        auto results = [&](auto ahead) {
            constexpr bool AHEAD = decltype(ahead)::value;
            constexpr int RV = F * MI * MI / 512;  // vectors of 8 of a fragment
            Addends<T, 8> with[RV];
            u32x4 rest[TM][RV];
#pragma unroll 1
            for (int f = 0; f < TNG / F * TM; ++f) {
                if (AHEAD && f % TM == 0)
#pragma unroll
                    for (int r = 0; r < RV; ++r) {
                        const int64_t n = q.n0 + nrow + f / TM * F * MI + nl + r * 16;
                        if (n < g.N) with[r].load_bias(g.e, n, (int)min((int64_t)8, g.N - n));
                        if (n + 8 <= g.N)
#pragma unroll
                            for (int j = 0; j < TM; ++j) {
                                const int64_t m = q.m0 + mrow + j * MI + (lane & (MI - 1));
                                if (m < g.M)
                                    __builtin_memcpy(&rest[j][r], reinterpret_cast<const T *>(g.e.R) + m * g.e.ldr + n, 16);
                            }
                    }
                Acc t[H][F];
                pick<TNG / F * TM>(f, [&](auto fc) {
                    constexpr int i = decltype(fc)::value / TM * F, j = decltype(fc)::value % TM;
#pragma unroll
                    for (int h = 0; h < H; ++h)
#pragma unroll
                        for (int k = 0; k < F; ++k) t[h][k] = acc[h * TNG + i + k][j];
                });
                const int64_t m = q.m0 + mrow + f % TM * MI + (lane & (MI - 1));
                const int64_t nb = q.n0 + nrow + f / TM * F * MI + nl;
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (MI == 16) {
                            const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(t[h][0][e]), __float_as_uint(t[h][F - 1][e]),
                                                                            false, false);
                            t[h][0][e] = __uint_as_float(w[0]);
                            t[h][F - 1][e] = __uint_as_float(w[1]);
                        } else {
#pragma unroll
                            for (int r = 0; r < 16; r += 8) {
                                const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(t[h][0][r + e]),
                                                                                __float_as_uint(t[h][0][r + e + 4]), false, false);
                                t[h][0][r + e] = __uint_as_float(w[0]);
                                t[h][0][r + e + 4] = __uint_as_float(w[1]);
                            }
                        }
                    }
                if (m >= g.M) continue;
#pragma unroll
                for (int r = 0; r < F * MI * MI / 64; r += 8) {
                    const int64_t n = nb + r * 2;
                    float z[8], u[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        z[e] = MI == 16 ? t[0][e / 4 * (F - 1)][e % 4] : t[0][0][(r + e) % (MI * MI / 64)];
                        if constexpr (GATED) u[e] = MI == 16 ? t[GATED][e / 4 * (F - 1)][e % 4] : t[GATED][0][(r + e) % (MI * MI / 64)];
                    }
                    if (n >= g.N) continue;
                    if (a.part.split > 1) {
                        store_vec<float, 8>(partial_at(a.part, g, q.chunk, q.z, 0, m, n), z);
                        if constexpr (GATED) store_vec<float, 8>(partial_at(a.part, g, q.chunk, q.z, 1, m, n), u);
                    } else if constexpr (AHEAD) {
                        Addends<T, 8> w = with[r / 8];
                        w.has_r = n + 8 <= g.N;
                        u32x4 x = {};
#pragma unroll
                        for (int j = 0; j < TM; ++j) {
                            const u32x4 y = rest[j][r / 8];
                            x = f % TM == j ? y : x;
                        }
                        __builtin_memcpy(&w.r, &x, sizeof x);
                        finish<T, GATED, 8>(g.e, Y, m, n, (int)min((int64_t)8, g.N - n), z, u, w);
                    } else {
                        finish<T, GATED, 8>(g.e, Y, m, n, (int)min((int64_t)8, g.N - n), z, u);
                    }
                }
            }
        };
        if constexpr (!NA && !GATED) {
            if (g.e.R && !g.e.out_f32 && a.part.split == 1) results(std::true_type{});
            else results(std::false_type{});
        } else {
            results(std::false_type{});
        }
    }
    wait_vm<0>();  // the loads past the last stage still write to LDS
}

template <typename T, bool NA, bool MA, bool GATED, int BN, int BM, int WN, int WM, int BK, int S, int MI>
__global__ __launch_bounds__(WN *WM * 64, 2) void k_gemm(TileArgs a) {
    tile_product<T, NA, MA, GATED, BN, BM, WN, WM, BK, S, MI>(a, blockIdx.x);
}

// The two products of a gradient, dX (a) and dW (b), in one launch.  Alone, small ones
// leave half of a CU's LDS and most of its matrix cores idle, waiting for a stage's loads;
// together, each waits while the other works: gradients of 512 x 2048 x 2048 bfloat16 36
// us in two launches and 28 in one, of 256 x 1024 x 1229 float16 29.7 and 23.4.
template <typename T, int BM, int S>
__global__ __launch_bounds__(256, 2) void k_gemm_pair(TileArgs a, TileArgs b, int first_b) {
    if ((int)blockIdx.x < first_b) {
        if ((int)blockIdx.x < a.groups) tile_product<T, true, false, false, 128, BM, 2, 2, 64, S, 32>(a, blockIdx.x);
    } else {
        tile_product<T, true, true, false, 128, BM, 2, 2, 64, S, 32>(b, (int)blockIdx.x - first_b);
    }
}

// Matrices to copy to rows of whole 16-byte chunks.
struct Copies {
    static constexpr int kMax = kMaxProducts * 4;
    struct {
        const uint16_t *p;
        uint16_t *out;
        int64_t ld, ldo, chunks;
        int cols;
    } m[kMax];
};

// Workgroups (x, y): matrix y, a chunk per thread; the elements' type does not matter.
__global__ __launch_bounds__(256) void k_align_rows(Copies a) {
    typedef uint16_t vec __attribute__((ext_vector_type(8)));
    const auto &q = a.m[blockIdx.y];
    const uint32_t across = (uint32_t)(q.ldo / 8);
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < q.chunks; c += (int64_t)gridDim.x * 256) {
        // the long division only where the short one does not do
        const int64_t row = c >> 32 ? c / across : (uint32_t)c / across;
        const int k = (int)(c - row * across) * 8;
        const uint16_t *p = q.p + row * q.ld + k;
        vec v = {};
        if (k + 8 <= q.cols) __builtin_memcpy(&v, p, 16);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k + e < q.cols) v[e] = p[e];
        *reinterpret_cast<vec *>(q.out + c * 8) = v;
    }
}

// ---------------------------------------------------------------- host side
// Workgroups of `kern` (nt threads, lds bytes) that the GPU holds at once; raises
// the kernel's LDS limit on the first call per device.
int resident(const void *kern, int nt, int lds, int *groups) try {
    static std::mutex mu;
    static std::map<std::pair<const void *, int>, int> known;
    int dev = 0;
    if (int rc = check_hip(hipGetDevice(&dev), "matrix product: current device")) return rc;
    std::lock_guard<std::mutex> lock(mu);
    const auto it = known.find({kern, dev});
    if (it != known.end()) {
        *groups = it->second;
        return SA_OK;
    }
    if (int rc = check_hip(hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds), "matrix product: LDS"))
        return rc;
    int per_cu = 0, cus = 0;
    if (int rc = check_hip(hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kern, nt, lds), "matrix product: occupancy"))
        return rc;
    if (int rc = check_hip(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev), "matrix product: CU count"))
        return rc;
    *groups = std::max(1, per_cu) * std::max(1, cus);
    known[{kern, dev}] = *groups;
    return SA_OK;
} catch (const std::exception &) {  // no exception leaves a C entry
    return fail(SA_E_HIP, "matrix product: out of host memory");
}

// How a product runs: k_rows with 16, 32 or 64 rows of M per workgroup (kRows64x2: 32
// rows of the N side instead of 16), or k_gemm with tiles of 128 x 64, 128 x 128 or
// 256 x 256 (N side by M side).
enum Path { kRows16, kRows32, kRows64, kTile64, kTile128, kTile256, kRows64x2 };
struct Plan {
    Path path;
    int split;   // chunks of k
    float time;  // of the model, microseconds
};

// Time models, microseconds, fitted to 364 products (4 to 2048 rows, 512 to 19712 by 512
// to 9856, forward and both gradients, k in 1 to 32 chunks: 4382 launches; median error 3
// to 7% a kernel).  The model's choice takes 1.012 of the best one's time on average, 1.34
// at most.
struct TileModel {
    int bn, bm, slots;    // tile; workgroups that the 256 CUs hold
    float launch, round;  // a launch; a round of tiles
    float one, two;       // a stage of 64 k: one tile per CU, every slot taken
    float join, join_chunk, join_mb;  // partial sums: a split, a chunk, a MB of them
    float out_mb, in_mb;  // a MB of results, of operands
};
constexpr TileModel kTileModel[] = {
    {128, 64, 512, 5.34f, 0.142f, 0.276f, 0.488f, 1.615f, 0.308f, 0.429f, 0.316f, 0.0495f},
    {128, 128, 512, 5.27f, 0.0f, 0.573f, 0.710f, 1.620f, 0.319f, 0.359f, 0.327f, 0.0576f},
    {256, 256, 256, 10.28f, 2.10f, 1.072f, 1.072f, 0.0f, 0.244f, 0.297f, 0.278f, 0.0115f},
};
struct RowsModel {
    Path path;
    int gated, bn, bm, u;  // rows of the N and M side per workgroup, k steps of 32 in a block
    float launch, block;   // a launch; a block of a wavefront's k
    float step;            // a step of 32 k, for every 256 workgroups past the first
    float join, join_mb, in_mb;
};
constexpr RowsModel kRowsModel[] = {
    {kRows16, 0, 16, 16, 8, 2.36f, 1.93f, 0.159f, 3.24f, 0.167f, 0.0586f},
    {kRows16, 1, 16, 16, 4, 4.05f, 1.43f, 0.264f, 3.71f, 0.238f, 0.0520f},
    {kRows32, 0, 16, 32, 4, 3.68f, 1.04f, 0.166f, 2.90f, 0.940f, 0.0607f},
    {kRows32, 1, 16, 32, 4, 4.34f, 1.70f, 0.223f, 3.56f, 0.420f, 0.0612f},
    {kRows64, 0, 16, 64, 4, 4.85f, 1.18f, 0.179f, 2.56f, 0.115f, 0.0830f},
    {kRows64, 1, 16, 64, 2, 5.76f, 0.82f, 0.303f, 2.81f, 0.270f, 0.0747f},
    {kRows64x2, 0, 32, 64, 4, 6.29f, 2.24f, 0.387f, 1.17f, 0.684f, 0.0757f},
};

float tile_time(const TileModel &m, const Gemm &g, int split) {
    const int64_t nn = g.N * (g.gated ? 2 : 1);
    const int64_t tiles = ((g.M + m.bm - 1) / m.bm) * ((nn + m.bn - 1) / m.bn) * g.batch * split;
    const float stages = (float)((g.K + 63) / 64 * g.parts) / split;
    const int64_t rest = tiles % m.slots;
    const bool sparse = rest > 0 && rest <= 256;
    const float full = (float)(tiles / m.slots + (rest > 0 && !sparse ? 1 : 0)), last = sparse ? 1.0f : 0.0f;
    const float out = (float)g.M * nn * g.batch, in = ((float)g.M + nn) * g.K * g.parts * g.batch;
    float t = m.launch + m.round * (full + last) + stages * (m.one * last + m.two * full) + out * 2e-6f * m.out_mb +
              in * 2e-6f * m.in_mb;
    if (split > 1) t += m.join + m.join_chunk * split + m.join_mb * split * out * 4e-6f;
    return t;
}

float rows_time(const RowsModel &m, const Gemm &g, int split) {
    const float nt = (float)((g.N + m.bn - 1) / m.bn), mt = (float)((g.M + m.bm - 1) / m.bm), groups = nt * mt * split;
    const int64_t blocks = (g.K + 32 * m.u - 1) / (32 * m.u);
    const float mine = (float)(((blocks + split - 1) / split + 7) / 8);
    const float nn = (float)g.N * (g.gated ? 2 : 1), in = (nt * g.M + mt * nn) * g.K;
    float t = m.launch + m.block * mine + m.step * mine * m.u * std::max(0.0f, groups / 256 - 1) + in * 2e-6f * m.in_mb;
    if (split > 1) t += m.join + m.join_mb * split * g.M * nn * 4e-6f;
    return t;
}

Plan plan_of(const Gemm &g) {
    const int64_t nn = g.N * (g.gated ? 2 : 1), stages = (g.K + 63) / 64 * g.parts;
    Plan best{kTile64, 1, 3e38f};
    const auto consider = [&](Path path, int split, float t) {
        if (t < best.time) best = {path, split, t};
    };
    if (!g.n[0].across)
        for (const RowsModel &m : kRowsModel) {
            if (m.gated != g.gated || (m.path != kRows64 && m.path != kRows64x2 && g.M > m.bm)) continue;
            if (((g.N + m.bn - 1) / m.bn) * ((g.M + m.bm - 1) / m.bm) > 2048) continue;  // beyond the fitted range
            for (int split = 1; split == 1 || (split <= 32 && split * 16 <= stages && nn * split <= 65536); split *= 2)
                consider(m.path, split, rows_time(m, g, split));
            if (g.M <= 16) return best;  // faster than every tile: gated 16 x 9830 x 4096 37 and 68 us
        }
    for (int i = 0; i < 3; ++i) {
        const TileModel &m = kTileModel[i];
        const int64_t tiles = ((g.M + m.bm - 1) / m.bm) * ((nn + m.bn - 1) / m.bn) * g.batch;
        consider((Path)(kTile64 + i), 1, tile_time(m, g, 1));
        for (int split = 2; split <= 32 && tiles < 512 && tiles * split <= 2 * m.slots && split * 2 <= stages; split *= 2)
            consider((Path)(kTile64 + i), split, tile_time(m, g, split));
    }
    return best;
}

// A product in one piece or in two: whole rounds of 256 x 256 tiles, which fill the GPU,
// and what is left of M or N, which would fill part of a round, by a plan of its own
// (in one piece and in two: float16 gradients of 6000 x 5000 x 4000 519 and 460 us, gated
// 2500 x 4096 x 2048 94.7 and 86.2, bfloat16 dW of 8192 x 4096 x 9830 672 and 635).
struct Pieces {
    int n;
    bool cut_m;
    int64_t at;  // where M, or else N, is cut
    Plan plan[2];
};

// The part of a product from m0 and n0 on, M by N.
Gemm part_of(const Gemm &g, int64_t m0, int64_t n0, int64_t M, int64_t N) {
    Gemm p = g;
    p.M = M;
    p.N = N;
    const auto move = [](auto *&q, int64_t elements, int size) {
        if (q) q = reinterpret_cast<std::remove_reference_t<decltype(q)>>(reinterpret_cast<uintptr_t>(q) + elements * size);
    };
    for (int i = 0; i < 2; ++i) {
        move(p.m[i].p, g.m[i].across ? m0 : m0 * g.m[i].ld, 2);
        move(p.n[i].p, g.n[i].across ? n0 : n0 * g.n[i].ld, 2);
    }
    const int out = g.e.out_f32 ? 4 : 2;
    move(p.e.bias, n0, 4);
    move(p.e.bias2, n0, 4);
    move(p.e.R, m0 * g.e.ldr + n0, out);
    move(p.e.Y, m0 * g.e.ldy + n0, out);
    move(p.y1, m0 * g.e.ldy + n0, out);
    move(p.e.Z, m0 * g.e.ldz + n0, 2);
    move(p.e.Z2, m0 * g.e.ldz + n0, 2);
    return p;
}

Pieces pieces_of(const Gemm &g) {
    Pieces best{1, false, 0, {plan_of(g), {}}};
    const TileModel &m = kTileModel[kTile256 - kTile64];
    const int64_t bn = g.gated ? m.bn / 2 : m.bn, mt = (g.M + m.bm - 1) / m.bm, nt = (g.N + bn - 1) / bn;
    const int64_t rounds = mt * nt * g.batch / m.slots;
    if (rounds == 0) return best;
    float least = best.plan[0].time;
    for (int cut_m = 0; cut_m < 2; ++cut_m) {
        const int64_t across = (cut_m ? nt : mt) * g.batch, tiles = rounds * m.slots / across;
        if (tiles < 1 || tiles >= (cut_m ? mt : nt)) continue;
        const int64_t at = tiles * (cut_m ? m.bm : bn);
        Gemm first = g, rest = g;
        (cut_m ? first.M : first.N) = at;
        (cut_m ? rest.M : rest.N) -= at;
        const Plan one{kTile256, 1, tile_time(m, first, 1)}, two = plan_of(rest);
        if (one.time + two.time < least) {
            least = one.time + two.time;
            best = {2, cut_m == 1, at, {one, two}};
        }
    }
    return best;
}

// The pieces' products: the parts of g, whose operands may have been moved.
int parts_of(const Gemm &g, const Pieces &p, Gemm (&parts)[2]) {
    parts[0] = p.n == 1 ? g : part_of(g, 0, 0, p.cut_m ? p.at : g.M, p.cut_m ? g.N : p.at);
    if (p.n == 2) parts[1] = part_of(g, p.cut_m ? p.at : 0, p.cut_m ? 0 : p.at, g.M - (p.cut_m ? p.at : 0), g.N - (p.cut_m ? 0 : p.at));
    return p.n;
}

size_t partial_bytes(const Gemm &g, int split) {
    return split > 1 ? (size_t)split * g.batch * (g.gated ? 2 : 1) * g.M * round_up(g.N, 8) * sizeof(float) : 0;
}

template <typename T, bool GATED>
int join(const Gemm &g, const Partial &q, hipStream_t stream) {
    const int64_t blocks = (g.M * (q.pitch / 8) + 255) / 256;
    hipLaunchKernelGGL((k_join<T, GATED>), dim3((unsigned)blocks, g.batch), dim3(256), 0, stream, g, q);
    return check_hip(hipGetLastError(), "k_join");
}

// The tiles of a product; groups: at most that many workgroups.
int tile_args(TileArgs &a, const Gemm &g, const Partial &q, int bn, int bm, int groups) {
    const int64_t mt = (g.M + bm - 1) / bm, rows = g.gated ? bn / 2 : bn, nt = (g.N + rows - 1) / rows;
    if (mt * nt >= (int64_t(1) << 28)) return fail(SA_E_UNSUPPORTED, "matrix product of more than 2^28 tiles");
    a = TileArgs{g, q, (int)mt, (int)nt, (int)(mt * nt) * g.batch * q.split, 0};
    a.groups = std::min(a.tiles, groups);
    return SA_OK;
}

template <typename T, bool NA, bool MA, bool GATED, int BN, int BM, int WN, int WM, int BK, int S, int MI>
int launch(const Gemm &g, const Partial &q, hipStream_t stream) {
    using Cfg = TileCfg<BN, BM, WN, WM, BK, S, MI>;
    auto kern = k_gemm<T, NA, MA, GATED, BN, BM, WN, WM, BK, S, MI>;
    int groups = 0;
    if (int rc = resident(reinterpret_cast<const void *>(kern), Cfg::NT, Cfg::lds, &groups)) return rc;
    TileArgs a;
    if (int rc = tile_args(a, g, q, BN, BM, groups)) return rc;
    hipLaunchKernelGGL(kern, dim3(a.groups), dim3(Cfg::NT), Cfg::lds, stream, a);
    if (int rc = check_hip(hipGetLastError(), "k_gemm")) return rc;
    return q.split > 1 ? join<T, GATED>(g, q, stream) : SA_OK;
}

template <typename T, int BM, int S>
int launch_pair(const Gemm *g, const Partial *q, hipStream_t stream) {
    constexpr int lds = TileCfg<128, BM, 2, 2, 64, S, 32>::lds;
    auto kern = k_gemm_pair<T, BM, S>;
    int groups = 0;
    if (int rc = resident(reinterpret_cast<const void *>(kern), 256, lds, &groups)) return rc;
    TileArgs a, b;
    if (int rc = tile_args(a, g[0], q[0], 128, BM, groups)) return rc;
    if (int rc = tile_args(b, g[1], q[1], 128, BM, groups)) return rc;
    const int first_b = (int)round_up(a.groups, 8);  // workgroup b of the second runs on XCD b mod 8 too
    hipLaunchKernelGGL(kern, dim3(first_b + b.groups), dim3(256), lds, stream, a, b, first_b);
    if (int rc = check_hip(hipGetLastError(), "k_gemm_pair")) return rc;
    for (int i = 0; i < 2; ++i)
        if (q[i].split > 1)
            if (int rc = join<T, false>(g[i], q[i], stream)) return rc;
    return SA_OK;
}

// Do the products of a gradient run in one launch?  Those of up to three rounds of small
// tiles do (gated 300 x 5504 x 2048, 1376 tiles, 70 us in two launches and 61 in one);
// 5409 x 8064 from 77, whose 2709 tiles fill the GPU without help, takes 108 us
// by itself with the other after it and 115 with the other beside it.
bool is_pair(const Gemm *g, const Pieces *p) {
    if (!g[0].n[0].across || g[0].m[0].across || !g[1].m[0].across) return false;
    for (int i = 0; i < 2; ++i) {
        const Plan &plan = p[i].plan[0];
        if (g[i].M == 0 || g[i].N == 0 || p[i].n != 1 || (plan.path != kTile64 && plan.path != kTile128)) return false;
        const TileModel &m = kTileModel[plan.path - kTile64];
        if (((g[i].M + m.bm - 1) / m.bm) * ((g[i].N + m.bn - 1) / m.bn) * g[i].batch * plan.split > 3 * m.slots) return false;
    }
    return true;
}

// Tiles of one shape for both, the smaller where the plans differ: with one of each shape
// gradients of 1000 x 2458 x 1024 (gated) take 60 us, as in two launches, with the smaller
// 55.
template <typename T>
int run_pair(const Gemm *g, const Pieces *p, const Partial *q, hipStream_t stream) {
    if (p[0].plan[0].path == kTile128 && p[1].plan[0].path == kTile128) return launch_pair<T, 128, 2>(g, q, stream);
    return launch_pair<T, 64, 3>(g, q, stream);
}

template <typename T, bool GATED, int NF, int MF, int U>
int launch_rows(const Gemm &g, const Partial &q, hipStream_t stream) {
    hipLaunchKernelGGL((k_rows<T, GATED, NF, MF, U>), dim3((unsigned)((g.N + NF * 16 - 1) / (NF * 16)), q.split,
                       (unsigned)((g.M + MF * 16 - 1) / (MF * 16))), dim3(512), 0, stream, g, q);
    if (int rc = check_hip(hipGetLastError(), "k_rows")) return rc;
    return q.split > 1 ? join<T, GATED>(g, q, stream) : SA_OK;
}

template <typename T, bool NA, bool MA, bool GATED>
int by_size(const Gemm &g, const Plan &p, const Partial &q, hipStream_t stream) {
    if constexpr (!NA) {
        if (p.path == kRows16) return launch_rows<T, GATED, 1, 1, GATED ? 4 : 8>(g, q, stream);
        if (p.path == kRows32) return launch_rows<T, GATED, 1, 2, 4>(g, q, stream);
        if constexpr (!GATED)
            if (p.path == kRows64x2) return launch_rows<T, GATED, 2, 4, 4>(g, q, stream);
        if (p.path == kRows64) return launch_rows<T, GATED, 1, 4, GATED ? 2 : 4>(g, q, stream);
    }
    if (p.path == kTile256) return launch<T, NA, MA, GATED, 256, 256, 2, 4, 64, 2, 16>(g, q, stream);
    if (p.path == kTile64) return launch<T, NA, MA, GATED, 128, 64, 2, 2, 64, 3, 32>(g, q, stream);
    return launch<T, NA, MA, GATED, 128, 128, 2, 2, 64, 2, 32>(g, q, stream);
}

template <typename T>
int run(const Gemm &g, const Plan &p, const Partial &q, hipStream_t stream) {
    if (g.gated) return by_size<T, false, false, true>(g, p, q, stream);
    if (!g.n[0].across) return by_size<T, false, false, false>(g, p, q, stream);
    if (!g.m[0].across) return by_size<T, true, false, false>(g, p, q, stream);
    return by_size<T, true, true, false>(g, p, q, stream);
}

// Rows and columns of an operand as it is stored.
struct Shape {
    int64_t rows, cols;
};
Shape shape_of(const Operand &o, int64_t r, int64_t K) { return o.across ? Shape{K, r} : Shape{r, K}; }

// Do the rows start on 16-byte boundaries (a single row needs no pitch)?
bool rows_aligned(const Operand &o, const Shape &s) { return aligned(o.p, 16) && (s.rows <= 1 || o.ld % 8 == 0); }

// Do the product's paths read rows of any alignment?
bool any_rows(const Pieces &p) {
    const Path path = p.plan[0].path;
    return p.n == 1 && (path <= kRows64 || path == kRows64x2);
}

// Visits the operands that have to be copied to aligned rows.
template <typename F>
void each_copied(Gemm &g, F &&f) {
    const int nm = std::max(g.parts, g.batch), nn = g.gated ? 2 : g.parts;
    // the two of a side share one pitch, so both are copied if one is
    bool cm = false, cn = false;
    for (int i = 0; i < nm; ++i) cm |= !rows_aligned(g.m[i], shape_of(g.m[i], g.M, g.K));
    for (int i = 0; i < nn; ++i) cn |= !rows_aligned(g.n[i], shape_of(g.n[i], g.N, g.K));
    for (int i = 0; i < nm && cm; ++i) f(g.m[i], shape_of(g.m[i], g.M, g.K));
    for (int i = 0; i < nn && cn; ++i) f(g.n[i], shape_of(g.n[i], g.N, g.K));
}

int64_t aligned_pitch(const Shape &s) { return round_up(s.cols, 8); }

}  // namespace

size_t gemm_workspace(const Gemm &g0) {
    Gemm g = g0;
    if (g.M == 0 || g.N == 0) return 0;
    const Pieces p = pieces_of(g);
    Gemm parts[2];
    size_t need = 0;
    for (int i = 0, k = parts_of(g, p, parts); i < k; ++i) need += round_up(partial_bytes(parts[i], p.plan[i].split), 256);
    if (!any_rows(p))
        each_copied(g, [&](Operand &, const Shape &s) { need += (size_t)round_up(s.rows * aligned_pitch(s) * 2, 256); });
    return need;
}

int gemm(const Gemm *const *gs, void *const *ws, int n, hipStream_t stream) {
    Gemm gemms[kMaxProducts];
    Pieces pieces[kMaxProducts];
    uint8_t *free[kMaxProducts];  // of the workspaces, behind the copies
    Copies copies{};
    int ncopies = 0;
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        Gemm &g = gemms[i] = *gs[i];
        if (g.M == 0 || g.N == 0) continue;
        pieces[i] = pieces_of(g);
        uint8_t *&at = free[i] = static_cast<uint8_t *>(ws[i]);
        if (!any_rows(pieces[i]))
            each_copied(g, [&](Operand &o, const Shape &s) {
                const int64_t ldo = aligned_pitch(s);
                const int64_t chunks = s.rows * (ldo / 8);
                if (chunks > 0)
                    copies.m[ncopies++] = {static_cast<const uint16_t *>(o.p), reinterpret_cast<uint16_t *>(at), o.ld, ldo,
                                           chunks, (int)s.cols};
                most = std::max(most, chunks);
                o.p = at;
                o.ld = ldo;
                at += round_up(s.rows * ldo * 2, 256);
            });
        // a single row has no pitch: one of whole chunks keeps the loads' ranges whole
        const int64_t mr = g.m[0].across ? g.K : g.M, nr = g.n[0].across ? g.K : g.N;
        for (int j = 0; j < 2; ++j) {
            if (mr <= 1) g.m[j].ld = round_up(g.m[0].across ? g.M : g.K, 8);
            if (nr <= 1) g.n[j].ld = round_up(g.n[0].across ? g.N : g.K, 8);
        }
    }
    if (ncopies > 0) {
        hipLaunchKernelGGL(k_align_rows, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 4096), ncopies), dim3(256), 0, stream,
                           copies);
        if (int rc = check_hip(hipGetLastError(), "k_align_rows")) return rc;
    }
    if (n == 2 && is_pair(gemms, pieces)) {
        Partial q[2];
        for (int i = 0; i < 2; ++i) q[i] = Partial{reinterpret_cast<float *>(free[i]), round_up(gemms[i].N, 8), pieces[i].plan[0].split};
        return gemms[0].type == SA_BF16 ? run_pair<__bf16>(gemms, pieces, q, stream) : run_pair<_Float16>(gemms, pieces, q, stream);
    }
    for (int i = 0; i < n; ++i) {
        const Gemm &g = gemms[i];
        if (g.M == 0 || g.N == 0) continue;
        Gemm parts[2];
        for (int j = 0, k = parts_of(g, pieces[i], parts); j < k; ++j) {
            const Plan &p = pieces[i].plan[j];
            const Partial q{reinterpret_cast<float *>(free[i]), round_up(parts[j].N, 8), p.split};
            free[i] += round_up(partial_bytes(parts[j], p.split), 256);
            const int rc = g.type == SA_BF16 ? run<__bf16>(parts[j], p, q, stream) : run<_Float16>(parts[j], p, q, stream);
            if (rc) return rc;
        }
    }
    return SA_OK;
}

}  // namespace sa
