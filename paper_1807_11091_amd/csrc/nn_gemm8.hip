// 8-bit matrix products with block scales on the gfx950 matrix cores, and the entry points
// of the operators made of them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "nn_epilogue.h"
#include "nn_gemm8.h"
#include "nn_quant.h"
#include "nn_tile.h"
#include "nn_types.h"
#include "sa_host.h"

namespace sa {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight codes as bfloat16, which holds every e4m3 value.
__device__ inline Vec8<__bf16>::type widen(int lo, int hi) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const pair c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return Vec8<__bf16>::type{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A lane's 32 codes of 16 rows' block, as the bfloat16 instructions take them.
struct Wide {
    Vec8<__bf16>::type k[4];
    __device__ explicit Wide(i32x8 v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) k[q] = widen(v[2 * q], v[2 * q + 1]);
    }
    Wide() = default;
};

// A block's products of 16 rows with 16, a lane's 32 codes of each in a and b.  How k is
// spread over lanes and bytes does not matter as long as both operands agree.
//
// The codes are widened for the bfloat16 instructions, whose binary32 sums are good to
// 1e-8 here.
__device__ inline f32x4 block_products(const Wide &a, const Wide &b) {
    f32x4 c = {};
#pragma unroll
    for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.k[q], b.k[q], c, 0, 0, 0);
    return c;
}

// The same by one 8-bit instruction, which spans the block.  It cuts each product of 8
// consecutive k at 2^-13 of 2^e, e the largest sum of two codes' exponents among them (so do
// all that take e4m3): up to 2^-10 of 2^e for each 8 k.  Of the sum of the products' magnitudes
// that is at most a quarter of what the rounding to bfloat16 costs a result, and twice what
// the one to binary16 does; of normal operands 1.3e-5, where the roundings cost 1.7e-3 and
// 2.1e-4.  Sums of large products that cancel can lose all that is left.  Results of 16 bits
// take it for a time of 0.5 to 0.6, unless the caller asks for exact products; binary32 ones
// and the scales of 8-bit ones, where it would show at once, are always made of exact ones.
__device__ inline f32x4 block_products8(i32x8 a, i32x8 b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{}, 0, 0, 0, 0, 0, 0);
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
// take the blocks of k in turn, U at a time, and feed the matrix cores straight from memory.
// Their sums are joined through LDS in a fixed order.  Rows past M or N read the last row and
// are not stored.  What hides the memory's latency is the other wavefronts of the CU: PER of
// them a SIMD.  With the next blocks on their way in a second set of registers and two
// workgroups a CU instead of three, 1 x 4096 x 9830 took 11.0 us instead of 9.5 (4.3 TB/s of
// weights), 16 x 9830 x 4096 18.5 instead of 13.9, gated 23.0 instead of 19.9.
template <typename T, bool GATED, bool EXACT, int NF, int MF, int U, int PER>
__global__ __launch_bounds__(512, PER) void k_rows8(Gemm8 g, Partial8 q) {
    constexpr int NW = 8, H = GATED ? 2 : 1;
    static_assert(128 % (NF * 16) == 0, "one block row");
    __shared__ float sums[NW][NF * H * MF][256];
    const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
    const int r = lane & 15, kg = (lane >> 4) * 16;
    const int64_t n0 = (int64_t)blockIdx.x * NF * 16, m0 = (int64_t)blockIdx.z * MF * 16;
    const int K = (int)g.K, last = (K - 1) & ~15;  // the last chunk of a row that holds codes
    // blocks of k of this workgroup
    const int blocks = (K + kBlock - 1) / kBlock;
    const int b0 = (int)((int64_t)blocks * blockIdx.y / q.split), b1 = (int)((int64_t)blocks * (blockIdx.y + 1) / q.split);

    const uint8_t *wp[H * NF], *xp[MF];
    const float *sx[MF], *sw[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int f = 0; f < NF; ++f) wp[h * NF + f] = g.w[h].codes + min(n0 + f * 16 + r, g.N - 1) * g.w[h].ld;
        sw[h] = g.w[h].scales + n0 / kBlock * g.w[h].scale_row;
    }
#pragma unroll
    for (int j = 0; j < MF; ++j) {
        const int64_t m = min(m0 + j * 16 + r, g.M - 1);
        xp[j] = g.x.codes + m * g.x.ld;
        sx[j] = g.x.scales + m * g.x.scale_row;
    }

    struct Set {  // this lane's part of U blocks: chunks of 16 codes at kg and kg + 64, and scales
        i32x4 w[U][H * NF][2], x[U][MF][2];
        float cx[U][MF], cw[U][H];
    };
    auto fetch = [&](Set &s, int b) {  // blocks past the last one: the last one again
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = min(b + u * NW, b1 - 1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = min(at * kBlock + i * 64 + kg, last);
#pragma unroll
                for (int f = 0; f < H * NF; ++f) s.w[u][f][i] = *reinterpret_cast<const i32x4 *>(wp[f] + k);
#pragma unroll
                for (int j = 0; j < MF; ++j) s.x[u][j][i] = *reinterpret_cast<const i32x4 *>(xp[j] + k);
            }
#pragma unroll
            for (int j = 0; j < MF; ++j) s.cx[u][j] = sx[j][at * g.x.scale_col];
#pragma unroll
            for (int h = 0; h < H; ++h) s.cw[u][h] = sw[h][at * g.w[0].scale_col];
        }
    };
    f32x4 acc[H * NF][MF] = {};
    auto whole = [&](i32x4 (&c)[2], int k) {  // a lane's codes, zeros past K
        union {
            i32x4 h[2];
            i32x8 v;
        } o;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            o.h[i] = c[i];
            if (k + kBlock > K)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int have = K - k - i * 64 - kg - e * 4;
                    if (have < 4) o.h[i][e] = have <= 0 ? 0 : o.h[i][e] & ((1 << have * 8) - 1);
                }
        }
        return o.v;
    };
    auto work = [&](Set &s, int b) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b + u * NW >= b1) break;
            const int k = (b + u * NW) * kBlock;
            i32x8 x[MF];
#pragma unroll
            for (int j = 0; j < MF; ++j) x[j] = whole(s.x[u][j], k);
            if constexpr (EXACT) {
                Wide wx[MF];
#pragma unroll
                for (int j = 0; j < MF; ++j) wx[j] = Wide(x[j]);
#pragma unroll
                for (int f = 0; f < H * NF; ++f) {
                    const Wide w(whole(s.w[u][f], k));
#pragma unroll
                    for (int j = 0; j < MF; ++j) add_scaled(acc[f][j], block_products(w, wx[j]), s.cx[u][j] * s.cw[u][f / NF]);
                }
            } else {
#pragma unroll
                for (int f = 0; f < H * NF; ++f) {
                    const i32x8 w = whole(s.w[u][f], k);
#pragma unroll
                    for (int j = 0; j < MF; ++j) add_scaled(acc[f][j], block_products8(w, x[j]), s.cx[u][j] * s.cw[u][f / NF]);
                }
            }
        }
    };
    if (b0 + wave < b1) {
        Set set;
        for (int b = b0 + wave; b < b1; b += NW * U) {
            fetch(set, b);
            __builtin_amdgcn_sched_barrier(0);  // every load goes out before the first product
            work(set, b);
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
        if (q.keep) {
            *partial_at(q, g, blockIdx.y, 0, m, n) = z[0];
            if constexpr (GATED) *partial_at(q, g, blockIdx.y, 1, m, n) = u[0];
        } else {
            finish<T, GATED, 1>(g.e, g.e.Y, m, n, 1, z, u);
        }
    }
}

// ------------------------------------------------------------ tiled product
// k_tile8: BN x BM outputs (N side by M side) per workgroup of WN x WM wavefronts, a block
// of 128 k a stage.  Stages go through a ring of S LDS buffers, written by buffer_load ..
// lds: the codes, 128 bytes a row, the 16-byte chunks of a row XOR-swizzled so that the rows
// of a fragment read hit distinct banks (the swizzle is applied to the source address); for
// each wavefront the scales of its rows of X, and of its block row of W.  The weights are
// the row operand of the matrix instructions, so a lane's four sums are consecutive in n and
// share one scale.
//
// Workgroups are persistent and their loads run over the stages of all their tiles.
//
// 8192 x 4096 x 9830 with 16-bit results takes 287 us (2.3 PFLOP/s; 318 to 331 with bias and
// residual): the matrix cores are busy half the time, a third of the wavefronts wait for
// loads, LDS or the barrier and a third for their turn to issue, at a clock of 2.0 GHz (2.4
// in a copy without loads).  Exact products take 552 (1.2 PFLOP/s), bound by issue: the
// widening of the codes and the scaling of the blocks are 3.4 vector instructions beside each
// matrix instruction, which hides 2.  With two stages in flight, and arguments kept in
// registers that then spilled, they took 75 more.
template <bool GATED, int BN, int BM, int WN, int WM, int S>
struct TileCfg8 {
    static constexpr int NW = WN * WM, NT = NW * 64;
    static constexpr int scales_at = (BN + BM) * kBlock;
    static constexpr int scales = 256 + 16;                     // bytes a wavefront: X's, one a lane, then W's
    static constexpr int stage = scales_at + NW * scales;
    static constexpr int join_at = S * stage;                   // largest values of the results' rows
    static constexpr bool touches = BM == 256;                  // see touch()
    static constexpr int touch_at = join_at + WN * BM * 4;
    static constexpr int lds = touch_at + (touches ? 256 : 0);
    static_assert(lds <= kMaxLds, "LDS");
};

struct TileArgs8 {
    Gemm8 g;
    Partial8 part;
    int mtiles, ntiles, tiles, groups;  // tiles: of all parts of k; groups: workgroups
};

// One operand's part of a stage: B rows of 128 codes, NW wavefronts.
template <int B, int NW>
struct Side8 {
    static constexpr int bytes = B * kBlock;
    static constexpr int loads = bytes / 1024 / NW;  // per wavefront
    static_assert(bytes % (1024 * NW) == 0, "whole loads per wavefront");

    __device__ static int swz(int r) { return (r >> 1) & 7; }

    uint32_t off[loads];  // byte offset of each load from the tile's origin
    int kc;               // first k of this lane's chunks: the loads lie 8 rows apart or a multiple

    __device__ void setup(int64_t ld, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < loads; ++i) {
            const int at = (i * NW + wave) * 64 + lane, row = at >> 3;
            const int chunk = (at & 7) ^ swz(row);
            off[i] = (uint32_t)row * (uint32_t)ld + chunk * 16u;
            if (i == 0) kc = chunk * 16;
        }
        static_assert(NW % 2 == 0 || loads == 1, "one chunk per lane");
    }

    // Where the next stage's loads read.  Rows past the matrix and k past K read as 0; a
    // chunk that K cuts is completed by mend().  The range is rounded up to whole chunks:
    // the bytes past the matrix's end lie in the aligned 16 bytes that hold its last code.
    struct Cursor {
        i32x4 rs;
        uint32_t so;
    };
    // at k0 of the rows at p (the tile's first row; `rows` of them in the matrix)
    __device__ static Cursor open(const uint8_t *p, int64_t ld, int rows, int K, int k0) {
        const uint32_t range = ((uint32_t)(min(rows, B) - 1) * (uint32_t)ld + (uint32_t)K + 15u) & ~15u;
        return Cursor{buffer_at(reinterpret_cast<uint64_t>(p), range), (uint32_t)uni(k0)};
    }
    __device__ static void advance(Cursor &c) { c.so = uni(c.so + kBlock); }
    // Lanes whose chunk begins at `k` or past it read zeros from here on (offsets are below
    // 2^31, one with the top bit set lies past every range).
    __device__ void limit(int k) {
#pragma unroll
        for (int i = 0; i < loads; ++i) off[i] = kc < k ? off[i] & ~kInvalidOffset : off[i] | kInvalidOffset;
    }
    template <int I>
    __device__ void load(const Cursor &c, uint32_t lds) const {
        dma16<I * NW * 1024>(c.rs, off[I], c.so, lds);
    }

    // The chunk that holds k = K - 1, in LDS: its codes past K become 0 (after this
    // wavefront's loads have landed); n: k of K's last stage.
    __device__ void mend(uint8_t *lds, int n, int wave, int lane) const {
        if (kc != (n & ~15)) return;
#pragma unroll
        for (int i = 0; i < loads; ++i) {
            i32x4 *q = reinterpret_cast<i32x4 *>(lds + (i * NW + wave) * 1024 + lane * 16);
            i32x4 v = *q;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int have = (n & 15) - e * 4;
                if (have < 4) v[e] = have <= 0 ? 0 : v[e] & ((1 << have * 8) - 1);
            }
            *q = v;
        }
    }
};

// A lane's codes of a fragment of 16 rows from row0 on: chunks lane / 16 and 4 + lane / 16.
struct Reads8 {
    uint32_t fo[2];
    __device__ explicit Reads8(int lane) {
        const int r = lane & 15;
#pragma unroll
        for (int c = 0; c < 2; ++c) fo[c] = r * kBlock + (((c * 4 + (lane >> 4)) ^ (r >> 1)) & 7) * 16;
    }
    __device__ i32x4 chunk(const uint8_t *lds, int row0, int c) const {
        return *reinterpret_cast<const i32x4 *>(lds + fo[c] + row0 * kBlock);
    }
    __device__ i32x2 half(const uint8_t *lds, int row0, int c, int which) const {
        return *reinterpret_cast<const i32x2 *>(lds + fo[c] + row0 * kBlock + which * 8);
    }
    __device__ i32x8 operator()(const uint8_t *lds, int row0) const {
        union {
            i32x4 h[2];
            i32x8 v;
        } x;
        x.h[0] = chunk(lds, row0, 0);
        x.h[1] = chunk(lds, row0, 1);
        return x.v;
    }
};

template <typename T, bool GATED, bool EXACT, int BN, int BM, int WN, int WM, int S>
__global__ __launch_bounds__(WN *WM * 64, 2) void k_tile8(TileArgs8) {
    using Cfg = TileCfg8<GATED, BN, BM, WN, WM, S>;
    constexpr int MI = 16;  // rows of a fragment
    constexpr int NW = Cfg::NW, TN = BN / WN / MI, TM = BM / WM / MI, TNG = GATED ? TN / 2 : TN, H = GATED ? 2 : 1;
    constexpr int NROWS = GATED ? BN / 2 : BN;  // n of a tile; gated: one half of the N side per projection
    using NSide = Side8<NROWS, NW>;
    using MSide = Side8<BM, NW>;
    constexpr int NL = NSide::loads * H, ML = NL + MSide::loads, L = ML + 1 + H;  // loads of a stage
    constexpr int WROWS = NROWS / WN, MROWS = BM / WM;               // n and m of a wavefront
    static_assert(128 % WROWS == 0 && MROWS <= 64 && TNG % 2 == 0 && TN % 2 == 0 && L * (S - 1) < 64, "shape");
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];

    // The arguments are read anew where they are used, so that the loop over the stages has
    // the registers: kept in scalar registers from the start they spill into vector ones,
    // and those into memory, whose waits would be for the loads of the stages too.
    auto args = []() -> const TileArgs8 & {
        auto p = (const __attribute__((address_space(4))) TileArgs8 *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(p));
        return *(const TileArgs8 *)p;
    };
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int wn = wave % WN, wm = wave / WN;
    const int nrow = wn * WROWS, mrow = wm * MROWS;

    // Workgroup b runs on XCD b mod 8, which walks one contiguous range of tiles (its own
    // L2); its workgroups take the range's tiles in turn.
    int first, mine, stride;
    {
        const TileArgs8 &a = args();
        const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
        const int per = a.tiles >> 3, extra = a.tiles & 7;
        first = uni(xcd * per + min(xcd, extra) + local);
        const int end = uni((xcd + 1) * per + min(xcd + 1, extra));
        stride = uni((a.groups >> 3) + (xcd < (a.groups & 7) ? 1 : 0));
        if (first >= end) return;
        mine = (end - first + stride - 1) / stride;  // tiles of this workgroup
    }

    const int K = uni((int)args().g.K), ns = (K + kBlock - 1) / kBlock;  // stages of a tile
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;

    // A tile: bands of 8 M tiles, down each band first, so that neighbours share operands
    struct Tile {
        int64_t m0, n0;
        int chunk;
        int s0, s1;  // its stages
    };
    auto tile_at = [&](int i) {
        const TileArgs8 &a = args();
        int t = first + i * stride;
        const int one = a.mtiles * a.ntiles;
        Tile q;
        q.chunk = t / one;
        t -= q.chunk * one;
        q.s0 = uni((int)((int64_t)ns * q.chunk / a.part.split));
        q.s1 = uni((int)((int64_t)ns * (q.chunk + 1) / a.part.split));
        const int band = t / (8 * a.ntiles), in = t - band * 8 * a.ntiles;
        const int h = min(8, a.mtiles - band * 8);
        q.m0 = (int64_t)(band * 8 + in % h) * BM;
        q.n0 = (int64_t)(in / h) * NROWS;
        return q;
    };

    NSide nside;
    MSide mside;
    nside.setup(args().g.w[0].ld, wave, lane);
    mside.setup(args().g.x.ld, wave, lane);
    const Reads8 read(lane);

    // The loads run over the stages of all tiles without a break, S stages ahead of
    // the products.  A run of stages below K differs from stage to stage by one addition per
    // operand; what else there is to work out is done between runs.
    typename NSide::Cursor nc, nc1;
    typename MSide::Cursor mc;
    i32x4 xs, ws[H];  // the scales' buffers
    const uint32_t xoff = lane < MROWS ? (uint32_t)lane * (uint32_t)args().g.x.scale_row * 4u : kInvalidOffset;
    const uint64_t xstep = (uint64_t)args().g.x.scale_col * 4, wstep = (uint64_t)args().g.w[0].scale_col * 4;
    uint32_t lat = lds0 + wave * 1024, slat = lds0 + Cfg::scales_at + wave * Cfg::scales;
    int run = 0, lstage = 0, lend = 0, ltile = -1, lslot = 0;
    int cuts = 0;  // slots that hold, or will, a chunk which K cuts
    auto next_run = [&]() {
        if (lstage == lend) ++ltile;
        if (ltile >= mine) {  // past the last stage: the loads write zeros that are not used
            nc.rs[2] = nc1.rs[2] = mc.rs[2] = xs[2] = ws[0][2] = ws[H - 1][2] = 0;
            nc.so = nc1.so = mc.so = 0;
            run = 1;
            return;
        }
        const Tile q = tile_at(ltile);
        const Gemm8 &g = args().g;
        const int64_t nld = g.w[0].ld, mld = g.x.ld;
        if (lstage == lend) {
            lstage = q.s0;
            lend = q.s1;
        }
        const int nrows = uni((int)min(g.N - q.n0, (int64_t)NROWS)), mrows = uni((int)min(g.M - q.m0, (int64_t)BM));
        const int k0 = lstage * kBlock;
        nc = NSide::open(g.w[0].codes + q.n0 * nld, nld, nrows, K, k0);
        if constexpr (GATED) nc1 = NSide::open(g.w[1].codes + q.n0 * nld, nld, nrows, K, k0);
        mc = MSide::open(g.x.codes + q.m0 * mld, mld, mrows, K, k0);
        nside.limit(K - k0);
        mside.limit(K - k0);
        const int64_t m = q.m0 + mrow;
        const int have = uni((int)min(g.M - m, (int64_t)MROWS));
        xs = buffer_at(reinterpret_cast<uint64_t>(g.x.scales + m * g.x.scale_row + lstage * g.x.scale_col),
                       have > 0 ? ((uint32_t)(have - 1) * (uint32_t)g.x.scale_row + 1u) * 4u : 0u);
        const int64_t n = q.n0 + nrow;
#pragma unroll
        for (int h = 0; h < H; ++h)
            ws[h] = buffer_at(reinterpret_cast<uint64_t>(g.w[h].scales + n / kBlock * g.w[0].scale_row + lstage * g.w[0].scale_col),
                              n < g.N ? 4u : 0u);
        if (kBlock > K - k0 && (K & 15) != 0) cuts |= 1 << lslot;
        run = uni(kBlock <= K - k0 ? min(K / kBlock - lstage, lend - lstage) : 1);
        lstage += run;
    };
    // The stage that is loaded next: begin, its loads 0 .. L - 1, end.
    auto begin_stage = [&]() {
        if (run == 0) next_run();
        --run;
    };
    auto load = [&](auto which) {
        constexpr int i = decltype(which)::value;
        if constexpr (i < NSide::loads) nside.template load<i>(nc, lat);
        else if constexpr (i < NL) nside.template load<i - NSide::loads>(nc1, lat + NSide::bytes);
        else if constexpr (i < ML) mside.template load<i - NL>(mc, lat + BN * kBlock);
        else if constexpr (i == ML) dma4<0>(xs, xoff, 0, slat);
        else if constexpr (i < L) {
            if (lane == 0) dma4<256 + 4 * (i - ML - 1)>(ws[i - ML - 1], 0, 0, slat);
        }
    };
    auto move = [](i32x4 &rs, uint64_t by) {
        const uint64_t base = ((uint64_t)(uint32_t)rs[1] << 32 | (uint32_t)rs[0]) + by;
        rs[0] = uni((int)(uint32_t)base);
        rs[1] = uni((int)(uint32_t)(base >> 32));
    };
    auto end_stage = [&]() {
        NSide::advance(nc);
        if constexpr (GATED) NSide::advance(nc1);
        MSide::advance(mc);
        move(xs, xstep);
#pragma unroll
        for (int h = 0; h < H; ++h) move(ws[h], wstep);
        lslot = lslot + 1 == S ? 0 : lslot + 1;
        lat = lds0 + wave * 1024 + lslot * Cfg::stage;
        slat = lds0 + Cfg::scales_at + wave * Cfg::scales + lslot * Cfg::stage;
    };
    // zeros past K in the stage that has landed in `slot`
    const int tail = K & (kBlock - 1);
    auto mend = [&](int slot) {
        if (uni(cuts >> slot & 1) == 0) return;
        asm volatile("" ::: "memory");  // a branch of its own: nothing below is done without it
        cuts &= ~(1 << slot);
        uint8_t *at = smem + slot * Cfg::stage;
        nside.mend(at, tail, wave, lane);
        if constexpr (GATED) nside.mend(at + NSide::bytes, tail, wave, lane);
        mside.mend(at + BN * kBlock, tail, wave, lane);
    };

    f32x4 acc[TN][TM];
    int slot = 0;
    if (ns > 0) {
        for (int s = 0; s + 1 < S; ++s) {
            begin_stage();
            each<L>(load);
            end_stage();
        }
        wait_vm<L *(S - 2)>();
        mend(0);
        lds_barrier();
        begin_stage();
        each<L>(load);
        end_stage();
    }

    auto rows_n = [&](const uint8_t *st, int i) { return st + (GATED && i >= TNG ? NSide::bytes : 0); };
    auto row_n = [&](int i) { return nrow + i % TNG * MI; };  // row i of a stage's fragments of W
    auto rows_m = [&](const uint8_t *st) { return st + BN * kBlock; };
    // X's scales of a stage, read at its start into scale[0], and W's; joined beside the first
    // row's products, whose sums are the first to need them
    float scale[H][TM], wscale[H];
    auto fetch_scales = [&](const uint8_t *st) {
        const float *s = reinterpret_cast<const float *>(st + Cfg::scales_at + wave * Cfg::scales);
#pragma unroll
        for (int j = 0; j < TM; ++j) scale[0][j] = s[j * MI + (lane & (MI - 1))];
#pragma unroll
        for (int h = 0; h < H; ++h) wscale[h] = s[64 + h];
    };
    auto join_scales = [&]() {
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int h = H - 1; h >= 0; --h) scale[h][j] = scale[0][j] * wscale[h];
    };
    f32x4 part[TM];
    auto add = [&](int i, int j) {  // beside the next row's products, not after all of them
        add_scaled(acc[i][j], part[j], scale[GATED && i >= TNG][j]);
        asm volatile("" : "+v"(acc[i][j]));
    };
    auto join = [&]() {  // the next stage has landed, `slot` before it has been read by all
        wait_vm<L *(S - 2)>();
        mend(slot);
        lds_barrier();
        begin_stage();
    };

    // 8-bit instructions.  Up to four rows of W's codes are in registers, each replaced by the
    // one as many further on behind its last product; X's by the next stage's behind the last
    // row's.  Where all rows are, the stage's buffer is free from its begin on.
    constexpr int RING = TN > 4 ? 2 : TN;
    i32x8 fa[RING], fb[TM];
    auto fetch8 = [&]() {
        const uint8_t *st = smem + slot * Cfg::stage;
#pragma unroll
        for (int i = 0; i < RING; ++i) fa[i] = read(rows_n(st, i), row_n(i));
#pragma unroll
        for (int j = 0; j < TM; ++j) fb[j] = read(rows_m(st), mrow + j * MI);
        fetch_scales(st);
    };
    auto multiply8 = [&]() {
        constexpr int JOIN = TN - RING, RATE = (L + RING - 1) / RING;  // loads that go out with a row from JOIN on
        const uint8_t *cur = smem + slot * Cfg::stage;
        slot = slot + 1 == S ? 0 : slot + 1;
        const uint8_t *nxt = smem + slot * Cfg::stage;
        each<TN>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            if (i == JOIN) join();
            if constexpr (i >= JOIN) each<RATE>([&](auto e) { load(std::integral_constant<int, (i - JOIN) * RATE + decltype(e)::value>{}); });
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                if (i > 0) add(i - 1, j);
                part[j] = block_products8(fa[i % RING], fb[j]);
                if (i == TN - 1) fb[j] = read(rows_m(nxt), mrow + j * MI);
            }
            if (i == 0) join_scales();
            constexpr int next = (i + RING) % TN;
            fa[i % RING] = read(rows_n(i < JOIN ? cur : nxt, next), row_n(next));
            __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int j = 0; j < TM; ++j) add(TN - 1, j);
        fetch_scales(nxt);
        end_stage();
    };

    // Exact products, in four steps of 32 k a row.  X's codes are widened once a stage, the
    // next stage's in place beside the last row's products, W's a step ahead; W's codes are
    // read two rows ahead.
    typedef Vec8<__bf16>::type Vec;
    i32x8 ra[2];
    Vec wa[2];
    Wide wb[TM];
    auto fetch_exact = [&]() {
        const uint8_t *st = smem + slot * Cfg::stage;
#pragma unroll
        for (int i = 0; i < 2; ++i) ra[i] = read(rows_n(st, i), row_n(i));
#pragma unroll
        for (int j = 0; j < TM; ++j) wb[j] = Wide(read(rows_m(st), mrow + j * MI));
        wa[0] = widen(ra[0][0], ra[0][1]);
        fetch_scales(st);
    };
    auto multiply_exact = [&]() {
        constexpr int JOIN = TN - 2, RATE = (L + 1) / 2;  // loads that go out with each of the last two rows
        const uint8_t *cur = smem + slot * Cfg::stage;
        slot = slot + 1 == S ? 0 : slot + 1;
        const uint8_t *nxt = smem + slot * Cfg::stage;
        i32x4 raw[TM];  // half of X's codes of the next stage: steps 0 and 1, then 2 and 3 as they are used up
        each<TN>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            if (i == JOIN) join();
            if constexpr (i >= JOIN) each<RATE>([&](auto e) { load(std::integral_constant<int, (i - JOIN) * RATE + decltype(e)::value>{}); });
            each<4>([&](auto qc) {
                constexpr int q = decltype(qc)::value;
                if (i == TN - 2 && q == 3)
#pragma unroll
                    for (int j = 0; j < TM; ++j) raw[j] = read.chunk(rows_m(nxt), mrow + j * MI, 0);
#pragma unroll
                for (int j = 0; j < TM; ++j) {
                    if (i > 0 && q == 0) add(i - 1, j);
                    part[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[q & 1], wb[j].k[q], q ? part[j] : f32x4{}, 0, 0, 0);
                }
                const i32x8 &from = ra[q < 3 ? i & 1 : (i + 1) & 1];
                constexpr int at = (q + 1) % 4 * 2;
                wa[(q + 1) & 1] = widen(from[at], from[at + 1]);
                if (i == TN - 1)
#pragma unroll
                    for (int j = 0; j < TM; ++j) {
                        wb[j].k[q] = widen(raw[j][q % 2 * 2], raw[j][q % 2 * 2 + 1]);
                        if (q < 2) {
                            const i32x2 v = read.half(rows_m(nxt), mrow + j * MI, 1, q);
                            raw[j][q * 2] = v[0];
                            raw[j][q * 2 + 1] = v[1];
                        }
                    }
                if (i == 0 && q == 3) join_scales();
                constexpr int next = (i + 2) % TN;
                if (q == 3) ra[i & 1] = read(rows_n(i < JOIN ? cur : nxt, next), row_n(next));
                __builtin_amdgcn_sched_barrier(0);
            });
        });
#pragma unroll
        for (int j = 0; j < TM; ++j) add(TN - 1, j);
        fetch_scales(nxt);
        end_stage();
    };

    // The lines of a tile's residual, which the epilogue reads piece by piece, into the L2, a
    // stage before: 8192 x 4096 x 9830 took 337 us without.  The words read go to LDS and are
    // not used.  Not in smaller tiles, where it cost more than it gave (a binary32 result with a
    // residual 620 us, 633 with it), so the residual has 16 bits.
    auto touch = [&](const Tile &q) {
        const Gemm8 &g = args().g;
        if (!g.e.R || args().part.keep) return;
        constexpr int size = 2, per = NROWS * size / 128;  // lines a row
        const int rows = (int)min(g.M - q.m0, (int64_t)BM), bytes = (int)min(g.N - q.n0, (int64_t)NROWS) * size;
        const uint64_t at = reinterpret_cast<uint64_t>(g.e.R) + (q.m0 * g.e.ldr + q.n0) * size;
        const uint32_t pitch = (uint32_t)g.e.ldr * (uint32_t)size;
        const i32x4 rs = buffer_at(at & ~(uint64_t)3, uni((int)((uint32_t)(rows - 1) * pitch + (uint32_t)bytes) & ~3));
#pragma unroll 1  // side by side they would spill
        for (int c = 0; c < BM * per; c += Cfg::NT) {
            const int i = c + tid, row = i / per, in = (i - row * per) * 128;
            dma4<Cfg::touch_at>(rs, row < rows && in < bytes ? (uint32_t)row * pitch + (uint32_t)in & ~3u : kInvalidOffset, 0, lds0);
        }
    };
    constexpr int PN = TNG / 2;  // pairs of fragments
#pragma unroll 1
    for (int ti = 0; ti < mine; ++ti) {
        const Tile q = tile_at(ti);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{};
        if constexpr (EXACT) {
            if (q.s0 < q.s1) fetch_exact();
#pragma unroll 1
            for (int s = q.s0; s < q.s1; ++s) multiply_exact();
        } else {
            if (q.s0 < q.s1) fetch8();
#pragma unroll 1
            for (int s = q.s0; s < q.s1; ++s) {
                if constexpr (Cfg::touches)
                    if (s + 1 == q.s1) touch(q);
                multiply8();
            }
        }

        // Results straight from the registers.  A lane holds 4 consecutive n of every 16;
        // exchanging the odd rows of 16 lanes of one such group with the even ones of the next
        // leaves 8 consecutive n in each lane.  A row's pieces of 64 bytes follow each other
        // (binary32 results with a residual 640 us in columns of pieces, 620 so).
        const TileArgs8 &a = args();
        const Gemm8 &g = a.g;
        int el = lane;
        asm volatile("" : "+v"(el));  // what follows from it takes no registers before
        // this lane's first n of two fragments and its m
        const int nl = ((el >> 4) & 1) * 16 + (el >> 5) * 8, ml = el & 15;
        constexpr bool EIGHT = EXACT && NROWS % kBlock == 0;  // smaller tiles: k_join8
        const bool eight = EIGHT && a.part.keep == 0 && g.q.codes;
        float top[TM] = {};  // largest values of this lane's rows
#pragma unroll 1
        for (int f = 0; f < PN * TM; ++f) {
            float z[8], u[8];
            pick<PN * TM>(f, [&](auto fc) {
                constexpr int p = decltype(fc)::value % PN, j = decltype(fc)::value / PN;
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int e = 0; e < 8; ++e) (h ? u : z)[e] = acc[h * TNG + 2 * p + e / 4][j][e % 4];
                asm volatile("" ::"n"(j * PN + p));  // keeps the compiler from merging the branches, which would index registers
            });
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float *v = h ? u : z;
                    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[e]), __float_as_uint(v[e + 4]), false, false);
                    v[e] = __uint_as_float(w[0]);
                    v[e + 4] = __uint_as_float(w[1]);
                }
            const int64_t m = q.m0 + mrow + f / PN * MI + ml, n = q.n0 + nrow + f % PN * 32 + nl;
            const int cnt = m < g.M ? (int)max((int64_t)0, min((int64_t)8, g.N - n)) : 0;
            if (cnt > 0) {
                if (a.part.keep) {
                    store_vec<float, 8>(partial_at(a.part, g, q.chunk, 0, m, n), z);
                    if constexpr (GATED) store_vec<float, 8>(partial_at(a.part, g, q.chunk, 1, m, n), u);
                } else {
                    Addends<T, 8> with;
                    with.has_r = false;
                    with.load_bias(g.e, n, cnt);
                    finish_values<T, GATED, 8, true>(g.e, m, n, cnt, z, u, with);
                    if (g.e.Y) put_values<T, 8, true>(g.e, g.e.Y, m, n, cnt, z);
                }
            }
            if constexpr (!EIGHT) continue;
            if (!eight) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = e < cnt ? z[e] : 0.0f;
            const float most = largest(z);
            pick<PN * TM>(f, [&](auto fc) {
                constexpr int p = decltype(fc)::value % PN, j = decltype(fc)::value / PN;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[2 * p + e / 4][j][e % 4] = z[e];
                top[j] = fmaxf(top[j], most);
                asm volatile("" ::"n"(j * PN + p));
            });
        }
        if constexpr (!EIGHT) continue;
        if (!eight) continue;
        // a row's block lies in one wavefront, or in some neighbours
        float *all = reinterpret_cast<float *>(smem + Cfg::join_at);
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            top[j] = lanes_max<MI, 64>(top[j]);
            if (WROWS < kBlock && el < MI) all[wn * BM + mrow + j * MI + el] = top[j];
        }
        if constexpr (WROWS < kBlock) {
            constexpr int PER = kBlock / WROWS;  // wavefronts a block
            lds_barrier();
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int w = 1; w < PER; ++w)
                    top[j] = fmaxf(top[j], all[((wn ^ w) % WN) * BM + mrow + j * MI + ml]);
            lds_barrier();  // read before the next tile's are written
        }
        const int64_t nb = q.n0 + nrow;
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const int64_t m = q.m0 + mrow + j * MI + ml;
            const float s = block_scale(top[j]), inv = block_inverse(s);
            if (m >= g.M) continue;
            if (nb % kBlock == 0 && el < MI && nb < g.N) g.q.scales[m * g.q.scale_row + nb / kBlock * g.q.scale_col] = s;
            each<PN>([&](auto pc) {
                const int64_t n = nb + decltype(pc)::value * 32 + nl;
                const int cnt = (int)min((int64_t)8, g.N - n);
                if (cnt <= 0) return;
                float z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = acc[2 * decltype(pc)::value + e / 4][j][e % 4];
                store_codes(g.q.codes + m * g.q.ld + n, cnt, codes8(z, inv));
            });
        }
    }
    wait_vm<0>();  // the loads past the last stage still write to LDS
}

// ---------------------------------------------------------------- host side
// M x N x K by GPU time in bfloat16, us, the best split of k each:
//                            kRows16 kRows32 kRows64 kTile64 kTile128 kTile256 kTile256x256
//   16 x 9830 x 4096            14.0    16.2    19.8    14.9     18.7     18.3         26.1
//   16 x 4096 x 9830 exact      15.2    16.4    19.6    20.6     24.6     30.1
//   64 x 4096 x 9830                            29.0    17.8     21.8     23.0         33.1
//   256 x 9830 x 4096                           98.1    26.9     31.2     31.0         39.0
//   1000 x 9830 x 4096 exact                            99.9      102      119
//   2048 x 4096 x 9830                                   114     94.2     89.7          131
//   5571 x 1870 x 13720                                  243      212      211          206
//   8192 x 4096 x 9830                                                     314          284
enum Path8 { kRows16, kRows32, kRows64, kTile64, kTile128, kTile256, kTile256x256 };
struct Plan8 {
    Path8 path;
    int split;
    int keep;  // the epilogue runs in k_join8
};

// 8-bit instructions where every result has 16 bits and the caller leaves the choice
// (8192 x 4096 x 9830: 287 us, and 552 of exact products).
bool is_exact(const Gemm8 &g) { return g.exact || g.q.codes || g.e.out_f32; }

// n of a tile
int tile_rows(Path8 path, bool gated) { return (path >= kTile256 ? 256 : 128) / (gated ? 2 : 1); }

// Time models, microseconds, fitted to the GPU times of 23000 launches (440 sizes: 1 to 4096
// rows, 64 to 16384 by 64 to 16384, every path in 1 to 32 parts of k; median error 3 to 12% a
// kernel).  Over 140 other sizes the choice takes 1.02 of the best one's time on average,
// 1.3 at most.  Sets: plain and gated, of each 8-bit instructions and exact products.
struct RowsModel8 {
    float launch, block;              // a launch; a block of a wavefront's k
    float more;                       // the same for every 256 workgroups past the first
    float in_mb;                      // a MB of operands
    float join, join_part, join_mb;   // k_join8: a launch, a part of k, a MB of sums
};
constexpr int kRowsM8[3] = {16, 32, 64};
constexpr RowsModel8 kRowsModel8[3][4] = {
    {{2.41f, 0.583f, 0.399f, 0.0965f, 1.58f, 0.282f, 2.16f},
     {4.37f, 0.587f, 0.359f, 0.0971f, 0.00496f, 0.284f, 2.48f},
     {2.5f, 0.986f, 0.195f, 0.108f, 1.81f, 0.324f, 0.894f},
     {4.76f, 0.986f, 0.309f, 0.103f, 0.000364f, 0.329f, 0.942f}},
    {{2.45f, 0.763f, 0.38f, 0.1f, 1.59f, 0.285f, 0.829f},
     {4.5f, 0.771f, 0.369f, 0.101f, 0.000156f, 0.285f, 0.891f},
     {2.73f, 1.18f, 0.707f, 0.0914f, 1.87f, 0.335f, 0.623f},
     {5.03f, 1.2f, 0.683f, 0.0917f, 0.0f, 0.339f, 0.743f}},
    {{2.86f, 1.14f, 0.622f, 0.0909f, 1.65f, 0.289f, 0.455f},
     {2.95f, 1.1f, 0.674f, 0.0813f, 2.15f, 0.289f, 0.622f},
     {3.34f, 1.57f, 1.89f, 0.0726f, 1.91f, 0.343f, 0.729f},
     {0.722f, 1.58f, 1.94f, 0.0554f, 5.06f, 0.353f, 0.99f}},
};
struct TileModel8 {
    float launch, round;              // a launch; a round of tiles
    float one, two;                   // a stage: one tile per CU, every slot taken
    float out_mb, in_mb;              // a million results; a MB of operands
    float join, join_part, join_mb;
};
struct TileShape8 {
    int bn, bm, slots;                // tile; workgroups that the 256 CUs hold
};
constexpr TileShape8 kTileShape8[4] = {{128, 64, 512}, {128, 128, 512}, {256, 128, 256}, {256, 256, 256}};
constexpr TileModel8 kTileModel8[3][4] = {
    {{5.21f, 1.33f, 0.381f, 0.633f, 0.966f, 0.0442f, 1.53f, 0.285f, 0.296f},
     {6.74f, 1.23f, 0.698f, 1.07f, 1.13f, 0.0441f, 0.664f, 0.29f, 0.285f},
     {4.86f, 1.54f, 0.404f, 0.671f, 0.668f, 0.0464f, 1.86f, 0.32f, 0.333f},
     {0.0f, 0.603f, 0.711f, 1.08f, 0.447f, 0.0451f, 7.85f, 0.343f, 0.377f}},
    {{6.95f, 0.885f, 0.563f, 0.887f, 0.965f, 0.0684f, 1.3f, 0.276f, 0.292f},
     {9.59f, 1.22f, 1.01f, 1.66f, 1.12f, 0.0396f, 0.0f, 0.254f, 0.24f},
     {6.11f, 1.22f, 0.609f, 0.928f, 0.709f, 0.0599f, 1.65f, 0.316f, 0.308f},
     {8.42f, 0.454f, 1.04f, 1.7f, 0.604f, 0.0424f, 0.545f, 0.348f, 0.307f}},
    {{6.42f, 2.46f, 2.94f, 0.725f, 0.96f, 0.0456f, 1.54f, 0.274f, 0.313f},
     {8.48f, 3.03f, 15.3f, 1.52f, 1.19f, 0.0425f, 0.0f, 0.267f, 0.261f},
     {6.05f, 2.06f, 10.1f, 0.799f, 0.748f, 0.0538f, 2.0f, 0.313f, 0.323f},
     {7.52f, 2.27f, 22.0f, 1.62f, 0.885f, 0.052f, 1.23f, 0.321f, 0.29f}},
};
// 256 x 256: plain products by 8-bit instructions only
constexpr TileModel8 kTileModel256x256 = {7.66f, 4.73f, 5.79f, 1.37f, 1.0f, 0.0655f, 0.926f, 0.268f, 0.272f};

// Do the results of a path go through k_join8?
bool is_joined(const Gemm8 &g, Path8 path, int split) {
    return split > 1 || (g.q.codes && (path < kTile64 || tile_rows(path, g.gated) < kBlock));
}

float rows_time(const Gemm8 &g, int i, int split) {
    const RowsModel8 &m = kRowsModel8[i][(g.gated ? 2 : 0) + is_exact(g)];
    const float nt = (float)((g.N + 15) / 16), mt = (float)((g.M + kRowsM8[i] - 1) / kRowsM8[i]);
    const int64_t blocks = (g.K + kBlock - 1) / kBlock, mine = ((blocks + split - 1) / split + 7) / 8;
    const float nn = (float)g.N * (g.gated ? 2 : 1);
    float more = nt * mt * split / 256;
    if (i == 2) more = ceilf(more);
    float t = m.launch + mine * (m.block + m.more * std::max(0.0f, more - 1)) + (nt * g.M + mt * nn) * g.K * 1e-6f * m.in_mb;
    if (is_joined(g, (Path8)i, split)) t += m.join + m.join_part * split + m.join_mb * split * g.M * nn * 4e-6f;
    return t;
}

float tile_time(const Gemm8 &g, int i, int split) {
    const TileModel8 &m = i < 3 ? kTileModel8[i][(g.gated ? 2 : 0) + is_exact(g)] : kTileModel256x256;
    const TileShape8 &s = kTileShape8[i];
    const int64_t nn = g.N * (g.gated ? 2 : 1);
    const int64_t tiles = ((g.M + s.bm - 1) / s.bm) * ((nn + s.bn - 1) / s.bn) * split, rest = tiles % s.slots;
    const bool sparse = s.slots > 256 && rest > 0 && rest <= 256;
    const float full = (float)(tiles / s.slots + (rest > 0 && !sparse)), last = sparse ? 1.0f : 0.0f;
    const float stages = (float)((g.K + kBlock - 1) / kBlock) / split;
    float t = m.launch + m.round * (full + last) + stages * (m.one * last + m.two * full) + (float)g.M * nn * 1e-6f * m.out_mb +
              ((float)g.M + nn) * g.K * 1e-6f * m.in_mb;
    if (is_joined(g, (Path8)(kTile64 + i), split)) t += m.join + m.join_part * split + m.join_mb * split * g.M * nn * 4e-6f;
    return t;
}

Plan8 plan_of(const Gemm8 &g) {
    Plan8 best{kTile256, 1, 0};
    float least = 3e38f;
    const int64_t blocks = (g.K + kBlock - 1) / kBlock, nn = g.N * (g.gated ? 2 : 1);
    const auto consider = [&](Path8 path, int64_t groups, auto &&time) {  // groups: workgroups with k in one part
        for (int split = 1; split == 1 || (split <= 32 && split * 2 <= blocks && groups < 512 && groups * split <= 2048); split *= 2) {
            const float t = time(split);
            if (t < least) least = t, best = {path, split, is_joined(g, path, split)};
        }
    };
    for (int i = 0; i < 3; ++i)  // up to 256 rows, where the models were fitted, and as many as a workgroup takes
        if (g.M <= (i == 2 ? 256 : kRowsM8[i]))
            consider((Path8)i, ((g.N + 15) / 16) * ((g.M + kRowsM8[i] - 1) / kRowsM8[i]), [&](int split) { return rows_time(g, i, split); });
    for (int i = 0; i < (g.gated || is_exact(g) ? 3 : 4); ++i) {
        const TileShape8 &s = kTileShape8[i];
        consider((Path8)(kTile64 + i), ((g.M + s.bm - 1) / s.bm) * ((nn + s.bn - 1) / s.bn), [&](int split) { return tile_time(g, i, split); });
    }
    return best;
}

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

template <typename T, bool GATED, bool EXACT, int BN, int BM, int WN, int WM, int S>
int launch_tiles(const Gemm8 &g, const Partial8 &q, hipStream_t stream) {
    using Cfg = TileCfg8<GATED, BN, BM, WN, WM, S>;
    auto kern = k_tile8<T, GATED, EXACT, BN, BM, WN, WM, S>;
    int groups = 0;
    if (int rc = resident(reinterpret_cast<const void *>(kern), Cfg::NT, Cfg::lds, &groups)) return rc;
    constexpr int rows = GATED ? BN / 2 : BN;
    const int64_t mt = (g.M + BM - 1) / BM, nt = (g.N + rows - 1) / rows;
    if (mt * nt * q.split >= (int64_t(1) << 30)) return fail(SA_E_UNSUPPORTED, "matrix product of 2^30 tiles or more");
    TileArgs8 a{g, q, (int)mt, (int)nt, (int)(mt * nt) * q.split, 0};
    a.groups = std::min(a.tiles, groups);
    hipLaunchKernelGGL(kern, dim3(a.groups), dim3(Cfg::NT), Cfg::lds, stream, a);
    return check_hip(hipGetLastError(), "k_tile8");
}

template <typename T, bool GATED, bool EXACT, int NF, int MF, int U, int PER>
int launch_rows(const Gemm8 &g, const Partial8 &q, hipStream_t stream) {
    hipLaunchKernelGGL((k_rows8<T, GATED, EXACT, NF, MF, U, PER>), dim3((unsigned)((g.N + NF * 16 - 1) / (NF * 16)), q.split,
                       (unsigned)((g.M + MF * 16 - 1) / (MF * 16))), dim3(512), 0, stream, g, q);
    return check_hip(hipGetLastError(), "k_rows8");
}

template <typename T, bool GATED, bool EXACT>
int by_path(const Gemm8 &g, const Plan8 &p, const Partial8 &q, hipStream_t stream) {
    switch (p.path) {
    case kRows16: return launch_rows<T, GATED, EXACT, 1, 1, GATED ? 1 : 2, 6>(g, q, stream);
    case kRows32: return launch_rows<T, GATED, EXACT, 1, 2, 1, GATED ? 4 : 6>(g, q, stream);
    case kRows64: return launch_rows<T, GATED, EXACT, 1, 4, 1, GATED ? 2 : 4>(g, q, stream);
    case kTile64: return launch_tiles<T, GATED, EXACT, 128, 64, 2, 2, 3>(g, q, stream);
    case kTile128: return launch_tiles<T, GATED, EXACT, 128, 128, 2, 2, 2>(g, q, stream);
    case kTile256x256:
        if constexpr (!GATED && !EXACT) return launch_tiles<T, GATED, EXACT, 256, 256, 2, 4, 2>(g, q, stream);
    default: return launch_tiles<T, GATED, EXACT, 256, 128, 4, 2, 3>(g, q, stream);
    }
}

template <typename T, bool GATED>
int run(const Gemm8 &g, const Plan8 &p, const Partial8 &q, hipStream_t stream) {
    if (int rc = is_exact(g) ? by_path<T, GATED, true>(g, p, q, stream) : by_path<T, GATED, false>(g, p, q, stream)) return rc;
    return q.keep ? join<T, GATED>(g, q, stream) : SA_OK;
}

// Tiles store 16-bit results of 48 MB and more past the caches, which the operands need, where
// the rows' pieces of 64 bytes are halves of lines: 8192 x 4096 x 9830 takes 284 us instead of
// 307, 5120 x 6080 x 84 with residual and Z 61 instead of 98.  Smaller ones lose by it if the
// caches hold where they go (4096 x 4100 x 300 39 us instead of 31).  Cut pieces are better joined
// there (8192 x 6060 x 1000 128 us instead of 94; gated 8192 x 9830 x 4096 with pre-activations,
// 1365 instead of 1312, though 1262 where two sets of buffers take turns).  Binary32 results,
// two stores a lane, lose too (608 us, 584).
int past_caches(int64_t M, int64_t N, const void *Y, int64_t ldy, const void *Z, const void *Z2, int64_t ldz) {
    const int64_t at = (int64_t)reinterpret_cast<uintptr_t>(Y) | (Y ? ldy * 2 : 0) | (int64_t)reinterpret_cast<uintptr_t>(Z) |
                       (int64_t)reinterpret_cast<uintptr_t>(Z2) | (Z ? ldz * 2 : 0);
    return at % 64 == 0 && M * N >= int64_t(24) << 20;
}

Gemm8 product(const sa_linear8_desc &d) {
    return Gemm8{d.M, d.N, d.K, d.type, 0, d.X, {d.W, sa_matrix8{}},
                 Epilogue{d.act, d.out_type == SA_F32, d.bias, nullptr, d.R, d.ldr, d.Y, d.ldy, d.Z, nullptr, d.ldz,
                          past_caches(d.M, d.N, d.Y, d.ldy, d.Z, nullptr, d.ldz)}, d.Q, d.exact};
}

Gemm8 product(const sa_glu8_desc &d) {
    return Gemm8{d.M, d.N, d.K, d.type, 1, d.X, {d.Wg, d.Wu},
                 Epilogue{d.act, 0, d.bg, d.bu, nullptr, 0, d.H, d.ldh, d.G, d.U, d.ldgu,
                          past_caches(d.M, d.N, d.H, d.ldh, d.G, d.U, d.ldgu)}, d.Q, d.exact};
}

// The outputs choose the plan, so a query covers each call that it holds for: with these
// outputs or fewer, and before the outputs with any of them.
template <typename D>
size_t workspace(const D &d, const void *y) {
    Gemm8 with = product(d), without = with;
    if (!y && !with.q.codes) with.q.codes = reinterpret_cast<uint8_t *>(16);
    without.q.codes = nullptr;
    if (d.Q.codes && !y) return gemm8_workspace(with);
    if (y && !d.Q.codes) return gemm8_workspace(without);
    return std::max(gemm8_workspace(with), gemm8_workspace(without));
}

sa_product8_plan_info plan_info(const Gemm8 &g) {
    sa_product8_plan_info info{};
    if (g.M == 0 || g.N == 0) return info;
    const Plan8 p = plan_of(g);
    if (p.path < kTile64) {
        info.rows = kRowsM8[p.path];
    } else {
        info.tile_n = kTileShape8[p.path - kTile64].bn;
        info.tile_m = kTileShape8[p.path - kTile64].bm;
    }
    info.exact = is_exact(g);
    info.split = p.split;
    info.joined = p.keep;
    return info;
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

extern "C" int structadmm_linear8_plan(const sa_linear8_desc *desc, sa_product8_plan_info *info) {
    clear_error();
    if (!desc || !info) return fail(SA_E_ARG, "linear8_plan: desc and info are required");
    if (int rc = validate_linear8(*desc)) return rc;
    *info = plan_info(product(*desc));
    return SA_OK;
}

extern "C" int structadmm_glu8_plan(const sa_glu8_desc *desc, sa_product8_plan_info *info) {
    clear_error();
    if (!desc || !info) return fail(SA_E_ARG, "glu8_plan: desc and info are required");
    if (int rc = validate_glu8(*desc)) return rc;
    *info = plan_info(product(*desc));
    return SA_OK;
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
