// Matrix products of the feed-forward operators on the gfx950 matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <mutex>
#include <set>
#include <type_traits>
#include <utility>

#include "nn_gemm.h"
#include "nn_types.h"
#include "sa_conv_device.h"
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

// Eight (n < 8 at a row's end) consecutive outputs from their sums.
template <typename T>
__device__ inline void finish8(const Epilogue &e, bool gated, void *Y, int64_t m, int64_t n, int cnt, const float *s,
                               const float *s2) {
    float z[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = s[i];
    auto add = [&](const float *b, float (&v)[8]) {
        float t[8];
        if (cnt == 8) load_vec<float, 8>(b + n, t);
        else load_part<float, 8>(b + n, cnt, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += t[i];
    };
    auto put = [&](void *p, int64_t at, const float (&v)[8]) {
        if (cnt == 8) store_vec<T, 8>(reinterpret_cast<T *>(p) + at, v);
        else store_part<T, 8>(reinterpret_cast<T *>(p) + at, cnt, v);
    };
    if (e.bias) add(e.bias, z);
    if (e.Z) put(e.Z, m * e.ldz + n, z);
    if (e.act != SA_ACT_NONE)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = act_value(e.act, z[i]);
    if (gated) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = s2[i];
        if (e.bias2) add(e.bias2, u);
        if (e.Z2) put(e.Z2, m * e.ldz + n, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= u[i];
    }
    if (e.out_f32) {
        float *y = reinterpret_cast<float *>(Y) + m * e.ldy + n;
        if (e.R) add(reinterpret_cast<const float *>(e.R) + m * e.ldr, z);
        if (cnt == 8) store_vec<float, 8>(y, z);
        else store_part<float, 8>(y, cnt, z);
    } else {
        if (e.R) {
            const T *r = reinterpret_cast<const T *>(e.R) + m * e.ldr + n;
            if (cnt == 8) load_vec<T, 8>(r, u);
            else load_part<T, 8>(r, cnt, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] += u[i];
        }
        put(Y, m * e.ldy + n, z);
    }
}

// ------------------------------------------------------------ tiled product
// k_gemm: BN x BM outputs (N side by M side) per workgroup of WN x WM wavefronts.
// Operands travel in stages of BK k through a ring of S LDS buffers, written by
// buffer_load ... lds (16 bytes per lane, S - 1 stages ahead).  The N side is the
// row operand of the MFMAs, so a lane's four sums are consecutive in n.
//
// LDS layouts (bank conflicts: 64 banks of 4 bytes):
//   - an operand whose rows run along k: [row][BK], the 16-byte chunks of a row
//     XOR-swizzled so that the 16 rows of one fragment read hit 16 distinct chunks;
//   - an operand whose rows run across k: [k][rows], read by ds_read_b64_tr_b16,
//     which hands each lane 4 consecutive k of its row (16 lanes transpose a block
//     of 4 k by 16 rows); its 64-byte units are XOR-swizzled by k.
// The swizzle is applied to the source address (the DMA writes lanes in order).
// Rows of the N side are dealt to fragments so that two fragments hold 8
// consecutive n in each lane.

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxLds = 160 * 1024;

__device__ inline int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a raw buffer of `bytes` at base, both wavefront-uniform
__device__ inline i32x4 buffer_at(uint64_t base, uint32_t bytes) {
    return i32x4{uni((int)(uint32_t)base), uni((int)((uint32_t)(base >> 32) & 0xffffu)), uni((int)bytes), kRsrcWord3};
}

// 16 bytes per lane straight from memory to LDS: lane i's land at lds + 16 * i.
// Inline asm: after the compiler's own LDS-DMA builtin every LDS read waits for
// all loads in flight.  The statement has no outputs; the waits are wait_vm().
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void dma16(i32x4 r, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voff),
                 "s"(r), "s"(soff)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ inline void wait_vm() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// this wavefront's LDS accesses done, then the workgroup's barrier
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One operand's part of a stage: B rows by BK k, NW wavefronts.
template <typename T, bool ACROSS, bool NSIDE, int B, int BK, int NW>
struct Side {
    typedef typename Vec8<T>::type vec;
    static constexpr int bytes = B * BK * 2;
    static constexpr int loads = bytes / 1024 / NW;  // per wavefront
    static constexpr int pitch = ACROSS ? B * 2 : BK * 2;
    static constexpr int cpr = pitch / 16;           // 16-byte chunks of an LDS row
    static constexpr int units = B / 32;             // 64-byte units of a k (ACROSS)
    static_assert(bytes % (1024 * NW) == 0, "whole loads per wavefront");

    // swizzle of row r (rows along k) or of k (rows across)
    __device__ static int swz(int r) {
        if constexpr (ACROSS) return ((r & 3) | ((r >> 3) & 1) << 2) & (units - 1);
        else if constexpr (BK == 64) return NSIDE ? ((r >> 1) & 1) | ((r >> 3) & 3) << 1 : (r >> 1) & 7;
        else return NSIDE ? (r >> 3) & 3 : (r >> 2) & 3;
    }
    // This lane's LDS row in load 0 and its source chunk.  Load i lies `step` rows
    // further on, a multiple of the swizzle's period: its chunk is the same.
    static constexpr int step = NW * 64 / cpr;
    static_assert(step % (ACROSS ? 16 : NSIDE ? 32 : 16) == 0 || loads == 1, "one chunk per lane");
    __device__ static void place(int wave, int lane, int &row, int &chunk) {
        const int at = wave * 64 + lane;
        row = at / cpr;
        const int c = at % cpr;
        chunk = ACROSS ? (((c >> 2) ^ swz(row)) << 2) | (c & 3) : c ^ swz(row);
    }

    uint32_t off[loads];  // byte offset of each load from the tile's origin
    int kc;               // first k of this lane's chunk (rows along k)

    __device__ void setup(int64_t ld, int wave, int lane) {
        int row, chunk;
        place(wave, lane, row, chunk);
        kc = chunk * 8;
#pragma unroll
        for (int i = 0; i < loads; ++i) off[i] = (uint32_t)(row + i * step) * (uint32_t)ld * 2u + chunk * 16u;
    }

    // The loads of one stage: k0 .. k0 + BK of the rows at p (the tile's first row;
    // `rows` of them in the matrix).  Rows past the matrix and k past K read as 0;
    // a chunk that K cuts is completed by mend().  The buffer's range is rounded up
    // to whole chunks: the bytes past the matrix's end lie in the aligned 16 bytes
    // that hold its last element, and never reach a result.
    struct Stage {
        i32x4 rs;
        uint32_t so;
        bool in;  // this lane's chunk begins below K
    };
    __device__ Stage stage(const T *p, int64_t ld, int rows, int K, int k0) const {
        Stage st;
        const int r = min(rows, B);
        if constexpr (ACROSS) {
            const int n = min(K - k0, BK);
            const uint32_t range = (((uint32_t)(n - 1) * (uint32_t)ld + r) * 2u + 15u) & ~15u;
            st.rs = buffer_at(reinterpret_cast<uint64_t>(p) + (uint64_t)k0 * (uint64_t)ld * 2u, range);
            st.so = 0;
        } else {
            const uint32_t range = (((uint32_t)(r - 1) * (uint32_t)ld + (uint32_t)K) * 2u + 15u) & ~15u;
            st.rs = buffer_at(reinterpret_cast<uint64_t>(p), range);
            st.so = uni(k0 * 2);
            st.in = kc < K - k0;
        }
        return st;
    }
    __device__ void load(const Stage &st, int i, uint32_t lds, int wave) const {
        const uint32_t at = uni(lds + (i * NW + wave) * 1024);
        if constexpr (ACROSS) dma16(st.rs, off[i], st.so, at);
        else dma16(st.rs, st.in ? off[i] : kInvalidOffset, st.so, at);
    }

    // The chunk that holds k = K - 1 of a stage at k0, in LDS: its elements past K
    // become +0 (after this wavefront's loads have landed).
    __device__ void mend(uint8_t *lds, int K, int k0, int wave, int lane) const {
        if constexpr (!ACROSS) {
            const int n = K - k0;  // valid k of the stage
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

    // Lane offsets of fragment reads.  Fragment f holds 16 rows: rows 16 f + (0 .. 15)
    // of the M side, rows 32 (f / 2) + 4 (f % 2) + {0-3, 8-11, 16-19, 24-27} of the N side.
    static constexpr int nfo = ACROSS ? 1 : BK / 32;
    uint32_t fo[nfo];

    __device__ void setup_reads(int lane) {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (ACROSS) {
            const int k = g * 8 + (r >> 2), piece = lane & 3;
            fo[0] = k * pitch + (swz(k) << 6) + piece * (NSIDE ? 16 : 8);
        } else {
            const int row = NSIDE ? 8 * (r >> 2) + (r & 3) : r;
#pragma unroll
            for (int q = 0; q < BK / 32; ++q) fo[q] = row * pitch + (((q * 4 + g) ^ swz(row)) << 4);
        }
    }

    // fragment f (rows from `row0`, a multiple of 32) of k step q
    __device__ vec read(const uint8_t *lds, int row0, int f, int q) const {
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) s16x4 *ptr;
            const int unit = row0 / 32 + (f >> 1);
            const uint8_t *p = lds + (fo[0] ^ (unit << 6)) + (f & 1) * (NSIDE ? 8 : 32) + q * 32 * pitch;
            union {
                s16x4 h[2];
                vec v;
            } x;
            x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p));
            x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p + 4 * pitch));
            return x.v;
        } else {
            const int at = NSIDE ? 32 * (f >> 1) + 4 * (f & 1) : 16 * f;
            return *reinterpret_cast<const vec *>(lds + fo[q] + (row0 + at) * pitch);
        }
    }
};

template <int BN, int BM, int WN, int WM, int BK, int S>
struct TileCfg {
    static constexpr int NW = WN * WM, NT = NW * 64;
    static constexpr int TN = BN / WN / 16, TM = BM / WM / 16;  // fragments of a wavefront
    static constexpr int stage = (BN + BM) * BK * 2;
    static constexpr int rows = 16 * WM;                        // rows of an epilogue pass
    static constexpr int cpitch = BN + 4;                       // its pitch in binary32
    static constexpr int lds = S * stage > rows * cpitch * 4 ? S * stage : rows * cpitch * 4;
    static_assert(lds <= kMaxLds, "LDS");
};

struct TileArgs {
    Gemm g;
    int mtiles, ntiles;
};

template <typename T, bool NA, bool MA, bool GATED, int BN, int BM, int WN, int WM, int BK, int S>
__global__ __launch_bounds__(WN *WM * 64) void k_gemm(TileArgs a) {
    using Cfg = TileCfg<BN, BM, WN, WM, BK, S>;
    using NSide = Side<T, NA, true, GATED ? BN / 2 : BN, BK, Cfg::NW>;  // gated: one half per projection
    using MSide = Side<T, MA, false, BM, BK, Cfg::NW>;
    typedef typename Vec8<T>::type vec;
    constexpr int TN = Cfg::TN, TM = Cfg::TM, KS = BK / 32, TNG = GATED ? TN / 2 : TN;
    constexpr int L = NSide::loads * (GATED ? 2 : 1) + MSide::loads;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];

    const Gemm &g = a.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
    const int wn = wave % WN, wm = wave / WN;
    const int z = blockIdx.z;
    // XCD x walks one contiguous range of tiles; within it, bands of 8 M tiles
    int mt, nt;
    {
        const int t = xcd_remap(blockIdx.x, a.mtiles * a.ntiles);
        const int band = t / (8 * a.ntiles), in = t - band * 8 * a.ntiles;
        const int h = min(8, a.mtiles - band * 8);
        mt = uni(band * 8 + in % h);
        nt = uni(in / h);
    }
    constexpr int NROWS = GATED ? BN / 2 : BN;  // n of a tile
    const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * NROWS;
    const int K = uni((int)g.K), nrows = uni((int)min(g.N - n0, (int64_t)NROWS)), mrows = uni((int)min(g.M - m0, (int64_t)BM));
    const int sp = (K + BK - 1) / BK, ns = sp * uni(g.parts);  // stages of a part, of all
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;

    NSide nside;
    MSide mside;
    nside.setup(g.n[0].ld, wave, lane);
    mside.setup(g.m[0].ld, wave, lane);
    nside.setup_reads(lane);
    mside.setup_reads(lane);
    const int64_t nld = g.n[0].ld, mld = g.m[0].ld;  // parts and batches share their pitch
    const T *np0 = reinterpret_cast<const T *>(g.n[0].p) + (NA ? n0 : n0 * nld);
    const T *np1 = reinterpret_cast<const T *>(g.n[1].p) + (NA ? n0 : n0 * nld);
    const T *mp0 = reinterpret_cast<const T *>(z ? g.m[1].p : g.m[0].p) + (MA ? m0 : m0 * mld);
    const T *mp1 = reinterpret_cast<const T *>(g.m[1].p) + (MA ? m0 : m0 * mld);
    // the loads of a stage, in the order of their issue
    struct Loads {
        typename NSide::Stage n, n1;
        typename MSide::Stage m;
        uint32_t at;
    };
    auto stage = [&](int st, int slot) {
        const bool second = st >= sp;
        const int k0 = (second ? st - sp : st) * BK;
        Loads l;
        l.at = lds0 + slot * Cfg::stage;
        l.n = nside.stage(second ? np1 : np0, nld, nrows, K, k0);
        if constexpr (GATED) l.n1 = nside.stage(np1, nld, nrows, K, k0);
        l.m = mside.stage(second ? mp1 : mp0, mld, mrows, K, k0);
        return l;
    };
    auto load = [&](const Loads &l, int i) {
        constexpr int NL = NSide::loads, NT = GATED ? 2 * NL : NL;
        if (i < NL) nside.load(l.n, i, l.at, wave);
        else if (GATED && i < NT) nside.load(l.n1, i - NL, l.at + NSide::bytes, wave);
        else mside.load(l.m, i - NT, l.at + BN * BK * 2, wave);
    };
    const bool cut = (K & 7) != 0;
    auto mend = [&](int st, int slot) {
        const int k0 = (st >= sp ? st - sp : st) * BK;
        if (!cut || k0 + BK < K) return;
        uint8_t *at = smem + slot * Cfg::stage;
        nside.mend(at, K, k0, wave, lane);
        if constexpr (GATED) nside.mend(at + NSide::bytes, K, k0, wave, lane);
        mside.mend(at + BN * BK * 2, K, k0, wave, lane);
    };

    f32x4 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    if (ns > 0) {
        const int nrow = wn * (BN / WN) / (GATED ? 2 : 1), mrow = wm * (BM / WM);
        auto readn = [&](const uint8_t *st, int i, int q) {
            if constexpr (GATED) return nside.read(st + (i >= TNG ? NSide::bytes : 0), nrow, i % TNG, q);
            else return nside.read(st, nrow, i, q);
        };
        auto readm = [&](const uint8_t *st, int j, int q) { return mside.read(st + BN * BK * 2, mrow, j, q); };
        for (int s = 0; s < S && s < ns; ++s) {
            const Loads l = stage(s, s);
#pragma unroll
            for (int i = 0; i < L; ++i) load(l, i);
        }
        // stage 0 has landed when at most the later ones are outstanding
        if (ns >= S) wait_vm<L *(S - 1)>();
        else wait_vm<0>();
        mend(0, 0);
        lds_barrier();
        vec fa[TN], fb[2][TM];
#pragma unroll
        for (int j = 0; j < TM; ++j) fb[0][j] = readm(smem, j, 0);
#pragma unroll
        for (int i = 0; i < TN; ++i) fa[i] = readn(smem, i, 0);
        int slot = 0;
        // Stage s is multiplied; in its last step the fragments of stage s + 1 are read
        // (MORE) and stage s + S is loaded into this one's buffer (FULL).
        auto multiply = [&](int s, auto more, auto full) {
            constexpr bool MORE = decltype(more)::value, FULL = decltype(full)::value;
            const uint8_t *cur = smem + slot * Cfg::stage;
            const int here = slot;
            slot = slot + 1 == S ? 0 : slot + 1;
            const uint8_t *nxt = smem + slot * Cfg::stage;
            Loads l;
            if constexpr (FULL) l = stage(s + S, here);
#pragma unroll
            for (int q = 0; q < KS; ++q) {
                const bool last = q == KS - 1;
                const uint8_t *from = last ? nxt : cur;
                const int fq = last ? 0 : q + 1;
                constexpr int HOLD = 1;  // rows multiplied before the barrier
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    __builtin_amdgcn_s_setprio(1);
#pragma unroll
                    for (int j = 0; j < TM; ++j) acc[i][j] = mfma(fa[i], fb[q & 1][j], acc[i][j]);
                    __builtin_amdgcn_s_setprio(0);
                    if (i == HOLD && last && MORE) {
                        // the next stage has landed, this one has been read by all
                        if constexpr (FULL) wait_vm<L *(S - 2)>();
                        else wait_vm<0>();
                        mend(s + 1, slot);
                        lds_barrier();
                    }
                    if (i >= HOLD && (!last || MORE)) {
                        if (i == HOLD) {
#pragma unroll
                            for (int j = 0; j < TM; ++j) fb[(q + 1) & 1][j] = readm(from, j, fq);
#pragma unroll
                            for (int h = 0; h < HOLD; ++h) fa[h] = readn(from, h, fq);
                        }
                        fa[i] = readn(from, i, fq);
                    }
                    if constexpr (FULL) {
                        if (last && i >= HOLD) {  // the loads, spread over the remaining rows
                            constexpr int per = (L + TN - HOLD - 1) / (TN - HOLD);
#pragma unroll
                            for (int e = 0; e < per; ++e)
                                if ((i - HOLD) * per + e < L) load(l, (i - HOLD) * per + e);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (KS % 2 == 1) {
#pragma unroll
                for (int j = 0; j < TM; ++j) fb[0][j] = fb[1][j];
            }
        };
        int s = 0;
        for (; s + S < ns; ++s) multiply(s, std::true_type{}, std::true_type{});
        for (; s + 1 < ns; ++s) multiply(s, std::true_type{}, std::false_type{});
        multiply(s, std::false_type{}, std::false_type{});
    }

    // The sums go through LDS, 16 rows of each wavefront at a time, and out in
    // vectors of 8 consecutive n.
    float *sc = reinterpret_cast<float *>(smem);
    constexpr int CP = Cfg::cpitch, CHUNKS = NROWS / 8;
    void *Y = z ? g.y1 : g.e.Y;
    auto stage_sums = [&](auto jc) {
        constexpr int j = decltype(jc)::value;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int f = GATED ? i % TNG : i;
            const int n = (GATED ? (i >= TNG ? BN / 2 : 0) + wn * (BN / WN / 2) : wn * (BN / WN)) + 32 * (f >> 1) +
                          8 * (lane >> 4) + 4 * (f & 1);
            *reinterpret_cast<f32x4 *>(sc + (wm * 16 + (lane & 15)) * CP + n) = acc[i][j];
        }
    };
    static_assert(TM == 4, "the passes below");
#pragma unroll 1
    for (int j = 0; j < TM; ++j) {
        lds_barrier();
        if (j == 0) stage_sums(std::integral_constant<int, 0>{});
        else if (j == 1) stage_sums(std::integral_constant<int, 1>{});
        else if (j == 2) stage_sums(std::integral_constant<int, 2>{});
        else stage_sums(std::integral_constant<int, 3>{});
        lds_barrier();
        for (int c = tid; c < Cfg::rows * CHUNKS; c += Cfg::NT) {
            const int r = c / CHUNKS, nl = (c - r * CHUNKS) * 8;
            const int64_t m = m0 + (r >> 4) * (BM / WM) + j * 16 + (r & 15), n = n0 + nl;
            if (m < g.M && n < g.N)
                finish8<T>(g.e, GATED, Y, m, n, (int)min((int64_t)8, g.N - n), sc + r * CP + nl,
                           GATED ? sc + r * CP + BN / 2 + nl : nullptr);
        }
    }
}

// Copies a matrix to rows of whole 16-byte chunks.
template <typename T>
__global__ __launch_bounds__(256) void k_align_rows(const T *p, int64_t ld, int64_t rows, int cols, T *out, int64_t ldo) {
    const int chunks = (cols + 7) / 8;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < rows * chunks; c += (int64_t)gridDim.x * 256) {
        const int64_t r = c / chunks;
        const int k = (int)(c - r * chunks) * 8;
        typename Vec8<T>::type v = {};
        if (k + 8 <= cols) __builtin_memcpy(&v, p + r * ld + k, 16);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k + e < cols) v[e] = p[r * ld + k + e];
        *reinterpret_cast<typename Vec8<T>::type *>(out + r * ldo + k) = v;
    }
}

// ---------------------------------------------------------------- host side
// Raises the kernel's LDS limit once per kernel and device.
int allow_lds(const void *kern, int lds) {
    static std::mutex mu;
    static std::set<std::pair<const void *, int>> known;
    int dev = 0;
    if (int rc = check_hip(hipGetDevice(&dev), "matrix product: current device")) return rc;
    std::lock_guard<std::mutex> lock(mu);
    if (known.count({kern, dev})) return SA_OK;
    if (int rc = check_hip(hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds), "matrix product: LDS"))
        return rc;
    known.insert({kern, dev});
    return SA_OK;
}

template <typename T, bool NA, bool MA, bool GATED, int BN, int BM, int WN, int WM, int BK, int S>
int launch(const Gemm &g, hipStream_t stream) {
    using Cfg = TileCfg<BN, BM, WN, WM, BK, S>;
    TileArgs a{g, 0, 0};
    const int64_t mt = (g.M + BM - 1) / BM, nt = (g.N + (GATED ? BN / 2 : BN) - 1) / (GATED ? BN / 2 : BN);
    if (mt * nt >= (int64_t(1) << 28)) return fail(SA_E_UNSUPPORTED, "matrix product of more than 2^28 tiles");
    a.mtiles = (int)mt;
    a.ntiles = (int)nt;
    auto kern = k_gemm<T, NA, MA, GATED, BN, BM, WN, WM, BK, S>;
    if (int rc = allow_lds(reinterpret_cast<const void *>(kern), Cfg::lds)) return rc;
    hipLaunchKernelGGL(kern, dim3(a.mtiles * a.ntiles, 1, g.batch), dim3(Cfg::NT), Cfg::lds, stream, a);
    return check_hip(hipGetLastError(), "k_gemm");
}

template <typename T, bool NA, bool MA, bool GATED>
int by_size(const Gemm &g, hipStream_t stream) {
    const int64_t big = ((g.M + 255) / 256) * ((g.N * (GATED ? 2 : 1) + 255) / 256) * g.batch;
    if (big >= 128) return launch<T, NA, MA, GATED, 256, 256, 2, 4, 64, 2>(g, stream);
    return launch<T, NA, MA, GATED, 128, 128, 2, 2, 64, 2>(g, stream);
}

template <typename T>
int run(const Gemm &g, hipStream_t stream) {
    if (g.gated) return by_size<T, false, false, true>(g, stream);
    if (!g.n[0].across) return by_size<T, false, false, false>(g, stream);
    if (!g.m[0].across) return by_size<T, true, false, false>(g, stream);
    return by_size<T, true, true, false>(g, stream);
}

// Rows and columns of an operand as it is stored.
struct Shape {
    int64_t rows, cols;
};
Shape shape_of(const Operand &o, int64_t r, int64_t K) { return o.across ? Shape{K, r} : Shape{r, K}; }

// Do the rows start on 16-byte boundaries (a single row needs no pitch)?
bool rows_aligned(const Operand &o, const Shape &s) { return aligned(o.p, 16) && (s.rows <= 1 || o.ld % 8 == 0); }

// Visits the operands of a product with the length of their rows' axis.
template <typename F>
int each_operand(Gemm &g, F &&f) {
    const int nm = std::max(g.parts, g.batch), nn = g.gated ? 2 : g.parts;
    // the two of a side share one pitch, so both are copied if one is
    bool cm = false, cn = false;
    for (int i = 0; i < nm; ++i) cm |= !rows_aligned(g.m[i], shape_of(g.m[i], g.M, g.K));
    for (int i = 0; i < nn; ++i) cn |= !rows_aligned(g.n[i], shape_of(g.n[i], g.N, g.K));
    for (int i = 0; i < nm && cm; ++i)
        if (int rc = f(g.m[i], shape_of(g.m[i], g.M, g.K))) return rc;
    for (int i = 0; i < nn && cn; ++i)
        if (int rc = f(g.n[i], shape_of(g.n[i], g.N, g.K))) return rc;
    return SA_OK;
}

int64_t aligned_pitch(const Shape &s) { return round_up(s.cols, 8); }

}  // namespace

size_t gemm_workspace(const Gemm &g0) {
    Gemm g = g0;
    size_t need = 0;
    if (g.M == 0 || g.N == 0) return 0;
    each_operand(g, [&](Operand &, const Shape &s) {
        need += (size_t)round_up(s.rows * aligned_pitch(s) * 2, 256);
        return SA_OK;
    });
    return need;
}

int gemm(const Gemm &g0, void *ws, hipStream_t stream) {
    Gemm g = g0;
    if (g.M == 0 || g.N == 0) return SA_OK;
    uint8_t *at = static_cast<uint8_t *>(ws);
    int rc = each_operand(g, [&](Operand &o, const Shape &s) {
        const int64_t ldo = aligned_pitch(s), chunks = s.rows * (ldo / 8);
        if (chunks > 0) {
            // the element's type does not matter to a copy
            hipLaunchKernelGGL(k_align_rows<_Float16>, dim3((unsigned)std::min<int64_t>((chunks + 255) / 256, 8192)), dim3(256), 0,
                               stream, static_cast<const _Float16 *>(o.p), o.ld, s.rows, (int)s.cols,
                               reinterpret_cast<_Float16 *>(at), ldo);
            if (int e = check_hip(hipGetLastError(), "k_align_rows")) return e;
        }
        o.p = at;
        o.ld = ldo;
        at += round_up(s.rows * ldo * 2, 256);
        return SA_OK;
    });
    if (rc) return rc;
    // a single row has no pitch: one of whole chunks keeps the loads' ranges whole
    const int64_t mr = g.m[0].across ? g.K : g.M, nr = g.n[0].across ? g.K : g.N;
    for (int i = 0; i < 2; ++i) {
        if (mr <= 1) g.m[i].ld = round_up(g.m[0].across ? g.M : g.K, 8);
        if (nr <= 1) g.n[i].ld = round_up(g.n[0].across ? g.N : g.K, 8);
    }
    return g.type == SA_BF16 ? run<__bf16>(g, stream) : run<_Float16>(g, stream);
}

}  // namespace sa
