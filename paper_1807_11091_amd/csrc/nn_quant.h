// 8-bit floating point (e4m3) with a binary32 scale for each block: device helpers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "structadmm.h"

namespace sa {
namespace {

constexpr int kBlock = SA_BLOCK;  // columns of a block

// The scale of a block whose largest magnitude (NaN left out) is amax: amax / 448, the largest
// code, and at least the smallest normal number, which keeps its reciprocal finite.  The
// quotient is a product with the rounded reciprocal and one step with the exact remainder,
// which rounds it as a division does, for a third of the instructions: a tile of
// quantisation divides twice for each of its rows and columns.
__device__ inline float block_scale(float amax) {
    constexpr float r = 1.0f / 448.0f;
    const float q = amax * r, s = fmaf(fmaf(-q, 448.0f, amax), r, q);
    return amax < __builtin_inff() ? fmaxf(s, 0x1p-126f) : amax;
}

// 1 / scale in the same way; 0 of an infinite one.
__device__ inline float block_inverse(float s) {
    const float r = __builtin_amdgcn_rcpf(s);
    return s < __builtin_inff() ? fmaf(fmaf(-s, r, 1.0f), r, r) : 0.0f;
}

// Largest magnitude of V values; a NaN does not count.
template <int V>
__device__ inline float largest(const float (&v)[V]) {
    float a = fabsf(v[0]);
#pragma unroll
    for (int i = 1; i < V; ++i) a = fmaxf(a, fabsf(v[i]));
    return fmaxf(a, 0.0f);  // all of them NaN
}

// Largest over lanes that differ in the given bits of their number.
template <int FROM, int TO>
__device__ inline float lanes_max(float a) {
#pragma unroll
    for (int off = FROM; off < TO; off <<= 1) a = fmaxf(a, __shfl_xor(a, off, 64));
    return a;
}

// Codes of 8 values, value * inv to nearest even.  |v| * inv is at most 448 up to rounding,
// far below where the conversion leaves the range (464); infinities come as NaN.
__device__ inline uint2 codes8(const float (&v)[8], float inv) {
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    return make_uint2((unsigned)lo, (unsigned)hi);
}

// The first n of 8 codes to p, which is 8-byte aligned; past the caches.
__device__ inline void store_codes(uint8_t *p, int n, uint2 c) {
    if (n >= 8) {
        __builtin_nontemporal_store((uint64_t)c.y << 32 | c.x, reinterpret_cast<uint64_t *>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p[i] = (uint8_t)((i < 4 ? c.x : c.y) >> i % 4 * 8);
    }
}

// Sixteen neighbouring lanes hold the 128 columns of a row's block, 8 each, zeros past the
// row's end; n: of this lane's columns, those inside the row (0 and less: none).
__device__ inline void quantise_row(const float (&v)[8], int n, uint8_t *codes, float *scale) {
    const float s = block_scale(lanes_max<1, 16>(largest(v)));
    if (n <= 0) return;
    store_codes(codes, n, codes8(v, block_inverse(s)));
    if ((threadIdx.x & 15) == 0) *scale = s;
}

}  // namespace
}  // namespace sa
