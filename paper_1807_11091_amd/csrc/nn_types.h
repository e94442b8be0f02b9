// Element types, unaligned vector loads and stores, and the activations of the
// feed-forward operators.  All arithmetic is binary32; a value is rounded to a
// 16-bit type once, when it is stored.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "structadmm.h"

namespace sa {

template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

// V elements from anywhere an element may lie: gfx950 loads and stores 16 bytes
// at any address, so rows of odd pitch need no path of their own.
template <typename T, int V>
__device__ inline void load_vec(const T *p, float (&v)[V]) {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec x;
    __builtin_memcpy(&x, p, sizeof x);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)x[i];
}

template <typename T, int V>
__device__ inline void store_vec(T *p, const float (&v)[V]) {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (T)v[i];  // round to nearest even
    __builtin_memcpy(p, &x, sizeof x);
}

// The first n < V elements only (0 elsewhere).
template <typename T, int V>
__device__ inline void load_part(const T *p, int n, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
}

template <typename T, int V>
__device__ inline void store_part(T *p, int n, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) p[i] = (T)v[i];
}

// Sum over the 64 lanes of a wavefront in a fixed order; every lane receives it.
__device__ inline float wave_sum_f32(float x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

// The logistic function s(y) = 1 / (1 + exp(-y)) without a difference from 1 and without
// an exponential that overflows: with e = exp(-|y| / 2) and q = 1 / (1 + e^2),
// s(|y|) = q, s(-|y|) = e^2 q and s'(y) = (e q)^2.  e and not e^2, so that a product with
// both factors e keeps its bits down to the smallest normal number.
struct Logistic {
    float e, q;
    __device__ explicit Logistic(float y) {
        e = __expf(fabsf(y) * -0.5f);
        q = __builtin_amdgcn_rcpf(fmaf(e, e, 1.0f));  // within an ulp
    }
    __device__ float at(float y) const { return y < 0.0f ? e * (e * q) : q; }
    // x s(y) for x and y of one sign = max(x, 0) - |x| s(-|y|), given xe = x e, in which x
    // is bounded from above: at infinity it is 0, and the value infinity
    __device__ float times(float x, float xe) const { return fmaf(-fabsf(xe), e * q, fmaxf(x, 0.0f)); }
    static __device__ float bounded(float x) { return fminf(x, 128.0f); }
};
// s(y) for y > -87, below which the reciprocal has no normal result
__device__ inline float plain_logistic(float y) { return __builtin_amdgcn_rcpf(1.0f + __expf(-y)); }

constexpr float kInvSqrt2Pi = 0.39894228040143268f;

// The normal distribution's Phi(x) = P(X <= x), without the difference 1 - erf of its
// lower tail.  With a = |x| and e = exp(-x^2 / 4), Phi(-a) = e^2 h(a), where
// h(a) = exp(a^2 / 2) Phi(-a) falls smoothly from 1/2 to 1 / (a sqrt(2 pi)): t = 1 / (1 + a/4)
// times a polynomial in t of degree 9, fitted for the least relative error (3.4e-8; 4e-7 with
// the roundings of its evaluation).  e and not e^2, so that products with e * e keep their
// bits down to the smallest normal number (x = -13.1).  A product of 8192 x 4096 x 1024
// bfloat16 with it takes 105 us, with erff 118.
struct NormalTail {
    float e, h, xe;  // xe: x e, and 0 at +infinity
    __device__ explicit NormalTail(float x) {
        e = __expf(x * x * -0.25f);
        xe = fminf(x, 64.0f) * e;
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.25f, 1.0f));
        constexpr float c[] = {0.0997355655f, 0.0997364298f, 0.0934663564f, 0.0816031024f,  0.0589751787f,
                               0.0636990219f, -0.03171736f,  0.0955969095f, -0.0808772147f, 0.0197819863f};
        float s = c[9];
#pragma unroll
        for (int k = 8; k >= 0; --k) s = fmaf(s, t, c[k]);
        h = s * t;
    }
    // x Phi(x) = max(x, 0) - |x| Phi(-|x|), and its derivative; no branch
    __device__ float value(float x) const { return fmaxf(x, 0.0f) - fabsf(xe * (e * h)); }
    __device__ float slope(float x) const {
        const float tail = e * e * h;
        return fmaf(xe, e * kInvSqrt2Pi, x < 0.0f ? tail : 1.0f - tail);
    }
};

constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;
__device__ inline float gelu_tanh_y(float x) { return kTwoSqrt2OverPi * (x + kGeluCubic * x * x * x); }

// act(z) and, if asked for, act'(z).  The tanh form uses z/2 (1 + tanh q) = z sigmoid(2q).
// The choice of the activation stands outside the loop over the values, so that their
// chains of exponential and reciprocal run side by side.
template <bool SLOPE, int V>
__device__ inline void activate(int act, const float (&z)[V], float (&value)[V], float (&slope)[V]) {
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < V; ++i) f(z[i], value[i], slope[i]);
    };
    // Values alone need the careful form of s(y) only near the end of its range: silu over
    // 8192 x 4096 results of a product of 1024 terms 94.6 us with it everywhere, 87.4 so.
    auto any_below = [&](float bound) {
        float least = z[0];
#pragma unroll
        for (int i = 1; i < V; ++i) least = fminf(least, z[i]);
        return least < bound;
    };
    switch (act) {
    case SA_ACT_RELU:
        each([](float x, float &v, float &s) {
            v = x <= 0.0f ? 0.0f : x;
            if (SLOPE) s = x <= 0.0f ? 0.0f : (x > 0.0f ? 1.0f : x);
        });
        return;
    case SA_ACT_SIGMOID:
        if (!SLOPE && !any_below(-80.0f)) return each([](float x, float &v, float &) { v = plain_logistic(x); });
        each([](float x, float &v, float &s) {
            const Logistic l(x);
            v = l.at(x);
            if (SLOPE) s = (l.e * l.q) * (l.e * l.q);
        });
        return;
    case SA_ACT_SILU:
        if (!SLOPE && !any_below(-80.0f)) return each([](float x, float &v, float &) { v = x * plain_logistic(x); });
        each([](float x, float &v, float &s) {
            const Logistic l(x);
            const float xe = Logistic::bounded(x) * l.e;
            v = l.times(x, xe);
            if (SLOPE) s = fmaf(xe * l.q, l.e * l.q, l.at(x));
        });
        return;
    case SA_ACT_GELU:
        each([](float x, float &v, float &s) {
            const NormalTail tail(x);
            v = tail.value(x);
            if (SLOPE) s = tail.slope(x);
        });
        return;
    case SA_ACT_GELU_TANH:
        if (!SLOPE && !any_below(-9.0f)) return each([](float x, float &v, float &) { v = x * plain_logistic(gelu_tanh_y(x)); });
        each([](float x, float &v, float &s) {
            const float y = gelu_tanh_y(x);
            const Logistic l(y);
            if (!SLOPE) {
                v = l.times(x, Logistic::bounded(x) * l.e);
            } else {  // the limits at both infinities; x * x does not overflow
                const float b = fmaxf(Logistic::bounded(x), -128.0f);
                v = l.times(x, b * l.e);
                s = fmaf(b * l.e * l.q, l.e * l.q * (kTwoSqrt2OverPi * (1.0f + 3.0f * kGeluCubic * b * b)), l.at(y));
            }
        });
        return;
    default:
        each([](float x, float &v, float &s) {
            v = x;
            if (SLOPE) s = 1.0f;
        });
    }
}

}  // namespace sa
