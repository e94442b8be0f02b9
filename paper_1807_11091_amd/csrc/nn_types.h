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

// 1 / (1 + exp(-z)) with the hardware's reciprocal, which is within an ulp; a value
// below the smallest normal number becomes 0.
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

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

// act(z) and, if asked for, act'(z).  The tanh form uses z/2 (1 + tanh q) = z sigmoid(2q).
// The choice of the activation stands outside the loop over the values, so that their
// chains of exponential and reciprocal run side by side.
template <bool SLOPE, int V>
__device__ inline void activate(int act, const float (&z)[V], float (&value)[V], float (&slope)[V]) {
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < V; ++i) f(z[i], value[i], slope[i]);
    };
    switch (act) {
    case SA_ACT_RELU:
        each([](float x, float &v, float &s) {
            v = x <= 0.0f ? 0.0f : x;
            if (SLOPE) s = x <= 0.0f ? 0.0f : (x > 0.0f ? 1.0f : x);
        });
        return;
    case SA_ACT_SIGMOID:
        each([](float x, float &v, float &s) {
            v = sigmoid(x);
            if (SLOPE) s = v * (1.0f - v);
        });
        return;
    case SA_ACT_SILU:
        each([](float x, float &v, float &s) {
            const float p = sigmoid(x);
            v = x * p;
            if (SLOPE) s = p * (1.0f + x * (1.0f - p));
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
        each([](float x, float &v, float &s) {
            const float p = sigmoid(kTwoSqrt2OverPi * (x + kGeluCubic * x * x * x));
            v = x * p;
            if (SLOPE) {
                s = p + x * (p * (1.0f - p)) * (kTwoSqrt2OverPi * (1.0f + 3.0f * kGeluCubic * x * x));
                if (fabsf(x) > 30.0f) {  // the limits; x * x overflows further out
                    v = x > 0.0f ? x : 0.0f;
                    s = x > 0.0f ? 1.0f : 0.0f;
                }
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
