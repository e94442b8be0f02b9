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

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
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
            const float p = 0.5f * (1.0f + erff(x * kSqrtHalf));
            v = x * p;
            if (SLOPE) s = p + x * (kInvSqrt2Pi * __expf(-0.5f * x * x));
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
