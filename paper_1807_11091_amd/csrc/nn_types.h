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

__device__ inline float sigmoid(float z) { return 1.0f / (1.0f + __expf(-z)); }

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// act(z); the tanh form uses z/2 (1 + tanh q) = z / (1 + exp(-2q)).
__device__ inline float act_value(int act, float z) {
    switch (act) {
    case SA_ACT_RELU: return z <= 0.0f ? 0.0f : z;
    case SA_ACT_SIGMOID: return sigmoid(z);
    case SA_ACT_SILU: return z / (1.0f + __expf(-z));
    case SA_ACT_GELU: return 0.5f * z * (1.0f + erff(z * kSqrtHalf));
    case SA_ACT_GELU_TANH: return z / (1.0f + __expf(-kTwoSqrt2OverPi * (z + kGeluCubic * z * z * z)));
    default: return z;
    }
}

// act(z) and act'(z)
__device__ inline void act_both(int act, float z, float &value, float &slope) {
    switch (act) {
    case SA_ACT_RELU:
        value = z <= 0.0f ? 0.0f : z;
        slope = z <= 0.0f ? 0.0f : (z > 0.0f ? 1.0f : z);
        return;
    case SA_ACT_SIGMOID: {
        const float p = sigmoid(z);
        value = p;
        slope = p * (1.0f - p);
        return;
    }
    case SA_ACT_SILU: {
        const float p = sigmoid(z);
        value = z * p;
        slope = p * (1.0f + z * (1.0f - p));
        return;
    }
    case SA_ACT_GELU: {
        const float p = 0.5f * (1.0f + erff(z * kSqrtHalf));
        value = z * p;
        slope = p + z * (kInvSqrt2Pi * __expf(-0.5f * z * z));
        return;
    }
    case SA_ACT_GELU_TANH: {
        if (fabsf(z) > 30.0f) {  // the limits; z * z overflows further out
            value = z > 0.0f ? z : 0.0f;
            slope = z > 0.0f ? 1.0f : 0.0f;
            return;
        }
        const float p = sigmoid(kTwoSqrt2OverPi * (z + kGeluCubic * z * z * z));
        value = z * p;
        slope = p + z * (p * (1.0f - p)) * (kTwoSqrt2OverPi * (1.0f + 3.0f * kGeluCubic * z * z));
        return;
    }
    default:
        value = z;
        slope = 1.0f;
    }
}

}  // namespace sa
