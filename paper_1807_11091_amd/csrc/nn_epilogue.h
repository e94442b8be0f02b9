// From the sums of a matrix product to its results: bias, pre-activations kept,
// activation, gate, residual.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "nn_gemm.h"
#include "nn_types.h"

namespace sa {
namespace {

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

// V (the first cnt < V at a row's end) results to p; past: 16-bit ones past the caches.
template <bool PAST, typename E, int V>
__device__ inline void put_results(E *p, int cnt, const float (&v)[V], int past) {
    if (cnt < V) {
        store_part<E, V>(p, cnt, v);
    } else if (PAST && sizeof(E) == 2 && past) {
        // an empty statement on either side keeps the compiler from merging the branches, which
        // drops the hint
        asm volatile("" ::"n"(0));
        typedef E vec __attribute__((ext_vector_type(V)));
        typedef vec loose __attribute__((aligned(alignof(E))));
        vec x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (E)v[i];  // round to nearest even
        __builtin_nontemporal_store(x, reinterpret_cast<loose *>(p));
        asm volatile("" ::"n"(1));
    } else {
        store_vec<E, V>(p, v);
    }
}

// V (cnt < V at a row's end) results z to Y.
template <typename T, int V, bool PAST = false>
__device__ inline void put_values(const Epilogue &e, void *Y, int64_t m, int64_t n, int cnt, const float (&z)[V]) {
    if (e.out_f32) put_results<PAST>(reinterpret_cast<float *>(Y) + m * e.ldy + n, cnt, z, e.past);
    else put_results<PAST>(reinterpret_cast<T *>(Y) + m * e.ldy + n, cnt, z, e.past);
}

// V (cnt < V at a row's end) consecutive results, in z, from their sums z (and u); the
// pre-activations are stored.
template <typename T, bool GATED, int V, bool PAST = false>
__device__ inline void finish_values(const Epilogue &e, int64_t m, int64_t n, int cnt, float (&z)[V], float (&u)[V],
                                     const Addends<T, V> &with) {
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
    if (e.Z) put_results<PAST>(reinterpret_cast<T *>(e.Z) + m * e.ldz + n, cnt, z, e.past);
    if (e.act != SA_ACT_NONE) activate<false, V>(e.act, z, z, z);
    if constexpr (GATED) {
        if (e.bias2)
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] += with.bias2[i];
        if (e.Z2) put_results<PAST>(reinterpret_cast<T *>(e.Z2) + m * e.ldz + n, cnt, u, e.past);
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
}

template <typename T, bool GATED, int V>
__device__ inline void finish(const Epilogue &e, void *Y, int64_t m, int64_t n, int cnt, float (&z)[V], float (&u)[V],
                              const Addends<T, V> &with) {
    finish_values<T, GATED, V>(e, m, n, cnt, z, u, with);
    put_values<T, V>(e, Y, m, n, cnt, z);
}

template <typename T, bool GATED, int V>
__device__ inline void finish(const Epilogue &e, void *Y, int64_t m, int64_t n, int cnt, float (&z)[V], float (&u)[V]) {
    Addends<T, V> with;
    with.has_r = false;
    with.load_bias(e, n, cnt);
    finish<T, GATED, V>(e, Y, m, n, cnt, z, u, with);
}

}  // namespace
}  // namespace sa
