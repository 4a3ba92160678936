// Vectors of fp32, bf16 and fp16 values in global memory, for the kernels that take all three.
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace l1csr {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// the values of a 16-byte access
template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);

// V values at any alignment of T (the hardware takes unaligned 16-byte accesses)
template <typename T, int V>
__device__ __forceinline__ void load_values(const T *p, T (&x)[V]) {
    __builtin_memcpy(x, p, sizeof(T) * V);
}
// Loads that are used once and leave the caches to what is read again
template <typename T, int V>
__device__ __forceinline__ void load_past(const T *p, T (&x)[V]) {
    constexpr int bytes = (int)sizeof(T) * V;
    static_assert(bytes % 4 == 0, "whole words");
    typedef unsigned words __attribute__((ext_vector_type(bytes / 4), aligned(2)));
    const words w = __builtin_nontemporal_load(reinterpret_cast<const words *>(p));
    __builtin_memcpy(x, &w, bytes);
}
template <typename T, int V>
__device__ __forceinline__ void store_values(T *p, const T (&x)[V]) {
    __builtin_memcpy(p, x, sizeof(T) * V);
}

// The first n of V values (what is past them reads as 0)
template <typename T, int V>
__device__ __forceinline__ void load_some(const T *p, int64_t n, T (&x)[V]) {
    if (n >= V) {
        load_values<T, V>(p, x);
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = v < n ? p[v] : (T)0.f;
}
template <typename T, int V>
__device__ __forceinline__ void store_some(T *p, int64_t n, const T (&x)[V]) {
    if (n >= V) {
        store_values<T, V>(p, x);
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v < n) p[v] = x[v];
}

// Stores past the caches, for results that would only displace what is read
template <typename T, int V>
__device__ __forceinline__ void store_past(T *p, const T (&x)[V]) {
    constexpr int bytes = (int)sizeof(T) * V;
    if constexpr (bytes % 4 == 0) {
        typedef unsigned words __attribute__((ext_vector_type(bytes / 4), aligned(2)));
        words w;
        __builtin_memcpy(&w, x, bytes);
        __builtin_nontemporal_store(w, reinterpret_cast<words *>(p));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) __builtin_nontemporal_store(x[i], p + i);
    }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// element types of the calls' arguments as types: f(A{}, B{}) for two of them, the second fp32 or the first's
template <typename F>
hipError_t with_types(int first, int second, F f) {
    const bool same = first == second;
    if (first == kTypeF32) return f(float{}, float{});
    if (first == kTypeBF16) return same ? f(__bf16{}, __bf16{}) : f(__bf16{}, float{});
    return same ? f(_Float16{}, _Float16{}) : f(_Float16{}, float{});
}

}  // namespace l1csr
