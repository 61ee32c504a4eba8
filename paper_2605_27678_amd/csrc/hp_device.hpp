// What the operators' kernels share: element types, vectors of them as they lie
// in memory, and reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hp_error.hpp"

namespace hp {

constexpr int kWave = 64;
constexpr int kComputeUnits = 256;      // of an MI355X

inline bool hip_failed(hipError_t e) {
    if (e == hipSuccess) return false;
    note_hip_error((int)e);
    return true;
}

template <class T, int N> struct VecOf {
    typedef T type __attribute__((ext_vector_type(N)));
    // element-aligned only: gfx950 loads and stores of any width take any address
    typedef T mem __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T> struct VecOf<T, 1> { typedef T type; typedef T mem; };
template <class T, int N> using Vec = typename VecOf<T, N>::type;

// N elements, the first `valid` of them from memory and zeros behind (valid may be <= 0 or >= N)
template <int N, class T> __device__ __forceinline__ Vec<T, N> load(const T *p, int valid) {
    Vec<T, N> v;
    if constexpr (N == 1) {
        v = valid >= 1 ? *p : (T)0.0f;
    } else if (valid >= N) {
        v = *(const typename VecOf<T, N>::mem *)p;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < valid ? p[i] : (T)0.0f;
    }
    return v;
}

template <int N, class T> __device__ __forceinline__ void store(T *p, Vec<T, N> v, int valid) {
    if constexpr (N == 1) {
        if (valid >= 1) *p = v;
    } else if (valid >= N) {
        *(typename VecOf<T, N>::mem *)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = v[i];
    }
}

template <int N, class T> __device__ __forceinline__ float at(const Vec<T, N> &v, int i) {
    if constexpr (N == 1) return (float)v;
    else return (float)v[i];
}

template <int N, class T> __device__ __forceinline__ void put(Vec<T, N> &v, int i, float x) {
    if constexpr (N == 1) v = (T)x;      // to nearest even
    else v[i] = (T)x;
}

// Buffers for loads that write LDS themselves, or that bring zeros from beyond the end: an offset that is always outside,
// and the wait for all of a wave's loads but the last `loads`.
constexpr uint32_t kOutside = 0x80000000u;
constexpr int but(int loads) { return (loads & 15) | 0x0f70 | (loads >> 4) << 14; }            // s_waitcnt vmcnt(loads)

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = kWave / 2; d; d /= 2) x += __shfl_xor(x, d);
    return x;
}

}  // namespace hp
