// Element types of the operators on learned tables and layers, and loads and
// stores of runs of elements.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sqn.h"

namespace sqn {

inline size_t element_size(int32_t dtype) { return dtype == SQN_F32 ? 4 : 2; }

template <typename T>
__device__ __forceinline__ float to_f32(T v)
{
    return static_cast<float>(v);
}

// rounded to nearest, ties to even
template <typename T>
__device__ __forceinline__ T from_f32(float v)
{
    return static_cast<T>(v);
}

// N elements moved as one access of their total width.  The alignment is an
// element's: rows of any length and stride are read this way, and the vector
// memory path takes wide accesses at any element boundary.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Run {
    uint32_t word[N * sizeof(T) / 4];
};

template <typename T, int N>
__device__ __forceinline__ void load_run(const T* p, float v[N])
{
    if constexpr (N == 1) {
        v[0] = to_f32(*p);
    } else {
        const Run<T, N> r = *reinterpret_cast<const Run<T, N>*>(p);
        T e[N];
        __builtin_memcpy(e, &r, sizeof(e));
#pragma unroll
        for (int k = 0; k < N; ++k)
            v[k] = to_f32(e[k]);
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const float v[N])
{
    if constexpr (N == 1) {
        *p = from_f32<T>(v[0]);
    } else {
        T e[N];
#pragma unroll
        for (int k = 0; k < N; ++k)
            e[k] = from_f32<T>(v[k]);
        Run<T, N> r;
        __builtin_memcpy(&r, e, sizeof(e));
        *reinterpret_cast<Run<T, N>*>(p) = r;
    }
}

}  // namespace sqn
