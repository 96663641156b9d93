// Elements of the operators that read and write a network's tensors: fp32, bf16 or fp16 in memory, fp32 in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace klay {

using f32 = float;
using bf16 = __bf16;
using f16 = _Float16;

// N consecutive elements at p as floats.  `Aligned` says that p is a multiple of the N elements' size (a power of two up to 16 bytes);
// otherwise p is a multiple of one element's size only, which the memory pipeline of gfx950 takes in the same single access.
template <typename T, int N> struct Pieces {
    typedef T Vec __attribute__((ext_vector_type(N)));
    typedef Vec Loose __attribute__((aligned(sizeof(T))));
};
template <typename T> struct Pieces<T, 1> {
    typedef T Vec;
    typedef T Loose;
};

template <int N, typename T>
__device__ __forceinline__ void load_elements(float (&x)[N], const T* p) {
    if constexpr (N == 1) {
        x[0] = (float)*p;
    } else {
        const typename Pieces<T, N>::Vec v = *reinterpret_cast<const typename Pieces<T, N>::Loose*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)v[i];
    }
}

// One rounding to nearest even per element (v_cvt_pk_bf16_f32 for bf16).
template <int N, typename T>
__device__ __forceinline__ void store_elements(T* p, const float (&x)[N]) {
    if constexpr (N == 1) {
        *p = (T)x[0];
    } else {
        typedef float Floats __attribute__((ext_vector_type(N)));
        Floats f;
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = x[i];
        *reinterpret_cast<typename Pieces<T, N>::Loose*>(p) = __builtin_convertvector(f, typename Pieces<T, N>::Vec);
    }
}

}  // namespace klay
