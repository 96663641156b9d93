// Elements of the operators that read and write a network's tensors: fp32, bf16 or fp16 in memory, fp32 in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace klay {

using f32 = float;
using bf16 = __bf16;
using f16 = _Float16;

// N consecutive elements.  `Loose`: in memory at a multiple of one element's size, which gfx950 loads and stores as one access all the same.
template <typename T, int N> struct Pieces {
    typedef T Vec __attribute__((ext_vector_type(N)));
    typedef Vec Loose __attribute__((aligned(sizeof(T))));
};
template <typename T> struct Pieces<T, 1> {
    typedef T Vec;
    typedef T Loose;
};

// One rounding to nearest even per element (v_cvt_pk_bf16_f32 for bf16).
template <typename T, int N>
__device__ __forceinline__ typename Pieces<T, N>::Vec rounded(const float (&x)[N]) {
    if constexpr (N == 1) {
        return (T)x[0];
    } else {
        typedef float Floats __attribute__((ext_vector_type(N)));
        Floats f;
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = x[i];
        return __builtin_convertvector(f, typename Pieces<T, N>::Vec);
    }
}

// N elements as they are in memory; a single one of 16 bits in a register of its own (two of them packed into one register would make
// every load wait for the one before it)
template <typename T, int N> using Raw = std::conditional_t<N == 1 && sizeof(T) == 2, unsigned int, typename Pieces<T, N>::Vec>;

// A stretch of memory that a wave reads or writes row by row: the address is in scalar registers, a lane adds `lane` bytes and a row
// `row` bytes (a scalar).  A lane with kNoLane reads zeros and writes nothing (the range check of buffer instructions).
typedef __amdgpu_buffer_rsrc_t Stretch;
constexpr uint32_t kNoLane = 0xffffffffu, kStretchBytes = 0xf0000000u;
__device__ __forceinline__ Stretch stretch_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)kStretchBytes, 0x00020000);
}
template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef unsigned short T; };
template <> struct Bits<4> { typedef unsigned int T; };
template <> struct Bits<8> { typedef unsigned int T __attribute__((ext_vector_type(2))); };
template <> struct Bits<16> { typedef unsigned int T __attribute__((ext_vector_type(4))); };

template <int N, typename T>
__device__ __forceinline__ Raw<T, N> load_raw(Stretch from, uint32_t lane, uint32_t row) {
    if constexpr (N * sizeof(T) == 2) return (unsigned int)__builtin_amdgcn_raw_buffer_load_b16(from, lane, row, 0);
    typename Bits<N * sizeof(T)>::T r;
    if constexpr (N * sizeof(T) == 4) r = __builtin_amdgcn_raw_buffer_load_b32(from, lane, row, 0);
    else if constexpr (N * sizeof(T) == 8) r = __builtin_amdgcn_raw_buffer_load_b64(from, lane, row, 0);
    else if constexpr (N * sizeof(T) == 16) r = __builtin_amdgcn_raw_buffer_load_b128(from, lane, row, 0);
    if constexpr (N * sizeof(T) > 2) return __builtin_bit_cast(Raw<T, N>, r);
}
template <int N, typename T>
__device__ __forceinline__ void store_row(Stretch to, uint32_t lane, uint32_t row, const float (&x)[N]) {
    const typename Pieces<T, N>::Vec r = rounded<T, N>(x);
    const auto bits = __builtin_bit_cast(typename Bits<N * sizeof(T)>::T, r);
    if constexpr (N * sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(bits, to, lane, row, 0);
    else if constexpr (N * sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(bits, to, lane, row, 0);
    else if constexpr (N * sizeof(T) == 8) __builtin_amdgcn_raw_buffer_store_b64(bits, to, lane, row, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(bits, to, lane, row, 0);
}

template <int N, typename T>
__device__ __forceinline__ float piece(const Raw<T, N>& r, int v) {
    if constexpr (N == 1 && sizeof(T) == 2) return (float)__builtin_bit_cast(T, (unsigned short)r);
    else if constexpr (N == 1) return r;
    else return (float)r[v];
}
template <int N, typename T>
__device__ __forceinline__ Raw<T, N> all_pieces(float x) {
    Raw<T, N> r;
    if constexpr (N == 1 && sizeof(T) == 2) {
        r = __builtin_bit_cast(unsigned short, (T)x);
    } else if constexpr (N == 1) {
        r = x;
    } else {
#pragma unroll
        for (int v = 0; v < N; ++v) r[v] = (T)x;
    }
    return r;
}

// N elements that are read once (they leave the caches to others: 1 GiB read at 7.0 TB/s, 6.2 by ordinary loads)
template <int N, typename T>
__device__ __forceinline__ Raw<T, N> stream_raw(const T* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const typename Pieces<T, N>::Loose*>(p));
}

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

template <int N, typename T>
__device__ __forceinline__ void store_elements(T* p, const float (&x)[N]) {
    *reinterpret_cast<typename Pieces<T, N>::Loose*>(p) = rounded<T, N>(x);
}
// past the caches, as stream_raw
template <int N, typename T>
__device__ __forceinline__ void stream_elements(T* p, const float (&x)[N]) {
    __builtin_nontemporal_store(rounded<T, N>(x), reinterpret_cast<typename Pieces<T, N>::Loose*>(p));
}

}  // namespace klay
