// Rows of channels in 16-byte pieces, for the kernels that take rows of any
// width and alignment (scram_norm.hip, scram_rotary.hip).  Memory takes vectors
// at any element's address.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_device.h"

namespace scram {
namespace {

template <typename T>
constexpr int kChunk = 16 / static_cast<int>(sizeof(T));  // channels of a chunk of X

// V channels at any element's address.
template <typename T, int V>
using vec = T __attribute__((ext_vector_type(V), aligned(sizeof(T))));

template <typename T>
__device__ __forceinline__ float to_float(T x)
{
    if constexpr (std::is_same<T, float>::value)
        return x;
    else
        return __uint_as_float(static_cast<uint32_t>(x) << 16);
}

template <typename T>
__device__ __forceinline__ T from_float(float x)
{
    if constexpr (std::is_same<T, float>::value)
        return x;
    else
        return static_cast<T>(f32_to_bf16_rne(x));
}

// N channels at `row` into x from element o on (o a multiple of N below V, the same for every thread).
template <int N, typename T, int V>
__device__ __forceinline__ void load_piece(const T* row, int o, vec<T, V>& x)
{
    const vec<T, N> y = *reinterpret_cast<const vec<T, N>*>(row + o);
#pragma unroll
    for (int q = 0; q < V; q += N)
#pragma unroll
        for (int j = 0; j < N; ++j) x[q + j] = q == o ? static_cast<T>(y[j]) : static_cast<T>(x[q + j]);
}

template <int N, typename T, int V>
__device__ __forceinline__ void store_piece(T* row, int o, const vec<T, V>& x)
{
    vec<T, N> y(T(0));
#pragma unroll
    for (int q = 0; q < V; q += N)
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = q == o ? static_cast<T>(x[q + j]) : static_cast<T>(y[j]);
    *reinterpret_cast<vec<T, N>*>(row + o) = y;
}

template <typename T, int V>
__device__ __forceinline__ vec<T, V> load_vec(const T* p)
{
    return *reinterpret_cast<const vec<T, V>*>(p);
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, vec<T, V> x)
{
    *reinterpret_cast<vec<T, V>*>(p) = x;
}

// The first n < V channels at p (n the same for every thread that gets here), in pieces of 4, 2 and 1; zeros after them.
template <typename T, int V>
__device__ __forceinline__ vec<T, V> load_part(const T* p, int n)
{
    vec<T, V> x(T(0));
    if constexpr (V > 4)
        if (n & 4) load_piece<4, T, V>(p, 0, x);
    if (n & 2) load_piece<2, T, V>(p, n & 4, x);
    if (n & 1) load_piece<1, T, V>(p, n & 6, x);
    return x;
}

template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, int n, const vec<T, V>& x)
{
    if constexpr (V > 4)
        if (n & 4) store_piece<4, T, V>(p, 0, x);
    if (n & 2) store_piece<2, T, V>(p, n & 4, x);
    if (n & 1) store_piece<1, T, V>(p, n & 6, x);
}

}  // namespace
}  // namespace scram
