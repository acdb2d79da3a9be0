// Rows of bf16 or fp32 elements in pieces of 16 bytes a lane, at any address and of any length.
#pragma once

#include <type_traits>

#include "device_utils.h"

// 16 bytes at an address of any element: global memory takes such an access whole (a lane pays for a second line where its piece crosses one)
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));

template <typename T> constexpr int PIECE = 16 / int(sizeof(T));   // elements of a piece

// left: elements that are there from p on (any number, also none)
template <typename T> __device__ __forceinline__ u32x4 load_piece(const T* p, int left);
template <> __device__ __forceinline__ u32x4 load_piece<bf16_t>(const bf16_t* p, int left)
{
    if (left >= 8) return *reinterpret_cast<const u32x4_at2*>(p);
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) v[i >> 1] |= uint32_t(p[i]) << (16 * (i & 1));
    return v;
}
template <> __device__ __forceinline__ u32x4 load_piece<float>(const float* p, int left)
{
    if (left >= 4) return *reinterpret_cast<const u32x4_at4*>(p);
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) v[i] = __float_as_uint(p[i]);
    return v;
}

// the same in pieces of E elements: 8 bytes of bfloat16 (E = 4), or 16
template <typename T, int E> using Piece = std::conditional_t<(E * sizeof(T) == 8), u32x2, u32x4>;
template <int E, typename T> __device__ __forceinline__ Piece<T, E> load_some(const T* p, int left)
{
    if constexpr (E * sizeof(T) == 8) {
        typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
        if (left >= 4) return *reinterpret_cast<const u32x2_at2*>(p);
        u32x2 v = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < left) v[i >> 1] |= uint32_t(p[i]) << (16 * (i & 1));
        return v;
    } else
        return load_piece(p, left);
}

template <typename T> __device__ __forceinline__ float element(const u32x2& v, int i)
{
    static_assert(sizeof(T) == 2, "eight bytes of bfloat16");
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
}
template <typename T> __device__ __forceinline__ float element(const u32x4& v, int i);
template <> __device__ __forceinline__ float element<bf16_t>(const u32x4& v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
template <> __device__ __forceinline__ float element<float>(const u32x4& v, int i) { return __uint_as_float(v[i]); }

// N floats (4 or 8) to p; left as above
template <int N> __device__ __forceinline__ void store_piece(float* p, int left, const float* v)
{
    if (left >= N) {
#pragma unroll
        for (int j = 0; j < N; j += 4)
            *reinterpret_cast<u32x4_at4*>(p + j) = u32x4{__float_as_uint(v[j]), __float_as_uint(v[j + 1]), __float_as_uint(v[j + 2]), __float_as_uint(v[j + 3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
        if (i < left) p[i] = v[i];
}
template <int N> __device__ __forceinline__ void store_piece(bf16_t* p, int left, const float* v)
{
    typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
    if (left >= N) {
        if constexpr (N == 8)
            *reinterpret_cast<u32x4_at2*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        else
            *reinterpret_cast<u32x2_at2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
        if (i < left) p[i] = f32_to_bf16(v[i]);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
