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

// a piece without its first n elements of bfloat16 (0 to 8), zeros behind the others
__device__ __forceinline__ u32x4 without_first(const u32x4& v, int n)
{
    uint64_t lo = uint64_t(v[1]) << 32 | v[0], hi = uint64_t(v[3]) << 32 | v[2];
    lo = n >= 4 ? hi : lo;
    hi = n >= 4 ? 0 : hi;
    const int bits = (n & 3) * 16;
    lo = lo >> bits | hi << 1 << (63 - bits);
    hi >>= bits;
    return n >= 8 ? u32x4{0u, 0u, 0u, 0u} : u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
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

// Large results go past the caches and leave those to what is read meanwhile: from PAST bytes on, half of what the 256 MB of the memory's own cache take beside the operands.
// Smaller ones are read from there by the next call, and leave as usual.  With the readers of a training step behind it a gated layer gains at every size from PAST on (64 MB of out:
// 815 -> 797 us, 128: 1478 -> 1456, 256: 2888 -> 2850); rows out of 8 bits and layer norm's dx gain by themselves (65536 x 1024 bf16, 128 MB: dx 74 -> 58 us) and lose with a reader right
// behind them up to 128 MB (dx and back into 8 bits 107 -> 115; 64 MB 53 -> 57; 256 MB 217 -> 216).  Which of the two a caller has cannot be seen from a call.
// put(std::true_type) stores past them, put(std::false_type) does not; `past` is the same for all lanes, MAY false: it never is.  (The compiler would make one store of the two, and an ordinary one.)
constexpr int64_t PAST = 64 << 20;
template <bool MAY = true, class F>
__device__ __forceinline__ void put_past(bool past, F put)
{
    if constexpr (!MAY) put(std::false_type{});
    else if (past) {
        asm volatile("; past the caches" ::: "memory");
        put(std::true_type{});
        asm volatile("" ::: "memory");
    } else put(std::false_type{});
}

// a piece of 16 bytes past the caches, at any element's address
__device__ __forceinline__ void store_past(bf16_t* p, const float (&v)[8])
{
    __builtin_nontemporal_store(u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])}, reinterpret_cast<u32x4_at2*>(p));
}
__device__ __forceinline__ void store_past(float* p, const float (&v)[4])
{
    __builtin_nontemporal_store(u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, reinterpret_cast<u32x4_at4*>(p));
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
