// Small device helpers shared by the kernels of this library (gfx950 only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

typedef uint16_t bf16_t;   // raw bfloat16 bits

__device__ __forceinline__ float bf16_to_f32(bf16_t v) { return __uint_as_float(uint32_t(v) << 16); }

// round to nearest even; NaN stays NaN
__device__ __forceinline__ bf16_t f32_to_bf16(float f)
{
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return bf16_t((u >> 16) | 0x40u);
    u += 0x7fffu + ((u >> 16) & 1u);
    return bf16_t(u >> 16);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// two floats -> packed bf16 pair, round to nearest even (one v_cvt_pk_bf16_f32 on gfx950)
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// ReLU on a packed bf16 pair: a negative bf16 is a negative int16, so a signed max with 0 clears it
__device__ __forceinline__ uint32_t relu_bf16x2(uint32_t p)
{
    const i16x2 z = {0, 0};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, p), z));
}

template <typename T> __device__ __forceinline__ float load_f32(const T* p);
template <> __device__ __forceinline__ float load_f32<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load_f32<bf16_t>(const bf16_t* p) { return bf16_to_f32(*p); }

template <typename T> __device__ __forceinline__ void store_f32(T* p, float v);
template <> __device__ __forceinline__ void store_f32<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void store_f32<bf16_t>(bf16_t* p, float v) { *p = f32_to_bf16(v); }

// the value a tensor of type T would hold after storing v
template <typename T> __device__ __forceinline__ float round_to(float v);
template <> __device__ __forceinline__ float round_to<float>(float v) { return v; }
template <> __device__ __forceinline__ float round_to<bf16_t>(float v) { return bf16_to_f32(f32_to_bf16(v)); }

// Every store of this wave has been answered by the L2.  A workgroup-scope release and a barrier order a workgroup's accesses for its own
// waves and do not wait for this: without it a wave may come to the barrier with its stores under way, and the agent-scope release of
// another wave behind the barrier waits for that wave's only.
__device__ __forceinline__ void wait_for_stores()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");    // (the compiler, too, keeps earlier stores ahead of what follows)
    __builtin_amdgcn_s_waitcnt(0x0f70);                       // vmcnt(0)
}

// What this workgroup stored (each wave behind wait_for_stores and a barrier) is in memory, where every CU can see it: one thread calls this, then raises
// the flag.  The wait is written out, because an atomic with a release of its own does without it here: the compiler finds no load or store between the
// wait above and the atomic, does not count the write-back as one, and leaves out the wait behind it, so that the flag could be seen while the write-back was
// under way, and other L2s' workgroups read what memory held before.
__device__ __forceinline__ void release_to_chip()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");        // writes the L2's dirty lines back
    __builtin_amdgcn_s_waitcnt(0x0f70);                       // vmcnt(0): it has been answered
}
