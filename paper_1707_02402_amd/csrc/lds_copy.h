// Rows on their way from memory straight into LDS, and the waits that go with them.
#pragma once

#include "device_utils.h"

// A unit: 64 rows x 64 channels of a matrix, copied without registers on the way.  Eight neighbouring lanes copy 128 bytes of a row, in their order (in any other a
// request is answered lane by lane, 13.5 bytes a clock instead of 64); a unit is eight blocks of 8 rows.  What an LDS pass of a fragment's read takes
// together, 16 of its 32 rows (lanes 0-3, 12-15, 20-23, 24-27 or the others), are two rows of every block, an even and an odd one, and the blocks are 16 bytes
// further apart than their size: all banks.
constexpr int XBLOCK = 1040, XUNIT = 8 * XBLOCK;
// the row of its fragment (lane / 32) that lane `lane` copies into block `block`
__device__ __forceinline__ int copied_row(int block, int lane)
{
    const int odd = lane >> 3 & 1, g = lane >> 4 & 1;
    return (block >> 1) * 8 + (g ^ (block >> 1 & 1) ^ (block >> 2 & 1)) * 4 + (block & 1) * 2 + odd;
}
// where in a unit lane q + 32 hk reads row q of the first fragment (the second lies 512 bytes further), its half of K-step 0 (each next one 32 bytes further)
__device__ __forceinline__ uint32_t fragment_at(int q, int hk)
{
    return uint32_t(((q >> 3) * 2 + (q >> 1 & 1)) * XBLOCK + (((q >> 2 ^ q >> 3 ^ q >> 4) & 1) * 2 + (q & 1)) * 128 + hk * 16);
}
template <bool ONCE = false>                                   // ONCE: nobody else wants these bytes, they need not stay in any cache
__device__ __forceinline__ void lds_copy16(const char* base, uint32_t off, uint32_t lds_at)   // 64 lanes x 16 bytes -> LDS at lds_at, lane after lane
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    asm volatile("" : "+s"(base), "+v"(off));                                      // (a scalar base and a lane's offset, and no address of 64 bits per lane kept for every request)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(base + off),
                                     (__attribute__((address_space(3))) uint32_t*)(lds_raw + lds_at), 16, 0, ONCE ? 2 : 0);
}
using lds_ptr = __attribute__((address_space(3))) unsigned char*;
__device__ __forceinline__ void lds_copy16_to(const char* base, uint32_t off, lds_ptr lds)
{
    asm volatile("" : "+s"(base), "+v"(off));
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(base + off), (__attribute__((address_space(3))) uint32_t*)lds, 16, 0, 0);
}
// *p by the scalar unit: the address is the same for the whole wave, and nobody writes there during the kernel
__device__ __forceinline__ int32_t uniform_load(const int32_t* p)
{
    return __builtin_amdgcn_readfirstlane(*(const __attribute__((address_space(4))) int32_t*)(p));
}
// All but this wave's newest N requests and stores have been answered
template <int N> __device__ __forceinline__ void answered_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// (Not __syncthreads, which waits for all requests into LDS)
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
