// The gate of a gated layer: f(g) = g sigma(p), p = g (a + b g^2).  SiLU: a = 1, b = 0.  GELU in its tanh form, g (1 + tanh(c (g + 0.044715 g^3))) / 2 with c = sqrt(2 / pi):
// a = 2 c, b = 0.044715 a, since (1 + tanh(x)) / 2 = sigma(2 x).      f'(g) = sigma + g sigma (1 - sigma) (a + 3 b g^2)
// g^2 is taken of g kept within +-10^4: nothing overflows there, and beyond, sigma is 0 or 1 in fp32 either way.  f(-infinity) is NaN, as -infinity * 0 is.
#pragma once

#include "device_utils.h"

namespace {

struct GateForm {
    float a2, b2;             // a and b, times -log2(e): what exp2 takes
    float a, b3;              // a and 3 b
};
struct GateValue { float f, slope; };

__device__ __forceinline__ float within_1e4(float g) { return __builtin_amdgcn_fmed3f(g, -1e4f, 1e4f); }
// sigma: a reciprocal and an exponential to 1 ulp each, 2^-22 (2 + |p|) relative in all; what follows is rounded to 8 bits
__device__ __forceinline__ float gate_sigma(const GateForm& k, float g, float c2)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * (k.a2 + k.b2 * c2)));
}
__device__ __forceinline__ float gate_f(const GateForm& k, float g)
{
    const float c = within_1e4(g);
    return g * gate_sigma(k, g, c * c);
}
__device__ __forceinline__ float gate_silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f)); }
__device__ __forceinline__ GateValue gate_both(const GateForm& k, float g)
{
    const float c = within_1e4(g), c2 = c * c, s = gate_sigma(k, g, c2), w = k.a + k.b3 * c2;
    return GateValue{g * s, s + s * (c * (w - s * w))};
}

// What a gated layer keeps of its forward pass: gate and up of row r at pre + r * stride and h further on, in bfloat16 or in 8 bits with their scales
enum Keep { KEEP_NOTHING, KEEP_BF16, KEEP_8 };

struct NoGate { static constexpr bool ON = false; };
struct Gate {
    static constexpr bool ON = true;
    GateForm form;
    int h, keep;              // features of either part
    void* pre;
    int64_t pre_stride;
    bf16_t* scale;            // row r's blocks of gate at scale + r * scale_stride, up's blocks(h) further on
    int64_t scale_stride;
    bf16_t* hidden;           // backward: f(gate) up, or null
    int64_t hidden_stride;
    bool past;                // results go past the caches
    bool on_16;               // rows kept in 8 bits lie on borders of 16 bytes
    __device__ __forceinline__ int blocks() const { return (h + 31) / 32; }
};
template <int KEEP_> struct GateKeeping : Gate { static constexpr int KEEP = KEEP_; };         // ... in a kernel that is made for one way of keeping

}  // namespace
