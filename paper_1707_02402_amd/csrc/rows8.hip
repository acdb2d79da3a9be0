// Rows into 8 bits and back (the format: rows8.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"
#include "rows.h"
#include "rows8.h"

using dynb::fail;

namespace {

// A lane has 8 elements of a block, four neighbouring lanes a block.
template <typename T>
__global__ __launch_bounds__(256) void k_store8(const T* __restrict__ x, int64_t x_stride, int8_t* __restrict__ q, int64_t q_stride, bf16_t* __restrict__ scale, int64_t scale_stride, int d,
                                                int pieces, int64_t all)
{
    constexpr int P = PIECE<T>, N = 8 / P;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / pieces;
        const int c = int(i - row * pieces) * 8, left = d - c;
        const T* const from = x + row * x_stride + c;
        float v[8];
        uint32_t largest = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            u32x4 raw = {0u, 0u, 0u, 0u};
            if (left > n * P) raw = load_piece(from + n * P, left - n * P);
#pragma unroll
            for (int j = 0; j < P; ++j) largest = max(largest, magnitude(v[n * P + j] = element<T>(raw, j)));
        }
        largest = max(largest, uint32_t(__shfl_xor(int(largest), 1)));
        largest = max(largest, uint32_t(__shfl_xor(int(largest), 2)));
        const Scale8 s = scale8(largest);
        if (left > 0) {
            store_eight(q + row * q_stride + c, left, u32x2{pack8(v[0], v[1], v[2], v[3], s.inv), pack8(v[4], v[5], v[6], v[7], s.inv)});
            if (c % BLOCK8 == 0) scale[row * scale_stride + c / BLOCK8] = scale8_bits(s);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_load8(const int8_t* __restrict__ q, int64_t q_stride, const bf16_t* __restrict__ scale, int64_t scale_stride, T* __restrict__ x, int64_t x_stride, int d,
                                               int pieces, int64_t all, bool past)
{
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / pieces;
        const int c = int(i - row * pieces) * 8, left = d - c;
        const u32x2 raw = load_eight(q + row * q_stride + c, left);
        const float s = bf16_to_f32(scale[row * scale_stride + c / BLOCK8]);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = unpack8(raw[j >> 2], j & 3) * s;
        T* const to = x + row * x_stride + c;
        put_past(past, [&](auto past_) {
            if (decltype(past_)::value && sizeof(T) == 2 && left >= 8) {
                const u32x4 packed = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
                __builtin_nontemporal_store(packed, reinterpret_cast<u32x4_at2*>(to));
            } else store_piece<8>(to, left, v);
        });
    }
}

int check(const dynb_rows8_shape* s, const void* x, int64_t x_stride, const dynb_rows8* r, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    const int d = s->d, dtype = s->dtype;
    if (s->T < 0 || d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (dtype != DYNB_F32 && dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    if (d > 1 << 28) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^28 columns");
    if (s->T == 0) return DYNB_OK;
    if (!x || !r || !r->q || !r->scale) return fail(DYNB_E_INVAL, who + ": NULL argument");
    if (x_stride < d || r->q_stride < d || r->scale_stride < (int64_t(d) + BLOCK8 - 1) / BLOCK8) return fail(DYNB_E_INVAL, who + ": rows overlap (stride below their length)");
    if ((reinterpret_cast<uintptr_t>(x) & (dtype == DYNB_BF16 ? 1 : 3)) || (reinterpret_cast<uintptr_t>(r->scale) & 1)) return fail(DYNB_E_INVAL, who + ": misaligned pointer");
    return DYNB_OK;
}
int launched(const char* who)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    return DYNB_OK;
}
constexpr int64_t MOST_GROUPS = 1 << 16;

}  // namespace

extern "C" int dynb_store8(const dynb_rows8_shape* s, const void* x, int64_t x_stride, const dynb_rows8* rows, void* stream)
{
    const int rc = check(s, x, x_stride, rows, "dynb_store8");
    if (rc != DYNB_OK || s->T == 0) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int d = s->d, pieces = (d + 31) / 32 * 4;                      // whole blocks: the four lanes of one belong together
    const int64_t all = int64_t(s->T) * pieces;
    const dim3 grid(unsigned(std::min((all + 255) / 256, MOST_GROUPS)));
    if (s->dtype == DYNB_BF16) hipLaunchKernelGGL((k_store8<bf16_t>), grid, dim3(256), 0, st, static_cast<const bf16_t*>(x), x_stride, static_cast<int8_t*>(rows->q), rows->q_stride, static_cast<bf16_t*>(rows->scale), rows->scale_stride, d, pieces, all);
    else hipLaunchKernelGGL((k_store8<float>), grid, dim3(256), 0, st, static_cast<const float*>(x), x_stride, static_cast<int8_t*>(rows->q), rows->q_stride, static_cast<bf16_t*>(rows->scale), rows->scale_stride, d, pieces, all);
    return launched("dynb_store8");
}

extern "C" int dynb_load8(const dynb_rows8_shape* s, const dynb_rows8* rows, void* x, int64_t x_stride, void* stream)
{
    const int rc = check(s, x, x_stride, rows, "dynb_load8");
    if (rc != DYNB_OK || s->T == 0) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int d = s->d, pieces = (d + 7) / 8;
    const int64_t all = int64_t(s->T) * pieces;
    const bool past = s->dtype == DYNB_BF16 && int64_t(s->T) * d * 2 >= PAST;               // (fp32: a lane's 32 bytes are two stores, 100 us past the caches where 62 do)
    const dim3 grid(unsigned(std::min((all + 255) / 256, MOST_GROUPS)));
    if (s->dtype == DYNB_BF16) hipLaunchKernelGGL((k_load8<bf16_t>), grid, dim3(256), 0, st, static_cast<const int8_t*>(rows->q), rows->q_stride, static_cast<const bf16_t*>(rows->scale), rows->scale_stride, static_cast<bf16_t*>(x), x_stride, d, pieces, all, past);
    else hipLaunchKernelGGL((k_load8<float>), grid, dim3(256), 0, st, static_cast<const int8_t*>(rows->q), rows->q_stride, static_cast<const bf16_t*>(rows->scale), rows->scale_stride, static_cast<float*>(x), x_stride, d, pieces, all, past);
    return launched("dynb_load8");
}
