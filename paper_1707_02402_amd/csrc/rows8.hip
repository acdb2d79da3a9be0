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

// A lane has 8 elements of a block, four neighbouring lanes a block, who exchange their largest.  A row is read once and what is written is half of it or a quarter: memory bounds it
// (65536 x 1024: bf16 35 us, 200 MB at 5.9 TB/s, fp32 57, 338 MB at 5.8).
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

// A lane has what one store of 16 bytes takes, so that the stores of a wave lie side by side; large results go past the caches (65536 x 1024: bf16 31 us, 6.6 TB/s; fp32 47, 7.2, where 8
// elements a lane, in two stores, took 62, and past the caches 100; rows of 1001: 33 and 52).
template <typename T>
__global__ __launch_bounds__(256) void k_load8(const int8_t* __restrict__ q, int64_t q_stride, const bf16_t* __restrict__ scale, int64_t scale_stride, T* __restrict__ x, int64_t x_stride, int d,
                                               int pieces, int64_t all, bool past)
{
    constexpr int P = PIECE<T>;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / pieces;
        const int c = int(i - row * pieces) * P, left = d - c;
        const int8_t* const from = q + row * q_stride + c;
        u32x2 raw;
        if constexpr (P == 8) raw = load_eight(from, left);
        else raw = u32x2{load_four(from, left), 0u};
        const float s = bf16_to_f32(scale[row * scale_stride + c / BLOCK8]);
        float v[P];
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = unpack8(raw[j >> 2], j & 3) * s;
        T* const to = x + row * x_stride + c;
        put_past(past, [&](auto past_) {
            if (decltype(past_)::value && left >= P) store_past(to, v);
            else store_piece<P>(to, left, v);
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
    const int d = s->d, piece = s->dtype == DYNB_BF16 ? 8 : 4, pieces = (d + piece - 1) / piece;
    const int64_t all = int64_t(s->T) * pieces;
    const bool past = int64_t(s->T) * d * (s->dtype == DYNB_BF16 ? 2 : 4) >= PAST;
    const dim3 grid(unsigned(std::min((all + 255) / 256, MOST_GROUPS)));
    if (s->dtype == DYNB_BF16) hipLaunchKernelGGL((k_load8<bf16_t>), grid, dim3(256), 0, st, static_cast<const int8_t*>(rows->q), rows->q_stride, static_cast<const bf16_t*>(rows->scale), rows->scale_stride, static_cast<bf16_t*>(x), x_stride, d, pieces, all, past);
    else hipLaunchKernelGGL((k_load8<float>), grid, dim3(256), 0, st, static_cast<const int8_t*>(rows->q), rows->q_stride, static_cast<const bf16_t*>(rows->scale), rows->scale_stride, static_cast<float*>(x), x_stride, d, pieces, all, past);
    return launched("dynb_load8");
}
