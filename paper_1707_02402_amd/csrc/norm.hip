// Layer norm of rows and its gradients.
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) r gamma + beta
//   g = dy gamma, h = (x - m) r:  dx = r (g - mean(g) - h mean(g h)),  dgamma = sum over the rows of dy h,  dbeta = of dy
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"

using dynb::fail;

namespace {

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// of all 256 threads
__device__ __forceinline__ float group_sum(float v, float* room)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm(const T* __restrict__ x, int64_t x_stride, const float* __restrict__ gamma, const float* __restrict__ beta,
                                              T* __restrict__ y, int64_t y_stride, float* __restrict__ mean, float* __restrict__ rstd, int d, float eps)
{
    __shared__ float room[4];
    const T* const from = x + int64_t(blockIdx.x) * x_stride;
    T* const to = y + int64_t(blockIdx.x) * y_stride;
    float s = 0.f;
    for (int c = threadIdx.x; c < d; c += 256) s += load_f32(from + c);
    const float m = group_sum(s, room) / float(d);
    s = 0.f;
    for (int c = threadIdx.x; c < d; c += 256) { const float v = load_f32(from + c) - m; s += v * v; }
    const float r = 1.f / sqrtf(group_sum(s, room) / float(d) + eps);
    for (int c = threadIdx.x; c < d; c += 256)
        store_f32(to + c, (load_f32(from + c) - m) * r * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
    if (threadIdx.x == 0) {
        if (mean) mean[blockIdx.x] = m;
        if (rstd) rstd[blockIdx.x] = r;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_dx(const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, const float* __restrict__ gamma,
                                                 const float* __restrict__ mean, const float* __restrict__ rstd, T* __restrict__ dx, int64_t dx_stride, int d)
{
    __shared__ float room[4];
    const int64_t t = blockIdx.x;
    const float m = mean[t], r = rstd[t];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < d; c += 256) {
        const float g = load_f32(dy + t * dy_stride + c) * (gamma ? gamma[c] : 1.f), h = (load_f32(x + t * x_stride + c) - m) * r;
        s1 += g;
        s2 += g * h;
    }
    s1 = group_sum(s1, room) / float(d);
    s2 = group_sum(s2, room) / float(d);
    for (int c = threadIdx.x; c < d; c += 256) {
        const float g = load_f32(dy + t * dy_stride + c) * (gamma ? gamma[c] : 1.f), h = (load_f32(x + t * x_stride + c) - m) * r;
        store_f32(dx + t * dx_stride + c, r * (g - s1 - h * s2));
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_dparams(const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride, const float* __restrict__ mean,
                                                      const float* __restrict__ rstd, float* __restrict__ dgamma, float* __restrict__ dbeta, int n, int d)
{
    __shared__ float room[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sg = 0.f, sb = 0.f;
    if (c < d)
        for (int64_t t = wave; t < n; t += 4) {
            const float v = load_f32(dy + t * dy_stride + c);
            sg += v * (load_f32(x + t * x_stride + c) - mean[t]) * rstd[t];
            sb += v;
        }
    room[0][wave][lane] = sg;
    room[1][wave][lane] = sb;
    __syncthreads();
    if (wave != 0 || c >= d) return;
    if (dgamma) dgamma[c] = (room[0][0][lane] + room[0][1][lane]) + (room[0][2][lane] + room[0][3][lane]);
    if (dbeta) dbeta[c] = (room[1][0][lane] + room[1][1][lane]) + (room[1][2][lane] + room[1][3][lane]);
}

int check(const dynb_norm_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->T < 0 || s->d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (!(s->eps >= 0.f)) return fail(DYNB_E_INVAL, who + ": eps must not be negative");
    if (s->dtype != DYNB_F32 && s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    return DYNB_OK;
}
bool misaligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == DYNB_BF16 ? 1 : 3)) != 0; }

}  // namespace

extern "C" int dynb_layer_norm(const dynb_norm_shape* s, const void* x, int64_t x_stride, const float* gamma, const float* beta, void* y, int64_t y_stride,
                               float* mean, float* rstd, void* stream)
{
    const int rc = check(s, "dynb_layer_norm");
    if (rc != DYNB_OK) return rc;
    if (s->T == 0) return DYNB_OK;
    if (!x || !y) return fail(DYNB_E_INVAL, "dynb_layer_norm: NULL argument");
    if (x_stride < s->d || y_stride < s->d) return fail(DYNB_E_INVAL, "dynb_layer_norm: rows overlap (stride below d)");
    if (misaligned(x, s->dtype) || misaligned(y, s->dtype) || misaligned(gamma, DYNB_F32) || misaligned(beta, DYNB_F32) || misaligned(mean, DYNB_F32) ||
        misaligned(rstd, DYNB_F32))
        return fail(DYNB_E_INVAL, "dynb_layer_norm: misaligned pointer");
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto in) {
        using T = decltype(in);
        hipLaunchKernelGGL((k_norm<T>), dim3(unsigned(s->T)), dim3(256), 0, st, static_cast<const T*>(x), x_stride, gamma, beta, static_cast<T*>(y), y_stride, mean, rstd, s->d, s->eps);
    };
    if (s->dtype == DYNB_BF16) launch(bf16_t{});
    else launch(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_layer_norm: ") + hipGetErrorString(e));
    return DYNB_OK;
}

extern "C" size_t dynb_layer_norm_backward_workspace_bytes(const dynb_norm_shape* s)
{
    if (check(s, "dynb_layer_norm_backward_workspace_bytes") != DYNB_OK) return 0;
    return 256;
}

extern "C" int dynb_layer_norm_backward(const dynb_norm_shape* s, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const float* gamma, const float* mean,
                                        const float* rstd, void* dx, int64_t dx_stride, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check(s, "dynb_layer_norm_backward");
    if (rc != DYNB_OK) return rc;
    if (!workspace || (s->T > 0 && (!dy || !x || !mean || !rstd))) return fail(DYNB_E_INVAL, "dynb_layer_norm_backward: NULL argument");
    if (dy_stride < s->d || x_stride < s->d || (dx && dx_stride < s->d)) return fail(DYNB_E_INVAL, "dynb_layer_norm_backward: rows overlap (stride below d)");
    if (workspace_bytes < dynb_layer_norm_backward_workspace_bytes(s)) return fail(DYNB_E_WORKSPACE, "dynb_layer_norm_backward: workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, "dynb_layer_norm_backward: workspace not 256-byte aligned");
    if (misaligned(dy, s->dtype) || misaligned(x, s->dtype) || misaligned(dx, s->dtype) || misaligned(gamma, DYNB_F32) || misaligned(mean, DYNB_F32) ||
        misaligned(rstd, DYNB_F32) || misaligned(dgamma, DYNB_F32) || misaligned(dbeta, DYNB_F32))
        return fail(DYNB_E_INVAL, "dynb_layer_norm_backward: misaligned pointer");
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto in) {
        using T = decltype(in);
        const T *a = static_cast<const T*>(dy), *b = static_cast<const T*>(x);
        if (dx && s->T > 0) hipLaunchKernelGGL((k_norm_dx<T>), dim3(unsigned(s->T)), dim3(256), 0, st, a, dy_stride, b, x_stride, gamma, mean, rstd, static_cast<T*>(dx), dx_stride, s->d);
        if (dgamma || dbeta)
            hipLaunchKernelGGL((k_norm_dparams<T>), dim3(unsigned((s->d + 63) / 64)), dim3(256), 0, st, a, dy_stride, b, x_stride, mean, rstd, dgamma, dbeta, s->T, s->d);
    };
    if (s->dtype == DYNB_BF16) launch(bf16_t{});
    else launch(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_layer_norm_backward: ") + hipGetErrorString(e));
    return DYNB_OK;
}
