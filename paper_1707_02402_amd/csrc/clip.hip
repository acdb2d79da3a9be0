// The norm of many gradient tensors together, and the gradients scaled down to a largest norm.
//   norm = sqrt(sum over all tensors of g^2);  out = g * (max_norm / norm if norm is finite and > max_norm, else 1)
// The squares are added up in fp64: no fp32 gradient over- or underflows there, and the order (fixed) hardly matters.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"

using dynb::fail;

namespace {

constexpr int CLIP_GRID = 1024;

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double room[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}

// sum of one tensor's squares, workgroup by workgroup, on top of what is there
template <typename T>
__global__ __launch_bounds__(256) void k_squares(const T* __restrict__ g, int64_t n, double* __restrict__ partial, int first)
{
    double s = 0.0;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(CLIP_GRID) * 256) { const double v = double(load_f32(g + i)); s += v * v; }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = (first ? 0.0 : partial[blockIdx.x]) + s;
}

__global__ __launch_bounds__(256) void k_norm_of(const double* __restrict__ partial, float* __restrict__ norm, int none)
{
    double s = 0.0;
    if (!none)
        for (int i = threadIdx.x; i < CLIP_GRID; i += 256) s += partial[i];
    s = block_sum(s);
    if (threadIdx.x == 0) *norm = float(sqrt(s));
}

template <typename T>
__global__ __launch_bounds__(256) void k_scale(const T* g, T* out, int64_t n, const float* __restrict__ norm, float max_norm)
{
    const float v = *norm;
    const float factor = v > max_norm && v < INFINITY ? max_norm / v : 1.f;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(CLIP_GRID) * 256) store_f32(out + i, load_f32(g + i) * factor);
}

}  // namespace

extern "C" size_t dynb_clip_workspace_bytes(void) { return CLIP_GRID * sizeof(double); }

extern "C" int dynb_clip_gradients(const dynb_grad_tensor* tensors, int32_t n, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (n < 0 || (n > 0 && !tensors) || !norm || !workspace) return fail(DYNB_E_INVAL, "dynb_clip_gradients: NULL argument or negative number of tensors");
    if (!(max_norm > 0.f)) return fail(DYNB_E_INVAL, "dynb_clip_gradients: max_norm must be positive");
    if (workspace_bytes < dynb_clip_workspace_bytes()) return fail(DYNB_E_WORKSPACE, "dynb_clip_gradients: workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, "dynb_clip_gradients: workspace not 256-byte aligned");
    for (int i = 0; i < n; ++i) {
        const dynb_grad_tensor& t = tensors[i];
        if (t.count < 0 || (t.count > 0 && !t.grad)) return fail(DYNB_E_INVAL, "dynb_clip_gradients: tensor " + std::to_string(i) + " has no data");
        if (t.dtype != DYNB_F32 && t.dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, "dynb_clip_gradients: tensor " + std::to_string(i) + " has an unknown dtype");
        if ((reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.out)) & (t.dtype == DYNB_BF16 ? 1 : 3))
            return fail(DYNB_E_INVAL, "dynb_clip_gradients: tensor " + std::to_string(i) + " is misaligned");
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    int first = 1;
    for (int i = 0; i < n; ++i) {
        const dynb_grad_tensor& t = tensors[i];
        if (t.count == 0) continue;
        if (t.dtype == DYNB_BF16) hipLaunchKernelGGL((k_squares<bf16_t>), dim3(CLIP_GRID), dim3(256), 0, st, static_cast<const bf16_t*>(t.grad), t.count, partial, first);
        else hipLaunchKernelGGL((k_squares<float>), dim3(CLIP_GRID), dim3(256), 0, st, static_cast<const float*>(t.grad), t.count, partial, first);
        first = 0;
    }
    hipLaunchKernelGGL(k_norm_of, dim3(1), dim3(256), 0, st, partial, norm, first);
    for (int i = 0; i < n; ++i) {
        const dynb_grad_tensor& t = tensors[i];
        if (t.count == 0 || !t.out) continue;
        if (t.dtype == DYNB_BF16) hipLaunchKernelGGL((k_scale<bf16_t>), dim3(CLIP_GRID), dim3(256), 0, st, static_cast<const bf16_t*>(t.grad), static_cast<bf16_t*>(t.out), t.count, norm, max_norm);
        else hipLaunchKernelGGL((k_scale<float>), dim3(CLIP_GRID), dim3(256), 0, st, static_cast<const float*>(t.grad), static_cast<float*>(t.out), t.count, norm, max_norm);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_clip_gradients: ") + hipGetErrorString(e));
    return DYNB_OK;
}
