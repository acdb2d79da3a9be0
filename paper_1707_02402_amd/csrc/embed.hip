// Token embeddings: rows of a table by token, scaled, and the table's gradient.
//   out[t] = scale * table[tokens[t]]              dtable[v] = scale * sum over t with tokens[t] = v of dout[t]
// A token outside [0, V) (padding) has a row of zeros and gives no gradient.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"

using dynb::fail;

namespace {

template <typename T>
__global__ __launch_bounds__(256) void k_embed(const int32_t* __restrict__ tokens, const T* __restrict__ table, T* __restrict__ out, int V, int d,
                                               int64_t out_stride, float scale)
{
    const int32_t tok = tokens[blockIdx.x];
    const bool known = tok >= 0 && tok < V;
    const T* const from = table + size_t(known ? tok : 0) * size_t(d);
    T* const to = out + int64_t(blockIdx.x) * out_stride;
    for (int c = threadIdx.x; c < d; c += 256) store_f32(to + c, known ? load_f32(from + c) * scale : 0.f);
}

// one workgroup for 256 columns of a row of the table: it looks through all tokens in their order
template <typename T, typename TG>
__global__ __launch_bounds__(256) void k_embed_grad(const int32_t* __restrict__ tokens, const T* __restrict__ dout, TG* __restrict__ dtable, int n, int d,
                                                    int64_t dout_stride, float scale)
{
    __shared__ int32_t tok[256];
    const int v = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
    float sum = 0.f;
    for (int t0 = 0; t0 < n; t0 += 256) {
        const int t = t0 + int(threadIdx.x);
        tok[threadIdx.x] = t < n ? tokens[t] : -1;
        __syncthreads();
        for (int i = 0; i < min(256, n - t0); ++i)
            if (tok[i] == v && c < d) sum += load_f32(dout + int64_t(t0 + i) * dout_stride + c);
        __syncthreads();
    }
    if (c < d) store_f32(dtable + size_t(v) * size_t(d) + c, sum * scale);
}

int check(const dynb_embed_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->T < 0 || s->V <= 0 || s->d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_F32 && s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    return DYNB_OK;
}
bool misaligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == DYNB_BF16 ? 1 : 3)) != 0; }

}  // namespace

extern "C" int dynb_embed(const dynb_embed_shape* s, const int32_t* tokens, const void* table, void* out, int64_t out_stride, void* stream)
{
    const int rc = check(s, "dynb_embed");
    if (rc != DYNB_OK) return rc;
    if (s->T == 0) return DYNB_OK;
    if (!tokens || !table || !out) return fail(DYNB_E_INVAL, "dynb_embed: NULL argument");
    if (out_stride < s->d) return fail(DYNB_E_INVAL, "dynb_embed: rows overlap (stride below d)");
    if (misaligned(tokens, DYNB_F32) || misaligned(table, s->dtype) || misaligned(out, s->dtype)) return fail(DYNB_E_INVAL, "dynb_embed: misaligned pointer");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (s->dtype == DYNB_BF16)
        hipLaunchKernelGGL((k_embed<bf16_t>), dim3(unsigned(s->T)), dim3(256), 0, st, tokens, static_cast<const bf16_t*>(table), static_cast<bf16_t*>(out), s->V, s->d, out_stride, s->scale);
    else
        hipLaunchKernelGGL((k_embed<float>), dim3(unsigned(s->T)), dim3(256), 0, st, tokens, static_cast<const float*>(table), static_cast<float*>(out), s->V, s->d, out_stride, s->scale);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_embed: ") + hipGetErrorString(e));
    return DYNB_OK;
}

extern "C" size_t dynb_embed_backward_workspace_bytes(const dynb_embed_shape* s)
{
    if (check(s, "dynb_embed_backward_workspace_bytes") != DYNB_OK) return 0;
    return 256;
}

extern "C" int dynb_embed_backward(const dynb_embed_shape* s, const int32_t* tokens, const void* dout, int64_t dout_stride, void* dtable, int32_t grad_dtype,
                                   void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check(s, "dynb_embed_backward");
    if (rc != DYNB_OK) return rc;
    if (grad_dtype != DYNB_F32 && grad_dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, "dynb_embed_backward: unknown dtype of the gradient");
    if (!dtable || !workspace || (s->T > 0 && (!tokens || !dout))) return fail(DYNB_E_INVAL, "dynb_embed_backward: NULL argument");
    if (dout_stride < s->d) return fail(DYNB_E_INVAL, "dynb_embed_backward: rows overlap (stride below d)");
    if (workspace_bytes < dynb_embed_backward_workspace_bytes(s)) return fail(DYNB_E_WORKSPACE, "dynb_embed_backward: workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, "dynb_embed_backward: workspace not 256-byte aligned");
    if (misaligned(tokens, DYNB_F32) || misaligned(dout, s->dtype) || misaligned(dtable, grad_dtype)) return fail(DYNB_E_INVAL, "dynb_embed_backward: misaligned pointer");
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid(unsigned(s->V), unsigned((s->d + 255) / 256));
    auto launch = [&](auto in, auto grad) {
        using T = decltype(in);
        using TG = decltype(grad);
        hipLaunchKernelGGL((k_embed_grad<T, TG>), grid, dim3(256), 0, st, tokens, static_cast<const T*>(dout), static_cast<TG*>(dtable), s->T, s->d, dout_stride, s->scale);
    };
    if (s->dtype == DYNB_BF16 && grad_dtype == DYNB_BF16) launch(bf16_t{}, bf16_t{});
    else if (s->dtype == DYNB_BF16) launch(bf16_t{}, float{});
    else if (grad_dtype == DYNB_BF16) launch(float{}, bf16_t{});
    else launch(float{}, float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_embed_backward: ") + hipGetErrorString(e));
    return DYNB_OK;
}
