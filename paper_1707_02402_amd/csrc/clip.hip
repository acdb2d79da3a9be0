// The norm of many gradient tensors together, and the gradients scaled down to a largest norm.
//   norm = sqrt(sum over all tensors of g^2);  out = g * (max_norm / norm if norm is finite and > max_norm, else 1)
// The squares are added up in fp64: the square of no fp32 number over- or underflows there.
//
// Two passes, the second of which starts where the first one ended (the last 256 MB that went by are still in the cache beside the memory).  Both
// take the tensors as one row of chunks; a launch's list of up to CLIP_LIST tensors comes with its arguments, so that a call neither copies nor keeps a table.
// The norm itself has no launch: every workgroup of the second pass adds up the first one's partial sums, in one order.
//
// Bound by memory: 2 GB of bfloat16 in 12 tensors 350 us (5.7 TB/s) and 768 (5.2 TB/s of what is read and written).  240 tensors of 56 MB in all are two lists, so four
// launches: 8 us each for the squares, 12 for the scaling, of which the bytes account for 24 in all.  Many small tensors are bound by their lists' launches: 1000 of 1000
// elements are eight lists, 88 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"
#include "rows.h"

using dynb::fail;

namespace {

constexpr int CLIP_GRID = 1024;                                // workgroups of a launch, partial sums
constexpr int CLIP_LIST = 128;                                 // tensors of a launch (4 KB of arguments hold 144)
constexpr int CLIP_STEP = 4;                                   // pieces of 16 bytes that a thread has under way
constexpr int64_t CLIP_CHUNK = 256 * CLIP_STEP * 16;           // bytes of a chunk

struct List {
    const void* grad[CLIP_LIST];
    void* out[CLIP_LIST];
    int64_t count[CLIP_LIST];                                  // elements, the type in the last bit
    uint32_t first[CLIP_LIST];                                 // a tensor's first chunk
    uint32_t chunks;                                           // of all of them
    int32_t n;
};

// the tensor of a chunk: the last whose first chunk is not behind it
__device__ __forceinline__ int tensor_of(const List& l, uint32_t chunk)
{
    int lo = 0, n = l.n;
    while (n > 1) {
        const int half = n >> 1;
        if (l.first[lo + half] <= chunk) { lo += half; n -= half; }
        else n = half;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double room[4];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}

template <typename T>
__device__ __forceinline__ void load_chunk(const T* p, int64_t left, u32x4 (&raw)[CLIP_STEP])
{
    constexpr int P = PIECE<T>;
    if (left >= CLIP_CHUNK / int64_t(sizeof(T))) {
#pragma unroll
        for (int i = 0; i < CLIP_STEP; ++i) raw[i] = load_piece(p + (i * 256 + int(threadIdx.x)) * P, P);
        return;
    }
#pragma unroll
    for (int i = 0; i < CLIP_STEP; ++i) {
        const int at = (i * 256 + int(threadIdx.x)) * P;
        raw[i] = load_piece(p + at, int(left) - at);
    }
}

template <typename T>
__device__ __forceinline__ double squares(const T* p, int64_t left)
{
    u32x4 raw[CLIP_STEP];
    load_chunk(p, left, raw);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < CLIP_STEP; ++i)
#pragma unroll
        for (int j = 0; j < PIECE<T>; ++j) {
            const double v = double(element<T>(raw[i], j));
            s = fma(v, v, s);
        }
    return s;
}

// partial[workgroup] = (with `add`: what is there +) the squares of its chunks
__global__ __launch_bounds__(256) void k_clip_squares(const List l, double* __restrict__ partial, int add)
{
    double s = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < l.chunks; chunk += CLIP_GRID) {
        const int t = tensor_of(l, chunk);
        const bool bf = l.count[t] & 1;
        const int64_t at = int64_t(chunk - l.first[t]) * (CLIP_CHUNK / (bf ? 2 : 4)), left = (l.count[t] >> 1) - at;
        s += bf ? squares(static_cast<const bf16_t*>(l.grad[t]) + at, left) : squares(static_cast<const float*>(l.grad[t]) + at, left);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + s : s;
}

template <typename T, typename F>
__device__ __forceinline__ void scale(const T* p, T* to, int64_t left, F factor)
{
    constexpr int P = PIECE<T>;
    u32x4 raw[CLIP_STEP];
    load_chunk(p, left, raw);
#pragma unroll
    for (int i = 0; i < CLIP_STEP; ++i) {
        const int at = (i * 256 + int(threadIdx.x)) * P;
        float v[P];
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = float(F(element<T>(raw[i], j)) * factor);
        store_piece<P>(to + at, left >= CLIP_CHUNK / int64_t(sizeof(T)) ? P : int(left) - at, v);
    }
}

__global__ __launch_bounds__(256) void k_clip_scale(const List l, const double* __restrict__ partial, float* __restrict__ norm, float max_norm)
{
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < CLIP_GRID / 256; ++i) s += partial[i * 256 + int(threadIdx.x)];
    const float v = float(sqrt(block_sum(s)));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    const bool down = v > max_norm && v < INFINITY;
    const float factor = down ? max_norm / v : 1.f;
    // (a factor below fp32's normal range, of a norm above 10^37 or so, has lost digits, or all of them: fp64 then)
    const bool tiny = factor < 0x1p-126f;
    const double tiny_factor = double(max_norm) / double(v);
    for (uint32_t c = blockIdx.x; c < l.chunks; c += CLIP_GRID) {
        const uint32_t chunk = l.chunks - 1 - c;
        const int t = tensor_of(l, chunk);
        if (!l.out[t] || (!down && l.out[t] == l.grad[t])) continue;      // (nothing is wanted, or nothing changes)
        const bool bf = l.count[t] & 1;
        const int64_t at = int64_t(chunk - l.first[t]) * (CLIP_CHUNK / (bf ? 2 : 4)), left = (l.count[t] >> 1) - at;
        auto scaled = [&](auto type) {
            using T = decltype(type);
            const T* const from = static_cast<const T*>(l.grad[t]) + at;
            T* const to = static_cast<T*>(l.out[t]) + at;
            if (tiny) scale(from, to, left, tiny_factor);
            else scale(from, to, left, factor);
        };
        if (bf) scaled(bf16_t{});
        else scaled(float{});
    }
}

int64_t chunks_of(const dynb_grad_tensor& t) { return (t.count * (t.dtype == DYNB_BF16 ? 2 : 4) + CLIP_CHUNK - 1) / CLIP_CHUNK; }

}  // namespace

extern "C" size_t dynb_clip_workspace_bytes(void) { return CLIP_GRID * sizeof(double); }

extern "C" int dynb_clip_gradients(const dynb_grad_tensor* tensors, int32_t n, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (n < 0 || (n > 0 && !tensors) || !norm || !workspace) return fail(DYNB_E_INVAL, "dynb_clip_gradients: NULL argument or negative number of tensors");
    if (!(max_norm > 0.f)) return fail(DYNB_E_INVAL, "dynb_clip_gradients: max_norm must be positive");
    if (workspace_bytes < dynb_clip_workspace_bytes()) return fail(DYNB_E_WORKSPACE, "dynb_clip_gradients: workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, "dynb_clip_gradients: workspace not 256-byte aligned");
    if (reinterpret_cast<uintptr_t>(norm) & 3) return fail(DYNB_E_INVAL, "dynb_clip_gradients: norm is misaligned");
    for (int i = 0; i < n; ++i) {
        const dynb_grad_tensor& t = tensors[i];
        if (t.count < 0 || (t.count > 0 && !t.grad)) return fail(DYNB_E_INVAL, "dynb_clip_gradients: tensor " + std::to_string(i) + " has no data");
        if (t.count > int64_t(1) << 42) return fail(DYNB_E_UNSUPPORTED, "dynb_clip_gradients: tensor " + std::to_string(i) + " has more than 2^42 elements");
        if (t.dtype != DYNB_F32 && t.dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, "dynb_clip_gradients: tensor " + std::to_string(i) + " has an unknown dtype");
        if ((reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.out)) & (t.dtype == DYNB_BF16 ? 1 : 3))
            return fail(DYNB_E_INVAL, "dynb_clip_gradients: tensor " + std::to_string(i) + " is misaligned");
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    // the list of a launch, from tensor i on (forwards) or back to front; returns the next tensor
    List l;
    auto add = [&](const dynb_grad_tensor& t) {
        const uint32_t chunks = uint32_t(chunks_of(t));        // (at most 2^30: two of them fit)
        if (chunks == 0) return true;
        if (l.n == CLIP_LIST || (l.n > 0 && uint64_t(l.chunks) + chunks > 0xffffffffull - CLIP_GRID)) return false;
        l.grad[l.n] = t.grad;
        l.out[l.n] = t.out;
        l.count[l.n] = t.count * 2 + (t.dtype == DYNB_BF16);
        l.first[l.n] = l.chunks;
        l.chunks += chunks;
        ++l.n;
        return true;
    };
    for (int i = 0, first = 1; i < n || first; first = 0) {
        l.n = 0;
        l.chunks = 0;
        while (i < n && add(tensors[i])) ++i;
        hipLaunchKernelGGL(k_clip_squares, dim3(CLIP_GRID), dim3(256), 0, st, l, partial, first ? 0 : 1);
    }
    for (int i = n, first = 1; i > 0 || first; first = 0) {
        l.n = 0;
        l.chunks = 0;
        while (i > 0 && add(tensors[i - 1])) --i;
        // (chunks are taken from the list's end: of the tensors that come last, here the list's first ones, the last chunks should come first)
        std::reverse(l.grad, l.grad + l.n);
        std::reverse(l.out, l.out + l.n);
        std::reverse(l.count, l.count + l.n);
        uint32_t at = 0;
        for (int j = 0; j < l.n; ++j) {
            l.first[j] = at;
            const int64_t bytes = (l.count[j] >> 1) * (l.count[j] & 1 ? 2 : 4);
            at += uint32_t((bytes + CLIP_CHUNK - 1) / CLIP_CHUNK);
        }
        const unsigned grid = std::max(1u, std::min<unsigned>(l.chunks, CLIP_GRID));
        hipLaunchKernelGGL(k_clip_scale, dim3(grid), dim3(256), 0, st, l, partial, norm, max_norm);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_clip_gradients: ") + hipGetErrorString(e));
    return DYNB_OK;
}
