// Matrix products of rows that are stacked by expert, each group with its expert's matrix, in the three directions of a layer:
//   out[r] = in[row(r)] W_e^T (optionally ReLU)      din[r] = (dout[r] W_e) (where act > 0)      dW_e = sum over the group of dout[r]^T in[row(r)]
// W_e is [N][K].  The groups are known on the device only (offsets): nothing is read back.  Every kernel covers them with units of work that a
// workgroup finds by itself: group e's units begin at  floor(offsets[e] / P) + e,  which leaves room for the ceil(rows / P) pieces of P rows that
// the group has (and one for an empty group), since  ceil((b - a) / P) <= floor(b / P) - floor(a / P) + 1.  floor(M / P) + E + 1 units hold all groups
// and what lies behind the last one, whose rows of results are zeros.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "device_utils.h"
#include "plan_internal.h"

using dynb::fail;

namespace {

struct Groups {
    const int32_t* offsets;   // [E + 1]; the first is taken as 0, and all are kept within 0 .. M
    const int32_t* perm;      // row r of the groups is row perm[r] / k of the gathered tensor, or null
    int32_t k, rows;          // ... which has `rows` rows
    int32_t M, E;
    __device__ __forceinline__ int begin(int e) const { return e <= 0 ? 0 : e > E ? M : min(max(offsets[e], 0), M); }
    __device__ __forceinline__ int64_t row(int r) const
    {
        if (!perm) return r;
        return min(uint32_t(perm[r]) / uint32_t(k), uint32_t(rows - 1));
    }
};

struct Piece { int e, begin, rows, part, parts; };             // rows begin .. of group e (E: what lies behind the last group)

// the unit's group and its piece of at most P rows; parts: how many the group has (0: it is empty).  All 64 lanes of a wave call it.
__device__ __forceinline__ Piece find_piece(const Groups& g, int P, int unit)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = g.E + 1;                                   // the group is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64, e = lo + lane * step;
        const bool here = lane * step < n && g.begin(e) / P + e <= unit;
        const int last = 63 - __builtin_clzll(__ballot(here) | 1ull);
        lo += last * step;
        n = min(step, n - last * step);
    }
    Piece p;
    p.e = __builtin_amdgcn_readfirstlane(lo);
    const int a = g.begin(p.e), rows = g.begin(p.e + 1) - a;
    p.part = unit - (a / P + p.e);
    p.parts = rows > 0 ? (rows - 1) / P + 1 : 0;
    p.begin = a + p.part * P;
    p.rows = p.part < p.parts ? min(P, rows - p.part * P) : 0;
    return p;
}

struct Args {
    Groups g;
    const bf16_t *a, *b;      // what gives the results' columns, and their rows
    int64_t a_stride, b_stride;
    const bf16_t* act;
    int64_t act_stride;
    void* out;
    int64_t out_stride;
    int K, N, relu;
};

enum { FORWARD, GRAD_INPUT, GRAD_WEIGHT };

// Any size, stride and address: tiles of 64 x 64 results, sums in pieces of 32 elements that are loaded one element at a time (the direction in memory
// goes over the lanes) and multiplied by 32x32x16 MFMAs from LDS.
constexpr int ANY = 64, ANY_C = 32, ANY_P = ANY_C + 8;

template <int DIR, typename TO>
__global__ __launch_bounds__(256) void k_product_any(Args p)
{
    __shared__ __attribute__((aligned(16))) bf16_t tile[2][ANY * ANY_P];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, q = lane & 31, hk = lane >> 5;
    const int cols = DIR == FORWARD ? p.N : p.K, ct = (cols + ANY - 1) / ANY, rt = DIR == GRAD_WEIGHT ? (p.N + ANY - 1) / ANY : 1;
    const int c0 = int(blockIdx.x) % ct * ANY, r0 = int(blockIdx.x) / ct % rt * ANY, unit = int(blockIdx.x) / ct / rt;
    const Piece at = find_piece(p.g, DIR == GRAD_WEIGHT ? 0x7fffffff : ANY, unit);
    if (DIR == GRAD_WEIGHT ? at.e >= p.g.E : at.rows == 0) return;
    const int rows = DIR == GRAD_WEIGHT ? p.N : at.rows;
    const int depth = DIR == FORWARD ? p.K : DIR == GRAD_INPUT ? p.N : at.rows;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    const size_t w = size_t(at.e) * size_t(p.N) * size_t(p.K);
    // element (index i of the results' side, place z of the sum)
    auto col_at = [&](int i, int z) -> bf16_t {
        if (i >= cols || z >= depth) return 0;
        if (DIR == FORWARD) return p.a[w + size_t(i) * p.K + z];
        if (DIR == GRAD_INPUT) return p.a[w + size_t(z) * p.K + i];
        return p.a[p.g.row(at.begin + z) * p.a_stride + i];
    };
    auto row_at = [&](int i, int z) -> bf16_t {
        if (i >= rows || z >= depth) return 0;
        if (DIR == FORWARD) return p.b[p.g.row(at.begin + i) * p.b_stride + z];
        if (DIR == GRAD_INPUT) return p.b[int64_t(at.begin + i) * p.b_stride + z];
        return p.b[int64_t(at.begin + z) * p.b_stride + i];
    };
    if (at.e < p.g.E)
        for (int z0 = 0; z0 < depth; z0 += ANY_C) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < ANY * ANY_C / 256; ++j) {
                const int v = tid + j * 256, along_i = v % ANY, along_z = v / ANY, z = v % ANY_C, i = v / ANY_C;
                if (DIR == FORWARD) tile[0][i * ANY_P + z] = col_at(c0 + i, z0 + z);
                else tile[0][along_i * ANY_P + along_z] = col_at(c0 + along_i, z0 + along_z);
                if (DIR == GRAD_WEIGHT) tile[1][along_i * ANY_P + along_z] = row_at(r0 + along_i, z0 + along_z);
                else tile[1][i * ANY_P + z] = row_at(r0 + i, z0 + z);
            }
            __syncthreads();
#pragma unroll
            for (int ks = 0; ks < ANY_C; ks += 16) {
                const bf16x8 a = *reinterpret_cast<const bf16x8*>(&tile[0][((wave & 1) * 32 + q) * ANY_P + ks + 8 * hk]);
                const bf16x8 b = *reinterpret_cast<const bf16x8*>(&tile[1][((wave >> 1) * 32 + q) * ANY_P + ks + 8 * hk]);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
            }
        }
    const int r = r0 + (wave >> 1) * 32 + q;
    if (r >= rows) return;
    TO* const to = static_cast<TO*>(p.out) + (DIR == GRAD_WEIGHT ? int64_t(w) + int64_t(r) * p.K : int64_t(at.begin + r) * p.out_stride);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = c0 + (wave & 1) * 32 + (i >> 2) * 8 + hk * 4 + (i & 3);
        if (c >= cols) continue;
        float v = acc[i];
        if (DIR == FORWARD && p.relu) v = v < 0.f ? 0.f : v;   // (a NaN stays one)
        if (DIR == GRAD_INPUT && p.act && !(bf16_to_f32(p.act[int64_t(at.begin + r) * p.act_stride + c]) > 0.f)) v = 0.f;
        store_f32(to + c, v);
    }
}

int check(const moe_product_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->M < 0 || s->K <= 0 || s->N <= 0 || s->E <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": only DYNB_BF16");
    if (s->flags & ~uint32_t(MOE_PRODUCT_RELU)) return fail(DYNB_E_UNSUPPORTED, who + ": unknown flag");
    if (s->M > 1 << 30 || s->E > 1 << 20 || s->K > 1 << 22 || s->N > 1 << 22) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^30 rows, 2^22 channels or 2^20 experts");
    return DYNB_OK;
}
int check_groups(const moe_product_shape* s, const moe_groups* g, bool gathers, const std::string& who)
{
    if (!g || !g->offsets) return fail(DYNB_E_INVAL, who + ": NULL groups");
    if (g->perm && !gathers) return fail(DYNB_E_INVAL, who + ": its rows are not gathered (perm must be NULL)");
    if (g->perm && (g->k <= 0 || (s->M > 0 && g->rows <= 0))) return fail(DYNB_E_INVAL, who + ": perm needs k and the number of rows it points into");
    if ((reinterpret_cast<uintptr_t>(g->offsets) | reinterpret_cast<uintptr_t>(g->perm)) & 3) return fail(DYNB_E_INVAL, who + ": misaligned pointer");
    return DYNB_OK;
}
int64_t tiles(int n) { return (int64_t(n) + ANY - 1) / ANY; }
constexpr int64_t MOST_GROUPS = (1 << 24) - 1;                 // workgroups of 256 threads in a launch
bool odd(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 1) != 0; }

int launched(const char* who)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    return DYNB_OK;
}

Groups groups_of(const moe_product_shape* s, const moe_groups* g) { return Groups{g->offsets, g->perm, std::max(g->k, 1), g->perm ? g->rows : s->M, s->M, s->E}; }

}  // namespace

extern "C" int moe_product(const moe_product_shape* s, const moe_groups* g, const void* in, int64_t in_stride, const void* W, void* out, int64_t out_stride, void* stream)
{
    int rc = check(s, "moe_product");
    if (rc == DYNB_OK) rc = check_groups(s, g, true, "moe_product");
    if (rc != DYNB_OK) return rc;
    if (s->M == 0) return DYNB_OK;
    if (!in || !W || !out) return fail(DYNB_E_INVAL, "moe_product: NULL argument");
    if (in_stride < s->K || out_stride < s->N) return fail(DYNB_E_INVAL, "moe_product: rows overlap (stride below their length)");
    if (odd(in) || odd(W) || odd(out)) return fail(DYNB_E_INVAL, "moe_product: misaligned pointer");
    const Args p = {groups_of(s, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(in), 0, in_stride, nullptr, 0, out, out_stride, s->K, s->N, int(s->flags & MOE_PRODUCT_RELU)};
    const int64_t grid = tiles(s->N) * (s->M / ANY + s->E + 1);
    if (grid > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, "moe_product: too many results");
    hipLaunchKernelGGL((k_product_any<FORWARD, bf16_t>), dim3(unsigned(grid)), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    return launched("moe_product");
}

extern "C" int moe_product_grad_input(const moe_product_shape* s, const moe_groups* g, const void* dout, int64_t dout_stride, const void* W, const void* act, int64_t act_stride,
                                      void* din, int64_t din_stride, void* stream)
{
    int rc = check(s, "moe_product_grad_input");
    if (rc == DYNB_OK) rc = check_groups(s, g, false, "moe_product_grad_input");
    if (rc != DYNB_OK) return rc;
    if (s->M == 0) return DYNB_OK;
    if (!dout || !W || !din) return fail(DYNB_E_INVAL, "moe_product_grad_input: NULL argument");
    if (dout_stride < s->N || din_stride < s->K || (act && act_stride < s->K)) return fail(DYNB_E_INVAL, "moe_product_grad_input: rows overlap (stride below their length)");
    if (odd(dout) || odd(W) || odd(act) || odd(din)) return fail(DYNB_E_INVAL, "moe_product_grad_input: misaligned pointer");
    const Args p = {groups_of(s, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(dout), 0, dout_stride, static_cast<const bf16_t*>(act), act_stride, din, din_stride, s->K, s->N, 0};
    const int64_t grid = tiles(s->K) * (s->M / ANY + s->E + 1);
    if (grid > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, "moe_product_grad_input: too many results");
    hipLaunchKernelGGL((k_product_any<GRAD_INPUT, bf16_t>), dim3(unsigned(grid)), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    return launched("moe_product_grad_input");
}

extern "C" size_t moe_product_grad_weight_workspace_bytes(const moe_product_shape* s)
{
    if (check(s, "moe_product_grad_weight_workspace_bytes") != DYNB_OK) return 0;
    return 256;
}

extern "C" int moe_product_grad_weight(const moe_product_shape* s, const moe_groups* g, const void* dout, int64_t dout_stride, const void* in, int64_t in_stride, void* dW,
                                       int32_t grad_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check(s, "moe_product_grad_weight");
    if (rc == DYNB_OK) rc = check_groups(s, g, true, "moe_product_grad_weight");
    if (rc != DYNB_OK) return rc;
    if (grad_dtype != DYNB_F32 && grad_dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, "moe_product_grad_weight: unknown dtype of the gradient");
    if (!dW || !workspace || (s->M > 0 && (!dout || !in))) return fail(DYNB_E_INVAL, "moe_product_grad_weight: NULL argument");
    if (dout_stride < s->N || in_stride < s->K) return fail(DYNB_E_INVAL, "moe_product_grad_weight: rows overlap (stride below their length)");
    if (odd(dout) || odd(in) || (reinterpret_cast<uintptr_t>(dW) & (grad_dtype == DYNB_BF16 ? 1 : 3))) return fail(DYNB_E_INVAL, "moe_product_grad_weight: misaligned pointer");
    if (workspace_bytes < moe_product_grad_weight_workspace_bytes(s)) return fail(DYNB_E_WORKSPACE, "moe_product_grad_weight: workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, "moe_product_grad_weight: workspace not 256-byte aligned");
    const Args p = {groups_of(s, g), static_cast<const bf16_t*>(in), static_cast<const bf16_t*>(dout), in_stride, dout_stride, nullptr, 0, dW, 0, s->K, s->N, 0};
    const int64_t grid = tiles(s->K) * tiles(s->N) * s->E;
    if (grid > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, "moe_product_grad_weight: too many results");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (grad_dtype == DYNB_BF16) hipLaunchKernelGGL((k_product_any<GRAD_WEIGHT, bf16_t>), dim3(unsigned(grid)), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_product_any<GRAD_WEIGHT, float>), dim3(unsigned(grid)), dim3(256), 0, st, p);
    return launched("moe_product_grad_weight");
}
