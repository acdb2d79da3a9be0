// Layer norm of rows and its gradients.
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) r gamma + beta
//   g = dy gamma, h = (x - m) r:  dx = r (g - mean(g) - h mean(g h)),  dgamma = sum over the rows of dy h,  dbeta = of dy
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "device_utils.h"
#include "plan_internal.h"
#include "rows.h"
#include "rows8.h"

using dynb::fail;

namespace {

// A lane keeps up to 16 elements of a row, so that it is read once: the mean, then the squares of what differs from it, from registers.  Rows of up to
// 1024 elements are a wave's each, up to 16384 a workgroup's of 4 or 16 waves.  Longer ones are read three times (k_norm_long and its like).
// Bound by memory where rows fill their lanes: a row in, a row out, no more.  65536 x 1024 bf16 51 us (5.3 TB/s; a large copy here 4.8), fp32 96 (5.6); 37 x 512
// takes 3.4 us, a launch's own time.  Narrower rows have a wave each all the same, most of whose lanes have nothing to do, and are bound by the waves:
// 65536 x 256 bf16 27 us (2.5 TB/s), fp32 25 (5.3); 65536 x 64 bf16 25 us (0.7 TB/s), fp32 20 (1.7).
// The variance from registers, and not the mean of squares less the squared mean, which would lose all digits where the mean is large.
constexpr int LANE = 16;

// the sum over a row's waves (WAVES > 1: all threads call it, `room` is free)
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* room)
{
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += room[i];
    }
    return v;
}

template <typename T, int NV, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void k_norm(const T* x, int64_t x_stride, const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                                                                        int64_t y_stride, float* __restrict__ mean, float* __restrict__ rstd, int n, int d, float eps)
{
    constexpr int P = PIECE<T>, NL = WAVES * 64;               // lanes of a row
    __shared__ float room[2][WAVES > 1 ? WAVES : 1];
    const int row = WAVES == 1 ? int(blockIdx.x) * 4 + int(threadIdx.x >> 6) : int(blockIdx.x);
    if (row >= n) return;
    const int lane = threadIdx.x & (NL - 1);
    const T* const from = x + row * x_stride;
    u32x4 raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = load_piece(from + (i * NL + lane) * P, d - (i * NL + lane) * P);
    float v[NV][P], s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j) s += v[i][j] = element<T>(raw[i], j);
    const float m = row_sum<WAVES>(s, room[0]) / float(d);
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            v[i][j] -= m;
            if ((i * NL + lane) * P + j < d) s += v[i][j] * v[i][j];
        }
    const float r = 1.f / sqrtf(row_sum<WAVES>(s, room[1]) / float(d) + eps);
    T* const to = y + row * y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * NL + lane) * P, left = d - c;
        float w[P];
#pragma unroll
        for (int j = 0; j < P; ++j) w[j] = v[i][j] * r;
        if (gamma) {
#pragma unroll
            for (int h = 0; h < P; h += 4) {
                const u32x4 g = load_piece(gamma + c + h, left - h);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[h + j] *= element<float>(g, j);
            }
        }
        if (beta) {
#pragma unroll
            for (int h = 0; h < P; h += 4) {
                const u32x4 b = load_piece(beta + c + h, left - h);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[h + j] += element<float>(b, j);
            }
        }
        store_piece<P>(to + c, left, w);
    }
    if (lane == 0) {
        if (mean) mean[row] = m;
        if (rstd) rstd[row] = r;
    }
}

// The sum over a wave without LDS: neighbours, quads, halves of 16 lanes and 16 lanes by lanes' permutations, then the two 16s and the two halves change places.  (By way of
// LDS it is six round trips of 100 clocks and more, which a row's wave does not hide.)
__device__ __forceinline__ float wave_sum_in_registers(float v)
{
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, true));              // lanes 1 0 3 2
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, true));              // lanes 2 3 0 1
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));             // eight lanes backwards
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true));             // sixteen lanes backwards
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The backward pass's x as it lies (RowsOf), or in 8 bits (Rows8).  From 8 bits 65536 x 1024 bf16 take 57 us (340 MB, 6.0 TB/s) where x in bf16 takes 74, 65536 x 1000 fp32 111 (595 MB, 5.3; 152);
// 4097 x 777 fp32, which wait for their rows' loads, 11.
template <typename T>
struct RowsOf {
    static constexpr bool WHOLE = false;
    const T* x;
    int64_t stride;
    using Raw = u32x4;
    __device__ __forceinline__ Raw load(int64_t row, int c, int, int d) const { return load_piece(x + row * stride + c, d - c); }
    static __device__ __forceinline__ float value(const Raw& v, int j) { return element<T>(v, j); }
    static __device__ __forceinline__ float sum(float v) { return wave_sum(v); }
    __device__ __forceinline__ float at(int64_t row, int c) const { return load_f32(x + row * stride + c); }
};
// WHOLE: d is a piece's elements or more, and every load is a whole piece: a lane whose piece would reach over the row's end takes the row's last one instead, and of that only the
// elements that no other lane has (65536 x 1001 bf16: 131 us element by element, 61 so)
template <typename T, bool WHOLE_>
struct Rows8 {
    static constexpr bool WHOLE = WHOLE_;
    const int8_t* q;
    int64_t stride;
    const bf16_t* scale;
    int64_t scale_stride;
    bool past;                // dx goes past the caches
    struct Raw { u32x2 q; float s; };
    // the piece from c, in its own place the one from `own`
    __device__ __forceinline__ Raw load(int64_t row, int c, int own, int d) const
    {
        if (!WHOLE && c >= d) return Raw{{0u, 0u}, 0.f};
        const int left = WHOLE ? 8 : d - c;
        const float s = bf16_to_f32(scale[row * scale_stride + min(own, d - 1) / BLOCK8]);
        if constexpr (PIECE<T> == 8) return Raw{load_eight(q + row * stride + c, left), s};
        else return Raw{{load_four(q + row * stride + c, left), 0u}, s};
    }
    static __device__ __forceinline__ float value(const Raw& v, int j) { return unpack8(v.q[j >> 2], j & 3) * v.s; }
    static __device__ __forceinline__ float sum(float v) { return wave_sum_in_registers(v); }
    __device__ __forceinline__ float at(int64_t row, int c) const { return float(q[row * stride + c]) * bf16_to_f32(scale[row * scale_stride + c / BLOCK8]); }
};
// said to be other numbers, so that what follows from them is made anew
__device__ __forceinline__ void anew(u32x4& v) { asm volatile("" : "+v"(v)); }
template <typename R> __device__ __forceinline__ void anew(R& v) { asm volatile("" : "+v"(v.q), "+v"(v.s)); }

// The backward pass reads dy and x once: a lane has the same columns of every row that its wave (workgroup) goes through and adds up their share of the
// parameters' gradients in registers.  A workgroup's shares are added in LDS and leave as one line of `partial` ([workgroup][2][d]), which k_norm_join adds up,
// so that every sum has one order.  The next row is on its way while one is worked on.  65536 x 1024 bf16: 74 us (403 MB, 5.5 TB/s) and 4.6 for k_norm_join; with a
// pass of its own for the parameters' gradients dy and x would be read twice.  Narrow rows as above (65536 x 256: bf16 44 us, 2.3 TB/s, fp32 35, 5.7; 65536 x 64:
// 42 and 33 us, 0.6 and 1.5 TB/s); sixteen waves, 8192 x 12288: bf16 130 us, 4.6 TB/s, fp32 231, 5.2.  Small ones (4097 x 777
// fp32: 11.6 us and 3.9) wait for their rows' few loads, and for the second launch.
template <typename T, class X, int NV, int WAVES>
__device__ __forceinline__ void norm_grad_rows(const T* dy, int64_t dy_stride, X x, const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                               int64_t dx_stride, float* __restrict__ partial, int n, int d)
{
    constexpr int P = PIECE<T>, NL = WAVES * 64, AT_ONCE = WAVES == 1 ? 4 : 1;
    // Sixteen waves have 128 registers each, which hold gamma, both sums and dy and x as they were loaded, of 16 columns.  y, h and y gamma, which the compiler would
    // keep, too, until the row's end, are made anew there: 58 to 75 registers were spilled (8192 rows of 12288: 190 us in bf16 and 308 in fp32, 130 and 231 so).
    constexpr bool TIGHT = WAVES == 16 && NV * P == LANE;
    __shared__ float room[2][2][WAVES > 1 ? WAVES : 1];
    __shared__ float share[WAVES == 1 ? 3 : 1][WAVES == 1 ? 64 * NV * P : 1];
    const int lane = threadIdx.x & (NL - 1), wave = threadIdx.x >> 6;
    // a lane's columns of piece i; WHOLE: where they begin, and which of them are its own
    auto own = [&](int i) { return (i * NL + lane) * P; };
    auto at = [&](int i) { return X::WHOLE ? min(own(i), d - P) : own(i); };
    u32x4 mine_of[X::WHOLE ? NV : 1];
    if constexpr (X::WHOLE)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int skip = own(i) < d ? own(i) - at(i) : P;
                mine_of[i][w] = P == 4 ? (w >= skip ? ~0u : 0u) : (2 * w >= skip ? 0xffffu : 0u) | (2 * w + 1 >= skip ? 0xffff0000u : 0u);
            }
    float g_[NV][P], dg[NV][P], db[NV][P];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int h = 0; h < P; h += 4) {
            const int c = at(i) + h;
            const u32x4 g = gamma ? load_piece(gamma + c, d - c) : u32x4{0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g_[i][h + j] = element<float>(g, j);
                dg[i][h + j] = db[i][h + j] = 0.f;
            }
        }
    const int step = int(gridDim.x) * AT_ONCE;
    u32x4 a[NV];
    typename X::Raw b[NV];
    float m = 0.f, r = 0.f;
    auto load = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = at(i);
            a[i] = load_piece(dy + row * dy_stride + c, X::WHOLE ? P : d - c);
            b[i] = x.load(row, c, own(i), d);
        }
        m = mean[row];
        r = rstd[row];
    };
    int64_t row = int(blockIdx.x) * AT_ONCE + (WAVES == 1 ? wave : 0);
    if (row < n) load(row);
    int turn = 0;
    for (; row < n; row += step) {
        float v[NV][P], h[NV][P], s1 = 0.f, s2 = 0.f;
        if constexpr (X::WHOLE)
#pragma unroll
            for (int i = 0; i < NV; ++i) a[i] &= mine_of[i];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                // (what lies behind the row must not count, whatever mean and rstd are.  WHOLE: it is another column of the row, and its dy is taken for 0)
                const bool on = X::WHOLE || (i * NL + lane) * P + j < d;
                h[i][j] = on ? (X::value(b[i], j) - m) * r : 0.f;
                const float y = element<T>(a[i], j);
                dg[i][j] += y * h[i][j];
                db[i][j] += y;
                if constexpr (TIGHT) asm volatile("" : "+v"(dg[i][j]), "+v"(db[i][j]));              // added here, not where the loop ends
                v[i][j] = y * g_[i][j];
                s1 += v[i][j];
                s2 += v[i][j] * h[i][j];
            }
        const float m0 = m, r0 = r;
        const int64_t here = row;
        if (WAVES < 16 && row < n - step) load(row + step);
        if constexpr (WAVES == 1) {
            s1 = X::sum(s1);
            s2 = X::sum(s2);
        } else {
            // (one meeting for both; the next row's sums lie in the other half)
            s1 = X::sum(s1);
            s2 = X::sum(s2);
            if ((threadIdx.x & 63) == 0) { room[turn][0][wave] = s1; room[turn][1][wave] = s2; }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) { s1 += room[turn][0][i]; s2 += room[turn][1][i]; }
            turn ^= 1;
        }
        if (dx) {
            const float m1 = s1 / float(d), m2 = s2 / float(d);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * NL + lane) * P;
                if constexpr (TIGHT) {
                    anew(a[i]);
                    anew(b[i]);
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        v[i][j] = element<T>(a[i], j) * g_[i][j];
                        h[i][j] = (X::value(b[i], j) - m0) * r0;
                    }
                }
#pragma unroll
                for (int j = 0; j < P; ++j) v[i][j] = r0 * (v[i][j] - m1 - h[i][j] * m2);
                if constexpr (X::WHOLE) {
                    T* const to = dx + here * dx_stride + at(i);
                    if (own(i) <= d - P)
                        put_past(x.past, [&](auto past) {
                            if constexpr (decltype(past)::value) store_past(to, v[i]);
                            else store_piece<P>(to, P, v[i]);
                        });
                    else
#pragma unroll
                        for (int j = 1; j < P; ++j)
                            if (at(i) + j >= own(i)) store_f32(to + j, v[i][j]);
                } else store_piece<P>(dx + here * dx_stride + c, d - c, v[i]);
            }
        }
        if (WAVES == 16 && row < n - step) load(row + step);   // (sixteen waves have half the registers: no room for two rows)
    }
    if (!partial) return;
    float* const mine = partial + size_t(blockIdx.x) * 2 * size_t(d);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        auto& sum = which ? db : dg;
        if constexpr (WAVES == 1) {
            __syncthreads();
            if (wave > 0)
#pragma unroll
                for (int i = 0; i < NV * P; ++i) share[wave - 1][i * 64 + lane] = sum[i / P][i % P];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int i = 0; i < NV * P; ++i) sum[i / P][i % P] = (sum[i / P][i % P] + share[0][i * 64 + lane]) + (share[1][i * 64 + lane] + share[2][i * 64 + lane]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * NL + lane) * P;
            if constexpr (X::WHOLE) {
#pragma unroll
                for (int j = 0; j < P; ++j)
                    if (own(i) < d && at(i) + j >= own(i)) mine[size_t(which) * size_t(d) + size_t(at(i) + j)] = sum[i][j];
            } else store_piece<P>(mine + size_t(which) * size_t(d) + c, d - c, sum[i]);
        }
    }
}

template <typename T, int NV, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void k_norm_grad(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, const float* __restrict__ gamma,
                                                                             const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t dx_stride,
                                                                             float* __restrict__ partial, int n, int d)
{
    norm_grad_rows<T, RowsOf<T>, NV, WAVES>(dy, dy_stride, RowsOf<T>{x, x_stride}, gamma, mean, rstd, dx, dx_stride, partial, n, d);
}
template <typename T, int NV, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void k_norm8_grad(const T* dy, int64_t dy_stride, Rows8<T, WHOLE> x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                                              const float* __restrict__ rstd, T* dx, int64_t dx_stride, float* __restrict__ partial, int n, int d)
{
    norm_grad_rows<T, Rows8<T, WHOLE>, NV, WAVES>(dy, dy_stride, x, gamma, mean, rstd, dx, dx_stride, partial, n, d);
}

// dgamma and dbeta, as they lie one behind the other in a line of `partial`
__global__ __launch_bounds__(1024) void k_norm_join(const float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int lines, int d)
{
    __shared__ float room[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = (lines + 15) / 16;
    const int64_t c = int64_t(blockIdx.x) * 64 + lane;
    float s = 0.f;
    if (c < 2 * int64_t(d)) {
        const int end = min(lines, (wave + 1) * per);
#pragma unroll 8
        for (int i = wave * per; i < end; ++i) s += partial[int64_t(i) * 2 * d + c];
    }
    room[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= 2 * int64_t(d)) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += room[i][lane];
    if (c < d) { if (dgamma) dgamma[c] = s; }
    else if (dbeta) dbeta[c - d] = s;
}

// ------------------------------------------------------------------------------------------ rows of more than 16384 elements
// A workgroup a row, which it reads again for every sum: the simple form, for widths that no register file holds (8192 x 20000 bf16: 419 us, backward 1294;
// 1.6 and 0.8 TB/s of what the operator has to move).
// the sum over 256 threads
__device__ __forceinline__ float group_sum(float v, float* room)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void k_norm_long(const T* x, int64_t x_stride, const float* __restrict__ gamma, const float* __restrict__ beta,
                                              T* y, int64_t y_stride, float* __restrict__ mean, float* __restrict__ rstd, int d, float eps)
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

template <typename T, class X>
__device__ __forceinline__ void norm_dx_long(const T* dy, int64_t dy_stride, X x, const float* __restrict__ gamma, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                             int64_t dx_stride, int d)
{
    __shared__ float room[4];
    const int64_t t = blockIdx.x;
    const float m = mean[t], r = rstd[t];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < d; c += 256) {
        const float g = load_f32(dy + t * dy_stride + c) * (gamma ? gamma[c] : 1.f), h = (x.at(t, c) - m) * r;
        s1 += g;
        s2 += g * h;
    }
    s1 = group_sum(s1, room) / float(d);
    s2 = group_sum(s2, room) / float(d);
    for (int c = threadIdx.x; c < d; c += 256) {
        const float g = load_f32(dy + t * dy_stride + c) * (gamma ? gamma[c] : 1.f), h = (x.at(t, c) - m) * r;
        store_f32(dx + t * dx_stride + c, r * (g - s1 - h * s2));
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm_dx_long(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, const float* __restrict__ gamma,
                                                 const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t dx_stride, int d)
{
    norm_dx_long<T>(dy, dy_stride, RowsOf<T>{x, x_stride}, gamma, mean, rstd, dx, dx_stride, d);
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm8_dx_long(const T* dy, int64_t dy_stride, Rows8<T, false> x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                       const float* __restrict__ rstd, T* dx, int64_t dx_stride, int d)
{
    norm_dx_long<T>(dy, dy_stride, x, gamma, mean, rstd, dx, dx_stride, d);
}

template <typename T, class X>
__device__ __forceinline__ void norm_dparams_long(const T* dy, int64_t dy_stride, X x, const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ dgamma,
                                                  float* __restrict__ dbeta, int n, int d)
{
    __shared__ float room[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sg = 0.f, sb = 0.f;
    if (c < d)
        for (int64_t t = wave; t < n; t += 4) {
            const float v = load_f32(dy + t * dy_stride + c);
            sg += v * (x.at(t, c) - mean[t]) * rstd[t];
            sb += v;
        }
    room[0][wave][lane] = sg;
    room[1][wave][lane] = sb;
    __syncthreads();
    if (wave != 0 || c >= d) return;
    if (dgamma) dgamma[c] = (room[0][0][lane] + room[0][1][lane]) + (room[0][2][lane] + room[0][3][lane]);
    if (dbeta) dbeta[c] = (room[1][0][lane] + room[1][1][lane]) + (room[1][2][lane] + room[1][3][lane]);
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm_dparams_long(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, const float* __restrict__ mean,
                                                      const float* __restrict__ rstd, float* __restrict__ dgamma, float* __restrict__ dbeta, int n, int d)
{
    norm_dparams_long<T>(dy, dy_stride, RowsOf<T>{x, x_stride}, mean, rstd, dgamma, dbeta, n, d);
}
template <typename T>
__global__ __launch_bounds__(256) void k_norm8_dparams_long(const T* dy, int64_t dy_stride, Rows8<T, false> x, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta, int n, int d)
{
    norm_dparams_long<T>(dy, dy_stride, x, mean, rstd, dgamma, dbeta, n, d);
}

int check(const dynb_norm_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->T < 0 || s->d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (!(s->eps >= 0.f)) return fail(DYNB_E_INVAL, who + ": eps must not be negative");
    if (s->dtype != DYNB_F32 && s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    if (s->d > 1 << 28) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^28 columns");
    return DYNB_OK;
}
constexpr int64_t MOST_ROWS = 1 << 21;                         // of a launch (which has room for 2^32 threads)
// pieces of a lane and waves of a row (0: long rows)
int row_waves(int d) { return d <= 64 * LANE ? 1 : d <= 256 * LANE ? 4 : d <= 1024 * LANE ? 16 : 0; }
template <typename T, typename F>
void by_width(T in, int d, F&& launch)
{
    auto with = [&](auto waves) {
        constexpr int W = decltype(waves)::value, P = PIECE<T>;
        if (d <= W * 64 * P) launch(in, std::integral_constant<int, 1>{}, waves);
        else if (P * 2 == LANE || d <= W * 64 * P * 2) launch(in, std::integral_constant<int, 2>{}, waves);
        else launch(in, std::integral_constant<int, LANE / P>{}, waves);
    };
    switch (row_waves(d)) {
    case 1: with(std::integral_constant<int, 1>{}); break;
    case 4: with(std::integral_constant<int, 4>{}); break;
    case 16: with(std::integral_constant<int, 16>{}); break;
    default: launch(in, std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{});
    }
}
// workgroups of the backward pass, a line of partial sums each
int grad_lines(const dynb_norm_shape* s)
{
    const int waves = row_waves(s->d);
    if (waves == 0) return 0;
    return waves == 1 ? int(std::min<int64_t>((int64_t(s->T) + 3) / 4, 512)) : std::min(s->T, waves == 4 ? 512 : 256);
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
    auto launch = [&](auto in, auto nv, auto waves) {
        using T = decltype(in);
        constexpr int NV = decltype(nv)::value, WAVES = decltype(waves)::value;
        const T* const a = static_cast<const T*>(x);
        T* const b = static_cast<T*>(y);
        for (int64_t t = 0; t < s->T; t += MOST_ROWS) {
            const int n = int(std::min<int64_t>(s->T - t, MOST_ROWS));
            float *const m = mean ? mean + t : nullptr, *const r = rstd ? rstd + t : nullptr;
            if constexpr (WAVES == 0)
                hipLaunchKernelGGL((k_norm_long<T>), dim3(unsigned(n)), dim3(256), 0, st, a + t * x_stride, x_stride, gamma, beta, b + t * y_stride, y_stride, m, r, s->d, s->eps);
            else
                hipLaunchKernelGGL((k_norm<T, NV, WAVES>), dim3(unsigned(WAVES == 1 ? (n + 3) / 4 : n)), dim3(WAVES == 1 ? 256 : WAVES * 64), 0, st, a + t * x_stride, x_stride, gamma,
                                   beta, b + t * y_stride, y_stride, m, r, n, s->d, s->eps);
        }
    };
    if (s->dtype == DYNB_BF16) by_width(bf16_t{}, s->d, launch);
    else by_width(float{}, s->d, launch);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_layer_norm: ") + hipGetErrorString(e));
    return DYNB_OK;
}

extern "C" size_t dynb_layer_norm_backward_workspace_bytes(const dynb_norm_shape* s)
{
    if (check(s, "dynb_layer_norm_backward_workspace_bytes") != DYNB_OK) return 0;
    const size_t lines = size_t(grad_lines(s));
    return std::max<size_t>(lines * 2 * size_t(s->d) * 4, 256);
}

namespace {

// x: as it lies, or null and `rows` in 8 bits
int norm_backward(const dynb_norm_shape* s, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const dynb_rows8* rows, const float* gamma, const float* mean,
                  const float* rstd, void* dx, int64_t dx_stride, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream, const std::string& who)
{
    const int rc = check(s, who);
    if (rc != DYNB_OK) return rc;
    const bool there = x || (rows && rows->q && rows->scale);
    if (!workspace || (s->T > 0 && (!dy || !there || !mean || !rstd))) return fail(DYNB_E_INVAL, who + ": NULL argument");
    if (dy_stride < s->d || (dx && dx_stride < s->d) || (rows ? rows->q_stride < s->d || rows->scale_stride < (int64_t(s->d) + BLOCK8 - 1) / BLOCK8 : x_stride < s->d))
        return fail(DYNB_E_INVAL, who + ": rows overlap (stride below d)");
    if (workspace_bytes < dynb_layer_norm_backward_workspace_bytes(s)) return fail(DYNB_E_WORKSPACE, who + ": workspace too small");
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(DYNB_E_INVAL, who + ": workspace not 256-byte aligned");
    if (misaligned(dy, s->dtype) || misaligned(x, s->dtype) || misaligned(dx, s->dtype) || misaligned(gamma, DYNB_F32) || misaligned(mean, DYNB_F32) ||
        misaligned(rstd, DYNB_F32) || misaligned(dgamma, DYNB_F32) || misaligned(dbeta, DYNB_F32) || (rows && misaligned(rows->scale, DYNB_BF16)))
        return fail(DYNB_E_INVAL, who + ": misaligned pointer");
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* const partial = dgamma || dbeta ? static_cast<float*>(workspace) : nullptr;
    const int lines = grad_lines(s);
    auto launch = [&](auto in, auto nv, auto waves) {
        using T = decltype(in);
        constexpr int NV = decltype(nv)::value, WAVES = decltype(waves)::value;
        const T *a = static_cast<const T*>(dy), *b = static_cast<const T*>(x);
        using Eight = Rows8<T, false>;
        const Eight r = rows ? Eight{static_cast<const int8_t*>(rows->q), rows->q_stride, static_cast<const bf16_t*>(rows->scale), rows->scale_stride, false} : Eight{};
        T* const to = static_cast<T*>(dx);
        if constexpr (WAVES > 0) {
            const dim3 threads(WAVES == 1 ? 256 : WAVES * 64);
            constexpr bool WHOLE = !(WAVES == 16 && NV * PIECE<T> == LANE);                  // (there is no room for the masks there)
            if (lines > 0 && rows && WHOLE && s->d >= PIECE<T>)
                hipLaunchKernelGGL((k_norm8_grad<T, NV, WAVES, WHOLE>), dim3(unsigned(lines)), threads, 0, st, a, dy_stride, Rows8<T, WHOLE>{r.q, r.stride, r.scale, r.scale_stride, int64_t(s->T) * s->d * int64_t(sizeof(T)) >= PAST}, gamma, mean, rstd,
                                   to, dx_stride, partial, s->T, s->d);
            else if (lines > 0 && rows)
                hipLaunchKernelGGL((k_norm8_grad<T, NV, WAVES, false>), dim3(unsigned(lines)), threads, 0, st, a, dy_stride, r, gamma, mean, rstd, to, dx_stride, partial, s->T, s->d);
            else if (lines > 0)
                hipLaunchKernelGGL((k_norm_grad<T, NV, WAVES>), dim3(unsigned(lines)), threads, 0, st, a, dy_stride, b, x_stride, gamma, mean, rstd, to, dx_stride, partial, s->T, s->d);
            if (partial) hipLaunchKernelGGL(k_norm_join, dim3(unsigned((2 * int64_t(s->d) + 63) / 64)), dim3(1024), 0, st, partial, dgamma, dbeta, lines, s->d);
            return;
        }
        // (the parameters' first: dx may be dy or x)
        const dim3 columns(unsigned((s->d + 63) / 64));
        if ((dgamma || dbeta) && rows) hipLaunchKernelGGL((k_norm8_dparams_long<T>), columns, dim3(256), 0, st, a, dy_stride, r, mean, rstd, dgamma, dbeta, s->T, s->d);
        else if (dgamma || dbeta) hipLaunchKernelGGL((k_norm_dparams_long<T>), columns, dim3(256), 0, st, a, dy_stride, b, x_stride, mean, rstd, dgamma, dbeta, s->T, s->d);
        for (int64_t t = 0; t < s->T && dx; t += MOST_ROWS) {
            const dim3 n(unsigned(std::min<int64_t>(s->T - t, MOST_ROWS)));
            if (rows)
                hipLaunchKernelGGL((k_norm8_dx_long<T>), n, dim3(256), 0, st, a + t * dy_stride, dy_stride, Eight{r.q + t * r.stride, r.stride, r.scale + t * r.scale_stride, r.scale_stride, false},
                                   gamma, mean + t, rstd + t, to + t * dx_stride, dx_stride, s->d);
            else
                hipLaunchKernelGGL((k_norm_dx_long<T>), n, dim3(256), 0, st, a + t * dy_stride, dy_stride, b + t * x_stride, x_stride, gamma, mean + t, rstd + t, to + t * dx_stride, dx_stride,
                                   s->d);
        }
    };
    if (s->dtype == DYNB_BF16) by_width(bf16_t{}, s->d, launch);
    else by_width(float{}, s->d, launch);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, who + ": " + hipGetErrorString(e));
    return DYNB_OK;
}

}  // namespace

extern "C" int dynb_layer_norm_backward(const dynb_norm_shape* s, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const float* gamma, const float* mean,
                                        const float* rstd, void* dx, int64_t dx_stride, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream)
{
    return norm_backward(s, dy, dy_stride, x, x_stride, nullptr, gamma, mean, rstd, dx, dx_stride, dgamma, dbeta, workspace, workspace_bytes, stream, "dynb_layer_norm_backward");
}

extern "C" int dynb_layer_norm_backward8(const dynb_norm_shape* s, const void* dy, int64_t dy_stride, const dynb_rows8* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                                         int64_t dx_stride, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream)
{
    const dynb_rows8 none = {};
    return norm_backward(s, dy, dy_stride, nullptr, 0, x ? x : &none, gamma, mean, rstd, dx, dx_stride, dgamma, dbeta, workspace, workspace_bytes, stream, "dynb_layer_norm_backward8");
}
