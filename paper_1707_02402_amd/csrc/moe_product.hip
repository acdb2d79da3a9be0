// Matrix products of rows that are stacked by expert, each group with its expert's matrix, in the three directions of a layer:
//   out[r] = in[row(r)] W_e^T (optionally ReLU)      din[r] = (dout[r] W_e) (where act > 0)      dW_e = sum over the group of dout[r]^T in[row(r)]
// W_e is [N][K].  The groups are known on the device only (offsets): nothing is read back.  Every kernel covers them with units of work that a
// workgroup finds by itself: group e's units begin at  floor(offsets[e] / P) + e,  which leaves room for the ceil(rows / P) pieces of P rows that
// the group has (and one for an empty group), since  ceil((b - a) / P) <= floor(b / P) - floor(a / P) + 1.  floor(M / P) + E + 1 units hold all groups
// and what lies behind the last one, whose rows of results are zeros.
//
// What bounds them: few rows an expert, the weights' way from memory (8192 rows of 256 experts, 512 -> 1024: 64 to 68 us for 309 MB, 4.7 TB/s); many, the matrix
// instructions and what feeds them (65536 rows, 1024 -> 2048, 64 experts: forward 336 us, 818 TFLOP/s, the weights' gradient 408, 361 into bfloat16;
// 8192 rows, channels and features, one expert: forward 782 us, 1.41 PFLOP/s; one library product of that size 807).  Sums as short as 1024 pay for their tiles'
// ends: with even loads the time is 1.73 us for each chunk of 64 places of a workgroup's tile, 1.24 PFLOP/s, and 9 us for every tile, in which its results leave
// and nothing is multiplied (the weights' gradient into fp32: 13 us); uneven loads by Zipf's law with exponent 0.6 add 14 % (the weights' gradient: 20 %).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <string>
#include <type_traits>

#include "moe_tiles.h"

namespace {

template <int DIR, typename TO, class S, bool FUSED>
__global__ __launch_bounds__(S::THREADS, S::SIMD) void k_product(Args p, int units, int ct, int rt, Shares shares, float* __restrict__ partial)
{
    product_tiles<DIR, TO, S, FUSED>(p, NoGate{}, units, ct, rt, shares, partial);
}

// ------------------------------------------------------------------------------------------ any size, stride and address
// Mid's tiles and its places in LDS, by way of registers: pieces of 16 bytes are loaded from wherever they lie (rows of odd length lie between the borders that a copy
// straight into LDS keeps to), the last of a row element by element, a chunk ahead.  65536 rows, 1001 -> 1501, one expert: 465 us forward, 485 the input's
// gradient, 855 the weights', where 1000 -> 1504 takes 231, 207 and 241 through k_product, whose tiles
// of 256 x 256 read either operand half as often and have their next chunk on its way without registers (what share each has was not taken apart).
template <int DIR, typename TO>
__global__ __launch_bounds__(256, 2) void k_product_any(Args p, int units, int ct, int rt, Shares shares, float* __restrict__ partial)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    using S = Mid;
    constexpr bool A_ACROSS = DIR != FORWARD, B_ACROSS = DIR == GRAD_WEIGHT;
    constexpr int U = 2, EACH = 2, UA = A_ACROSS ? YUNIT : XUNIT, UB = B_ACROSS ? YUNIT : XUNIT;
    constexpr uint32_t BUF = BUF_BYTES<DIR, S>;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, q = lane & 31, hk = lane >> 5, cg = wave % 2, rg = wave / 2;
    const int cols = DIR == FORWARD ? p.N : p.K;
    const lds_ptr lds = (lds_ptr)lds_raw;
    using lds_u32x4 = __attribute__((address_space(3))) u32x4;

    u32x4 a_piece[U][EACH], b_piece[U][EACH];
    auto load = [&](const Tile& t, int z0) {
        const u32x4 none = {0u, 0u, 0u, 0u};
        const size_t w = size_t(t.e) * size_t(p.N) * size_t(p.K);
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int block = wave + j * S::WAVES, s_q = copied_row(block, lane), z = z0 + copied_place(block, lane), along = z0 + (lane & 7) * 8, rest = t.depth - along;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int a_col = t.c0 + i * 64 + (lane & 7) * 8, row = i * 64 + (lane >> 5) * 32 + s_q;
                if constexpr (DIR == FORWARD) {                // (the features in the order that gives a lane 16 neighbours)
                    const int feature = t.c0 + i * 64 + (lane >> 5) * 32 + (s_q >> 2 & 1) * 16 + (s_q >> 3) * 4 + (s_q & 3);
                    a_piece[i][j] = feature < cols && rest > 0 ? load_piece(p.a + w + size_t(feature) * size_t(p.K) + along, rest) : none;
                    b_piece[i][j] = row < t.rows && rest > 0 ? load_piece(p.b + p.g.row(t.begin + row) * p.b_stride + along, rest) : none;
                } else if constexpr (DIR == GRAD_INPUT) {
                    a_piece[i][j] = z < t.depth && a_col < cols ? load_piece(p.a + w + size_t(z) * size_t(p.K) + a_col, cols - a_col) : none;
                    b_piece[i][j] = row < t.rows && rest > 0 ? load_piece(p.b + int64_t(t.begin + row) * p.b_stride + along, rest) : none;
                } else {
                    const int b_col = t.r0 + i * 64 + (lane & 7) * 8;
                    a_piece[i][j] = z < t.depth && a_col < cols ? load_piece(p.a + p.g.row(t.begin + z) * p.a_stride + a_col, cols - a_col) : none;
                    b_piece[i][j] = z < t.depth && b_col < p.N ? load_piece(p.b + int64_t(t.begin + z) * p.b_stride + b_col, p.N - b_col) : none;
                }
            }
        }
    };
    auto write = [&](lds_ptr to) {
#pragma unroll
        for (int j = 0; j < EACH; ++j)
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int block = wave + j * S::WAVES;
                *(lds_u32x4*)(to + uint32_t(i * UA + block * (A_ACROSS ? YBLOCK : XBLOCK) + lane * 16)) = a_piece[i][j];
                *(lds_u32x4*)(to + uint32_t(U * UA + i * UB + block * (B_ACROSS ? YBLOCK : XBLOCK) + lane * 16)) = b_piece[i][j];
            }
    };
    const uint32_t a_slot = uint32_t(cg * UA) + (A_ACROSS ? places_at(lane, false) : fragment_at(q, hk));
    const uint32_t b_slot = uint32_t(U * UA) + uint32_t(rg * (B_ACROSS ? 64 : 512)) + (B_ACROSS ? places_at(lane, true) : fragment_at(q, hk));

    auto work = [&](const Tile& t) {
        f32x16 acc[2][2];
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i >> 5][i >> 4 & 1][i & 15] = 0.f;
        if (t.depth > 0) load(t, 0);
        uint32_t at = 0;
        for (int z0 = 0; z0 < t.depth; z0 += 64) {
            write(lds + at);
            __syncthreads();                                   // (who is still at the other place's chunk has not written this one's successor)
            if (z0 + 64 < t.depth) load(t, z0 + 64);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                bf16x8 af[2], bf[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // (rows: block i of this wave is the i-th unit's fragment rg)
                    if constexpr (A_ACROSS) af[i] = read_across(lds + at + a_slot + uint32_t(i * 64 + ks * 2 * YBLOCK));
                    else af[i] = read_along(lds + at + a_slot + uint32_t(i * 512 + ks * 32));
                    if constexpr (B_ACROSS) bf[i] = read_across(lds + at + b_slot + uint32_t(i * UB + ks * 2 * YBLOCK));
                    else bf[i] = read_along(lds + at + b_slot + uint32_t(i * UB + ks * 32));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i & 1][i >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[i & 1], bf[i >> 1], acc[i & 1][i >> 1], 0, 0, 0);
            }
            at = BUF - at;
        }
        __syncthreads();
        const lds_ptr mine_at = lds + uint32_t(wave) * (2 * BUF / S::WAVES / 16 * 16);
        auto put = [&](auto* to, int64_t pitch) {
            using T = std::remove_pointer_t<decltype(to)>;
            constexpr int P = PIECE<T>, LANES = 64 / P, AT_ONCE = 64 / LANES, PITCH = 64 * int(sizeof(T)) + 16;
            static_assert(32 * PITCH <= int(2 * BUF / S::WAVES), "room");
            const int col = lane % LANES * P, row = lane / LANES, first = t.c0 + cg * 64, left = cols - first - col;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float v = acc[i >> 4][b][i & 15];
                    if (DIR == FORWARD && p.relu) v = v < 0.f ? 0.f : v;                                     // (a NaN stays one)
                    const lds_ptr here = mine_at + uint32_t(q * PITCH + ((i >> 4) * 32 + 16 * hk + (i & 15)) * int(sizeof(T)));
                    if constexpr (sizeof(T) == 4) *(__attribute__((address_space(3))) float*)here = v;
                    else *(__attribute__((address_space(3))) bf16_t*)here = f32_to_bf16(v);
                }
                wave_sync();
                for (int i = 0; i < 32; i += AT_ONCE) {
                    const int r = (b * 2 + rg) * 32 + row + i;
                    if (r >= t.rows || left <= 0) continue;
                    const u32x4 v = *(const lds_u32x4*)(mine_at + uint32_t((row + i) * PITCH + col * int(sizeof(T))));
                    u32x4 act;
                    const bool masked = DIR == GRAD_INPUT && p.act;
                    if (masked) act = load_piece(p.act + int64_t(t.begin + r) * p.act_stride + first + col, left);
                    float w[P];
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        w[j] = element<T>(v, j);
                        if (masked && !(element<bf16_t>(act, j) > 0.f)) w[j] = 0.f;
                    }
                    store_piece<P>(to + int64_t(r) * pitch + first + col, left, w);
                }
                wave_sync();
            }
        };
        if constexpr (DIR == GRAD_WEIGHT) {
            const size_t all = size_t(p.N) * size_t(p.K), row = size_t(t.r0) * size_t(p.K);
            if (t.slot >= 0) put(partial + size_t(t.slot) * all + row, p.K);
            else put(static_cast<TO*>(p.out) + size_t(t.e) * all + row, p.K);
        } else put(static_cast<TO*>(p.out) + int64_t(t.begin) * p.out_stride, p.out_stride);
        __syncthreads();
    };
    if constexpr (DIR == GRAD_WEIGHT) {
        const int w_lane = int(blockIdx.x) / (ct * rt);
        const Place at = walk<4>(int(blockIdx.x) % (ct * rt), rt, ct);
        const int64_t from = shares.each * w_lane, to = from + shares.each;
        for (int e = group_at(p.g, shares, from); e < p.g.E && start_of(p.g, shares, e) < to; ++e) {
            const int a = p.g.begin(e), n = max(p.g.begin(e + 1) - a, 0);
            const int64_t s = start_of(p.g, shares, e), first = s + shares.extra;
            const int lo = int(min(max(from - first, int64_t(0)), int64_t(n))), hi = int(min(max(to - first, int64_t(0)), int64_t(n)));
            if (n == 0 ? s < from : hi <= lo) continue;
            work(Tile{e, a + lo, min(p.N - at.row * S::ROWS, S::ROWS), at.col * S::COLS, at.row * S::ROWS, hi - lo, hi - lo == n ? -1 : 2 * w_lane + (lo > 0 ? 0 : 1)});
        }
    } else {
        const Place w = walk<1>(int(blockIdx.x), units / ct, ct);
        const Piece at = counted(p.g.M, p.g.E) ? count_pieces(p.g, S::ROWS, w.row, reinterpret_cast<int*>(lds_raw)) : find_piece(p.g, S::ROWS, w.row);
        if (at.rows > 0) work(Tile{at.e, at.begin, at.rows, w.col * S::COLS, 0, at.e < p.g.E ? (DIR == FORWARD ? p.K : p.N) : 0, -1});
    }
}

// Gradients whose sum a border between two lanes cuts: their parts, in order.  A workgroup looks after a share of the elements for one border, and only for the
// first one inside a group.  Few parts: a wave adds up all parts of 256 elements; many (one crowded expert, small matrices): a quarter of the parts each, or the
// loads' chain is what it takes (65536 rows, 256 x 256: 128 parts, 59 us a pass with a wave for all parts, 40 so).
constexpr int JOIN_FEW = 8;
template <typename TO>
__global__ __launch_bounds__(256) void k_join(Groups g, Shares s, const float* __restrict__ partial, TO* __restrict__ out, int64_t elements, int per_border)
{
    __shared__ f32x4 room[3][64];
    const int border = int(blockIdx.x) / per_border + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t x = s.each * border;
    const int e = group_at(g, s, x), n = max(g.begin(e + 1) - g.begin(e), 0);
    const int64_t first = start_of(g, s, e) + s.extra;
    if (x <= first || x >= first + n || x - s.each > first) return;
    int last = border;
    while (last + 1 < s.lanes && s.each * (last + 1) < first + n) ++last;
    const int parts = last - border + 2;                       // slot 2 * border - 1, then 2 * border, 2 * border + 2 ..
    auto sum = [&](int64_t i, int from, int to) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int j = from; j < to; ++j) v += __builtin_bit_cast(f32x4, load_piece(partial + int64_t(j == 0 ? 2 * border - 1 : 2 * (border + j - 1)) * elements + i, int(min(elements - i, int64_t(4)))));
        return v;
    };
    auto put = [&](int64_t i, const f32x4& v) {
        const float w[4] = {v[0], v[1], v[2], v[3]};
        store_piece<4>(out + int64_t(e) * elements + i, int(min(elements - i, int64_t(4))), w);
    };
    const int64_t share = int64_t(blockIdx.x) % per_border;
    if (parts <= JOIN_FEW) {
        for (int64_t i = (share * 256 + threadIdx.x) * 4; i < elements; i += int64_t(per_border) * 1024) put(i, sum(i, 0, parts));
        return;
    }
    for (int64_t i0 = share * 256; i0 < elements; i0 += int64_t(per_border) * 256) {
        const int64_t i = i0 + lane * 4;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (i < elements) v = sum(i, parts * wave / 4, parts * (wave + 1) / 4);
        if (wave > 0) room[wave - 1][lane] = v;
        __syncthreads();
        if (wave == 0 && i < elements) put(i, ((v + room[0][lane]) + room[1][lane]) + room[2][lane]);
        __syncthreads();
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
using Kernel = void (*)(Args, int, int, int, Shares, float*);
template <int DIR, class S>
int launch_kernel(Kernel kernel, const Args& p, int64_t grid, int64_t units, int ct, int rt, const Shares& shares, float* partial, hipStream_t st, const char* who)
{
    // LDS beyond 64 KB has to be asked for; a kernel is asked for once on every device (beyond DEVICES and KERNELS, at every call)
    constexpr int DEVICES = 64, KERNELS = 4;
    static std::atomic<Kernel> asked[DEVICES][KERNELS];
    int dev = 0, slot = 0;
    hipError_t e = hipGetDevice(&dev);
    std::atomic<Kernel>* const mine = asked[dev >= 0 && dev < DEVICES ? dev : 0];
    while (slot < KERNELS && mine[slot].load() && mine[slot].load() != kernel) ++slot;
    if (e == hipSuccess && (dev >= DEVICES || slot == KERNELS || !mine[slot].load())) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(LDS_BYTES<DIR, S>));
        Kernel none = nullptr;                                 // (two threads at once: one of them asks again at its next call)
        if (e == hipSuccess && dev < DEVICES && slot < KERNELS) mine[slot].compare_exchange_strong(none, kernel);
    }
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(S::THREADS), (LDS_BYTES<DIR, S>), st, p, int(units), ct, rt, shares, partial);
    return launched(who);
}

// forward and the input's gradient
template <int DIR>
int launch_rows(const moe_product_shape* s, const Args& p, bool fast, hipStream_t st, const char* who)
{
    const int cols = DIR == FORWARD ? s->N : s->K;
    auto launch = [&](auto kind) {
        using S = decltype(kind);
        const int ct = (cols + S::COLS - 1) / S::COLS;
        const int64_t units = (S::BIG ? int64_t(s->M) / S::ROWS + s->E + 1 : most_pieces(s->M, s->E, S::ROWS)) * ct;
        if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
        return launch_kernel<DIR, S>(p.relu || p.act ? k_product<DIR, bf16_t, S, true> : k_product<DIR, bf16_t, S, false>, p, S::BIG ? std::min<int64_t>(units, CUS) : units, units, ct, 1,
                                     Shares{}, nullptr, st, who);
    };
    if (fast) switch (kind_of(s, cols, DIR == FORWARD ? s->K : s->N)) {
        case BIG: return launch(Big{});
        case MID: return launch(Mid{});
        default: return launch(Few{});
        }
    const int ct = (cols + Mid::COLS - 1) / Mid::COLS;
    const int64_t units = most_pieces(s->M, s->E, Mid::ROWS) * ct;
    if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
    return launch_kernel<DIR, Mid>(k_product_any<DIR, bf16_t>, p, units, units, ct, 1, Shares{}, nullptr, st, who);
}

// How the weights' gradient runs: the kind of tile, and as many lanes as give the least work to the workgroup that has the most, with what adding up
// the lanes' parts takes.  In rows' time of a tile, 16 ns: a tile's way to memory is 512 of them, and a lane's two parts move some
// 2.5 times the gradient's size at 5 TB/s.
struct WeightPlan {
    bool big;
    int ct, rt;
    Shares shares;
    size_t bytes;                                              // of partial sums
};
WeightPlan weight_plan(const moe_product_shape* s, bool fast)
{
    WeightPlan w = {};
    // us, Big / Mid, into fp32 and into bfloat16, by rows, K, N, experts: 65536 x 1024 x 2048, 64 398 / 479 and 357 / 413, 256 764 / 893 and 582 / 673;
    // 65536 x 512 x 1024, 64 139 / 145 and 129 / 130; 65536 x 512 x 512, 64 94 / 63 and 74 / 63; 8192 x 4096 x 4096, 1 222 / 257 and 218 / 253;
    // 3000 x 2048 x 2048, 1 54 / 45 and 55 / 46; 16384 x 512 x 1024, 256 165 / 160 and 133 / 134; 74 x 512 x 1024, 256 108 / 102 and 61 / 52
    w.big = fast && int64_t(s->M) / 64 * ((s->K + 255) / 256) * ((s->N + 255) / 256) >= 8192;
    const int side = w.big ? 256 : 128, slots = w.big ? CUS : 2 * CUS;
    w.ct = (s->K + side - 1) / side;
    w.rt = (s->N + side - 1) / side;
    w.shares.extra = 512;
    const int64_t tiles_ = int64_t(w.ct) * w.rt, all = int64_t(s->M) + int64_t(w.shares.extra) * s->E;
    const double join = 2.5 * 4.0 * double(s->K) * double(s->N) / 5e6 / 0.016;
    double best = 0.0;
    w.shares.lanes = 1;
    for (int lanes = 1; lanes <= slots && int64_t(lanes) * 256 <= all; ++lanes) {
        const double cost = double((tiles_ * lanes + slots - 1) / slots) * double(all) / lanes + (lanes - 1) * join;
        if (lanes == 1 || cost < best) { best = cost; w.shares.lanes = lanes; }
    }
    w.shares.each = (all + w.shares.lanes - 1) / w.shares.lanes;
    w.bytes = w.shares.lanes > 1 ? size_t(w.shares.lanes) * 2 * size_t(s->K) * size_t(s->N) * 4 : 0;
    return w;
}


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
    const bool fast = s->K % 8 == 0 && s->N % 8 == 0 && in_stride % 8 == 0 && out_stride % 8 == 0 && on_16({in, W, out}) && reached(g, in_stride, 0);
    return launch_rows<FORWARD>(s, p, fast, static_cast<hipStream_t>(stream), "moe_product");
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
    const bool fast = s->K % 8 == 0 && s->N % 8 == 0 && dout_stride % 8 == 0 && act_stride % 8 == 0 && din_stride % 8 == 0 && on_16({dout, W, act, din}) && reached(g, 0, dout_stride);
    return launch_rows<GRAD_INPUT>(s, p, fast, static_cast<hipStream_t>(stream), "moe_product_grad_input");
}

extern "C" size_t moe_product_grad_weight_workspace_bytes(const moe_product_shape* s)
{
    if (check(s, "moe_product_grad_weight_workspace_bytes") != DYNB_OK) return 0;
    // (which of the two runs depends on addresses, too)
    return std::max<size_t>({weight_plan(s, true).bytes, weight_plan(s, false).bytes, 256});
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
    const bool fast = s->K % 8 == 0 && s->N % 8 == 0 && dout_stride % 8 == 0 && in_stride % 8 == 0 && on_16({dout, in, dW}) && reached(g, in_stride, dout_stride);
    const WeightPlan w = weight_plan(s, fast);
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* const partial = static_cast<float*>(workspace);
    const int64_t grid = int64_t(w.ct) * w.rt * w.shares.lanes, elements = int64_t(s->K) * s->N;
    if (grid > MOST_GROUPS / 2) return fail(DYNB_E_UNSUPPORTED, "moe_product_grad_weight: too many results");
    auto launch = [&](auto to) {
        using TO = decltype(to);
        const char* const who = "moe_product_grad_weight";
        const int done = w.big ? launch_kernel<GRAD_WEIGHT, Big>(k_product<GRAD_WEIGHT, TO, Big, false>, p, grid, 0, w.ct, w.rt, w.shares, partial, st, who)
                               : launch_kernel<GRAD_WEIGHT, Mid>(fast ? k_product<GRAD_WEIGHT, TO, Mid, false> : k_product_any<GRAD_WEIGHT, TO>, p, grid, 0, w.ct, w.rt, w.shares, partial, st, who);
        if (done != DYNB_OK || w.shares.lanes == 1) return done;
        const int per_border = int(std::min<int64_t>((elements + 255) / 256, std::max(64, 2048 / (w.shares.lanes - 1))));
        hipLaunchKernelGGL((k_join<TO>), dim3(unsigned((w.shares.lanes - 1) * per_border)), dim3(256), 0, st, p.g, w.shares, partial, static_cast<TO*>(dW), elements, per_border);
        return launched(who);
    };
    return grad_dtype == DYNB_BF16 ? launch(bf16_t{}) : launch(float{});
}
