// The first half of a gated feed-forward layer of experts, out = f(in Wg_e^T) (in Wu_e^T), and the gradients of its gate and up through the second layer's product:
// dact = dout W_e, dgate = dact up f'(gate), dup = dact f(gate).  W is [E][2][h][K], so that [dgate, dup] and W are an ordinary layer's (N = 2 h) for the products that remain.
//
// Either is one launch: the products are the tiles of moe_tiles.h, and the gate is where a tile leaves, on sums in fp32.  A wave has gate and up of the same features in the same lane
// (pair_feature), so the forward pass writes h numbers a row where a product and a gate of its own would write 2 h, read them and write h; what the backward pass needs is written
// beside, in bfloat16 or 8 bits.  Backward a tile's dact never leaves the CU.
// Bounds: products where a group has hundreds of rows, the weights' bytes where it has few.  us on this card (products by hipBLASLt reach 1.36 PFLOP/s, copies 4.8 TB/s):
//   forward, 8192 rows, 2048 -> 2 x 4096, one expert       224 (1.23 PFLOP/s), with the pair in bf16 236, in 8 bits 243.  206 of them are the tiles' loop
//   forward, 65536 rows, 1024 -> 2 x 2048, 64 experts      585 (0.94 PFLOP/s), 640, 685.  505 are the loop: 16 chunks a tile, and one wave a SIMD, which multiplies nothing while a
//                                                          tile leaves; of the rest the stores are 15 without a pair, the arithmetic in 8 bits 40
//   backward, 65536 rows, 1024 x 2048, 64 experts          490 from bf16, 467 from 8 bits: 275 GFLOP and 1.4 GB; without the stores 340
//   forward, 148 rows, 256 experts, 1024 -> 2 x 2048       91 (504 MB of weights at 5.5 TB/s)
//   forward, one row, 2048 -> 2 x 4096                     7.4 (33.6 MB), 8192 -> 2 x 8192 42 (6.4 TB/s)
//   backward, 8192 rows, 256 experts, 512 x 1024           78 to 82 (360 MB at 4.5 TB/s)
#include "moe_tiles.h"

namespace {

// ------------------------------------------------------------------------------------------ any size, stride and address
// 128 columns (64 features' gate and up) by 128 or 64 rows, by way of registers: pieces of 16 bytes are loaded from wherever they lie and wait there, DEPTH chunks of 64 places of the sum
// ahead, then go where a copy would have put them.  Places of rows and features are found once a tile; behind a tile's last row or feature the last one is loaded again, and the
// results that it gives go nowhere.  Only the last chunk looks where its rows end.  A chunk's arithmetic (16 products a wave) covers a fraction of
// memory's latency: with one chunk ahead 3001 rows, 777 -> 2 x 1001, 8 experts, the pair in bf16 take 47 us, with three 28 (776 -> 2 x 1000 by the kernels below: 22).
template <int DIR, class S, int KEEP>
__device__ __forceinline__ void gated_any(const Args& p, const Gate& gate, const Tile& t, lds_ptr lds)
{
    constexpr bool A_ACROSS = DIR != FORWARD;
    constexpr int DEPTH = 3, AU = S::COLS / 64, BU = S::ROWS / 64, EACH = 8 / S::WAVES, UA = A_ACROSS ? YUNIT : XUNIT, UB = XUNIT, FA = S::FA, NB = S::NB;
    constexpr uint32_t BUF = BUF_BYTES<DIR, S>;
    using lds_u32x4 = __attribute__((address_space(3))) u32x4;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, q = lane & 31, hk = lane >> 5, cg = wave % S::CG, rg = wave / S::CG;
    const int h = gate.h, nchunk = (t.depth + 63) / 64, along = (lane & 7) * 8;
    const bf16_t *a_at[AU][EACH], *b_at[BU][EACH];
    int a_left[AU];                                            // backward: columns from the piece's first
    const bf16_t* const w = p.a + size_t(t.e) * size_t(p.N) * size_t(p.K);
    if (nchunk > 0) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int block = wave + j * S::WAVES, s_q = copied_row(block, lane);
#pragma unroll
            for (int i = 0; i < AU; ++i) {
                if constexpr (DIR == FORWARD) {
                    const int feature = min(t.c0 + (i * 2 + (lane >> 5)) * 16 + pair_feature(s_q), h - 1);
                    a_at[i][j] = w + (size_t(s_q >> 4) * size_t(h) + size_t(feature)) * size_t(p.K) + along;
                } else {
                    const int col = t.c0 + i * 64 + along;
                    a_left[i] = h - col;
                    a_at[i][j] = w + size_t(min(copied_place(block, lane), t.depth - 1)) * size_t(p.K) + min(col, h - 1);
                }
            }
#pragma unroll
            for (int i = 0; i < BU; ++i) b_at[i][j] = p.b + p.g.row(t.begin + min(i * 64 + (lane >> 5) * 32 + s_q, t.rows - 1)) * p.b_stride + along;
        }
    }
    struct Chunk { u32x4 a[AU][EACH], b[BU][EACH]; } chunks[DEPTH];
    const u32x4 none = {0u, 0u, 0u, 0u};
    auto load = [&](Chunk& to, int c) {
        if (c >= nchunk) return;
        const size_t z = size_t(c) * 64;
        if (c < nchunk - 1 && (!A_ACROSS || h >= 8)) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                // (a piece of the weights that reaches over its row's end has the next row's beginning there, in columns that go nowhere; there is a next row, of eight columns or more)
#pragma unroll
                for (int i = 0; i < AU; ++i) to.a[i][j] = load_piece(a_at[i][j] + (A_ACROSS ? z * size_t(p.K) : z), 8);
#pragma unroll
                for (int i = 0; i < BU; ++i) to.b[i][j] = load_piece(b_at[i][j] + z, 8);
            }
            return;
        }
        const int rest = t.depth - int(z) - along;
        if (t.depth >= 8 && (!A_ACROSS || h >= 8)) {
            // Whole pieces all the same: one that would reach over its row's end is the row's last eight elements, without those that another lane has
            const int gone = min(max(8 - rest, 0), 8);
            const int64_t from = gone > 0 ? int64_t(t.depth) - 8 - along : int64_t(z);
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int place = int(z) + copied_place(wave + j * S::WAVES, lane), last = t.depth - 1;
#pragma unroll
                for (int i = 0; i < AU; ++i) {
                    if constexpr (!A_ACROSS) to.a[i][j] = without_first(load_piece(a_at[i][j] + from, 8), gone);
                    else {
                        // (over its end is the next row's beginning, in columns that go nowhere, but behind the last row)
                        const int left = max(a_left[i], 1);
                        const bool over = place >= last && left < 8;
                        const u32x4 v = load_piece(w + size_t(min(place, last)) * size_t(p.K) + (h - (over ? 8 : left)), 8);
                        to.a[i][j] = without_first(v, place > last ? 8 : over ? 8 - left : 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < BU; ++i) to.b[i][j] = without_first(load_piece(b_at[i][j] + from, 8), gone);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int place = int(z) + copied_place(wave + j * S::WAVES, lane);
#pragma unroll
            for (int i = 0; i < AU; ++i) {
                if constexpr (!A_ACROSS) to.a[i][j] = rest > 0 ? load_piece(a_at[i][j] + z, rest) : none;
                else to.a[i][j] = place < t.depth && a_left[i] > 0 ? load_piece(w + size_t(place) * size_t(p.K) + (h - a_left[i]), a_left[i]) : none;
            }
#pragma unroll
            for (int i = 0; i < BU; ++i) to.b[i][j] = rest > 0 ? load_piece(b_at[i][j] + z, rest) : none;
        }
    };
    auto write = [&](const Chunk& from, lds_ptr to) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int block = wave + j * S::WAVES;
#pragma unroll
            for (int i = 0; i < AU; ++i) *(lds_u32x4*)(to + uint32_t(i * UA + block * (A_ACROSS ? YBLOCK : XBLOCK) + lane * 16)) = from.a[i][j];
#pragma unroll
            for (int i = 0; i < BU; ++i) *(lds_u32x4*)(to + uint32_t(AU * UA + i * UB + block * XBLOCK + lane * 16)) = from.b[i][j];
        }
    };
    const uint32_t a_slot = uint32_t(cg * FA / 2 * UA) + (A_ACROSS ? places_at(lane, false) : fragment_at(q, hk)), b_slot = uint32_t(AU * UA) + fragment_at(q, hk);
    f32x16 acc[FA][NB];
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
#pragma unroll
    for (int n = 0; n < DEPTH; ++n) load(chunks[n], n);
    uint32_t at = 0;
    auto one = [&](Chunk& chunk, int c) {
        if (c >= nchunk) return;
        write(chunk, lds + at);
        meet();                                                // (who is still at the other place's chunk has not written this one's successor)
        load(chunk, c + DEPTH);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            bf16x8 af[FA], bf[NB];
#pragma unroll
            for (int a = 0; a < FA; ++a) {
                if constexpr (A_ACROSS) af[a] = read_across(lds + (at + a_slot + uint32_t(a / 2 * UA + a % 2 * 64 + ks * 2 * YBLOCK)));
                else af[a] = read_along(lds + (at + a_slot + uint32_t(a / 2 * UA + a % 2 * 512 + ks * 32)));
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) bf[b] = read_along(lds + (at + b_slot + uint32_t((b * S::RG + rg) / 2 * UB + (b * S::RG + rg) % 2 * 512 + ks * 32)));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int a = 0; a < FA; ++a) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[a], bf[b], acc[a][b], 0, 0, 0);
        }
        at = BUF - at;
    };
#pragma unroll 1
    for (int c = 0; c < nchunk; c += DEPTH)
#pragma unroll
        for (int n = 0; n < DEPTH; ++n) one(chunks[n], c + n);
    meet();
    constexpr int ROOM = int(2 * BUF / S::WAVES / 16 * 16);
    if constexpr (DIR == FORWARD) leave_pairs<S, NB, KEEP, false, ROOM>(acc, gate, p, t, lds + uint32_t(wave * ROOM), nchunk > 0, lane, cg, rg);
    else leave_grads<S, NB, KEEP, false, ROOM>(acc, gate, p, t, lds + uint32_t(wave * ROOM), nchunk > 0, lane, cg, rg);
}
template <int DIR, class S, int KEEP>
__global__ __launch_bounds__(S::THREADS, S::SIMD) void k_gated_any(Args p, GateKeeping<KEEP> gate, int units, int ct)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    const Place w = walk<1>(int(blockIdx.x), units / ct, ct);
    const Piece at = counted(p.g.M, p.g.E) ? count_pieces(p.g, S::ROWS, w.row, reinterpret_cast<int*>(lds_raw)) : find_piece(p.g, S::ROWS, w.row);
    if (at.rows > 0)
        gated_any<DIR, S, KEEP>(p, gate, Tile{at.e, at.begin, at.rows, w.col * (DIR == FORWARD ? S::COLS / 2 : S::COLS), 0, at.e < p.g.E ? (DIR == FORWARD ? p.K : p.N) : 0, -1}, (lds_ptr)lds_raw);
}

// ------------------------------------------------------------------------------------------ K and h multiples of 8, rows on 16-byte borders
template <int DIR, class S, int KEEP>
__global__ __launch_bounds__(S::THREADS, S::SIMD) void k_gated(Args p, GateKeeping<KEEP> gate, int units, int ct)
{
    product_tiles<DIR, bf16_t, S, false>(p, gate, units, ct, 1, Shares{}, nullptr);
}

// ------------------------------------------------------------------------------------------ few rows, nothing kept
// Tokens that are being answered: their experts' weights are read once, and that is all there is to do.  A workgroup takes NA blocks of 8 features, each 16 rows of weights (of four
// neighbours: gate's of two features, up's of the same, which are a lane's four sums), and up to 16 rows of one group: the matrix instructions take 16 rows in the time of one.  Its waves take every
// WAVES-th 64 channels each, straight into registers with DEPTH of them on their way at once, and their sums meet in LDS and are added up in order.  A lane has 32 neighbouring bytes of a
// row's 64 channels, half of them in either product.
constexpr int ROWS_FEW = 16;
template <int NA, int DEPTH>
__global__ __launch_bounds__(256) void k_gated_few(Args p, Gate gate, int ct)
{
    constexpr int WAVES = 4;
    __shared__ __attribute__((aligned(16))) float sums[WAVES * NA * 256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane & 15, h = gate.h;
    const Place place = walk<1>(int(blockIdx.x), int(gridDim.x) / ct, ct);
    const Piece at = counted(p.g.M, p.g.E) ? count_pieces(p.g, ROWS_FEW, place.row, reinterpret_cast<int*>(sums)) : find_piece(p.g, ROWS_FEW, place.row);
    if (at.rows <= 0) return;
    const int f0 = place.col * NA * 8;
    f32x4 acc[NA] = {};
    if (at.e < p.g.E) {
        const bf16_t* w[NA];
#pragma unroll
        for (int n = 0; n < NA; ++n) w[n] = p.a + (size_t(at.e) * 2 * size_t(h) + (q & 2 ? size_t(h) : 0) + size_t(min(f0 + n * 8 + (q >> 2) * 2 + (q & 1), h - 1))) * size_t(p.K);
        const bf16_t* const x = p.b + p.g.row(at.begin + min(q, at.rows - 1)) * p.b_stride;
        for (int k0 = wave * 64; k0 < p.K; k0 += DEPTH * WAVES * 64) {
            u32x4 a[DEPTH][2][NA] = {}, b[DEPTH][2] = {};
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int k = k0 + d * WAVES * 64 + (lane >> 4) * 16 + s * 8;
                    if (k >= p.K) continue;
#pragma unroll
                    for (int n = 0; n < NA; ++n) a[d][s][n] = *reinterpret_cast<const u32x4*>(w[n] + k);
                    b[d][s] = *reinterpret_cast<const u32x4*>(x + k);
                }
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < NA; ++n)
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[d][s][n]), __builtin_bit_cast(bf16x8, b[d][s]), acc[n], 0, 0, 0);
        }
    }
#pragma unroll
    for (int n = 0; n < NA; ++n) *reinterpret_cast<f32x4*>(sums + (n * WAVES * 64 + tid) * 4) = acc[n];
    __syncthreads();
    if (wave >= NA || q >= at.rows) return;                    // (wave n leaves with block n of features)
    f32x4 sum = *reinterpret_cast<const f32x4*>(sums + (wave * WAVES * 64 + lane) * 4);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += *reinterpret_cast<const f32x4*>(sums + ((wave * WAVES + w) * 64 + lane) * 4);
    const int f = f0 + wave * 8 + (lane >> 4) * 2;
    bf16_t* const to = static_cast<bf16_t*>(p.out) + int64_t(at.begin + q) * p.out_stride + f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (f + i < h) to[i] = f32_to_bf16((gate.form.b2 == 0.f ? gate_silu(sum[i]) : gate_f(gate.form, sum[i])) * sum[2 + i]);
}

int check(const moe_gated_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->M < 0 || s->K <= 0 || s->h <= 0 || s->E <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": only DYNB_BF16");
    if (s->flags > MOE_GATE_GELU) return fail(DYNB_E_UNSUPPORTED, who + ": unknown flag");
    if (s->M > 1 << 30 || s->E > 1 << 20 || s->K > 1 << 22 || s->h > 1 << 21) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^30 rows, 2^22 channels, 2^21 hidden features or 2^20 experts");
    return DYNB_OK;
}
int check_pre(const moe_gated_shape* s, const moe_gated_pre* p, const std::string& who)
{
    if (p->dtype != DYNB_BF16 && p->dtype != DYNB_I8) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype of what is kept");
    if (!p->rows || (p->dtype == DYNB_I8 && !p->scale)) return fail(DYNB_E_INVAL, who + ": NULL pre");
    if (p->stride < 2 * int64_t(s->h) || (p->dtype == DYNB_I8 && p->scale_stride < 2 * ((int64_t(s->h) + BLOCK8 - 1) / BLOCK8)))
        return fail(DYNB_E_INVAL, who + ": rows of pre overlap (stride below their length)");
    if ((p->dtype == DYNB_BF16 && odd(p->rows)) || (p->dtype == DYNB_I8 && odd(p->scale))) return fail(DYNB_E_INVAL, who + ": misaligned pre");
    return DYNB_OK;
}
// written: bytes of results for a row's feature
Gate gate_of(const moe_gated_shape* s, const moe_gated_pre* p, void* hidden, int64_t hidden_stride, int written)
{
    constexpr double LOG2E = 1.4426950408889634, C = 1.5957691216057308;                   // 2 sqrt(2 / pi)
    const double a = s->flags == MOE_GATE_GELU ? C : 1.0, b = s->flags == MOE_GATE_GELU ? C * 0.044715 : 0.0;
    Gate g = {};
    g.form = GateForm{float(-LOG2E * a), float(-LOG2E * b), float(a), float(3 * b)};
    g.h = s->h;
    g.keep = !p ? KEEP_NOTHING : p->dtype == DYNB_BF16 ? KEEP_BF16 : KEEP_8;
    if (p) {
        g.pre = p->rows;
        g.pre_stride = p->stride;
        g.scale = static_cast<bf16_t*>(p->scale);
        g.scale_stride = p->scale_stride;
        g.on_16 = s->h % 16 == 0 && p->stride % 16 == 0 && on_16({p->rows});
    }
    g.hidden = static_cast<bf16_t*>(hidden);
    g.hidden_stride = hidden_stride;
    g.past = int64_t(s->M) * s->h * written >= PAST;
    return g;
}

// LDS beyond 64 KB has to be asked for: a kernel is asked for once on every device (beyond DEVICES, at every call)
template <class K, class... A>
int launch_with(K kernel, std::atomic<bool>* asked, uint32_t lds, int64_t grid, int threads, hipStream_t st, const char* who, A... args)
{
    constexpr int DEVICES = 64;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && (dev < 0 || dev >= DEVICES || !asked[dev].load())) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e == hipSuccess && dev >= 0 && dev < DEVICES) asked[dev].store(true);
    }
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(unsigned(threads)), lds, st, args...);
    return launched(who);
}

template <int DIR, class S, int KEEP, bool ANY>
int launch_kind(const moe_product_shape* s, const Args& p, const Gate& gate, hipStream_t st, const char* who)
{
    static std::atomic<bool> asked[64];
    const int wide = DIR == FORWARD ? S::COLS / 2 : S::COLS, ct = (gate.h + wide - 1) / wide;
    const int64_t units = (S::BIG ? int64_t(s->M) / S::ROWS + s->E + 1 : most_pieces(s->M, s->E, S::ROWS)) * ct;
    if (units > MOST_GROUPS) return fail(DYNB_E_UNSUPPORTED, std::string(who) + ": too many results");
    GateKeeping<KEEP> g = {};
    static_cast<Gate&>(g) = gate;
    const int64_t grid = S::BIG ? std::min<int64_t>(units, CUS) : units;
    if constexpr (ANY) return launch_with(k_gated_any<DIR, S, KEEP>, asked, 2 * BUF_BYTES<DIR, S>, grid, S::THREADS, st, who, p, g, int(units), ct);
    else return launch_with(k_gated<DIR, S, KEEP>, asked, LDS_BYTES<DIR, S>, grid, S::THREADS, st, who, p, g, int(units), ct);
}

// Few with waves of 64 columns and 32 rows: what is kept in 8 bits shares a scale among 32 features, which have to be a wave's (148 rows, 256 experts, 1024 -> 2 x 2048: 94 us, by
// Mid 104, Few without a pair 91)
using FewWide = Kind<2, 1, 2, 2, 3, 2>;
// Half of Few's columns: twice the workgroups where Few's leave half of the CUs without work.  What bounds those is the way of a workgroup's stream of weights into its CU (one row,
// 2048 -> 2 x 4096, the pair in bf16: 13.4 us by Few, 12.0 so; backward 14.8, 12.2; 64 rows, 1024 -> 2 x 2048: 8.9, 7.7; backward 11.0, 8.6; five chunks ahead instead of two: 12.8)
using Narrow = Kind<1, 1, 2, 2, 3, 2>;
using AnyMid = Kind<2, 2, 2, 2, 2, 2>;   // 128 x 128
using AnyFew = Kind<2, 1, 2, 2, 2, 2>;   // 128 columns x 64 rows

template <int DIR>
int launch_gated(const moe_product_shape* s, const Args& p, const Gate& gate, bool fast, hipStream_t st, const char* who)
{
    auto keeping = [&](auto kind, auto any) {
        using S = decltype(kind);
        constexpr bool ANY = decltype(any)::value;
        if (gate.keep == KEEP_8) return launch_kind<DIR, std::conditional_t<DIR == FORWARD && S::FA == 1, FewWide, S>, KEEP_8, ANY>(s, p, gate, st, who);
        if constexpr (DIR == FORWARD)
            if (gate.keep == KEEP_NOTHING) return launch_kind<DIR, S, KEEP_NOTHING, ANY>(s, p, gate, st, who);
        return launch_kind<DIR, S, KEEP_BF16, ANY>(s, p, gate, st, who);
    };
    // The products' rule.  us of the gated layer, forward without a pair / backward from bf16, by rows, K, h, experts, Zipf exponent:
    //                                   Big          Mid          Few
    //   1000 x 1024 x 512, 8, 0.5       29 / 42      14 / 14      10 / 9
    //   3000 x 2048 x 1024, 1           47 / 61      30 / 30      37 / 25
    //   4096 x 2048 x 1024, 16, 0.6     58 / 63      55 / 33      64 / 41
    //   8192 x 512 x 1024, 64, 0.8      52 / 57      39 / 33      42 / 32
    //   16384 x 512 x 1024, 256, 0.8   160 / 126    146 / 96     133 / 98
    //   16384 x 1024 x 1024, 64, 0.8   120 / 84     108 / 69     124 / 77
    //   32768 x 1024 x 1024, 32, 0.6   149 / 130    162 / 112    204 / 133
    //   65536 x 512 x 512, 64, 0.6      92 / 100     92 / 80     117 / 93
    //   65536 x 1024 x 1024, 256, 0.6  412 / 315    461 / 314    521 / 362
    //   65536 x 1024 x 2048, 64, 0.6   586 / 489    845 / 541   1207 / 679
    // (the rule takes the best of a line or one within 5 %; with the pair in 8 bits 16384 rows of 2048 -> 2 x 1024 take 170 by Big, 159 by Mid)
    const KindOf kind = kind_of(s, DIR == FORWARD ? s->N : s->K, DIR == FORWARD ? s->K : s->N);
    if (!fast) return kind == FEW ? keeping(AnyFew{}, std::true_type{}) : keeping(AnyMid{}, std::true_type{});
    switch (kind) {
    case BIG: return keeping(Big{}, std::false_type{});
    case MID: return keeping(Mid{}, std::false_type{});
    default: {
        const int wide = DIR == FORWARD ? Few::COLS / 2 : Few::COLS;
        return most_pieces(s->M, s->E, Few::ROWS) * ((gate.h + wide - 1) / wide) <= CUS / 2 ? keeping(Narrow{}, std::false_type{}) : keeping(Few{}, std::false_type{});
    }
    }
}

// Where this layer's tiles would leave CUs without work, and give the others one stream of weights after the other: up to 16 rows, and as many blocks of 8 features as start at once.  us, by rows, K, h,
// experts and the blocks that are launched:
//                                      tiles   1 block   2 blocks a workgroup
//   1 x 512 x 1024, 1           128      4.9     3.2       3.7
//   2 x 512 x 1024, 256         256      6.2     4.4       4.9
//   1 x 2048 x 4096, 1          512     11.9     7.5       7.6
//   16 x 2048 x 512, 1          128     11.1     6.1       7.9
//   8 x 4096 x 1024, 1          128     19.8     9.1      12.5
//   16 x 2048 x 4096, 1        1024     12.0    10.3       8.9
//   4 x 1024 x 2048, 64        1024      9.3     9.5       8.1
//   1 x 8192 x 8192, 1         1024     58.8    45.0      41.8
//   8 x 4096 x 1536, 128       1536     30.9    34.4      34.0
//   16 x 512 x 1024, 256       2048      6.9    12.2       7.3
template <int NA, int DEPTH>
int launch_few(const moe_product_shape* s, const Args& p, const Gate& gate, hipStream_t st)
{
    const int ct = (gate.h + NA * 8 - 1) / (NA * 8);
    hipLaunchKernelGGL((k_gated_few<NA, DEPTH>), dim3(unsigned(most_pieces(s->M, s->E, ROWS_FEW) * ct)), dim3(256), 0, st, p, gate, ct);
    return launched("moe_gated");
}

// whether what is kept lies on borders of 8 elements, and 32 rows of scales within 32 bits
bool kept_on_8(const moe_gated_pre* p)
{
    if (!p) return true;
    if (p->dtype == DYNB_BF16) return p->stride % 8 == 0 && on_16({p->rows});
    return p->stride % 8 == 0 && (reinterpret_cast<uintptr_t>(p->rows) & 7) == 0 && p->scale_stride <= 1 << 27;
}

}  // namespace

extern "C" int moe_gated(const moe_gated_shape* s, const moe_groups* g, const void* in, int64_t in_stride, const void* W, void* out, int64_t out_stride, const moe_gated_pre* pre, void* stream)
{
    int rc = check(s, "moe_gated");
    if (rc != DYNB_OK) return rc;
    const moe_product_shape as = {s->M, s->K, 2 * s->h, s->E, DYNB_BF16, 0};
    rc = check_groups(&as, g, true, "moe_gated");
    if (rc == DYNB_OK && pre && s->M > 0) rc = check_pre(s, pre, "moe_gated");
    if (rc != DYNB_OK || s->M == 0) return rc;
    if (!in || !W || !out) return fail(DYNB_E_INVAL, "moe_gated: NULL argument");
    if (in_stride < s->K || out_stride < s->h) return fail(DYNB_E_INVAL, "moe_gated: rows overlap (stride below their length)");
    if (odd(in) || odd(W) || odd(out)) return fail(DYNB_E_INVAL, "moe_gated: misaligned pointer");
    const Args p = {groups_of(&as, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(in), 0, in_stride, nullptr, 0, out, out_stride, as.K, as.N, 0};
    const Gate gate = gate_of(s, pre, nullptr, 0, !pre ? 2 : pre->dtype == DYNB_BF16 ? 6 : 4);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!pre && s->M <= ROWS_FEW && s->K % 8 == 0 && in_stride % 8 == 0 && on_16({in, W})) {
        const int64_t blocks = (most_pieces(s->M, s->E, ROWS_FEW) - 1) * ((s->h + 7) / 8);
        if (blocks <= 2 * CUS) return launch_few<1, 8>(&as, p, gate, st);
        if (blocks <= 4 * CUS) return launch_few<2, 4>(&as, p, gate, st);
    }
    // (32-bit offsets within an expert's two matrices: up's rows lie h rows behind gate's)
    const bool fast = s->K % 8 == 0 && s->h % 8 == 0 && in_stride % 8 == 0 && out_stride % 8 == 0 && on_16({in, W, out}) && kept_on_8(pre) && reached(g, in_stride, 0) &&
                      (int64_t(s->h) + 256) * s->K * 2 < int64_t(1) << 32;
    return launch_gated<FORWARD>(&as, p, gate, fast, st, "moe_gated");
}

extern "C" int moe_gated_grad(const moe_gated_shape* s, const moe_groups* g, const void* dout, int64_t dout_stride, const void* W, const moe_gated_pre* pre, void* dpre, int64_t dpre_stride,
                              void* hidden, int64_t hidden_stride, void* stream)
{
    int rc = check(s, "moe_gated_grad");
    if (rc != DYNB_OK) return rc;
    const moe_product_shape as = {s->M, s->h, s->K, s->E, DYNB_BF16, 0};
    rc = check_groups(&as, g, false, "moe_gated_grad");
    if (rc != DYNB_OK || s->M == 0) return rc;
    if (!dout || !W || !pre || !dpre) return fail(DYNB_E_INVAL, "moe_gated_grad: NULL argument");
    rc = check_pre(s, pre, "moe_gated_grad");
    if (rc != DYNB_OK) return rc;
    if (dout_stride < s->K || dpre_stride < 2 * int64_t(s->h) || (hidden && hidden_stride < s->h)) return fail(DYNB_E_INVAL, "moe_gated_grad: rows overlap (stride below their length)");
    if (odd(dout) || odd(W) || odd(dpre) || odd(hidden)) return fail(DYNB_E_INVAL, "moe_gated_grad: misaligned pointer");
    const Args p = {groups_of(&as, g), static_cast<const bf16_t*>(W), static_cast<const bf16_t*>(dout), 0, dout_stride, nullptr, 0, dpre, dpre_stride, as.K, as.N, 0};
    const bool fast = s->K % 8 == 0 && s->h % 8 == 0 && dout_stride % 8 == 0 && dpre_stride % 8 == 0 && hidden_stride % 8 == 0 && on_16({dout, W, dpre, hidden}) && kept_on_8(pre) &&
                      reached(g, 0, dout_stride);
    return launch_gated<GRAD_INPUT>(&as, p, gate_of(s, pre, hidden, hidden_stride, hidden ? 6 : 4), fast, static_cast<hipStream_t>(stream), "moe_gated_grad");
}
