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

#include "device_utils.h"
#include "lds_copy.h"
#include "plan_internal.h"
#include "rows.h"

using dynb::fail;

namespace {

struct Groups {
    const int32_t* offsets;   // [E + 1]; the first is taken as 0, and all are kept within 0 .. M
    const int32_t* perm;      // row r of the groups is row perm[r] / k of the gathered tensor, or null
    int32_t k, rows;          // ... which has `rows` rows
    int32_t M, E;
    __device__ __forceinline__ int begin(int e) const { return e <= 0 ? 0 : e > E ? M : min(max(offsets[e], 0), M); }
    __device__ __forceinline__ uint32_t row_of(int32_t use) const { return min(uint32_t(use) / uint32_t(k), uint32_t(rows - 1)); }
    __device__ __forceinline__ int64_t row(int r) const { return perm ? row_of(perm[r]) : r; }
};

struct Piece { int e, begin, rows; };                          // rows begin .. of group e (E: what lies behind the last group)

__device__ __forceinline__ Piece piece_of(int P, int unit, int e, int a, int b)
{
    Piece p;
    p.e = e;
    const int rows = b - a, part = unit - (a / P + e);
    p.begin = a + part * P;
    p.rows = rows > 0 && part <= (rows - 1) / P ? min(P, rows - part * P) : 0;
    return p;
}
// the unit's group and its piece of at most P rows (0: it has none).  All 64 lanes of a wave call it.
__device__ __forceinline__ Piece find_piece(const Groups& g, int P, int unit)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = g.E + 1;                                   // the group is one of lo .. lo + n - 1
    while (n > 63) {
        const int step = (n + 63) / 64, e = lo + lane * step;
        const bool here = lane * step < n && g.begin(e) / P + e <= unit;
        const int last = 63 - __builtin_clzll(__ballot(here) | 1ull);
        lo += last * step;
        n = min(step, n - last * step);
    }
    // (a lane a group, and one behind them: the group's borders need no further load)
    const int e = lo + lane, begin = g.begin(min(e, g.E + 1));
    const int last = 63 - __builtin_clzll(__ballot(lane < n && begin / P + e <= unit) | 1ull);
    return piece_of(P, unit, lo + last, __builtin_amdgcn_readlane(begin, last), __builtin_amdgcn_readlane(begin, last + 1));
}
// ... for every lane its own
__device__ __forceinline__ Piece find_piece_alone(const Groups& g, int P, int unit)
{
    int lo = 0, n = g.E + 1;
    while (n > 1) {
        const int half = n >> 1;
        if (g.begin(lo + half) / P + lo + half <= unit) { lo += half; n -= half; }
        else n = half;
    }
    return piece_of(P, unit, lo, g.begin(lo), g.begin(lo + 1));
}

// Fewer rows than groups: most groups are empty, and a launch with room for them all would be workgroups with nothing to do for the most part (74 rows, 256
// experts, K 512: 13.3 us, 9.8 with room for as many groups as rows).  The unit counts pieces then: every workgroup of 256 threads adds them up.
constexpr int COUNTED = 2048;            // most groups, eight a thread
__host__ __device__ __forceinline__ bool counted(int M, int E) { return M < E && E < COUNTED; }
__host__ __device__ __forceinline__ int64_t most_pieces(int M, int E, int P) { return int64_t(M) / P + (counted(M, E) ? M : E) + 1; }
// All 256 threads call it; room: 7 ints of LDS
__device__ __forceinline__ Piece count_pieces(const Groups& g, int P, int unit, int* room)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (g.E + 256) / 256, e0 = min(tid * per, g.E + 1), e1 = min(e0 + per, g.E + 1);
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += (max(g.begin(e + 1) - g.begin(e), 0) + P - 1) / P;
    int ahead = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(ahead, o);
        ahead += lane >= o ? v : 0;
    }
    if (lane == 63) room[wave] = ahead;
    if (tid == 0) room[6] = 0;
    __syncthreads();
    ahead -= mine;
    for (int w = 0; w < wave; ++w) ahead += room[w];
    if (unit >= ahead && unit < ahead + mine)
        for (int e = e0; e < e1; ++e) {
            const int a = g.begin(e), n = max(g.begin(e + 1) - a, 0), pieces = (n + P - 1) / P;
            if (unit < ahead + pieces) {
                room[4] = e;
                room[5] = a + (unit - ahead) * P;
                room[6] = min(P, n - (unit - ahead) * P);
                break;
            }
            ahead += pieces;
        }
    __syncthreads();
    const Piece p = {__builtin_amdgcn_readfirstlane(room[4]), __builtin_amdgcn_readfirstlane(room[5]), __builtin_amdgcn_readfirstlane(room[6])};
    __syncthreads();
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

// ------------------------------------------------------------------------------------------ K and N multiples of 8, rows on 16-byte borders
// Tiles of results whose operands go straight from memory into LDS, a chunk of 64 places of the sum at a time and at least one chunk ahead, and
// are multiplied by 32x32x16 MFMAs.  Both operands lie in LDS as they lie in memory.  One whose places of the sum are neighbours there ("along": the rows and the weights of
// the forward pass, the rows of the input's gradient) is read 16 bytes a lane; one whose places are rows ("across": the weights of the input's gradient, both
// operands of the weights' gradient) by the transposing LDS load, four places of one column a lane.
//
// An across unit is 64 places x 64 columns in eight blocks of 8 places (128 bytes each).  The four places that 32 lanes read together are two neighbours of an
// even and two of an odd block, and blocks are 64 bytes further apart than their size: all banks.
constexpr int YBLOCK = 1024 + 64, YUNIT = 8 * YBLOCK;
// the place of the sum that lane `lane` copies into block `block`
__device__ __forceinline__ int copied_place(int block, int lane) { return (block >> 1) * 16 + (lane >> 4) * 4 + (block & 1) * 2 + (lane >> 3 & 1); }
// where in a unit lane `lane` reads four places of its column of the first 32 (the others lie 64 bytes further), K-step 0: the second four lie 256 bytes, each
// next step 2 * YBLOCK further.  The 16 lanes of a group read 16 columns of four places, four columns of one place each; natural: lane q gets column q; else
// column 16 h + 4 b + c for q = 8 b + 4 h + c, so that a lane's results (rows 8 b + 4 h + c of the accumulators) are 16 neighbours.
__device__ __forceinline__ uint32_t places_at(int lane, bool natural)
{
    const int r = lane >> 2 & 3, g = lane >> 4 & 1, p = lane & 3, hk = lane >> 5;
    const int col = natural ? 16 * g + 4 * p : 16 * (p & 1) + 8 * g + 4 * (p >> 1);
    return uint32_t((r >> 1) * YBLOCK + hk * 512 + (r & 1) * 128 + col * 2);
}
__device__ __forceinline__ bf16x8 read_across(lds_ptr p)
{
    using lds_i16x4 = __attribute__((address_space(3))) i16x4;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(p));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(p + 256));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ bf16x8 read_along(lds_ptr p) { return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(p); }

// what this wave's lanes wrote to LDS is there for its other lanes
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A kind of tile: CG x RG waves, each with FA x 32 columns and NB x 32 rows of the results
template <int FA_, int NB_, int CG_, int RG_, int BUFS_, int SIMD_>
struct Kind {
    static constexpr bool BIG = FA_ * CG_ == 8;
    static constexpr int FA = FA_, NB = NB_, CG = CG_, RG = RG_, BUFS = BUFS_, SIMD = SIMD_, WAVES = CG * RG, THREADS = WAVES * 64, COLS = CG * FA * 32, ROWS = RG * NB * 32;
};
using Big = Kind<4, 4, 2, 2, 2, 1>;      // 256 x 256: an operand's bytes are multiplied 256 times
using Mid = Kind<2, 2, 2, 2, 2, 2>;      // 128 x 128, two workgroups a CU
using Few = Kind<1, 2, 4, 1, 3, 2>;      // 128 columns x 64 rows, two chunks ahead: a stream of weights

constexpr int LIST = 256;                // tiles that a staying workgroup looks up at once
constexpr int SORTED = 8192;             // groups whose counts fit where chunks go
template <int DIR, class S> constexpr uint32_t BUF_BYTES = uint32_t((S::COLS / 64) * (DIR == FORWARD ? XUNIT : YUNIT) + (S::ROWS / 64) * (DIR == GRAD_WEIGHT ? YUNIT : XUNIT));
template <int DIR, class S> constexpr uint32_t LDS_BYTES = BUF_BYTES<DIR, S> * S::BUFS + (DIR != GRAD_WEIGHT && S::BIG ? LIST * 16 + S::ROWS * 4 : 0);

// How the weights' gradient is shared out.  The sums run over the rows of a group; every tile of W_e's gradient is the work of one workgroup, or, where there are
// fewer tiles than CUs, of several ("lanes") that take a share of all rows each.  A group counts as its rows and `extra` more for its tile's way to memory;
// group e starts at  offsets[e] + extra * e  of the M + extra * E that are shared out evenly.  A group cut by a border leaves partial sums (slots 2 lane for a part
// that does not begin the group, 2 lane + 1 for one that does) that k_join adds up in order.
struct Shares {
    int lanes, extra;
    int64_t each;
};
__device__ __forceinline__ int64_t start_of(const Groups& g, const Shares& s, int e) { return int64_t(g.begin(e)) + int64_t(s.extra) * e; }
// the last group that starts at or ahead of x.  All 64 lanes of a wave call it.
__device__ __forceinline__ int group_at(const Groups& g, const Shares& s, int64_t x)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = g.E;
    while (n > 1) {
        const int step = (n + 63) / 64, e = lo + lane * step;
        const bool here = lane * step < n && start_of(g, s, e) <= x;
        const int last = 63 - __builtin_clzll(__ballot(here) | 1ull);
        lo += last * step;
        n = min(step, n - last * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

struct Tile {
    int e, begin, rows, c0, r0, depth;   // group; its first row here; rows of results; first column, row of W's gradient; places of the sum
    int slot;                            // of the partial sums, or -1
};

// Unit u of rows x ct tiles: TALL rows walk the columns together.  Four for Big, so that the workgroups of a die, which run 32 neighbours at a time, share both
// operands in its L2 (8 columns and 4 rows instead of 32 and 1; 8192 rows, channels and features, one expert: forward 1264 -> 805 us).  One for the others, whose rows
// are of different experts (1024 experts of 64 rows: 888 us, four 1049).
struct Place { int row, col; };
template <int TALL>
__device__ __forceinline__ Place walk(int u, int rows, int ct)
{
    const int group = u / (TALL * ct), in = u - group * TALL * ct, tall = min(TALL, rows - group * TALL);
    return Place{group * TALL + in % tall, in / tall};
}

template <int DIR, typename TO, class S, bool FUSED>
__global__ __launch_bounds__(S::THREADS, S::SIMD) void k_product(Args p, int units, int ct, int rt, Shares shares, float* __restrict__ partial)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    constexpr bool A_ACROSS = DIR != FORWARD, B_ACROSS = DIR == GRAD_WEIGHT, STAYS = S::BUFS == 2 && (S::BIG || DIR == GRAD_WEIGHT);
    constexpr int AU = S::COLS / 64, BU = S::ROWS / 64, UA = A_ACROSS ? YUNIT : XUNIT, UB = B_ACROSS ? YUNIT : XUNIT, EACH = 8 / S::WAVES, REQUESTS = (AU + BU) * EACH;
    constexpr uint32_t BUF = BUF_BYTES<DIR, S>;
    constexpr int AHEAD = S::BUFS - 1, FA = S::FA, NB = S::NB;
    static_assert(DIR != FORWARD || !STAYS || S::ROWS == S::THREADS, "a thread a row looks up");
    static_assert(AHEAD == 1 || !STAYS, "a tile's first chunk is asked for under the last one's last chunk");
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, q = lane & 31, hk = lane >> 5;
    const int cg = wave % S::CG, rg = wave / S::CG;
    const int cols = DIR == FORWARD ? p.N : p.K;
    const lds_ptr lds = (lds_ptr)lds_raw;

    // workgroups of a die (every eighth) are neighbours among the units: they share weights and rows in its L2
    // (counted units: those that there are come first, and go to all dies)
    const bool counts = !STAYS && counted(p.g.M, p.g.E);
    const int per_die = int(gridDim.x) / 8, place = !counts && int(blockIdx.x) < per_die * 8 ? int(blockIdx.x & 7) * per_die + int(blockIdx.x >> 3) : int(blockIdx.x);

    // ---- the tiles
    // forward, input's gradient: unit = piece of rows * ct + column; a workgroup that stays takes every gridDim.x-th unit, by the list.
    // Up to SORTED groups and LIST units a workgroup, the units are the pieces that there are, those of more than half of a tile's rows first: rests of up to
    // 128 rows, which take half as long, even out what is left over (65536 rows, 64 experts by Zipf's law, 8 columns of tiles: 8.6 tiles' time a workgroup on average,
    // 10 for the longest without, 9.1 so).  Beyond, find_piece's units.  (All workgroups go by one numbering: it is the most units of any of them that decides.)
    int count = DIR == GRAD_WEIGHT ? 0 : STAYS ? (units - place + int(gridDim.x) - 1) / int(gridDim.x) : 1;
    const bool sorted = DIR != GRAD_WEIGHT && STAYS && p.g.E < SORTED && (units + int(gridDim.x) - 1) / int(gridDim.x) <= LIST;
    int at_unit = -1;
    // weights' gradient: a lane's groups
    const int w_lane = place / (ct * rt);
    const Place w_tile = walk<4>(place % (ct * rt), rt, ct);
    const int64_t w_from = shares.each * w_lane, w_to = w_from + shares.each;
    int w_e = 0;
    auto tile_of = [&](const Piece& at, int col) {
        return Tile{at.e, at.begin, at.rows, col * S::COLS, 0, at.e < p.g.E ? (DIR == FORWARD ? p.K : p.N) : 0, -1};
    };
    auto put_unit = [&](int i, const Piece& at, int col) {
        *reinterpret_cast<u32x4*>(lds_raw + BUF * S::BUFS + i * 16) = u32x4{uint32_t(at.e), uint32_t(at.begin), uint32_t(at.rows), uint32_t(col)};
    };
    auto list_units = [&](int from) {
        meet();
        if (tid < LIST && from + tid < count) {
            const Place w = walk<4>(place + (from + tid) * int(gridDim.x), units / ct, ct);
            put_unit(tid, find_piece_alone(p.g, S::ROWS, w.row), w.col);
        }
        meet();
    };
    auto list_sorted = [&]() {
        // how many large and small pieces there are ahead of every group, where the first chunks will be; what lies behind the groups counts as small
        int2* const ahead = reinterpret_cast<int2*>(lds_raw);
        int* const sums = reinterpret_cast<int*>(lds_raw + BUF * S::BUFS);
        auto pieces = [&](int e) {
            const int n = max(p.g.begin(e + 1) - p.g.begin(e), 0), rest = n % S::ROWS;
            return e == p.g.E ? int2{0, (n + S::ROWS - 1) / S::ROWS} : int2{n / S::ROWS + (rest > S::ROWS / 2), rest > 0 && rest <= S::ROWS / 2};
        };
        const int per = (p.g.E + S::THREADS) / S::THREADS, e0 = min(tid * per, p.g.E + 1), e1 = min(e0 + per, p.g.E + 1);
        int2 mine = {0, 0};
        for (int e = e0; e < e1; ++e) {
            const int2 n = pieces(e);
            mine.x += n.x;
            mine.y += n.y;
        }
        int2 at = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(at.x, o), y = __shfl_up(at.y, o);
            at.x += lane >= o ? x : 0;
            at.y += lane >= o ? y : 0;
        }
        if (lane == 63) { sums[wave * 2] = at.x; sums[wave * 2 + 1] = at.y; }
        meet();
        int2 all = {0, 0};
        at.x -= mine.x;
        at.y -= mine.y;
#pragma unroll
        for (int w = 0; w < S::WAVES; ++w) {
            at.x += w < wave ? sums[w * 2] : 0;
            at.y += w < wave ? sums[w * 2 + 1] : 0;
            all.x += sums[w * 2];
            all.y += sums[w * 2 + 1];
        }
        for (int e = e0; e < e1; ++e) {
            ahead[e] = at;
            const int2 n = pieces(e);
            at.x += n.x;
            at.y += n.y;
        }
        meet();
        count = min(((all.x + all.y) * ct - place + int(gridDim.x) - 1) / int(gridDim.x), LIST);
        if (tid < count) {
            const int unit = place + tid * int(gridDim.x);
            const bool large = unit < all.x * ct;
            const Place w = walk<4>(large ? unit : unit - all.x * ct, large ? all.x : all.y, ct);
            int lo = 0, n = p.g.E + 1;                         // the last group with no more pieces ahead of it than w.row (those without pieces stand ahead of it)
            while (n > 1) {
                const int half = n >> 1;
                const int2 v = ahead[lo + half];
                if ((large ? v.x : v.y) <= w.row) { lo += half; n -= half; }
                else n = half;
            }
            const int a = p.g.begin(lo), rows = max(p.g.begin(lo + 1) - a, 0);
            const int part = large ? w.row - ahead[lo].x : lo == p.g.E ? w.row - ahead[lo].y : rows / S::ROWS;
            const bool there = part >= 0 && part <= (rows - 1) / S::ROWS && rows > 0;    // (else the offsets fall)
            put_unit(tid, there ? Piece{lo, a + part * S::ROWS, min(S::ROWS, rows - part * S::ROWS)} : Piece{lo, a, 0}, w.col);
        }
        meet();
    };
    // the next tile, if there is one (rows 0: none)
    auto next_tile = [&]() -> Tile {
        Tile t = {};
        if constexpr (DIR == GRAD_WEIGHT) {
            for (; w_e < p.g.E; ++w_e) {
                const int a = min(max(w_e ? uniform_load(p.g.offsets + w_e) : 0, 0), p.g.M), n = max(min(max(uniform_load(p.g.offsets + w_e + 1), 0), p.g.M) - a, 0);
                const int64_t s = int64_t(a) + int64_t(shares.extra) * w_e, first = s + shares.extra;
                if (s >= w_to) break;
                const int lo = int(min(max(w_from - first, int64_t(0)), int64_t(n))), hi = int(min(max(w_to - first, int64_t(0)), int64_t(n)));
                if (n == 0 ? s < w_from : hi <= lo) continue;
                t = Tile{w_e, a + lo, p.N - w_tile.row * S::ROWS, w_tile.col * S::COLS, w_tile.row * S::ROWS, hi - lo, hi - lo == n ? -1 : 2 * w_lane + (lo > 0 ? 0 : 1)};
                t.rows = min(t.rows, S::ROWS);
                ++w_e;
                break;
            }
        } else if constexpr (STAYS) {
            while (++at_unit < count) {
                if (!sorted && at_unit % LIST == 0) list_units(at_unit);
                const u32x4 v = *reinterpret_cast<const u32x4*>(lds_raw + BUF * S::BUFS + at_unit % LIST * 16);
                Piece at;
                at.e = __builtin_amdgcn_readfirstlane(v.x);
                at.begin = __builtin_amdgcn_readfirstlane(v.y);
                at.rows = __builtin_amdgcn_readfirstlane(v.z);
                if (at.rows > 0) { t = tile_of(at, __builtin_amdgcn_readfirstlane(v.w)); break; }
            }
        } else if (++at_unit == 0) {
            const Place w = walk<1>(place, units / ct, ct);
            t = tile_of(counts ? count_pieces(p.g, S::ROWS, w.row, reinterpret_cast<int*>(lds_raw)) : find_piece(p.g, S::ROWS, w.row), w.col);
        }
        return t;
    };
    if constexpr (DIR == GRAD_WEIGHT) {
        if (w_lane >= shares.lanes) return;
        w_e = group_at(p.g, shares, w_from);
    } else if (sorted) list_sorted();

    // ---- copying: wave w's blocks are w, w + WAVES ..; a request is a scalar base, which moves on with the chunks, and a lane's offset, which a tile keeps
    // (but for gathered rows as places of the sum).  Behind the end of a sum the last place that there is is copied again, and cleared in LDS before use.
    const uint32_t piece = uint32_t(lane & 7) * 16u;
    const char *a_base = nullptr, *b_base = nullptr;
    uint32_t a_off[AU][EACH], b_off[BU][EACH], more[EACH];
    const bool gathers = DIR != GRAD_INPUT && p.g.perm != nullptr;
    const size_t a_step = DIR == FORWARD ? 128 : DIR == GRAD_INPUT ? size_t(p.K) * 128 : gathers ? 0 : size_t(p.a_stride) * 128;
    const size_t b_step = B_ACROSS ? size_t(p.b_stride) * 128 : 128;
    int32_t uses[EACH];                                        // weights' gradient: `perm` at this lane's places of the chunk that is asked for next
    Tile asked = {};                                           // the tile that is asked for
    int z_asked = 0;                                           // ... and the chunk: its first place
    // forward: `perm` at the next tile's rows, into LDS (registers that a load is on its way to would be waited for under the next chunk's requests)
    constexpr uint32_t ROWS_AT = BUF * S::BUFS + LIST * 16;
    auto look_up_rows = [&](const Tile& t) {
        if constexpr (DIR == FORWARD && STAYS)
            if (gathers)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(p.g.perm + t.begin + min(wave * 64 + lane, t.rows - 1)),
                                                 (__attribute__((address_space(3))) uint32_t*)(lds + ROWS_AT + wave * 256), 4, 0, 0);
    };
    auto rows_looked_up = [&]() {
        if (DIR == FORWARD && STAYS && gathers) {
            answered_but<0>();
            meet();
        }
    };
    auto look_up_places = [&]() {
        if constexpr (DIR == GRAD_WEIGHT)
            if (gathers)
#pragma unroll
                for (int j = 0; j < EACH; ++j) uses[j] = p.g.perm[asked.begin + min(z_asked + copied_place(wave + j * S::WAVES, lane), asked.depth - 1)];
    };
    auto open_a = [&](const Tile& t) {
        asked = t;
        z_asked = 0;
        const size_t w = size_t(t.e) * size_t(p.N) * size_t(p.K);
        a_base = reinterpret_cast<const char*>(DIR == GRAD_WEIGHT ? p.a + (gathers ? 0 : t.begin * p.a_stride) : DIR == FORWARD ? p.a + w + size_t(t.c0) * size_t(p.K) : p.a + w);
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int block = wave + j * S::WAVES, s_q = copied_row(block, lane), z = copied_place(block, lane);
#pragma unroll
            for (int i = 0; i < AU; ++i) {
                const uint32_t col = uint32_t(min(t.c0 + i * 64 + (lane & 7) * 8, cols - 8)) * 2u;
                if constexpr (DIR == FORWARD)                  // (the features in the order that gives a lane 16 neighbours)
                    a_off[i][j] = uint32_t(min(i * 64 + (lane >> 5) * 32 + (s_q >> 2 & 1) * 16 + (s_q >> 3) * 4 + (s_q & 3), cols - 1 - t.c0)) * uint32_t(p.K) * 2u + piece;
                else if constexpr (DIR == GRAD_INPUT) a_off[i][j] = uint32_t(z) * uint32_t(p.K) * 2u + col;
                else a_off[i][j] = (gathers ? 0u : uint32_t(z) * uint32_t(p.a_stride) * 2u) + col;
            }
        }
    };
    auto open_b = [&](const Tile& t) {
        b_base = reinterpret_cast<const char*>(DIR == FORWARD && gathers ? p.b : p.b + t.begin * p.b_stride);
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int block = wave + j * S::WAVES, s_q = copied_row(block, lane), z = copied_place(block, lane);
#pragma unroll
            for (int i = 0; i < BU; ++i) {
                if constexpr (B_ACROSS) b_off[i][j] = uint32_t(z) * uint32_t(p.b_stride) * 2u + uint32_t(min(t.r0 + i * 64 + (lane & 7) * 8, p.N - 8)) * 2u;
                else {
                    uint32_t row = uint32_t(min(i * 64 + (lane >> 5) * 32 + s_q, t.rows - 1));
                    if (DIR == FORWARD && gathers) row = p.g.row_of(STAYS ? *(const __attribute__((address_space(3))) int32_t*)(lds + ROWS_AT + row * 4) : p.g.perm[t.begin + int(row)]);
                    b_off[i][j] = row * uint32_t(p.b_stride) * 2u + piece;
                }
            }
        }
    };
    auto open = [&](const Tile& t) {
        open_a(t);
        open_b(t);
        look_up_places();
    };
    // ahead of a chunk's requests
    auto prepare = [&](bool a_too = true, bool b_too = true) {
        const int rest = asked.depth - z_asked;
        if (rest < 64) {                                       // (the tile's last: its offsets are not used again)
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int z = copied_place(wave + j * S::WAVES, lane);
                const uint32_t places = uint32_t(max(z - (rest - 1), 0)), pieces = (lane & 7) * 8 >= rest ? piece : 0u;
#pragma unroll
                for (int i = 0; i < AU; ++i) if (a_too) a_off[i][j] -= DIR == FORWARD ? pieces : DIR == GRAD_INPUT ? places * uint32_t(p.K) * 2u : gathers ? 0u : places * uint32_t(p.a_stride) * 2u;
#pragma unroll
                for (int i = 0; i < BU; ++i) if (b_too) b_off[i][j] -= B_ACROSS ? places * uint32_t(p.b_stride) * 2u : pieces;
            }
        }
        if constexpr (DIR == GRAD_WEIGHT) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) more[j] = gathers ? p.g.row_of(uses[j]) * uint32_t(p.a_stride) * 2u : 0u;
        }
    };
    // requests i0 .. i1 of a chunk
    auto request = [&](lds_ptr to, int i0, int i1) {
#pragma unroll
        for (int n = 0; n < REQUESTS; ++n) {
            if (n < i0 || n >= i1) continue;
            const int i = n / EACH, j = n % EACH, block = wave + j * S::WAVES;
            if (i < AU) lds_copy16_to(a_base, DIR == GRAD_WEIGHT ? a_off[i % AU][j] + more[j] : a_off[i % AU][j], to + uint32_t(i * UA + block * (A_ACROSS ? YBLOCK : XBLOCK)));
            else lds_copy16_to(b_base, b_off[(i - AU + BU) % BU][j], to + uint32_t(AU * UA + (i - AU) * UB + block * (B_ACROSS ? YBLOCK : XBLOCK)));
        }
    };
    auto requested = [&]() {
        z_asked += 64;
        if (z_asked >= asked.depth) return;
        a_base += a_step;
        b_base += b_step;
        look_up_places();
    };
    // zeros behind the end of the sum, each wave in what it has copied
    auto clear = [&](lds_ptr at, int rest) {
#pragma unroll
        for (int n = 0; n < REQUESTS; ++n) {
            const int i = n / EACH, j = n % EACH, block = wave + j * S::WAVES;
            const bool is_a = i < AU;
            if (((is_a ? A_ACROSS : B_ACROSS) ? copied_place(block, lane) : (lane & 7) * 8) >= rest)
                *(__attribute__((address_space(3))) u32x4*)(at + uint32_t((is_a ? i * UA : AU * UA + (i - AU) * UB) + block * ((is_a ? A_ACROSS : B_ACROSS) ? YBLOCK : XBLOCK) + lane * 16)) =
                    u32x4{0u, 0u, 0u, 0u};
        }
        meet();
    };
    uint32_t fill = 0, take = 0;                               // the chunk's place in LDS that is filled next, and the one that is read
    auto next_place = [&](uint32_t at) { return at == AHEAD * BUF ? 0 : at + BUF; };

    // ---- a tile after the other
    const uint32_t a_slot = A_ACROSS ? places_at(lane, false) : fragment_at(q, hk), b_slot = B_ACROSS ? places_at(lane, true) : fragment_at(q, hk);
    Tile now = next_tile();
    bool primed = false;                                       // its first chunk has been asked for
    int stores = 0;                                            // of this wave, behind that request
    while (now.rows > 0) {
        const int nchunk = (now.depth + 63) / 64;
        // The mask's pieces, as the results will leave, ahead of everything (Big has no registers for them and loads them with the results).  8192 rows of 256 experts,
        // 512 features, 1024 channels: 65 us with loads at the end, 64 so, 57 without a mask.
        constexpr bool ACT_AHEAD = DIR == GRAD_INPUT && FUSED && !STAYS;
        constexpr int ACT_STORES = ACT_AHEAD ? FA * 2 : 1;     // pieces of a block of 32 rows
        u32x4 act_ahead[ACT_AHEAD ? NB : 1][ACT_STORES];
        if constexpr (ACT_AHEAD) {
            constexpr int LANES = FA * 4;
            const int col = min(now.c0 + cg * (FA * 32) + lane % LANES * 8, cols - 8);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < ACT_STORES; ++i) {
                    const int r = min((b * S::RG + rg) * 32 + lane / LANES + i * (64 / LANES), now.rows - 1);
                    act_ahead[b][i] = *reinterpret_cast<const u32x4*>(p.act + int64_t(now.begin + r) * p.act_stride + col);
                }
        }
        if (nchunk > 0 && !primed) {
            look_up_rows(now);
            fill = take;                                       // (what was asked for behind the last tile is overwritten)
            if constexpr (STAYS) {
                rows_looked_up();
                open(now);
                prepare();
                request(lds + fill, 0, REQUESTS);
                requested();
                fill = next_place(fill);
            } else {
                // the columns' pieces first, which need no look at `perm`
                open_a(now);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (half == 1) open_b(now);
#pragma unroll
                    for (int c = 0; c < AHEAD; ++c)
                        if (c < nchunk) {
                            z_asked = c * 64;
                            prepare(half == 0, half == 1);
                            request(lds + c * BUF, half ? AU * EACH : 0, half ? REQUESTS : AU * EACH);
                            (half ? b_base : a_base) += half ? b_step : a_step;
                        }
                }
                z_asked = min(AHEAD, nchunk) * 64;
                fill = uint32_t(min(AHEAD, nchunk)) % uint32_t(S::BUFS) * BUF;
            }
            stores = 0;
        }
        Tile then = {};
        const int blocks = (now.rows + 31) / 32;
        const int mine = now.c0 + cg * (FA * 32) < cols ? max(0, (blocks - rg + S::RG - 1) / S::RG) : 0;
        auto arrive = [&](int c) {                             // chunk c is there, and all waves are done with the one before
            if constexpr (AHEAD == 1) {
                if (c == 0 && stores > 0) {
                    if (stores >= 60) answered_but<60>();
                    else if (stores >= 32) answered_but<32>();
                    else if (stores >= 16) answered_but<16>();
                    else if (stores >= 8) answered_but<8>();
                    else answered_but<4>();
                } else answered_but<0>();
            } else {
                if (c == 0 && nchunk > 1) answered_but<BU * EACH>();       // (both chunks' columns were asked for ahead of the rows)
                else if (c + 1 < nchunk) answered_but<REQUESTS>();
                else answered_but<0>();
            }
            meet();
        };
        auto work = [&](auto nb_const) {
            constexpr int LIVE = decltype(nb_const)::value;
            f32x16 acc[FA][LIVE > 0 ? LIVE : 1];
#pragma unroll
            for (int a = 0; a < FA; ++a)
#pragma unroll
                for (int b = 0; b < LIVE; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
            // The last K-step of a chunk is multiplied behind the next one's arrival: under it the next chunk's first fragments come from LDS, and the requests are
            // made, one of each a product.  (Ahead of the first chunk, zeros.)  Nothing in a chunk branches.
            bf16x8 af[2][FA], bf[2][LIVE > 0 ? LIVE : 1];
#pragma unroll
            for (int a = 0; a < FA; ++a) af[1][a] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
#pragma unroll
            for (int b = 0; b < LIVE; ++b) bf[1][b] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
            // (what is read and what is filled are said to be apart: else every transposing read would wait for all requests)
            auto chunk = [&](const lds_ptr __restrict__ from, const lds_ptr __restrict__ to, auto asks) {
                constexpr int ASKS = decltype(asks)::value ? REQUESTS : 0;
                const lds_ptr au = from + (uint32_t((cg * FA / 2) * UA) + a_slot + uint32_t(FA == 1 ? (cg & 1) * (A_ACROSS ? 64 : 512) : 0));
                const lds_ptr bu = from + (uint32_t(AU * UA) + b_slot);
                // fragments i0 .. i1 of K-step ks
                auto read = [&](int ks, int i0, int i1) {
#pragma unroll
                    for (int a = 0; a < FA; ++a)
                        if (a >= i0 && a < i1) {
                            if constexpr (A_ACROSS) af[ks & 1][a] = read_across(au + uint32_t(a / 2 * UA + a % 2 * 64 + ks * 2 * YBLOCK));
                            else af[ks & 1][a] = read_along(au + (a / 2 * UA + a % 2 * 512 + ks * 32));
                        }
#pragma unroll
                    for (int b = 0; b < LIVE; ++b)
                        if (FA + b >= i0 && FA + b < i1) {
                            const lds_ptr at = bu + uint32_t((b * S::RG + rg) / 2 * UB + (b * S::RG + rg) % 2 * (B_ACROSS ? 64 : 512));
                            if constexpr (B_ACROSS) bf[ks & 1][b] = read_across(at + uint32_t(ks * 2 * YBLOCK));
                            else bf[ks & 1][b] = read_along(at + ks * 32);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                };
                // the products of K-step ks (-1: the chunk before's last); in the first half of them K-step ks + 1 is read, and with the first ones requests are made
                auto step = [&](int ks, int asks_before, int asks_behind) {
                    constexpr int PRODUCTS = FA * (LIVE > 0 ? LIVE : 1), FRAGMENTS = FA + LIVE;
#pragma unroll
                    for (int m = 0; m < PRODUCTS; ++m) {
                        const int a = m % FA, b = m / FA;
                        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[ks & 1][a], bf[ks & 1][b], acc[a][b], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                        if (ks < 3) read(ks + 1, min(FRAGMENTS, m * FRAGMENTS * 2 / PRODUCTS), min(FRAGMENTS, (m + 1) * FRAGMENTS * 2 / PRODUCTS));
                        request(to, asks_before + m * (asks_behind - asks_before) / PRODUCTS, asks_before + (m + 1) * (asks_behind - asks_before) / PRODUCTS);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if constexpr (LIVE == 0) request(to, 0, ASKS);
                else {
                    // (the last step's fragments are here, all waves have met behind their reads: said so, or they would be waited for behind the next ones)
#pragma unroll
                    for (int a = 0; a < FA; ++a) asm volatile("" : "+v"(af[1][a]));
#pragma unroll
                    for (int b = 0; b < LIVE; ++b) asm volatile("" : "+v"(bf[1][b]));
                    constexpr int FIRST = S::BUFS > 2 ? ASKS : ASKS / 2;       // (a stream of weights: all at once)
                    step(-1, 0, FIRST);
                    step(0, FIRST, ASKS);
                    step(1, ASKS, ASKS);
                    step(2, ASKS, ASKS);
                }
            };
            int c = 0;
            uint32_t last = take;                              // the last chunk's place
            auto through = [&](int end, auto asks) {
#pragma unroll 1
                for (; c < end; ++c) {
                    arrive(c);
                    if (c == nchunk - 1 && now.depth % 64 != 0) clear(lds + take, now.depth - c * 64);
                    if constexpr (STAYS) {
                        if (c == 0) {
                            then = next_tile();
                            if (then.depth > 0) look_up_rows(then);
                        }
                        // (behind the last tile the last chunk is asked for again)
                        if (nchunk == 1 && then.depth > 0) rows_looked_up();
                        if (c == nchunk - 1 && then.depth > 0) open(then);
                    }
                    if constexpr (decltype(asks)::value) {
                        if (z_asked < asked.depth) prepare();
                        chunk(lds + take, lds + fill, asks);
                        requested();
                        fill = next_place(fill);
                    } else chunk(lds + take, lds + fill, asks);
                    last = take;
                    take = next_place(take);
                }
            };
            if constexpr (STAYS) through(nchunk, std::true_type{});
            else {
                through(nchunk - AHEAD, std::true_type{});
                through(nchunk, std::false_type{});
            }
            // (without a chunk, zeros: a branch around this would have the accumulators copied)
#pragma unroll
            for (int m = 0; m < FA * LIVE; ++m) acc[m % FA][m / FA] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[1][m % FA], bf[1][m / FA], acc[m % FA][m / FA], 0, 0, 0);
            // A lane has 16 neighbouring columns of row q of every block.  They go by way of LDS, each wave its own share of the last chunk's place, and leave with all
            // lanes of a store side by side: 16 bytes of every row a lane took the stores' address unit 64 clocks each, 8 us of a tile's 37 (forward, 1024 channels).
            if (nchunk > 0) meet();                            // (all waves are done with that chunk)
            const lds_ptr mine_at = lds + last + uint32_t(wave) * (BUF / S::WAVES / 16 * 16);
            // to: row 0 of the tile, this wave's first column.  A bfloat16 weights' gradient has `part` beside it: null, or where this tile's sums go in fp32 instead.
            // Which of the two is asked anew for every piece that goes into LDS and comes out of it.  Asked once, with a way out each, it had 108 of the 256 x 256 kernel's
            // registers spilled, and their loads waited for the next tile's requests (65536 rows, 1024 -> 2048: 64 experts 377 us, 345 so; 256 experts 721, 575).
            auto put = [&](auto* to, float* part, int64_t pitch) {
                using T = std::remove_pointer_t<decltype(to)>;
                constexpr bool EITHER = DIR == GRAD_WEIGHT && sizeof(T) == 2;
                constexpr int P = 16 / int(sizeof(T)), LANES = FA * 32 / P, AT_ONCE = 64 / LANES, PITCH = FA * 32 * int(sizeof(T)) + 16, PART_PITCH = FA * 32 * 4 + 16;
                static_assert(32 * (EITHER ? PART_PITCH : PITCH) <= int(BUF / S::WAVES), "room");
                const bool parts = EITHER && part;
                const int size = parts ? 4 : int(sizeof(T)), in_pitch = parts ? PART_PITCH : PITCH;
                const int col = lane % LANES * P, row = lane / LANES;
                const bool on = now.c0 + cg * (FA * 32) + col < cols;
                // (one address each, the steps are constants or scalars: an address a store was one too many to keep)
                const lds_ptr in_at = mine_at + uint32_t(q * in_pitch + 16 * hk * size), out_at = mine_at + uint32_t(row * in_pitch + col * size);
                char* lane_to = (parts ? reinterpret_cast<char*>(part) : reinterpret_cast<char*>(to)) + (int64_t(rg * 32 + row) * pitch + col) * size;
                const int64_t step = AT_ONCE * pitch * size, to_next = S::RG * 32 * pitch * size;
                const char* act_at = nullptr;
                int64_t act_step = 0, act_next = 0;
                if constexpr (DIR == GRAD_INPUT && FUSED) {
                    act_at = reinterpret_cast<const char*>(p.act + (now.begin + rg * 32 + row) * p.act_stride + now.c0 + cg * (FA * 32) + col);
                    act_step = AT_ONCE * p.act_stride * 2;
                    act_next = S::RG * 32 * p.act_stride * 2;
                }
#pragma unroll
                for (int b = 0; b < LIVE; ++b) {
#pragma unroll
                    for (int a = 0; a < FA; ++a) {
                        if (nchunk == 0) break;                // (zeros, and LDS is the next tile's)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float v[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = acc[a][b][8 * h + i];
                            if (DIR == FORWARD && FUSED)
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];                  // (a NaN stays one)
                            using lds_u32x4 = __attribute__((address_space(3))) u32x4;
                            if (sizeof(T) == 4 || parts) {
                                const lds_ptr at = in_at + (a * 32 + 8 * h) * 4;
                                *(lds_u32x4*)at = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                                *(lds_u32x4*)(at + 16) = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
                            } else
                                *(lds_u32x4*)(in_at + (a * 32 + 8 * h) * 2) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
                        }
                        __builtin_amdgcn_sched_barrier(0);     // (all accumulators at once in other registers would have no room)
                    }
                    wave_sync();
                    constexpr int STORES = 32 / AT_ONCE;
                    u32x4 v[STORES], act[STORES];
                    if constexpr (ACT_AHEAD) {
                        static_assert(STORES == ACT_STORES, "the pieces that were loaded");
#pragma unroll
                        for (int i = 0; i < STORES; ++i) act[i] = act_ahead[b][i];
                    }
                    auto take_out = [&](int at, int lds_pitch) {
#pragma unroll
                        for (int i = 0; i < STORES; ++i) v[i] = *(const __attribute__((address_space(3))) u32x4*)(out_at + (i * AT_ONCE * lds_pitch + at));
                    };
                    const int left = now.rows - (b * S::RG + rg) * 32;
                    if constexpr (EITHER) {
                        if (parts) {                           // (which have rows, so chunks)
#pragma unroll
                            for (int h = 0; h < 32; h += 16) {                     // eight fp32 columns a lane, in two stores
                                take_out(h, PART_PITCH);
#pragma unroll
                                for (int i = 0; i < STORES; ++i)
                                    if (row + i * AT_ONCE < left && on) *reinterpret_cast<u32x4*>(lane_to + i * step + h) = v[i];
                            }
                        } else {
                            take_out(0, PITCH);
                            if (nchunk == 0)
#pragma unroll
                                for (int i = 0; i < STORES; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                            for (int i = 0; i < STORES; ++i)
                                if (row + i * AT_ONCE < left && on) *reinterpret_cast<u32x4*>(lane_to + i * step) = v[i];
                        }
                        lane_to += to_next;
                        wave_sync();
                        __builtin_amdgcn_sched_barrier(0);
                        continue;
                    }
                    take_out(0, PITCH);
                    if (nchunk == 0)
#pragma unroll
                        for (int i = 0; i < STORES; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
                    auto one = [&](int i) {
                        if constexpr (DIR == GRAD_INPUT && FUSED)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                v[i][j] = (__uint_as_float(act[i][j] << 16) > 0.f ? v[i][j] & 0xffffu : 0u) | (__uint_as_float(act[i][j] & 0xffff0000u) > 0.f ? v[i][j] & 0xffff0000u : 0u);
                        *reinterpret_cast<u32x4*>(lane_to + i * step) = v[i];
                    };
                    if (left >= 32 && now.c0 + cg * (FA * 32) + FA * 32 <= cols) {
                        if constexpr (DIR == GRAD_INPUT && FUSED && !ACT_AHEAD)
#pragma unroll
                            for (int i = 0; i < STORES; ++i) act[i] = *reinterpret_cast<const u32x4*>(act_at + i * act_step);
#pragma unroll
                        for (int i = 0; i < STORES; ++i) one(i);
                    } else
#pragma unroll
                        for (int i = 0; i < STORES; ++i)
                            if (row + i * AT_ONCE < left && on) {
                                if constexpr (DIR == GRAD_INPUT && FUSED && !ACT_AHEAD) act[i] = *reinterpret_cast<const u32x4*>(act_at + i * act_step);
                                one(i);
                            }
                    lane_to += to_next;
                    act_at += act_next;
                    wave_sync();
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            const int first_col = now.c0 + cg * (FA * 32);
            if constexpr (DIR == GRAD_WEIGHT) {
                const size_t row = size_t(now.r0) * size_t(p.K) + size_t(first_col), all = size_t(p.N) * size_t(p.K);
                float* const part = now.slot >= 0 ? partial + size_t(now.slot) * all + row : nullptr;
                TO* const to = static_cast<TO*>(p.out) + size_t(now.e) * all + row;
                if constexpr (std::is_same_v<TO, float>) put(part ? part : to, nullptr, p.K);
                else put(to, part, p.K);
            } else put(static_cast<TO*>(p.out) + int64_t(now.begin) * p.out_stride + first_col, nullptr, p.out_stride);
            // (an end of its own for every size, so that the compiler keeps what is the same for all lanes in scalar registers)
            asm volatile("; %0" ::"n"(LIVE));
        };
        if (mine > NB / 2) work(std::integral_constant<int, NB>{});
        else if (mine > 0) work(std::integral_constant<int, NB / 2>{});
        else work(std::integral_constant<int, 0>{});
        if (!STAYS) return;
        if (nchunk == 0) then = next_tile();
        primed = nchunk > 0 && then.depth > 0;
        // (the fewest that there can have been: of the blocks that are whole)
        stores = now.c0 + cg * (FA * 32) + FA * 32 <= cols ? max(0, (now.rows / 32 - rg + S::RG - 1) / S::RG) * FA * (DIR == GRAD_WEIGHT ? int(sizeof(TO)) : 2) : 0;
        now = then;
    }
    answered_but<0>();                                         // (nothing is on its way to LDS that another workgroup may have next)
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
int check_groups(const moe_product_shape* s, const moe_groups* g, bool gathers, const std::string& who)
{
    if (!g || !g->offsets) return fail(DYNB_E_INVAL, who + ": NULL groups");
    if (g->perm && !gathers) return fail(DYNB_E_INVAL, who + ": its rows are not gathered (perm must be NULL)");
    if (g->perm && (g->k <= 0 || (s->M > 0 && g->rows <= 0))) return fail(DYNB_E_INVAL, who + ": perm needs k and the number of rows it points into");
    if ((reinterpret_cast<uintptr_t>(g->offsets) | reinterpret_cast<uintptr_t>(g->perm)) & 3) return fail(DYNB_E_INVAL, who + ": misaligned pointer");
    return DYNB_OK;
}
constexpr int CUS = 256;
constexpr int64_t MOST_GROUPS = (1 << 24) - 1;                 // workgroups of 256 threads in a launch
bool odd(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 1) != 0; }

int launched(const char* who)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
    return DYNB_OK;
}

// what k_product's 32-bit offsets reach: 255 rows from a tile's first, and gathered rows from the first of all
bool reached(const moe_groups* g, int64_t in_stride, int64_t other_stride)
{
    return in_stride <= 1 << 22 && other_stride <= 1 << 22 && (!g->perm || int64_t(g->rows) * in_stride * 2 < int64_t(1) << 32);
}
bool on_16(std::initializer_list<const void*> pointers)
{
    for (const void* p : pointers)
        if (reinterpret_cast<uintptr_t>(p) & 15) return false;
    return true;
}

// Few: rows that leave most of a larger tile empty, or too few tiles of 128 x 128 for the chip.  Big: where its tiles are many and long enough.  us, forward / the
// input's gradient, by rows, K, N, experts, Zipf exponent:
//                                   Big          Mid          Few
//   16 x 2048 x 512, 1              30 / 13      15 / 7       13 / 8
//   74 x 512 x 1024, 256, 1.1       18 / 24      10 / 14      10 / 10
//   1000 x 1024 x 1024, 8, 0.5      27 / 26      14 / 13      10 / 10
//   3000 x 2048 x 2048, 1           47 / 45      29 / 29      34 / 36
//   4096 x 2048 x 1024, 16, 0.6     49 / 35      28 / 31      35 / 34
//   8192 x 512 x 1024, 256, 1.1     81 / 88      56 / 57      52 / 53
//   8192 x 512 x 1024, 64, 0.8      35 / 32      21 / 18      22 / 22
//   16384 x 512 x 1024, 256, 0.8    88 / 94      66 / 65      62 / 62
//   16384 x 1024 x 2048, 64, 0.8   122 / 116    116 / 113    133 / 126
//   16384 x 2048 x 2048, 16, 0.6   144 / 142    143 / 142    192 / 206
//   32768 x 1024 x 2048, 32, 0.6   153 / 157    192 / 176    226 / 198
//   65536 x 512 x 1024, 64, 0.6     86 / 84      81 / 78     115 / 95
//   65536 x 512 x 2048, 16, 0.6    165 / 158    220 / 179    263 / 203
//   65536 x 1024 x 2048, 256, 0.6  421 / 390    434 / 411    506 / 484
//   65536 x 1024 x 2048, 512, 0.6  606 / 579    562 / 554    614 / 627
//   8192 x 8192 x 8192, 1          782 / 768   1319 / 1402  2367 / 2516
// (16 rows of one group: four workgroups, 32 chunks one after the other, so the latency of memory; the sum is not shared out)
enum KindOf { BIG, MID, FEW };
KindOf kind_of(const moe_product_shape* s, int cols, int depth)
{
    const int64_t each = s->M / s->E, chunks = (depth + 63) / 64;
    if (each >= 192 && s->M / 256 * ((cols + 255) / 256) * chunks >= 12288) return BIG;
    return each > 64 && (int64_t(s->M) + 127) / 128 * ((cols + 127) / 128) >= 256 ? MID : FEW;
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
