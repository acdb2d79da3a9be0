// Token embeddings: rows of a table by token, scaled, and the table's gradient.
//   out[t] = scale * table[tokens[t]]              dtable[v] = scale * sum over t with tokens[t] = v of dout[t]
// A token outside [0, V) (padding) has a row of zeros and gives no gradient.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "device_utils.h"
#include "plan_internal.h"
#include "rows.h"

using dynb::fail;

namespace {

// A wave a token; every row that is asked for is read and written once.  Bound by memory: 65536 tokens x 1024 bf16 40 us (6.7 TB/s); 37 x 512 takes 2 us, a launch's own time.
// Narrow rows leave lanes idle and are bound by the waves: 65536 x 128 bf16 12 us (2.9 TB/s), 65536 x 64 10 (1.8).
template <typename T>
__global__ __launch_bounds__(256) void k_embed(const int32_t* __restrict__ tokens, const T* __restrict__ table, T* __restrict__ out, int n, int V, int d,
                                               int64_t out_stride, float scale)
{
    constexpr int P = PIECE<T>;
    const int t = int(blockIdx.x) * 4 + int(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (t >= n) return;
    const int32_t tok = tokens[t];
    const bool known = tok >= 0 && tok < V;
    const T* const from = table + size_t(known ? tok : 0) * size_t(d);
    T* const to = out + int64_t(t) * out_stride;
#pragma unroll 2
    for (int c = lane * P; c < d; c += 64 * P) {
        const u32x4 raw = load_piece(from + c, d - c);
        float v[P];
#pragma unroll
        for (int j = 0; j < P; ++j) v[j] = known ? element<T>(raw, j) * scale : 0.f;
        store_piece<P>(to + c, d - c, v);
    }
}

// ------------------------------------------------------------------------------------------ gradient of the table
// The uses are brought into the order of their tokens (each token's in the order they stand in), so that a row's gradient is one sum, in one
// order; a row without uses is a row of zeros.  A wave sums the columns of a row that it reads in pieces of 16 bytes a lane (512 of bfloat16; others have
// the further ones), and a workgroup's waves share the uses of a row that has many.  Bound by memory where there is much of it: 65536 tokens, 50021 x 1024, bf16
// into fp32, 338 MB: 104 us, of which the sort's four launches take 22, the chunks' sums 18 to 25 and the rows 60; 4095 tokens, 20011 x 512 fp32, 49 MB: 15.3 us, 10 of
// them for the zeros (a fill takes 8), the rest a crowded row's.

// E: elements of a lane's piece.  Sums that leave in fp32 are stored 16 bytes a lane, lane by lane, so bfloat16 is then read in pieces of 8 bytes (pieces of 16
// would leave in two stores of 16 bytes of every 32: 50021 rows x 1024, each used once: 77 us instead of 66)
template <typename T, int E>
struct Sums {
    static constexpr int NV = PIECE<T> / E, COLS = 64 * PIECE<T>, STEP = 64 * E;
    float v[NV][E];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) v[i][j] = 0.f;
    }
    template <int K, typename At>
    __device__ __forceinline__ void add_some(const T* rows, int64_t stride, int c, int d, int u, At&& at)
    {
        Piece<T, E> raw[K][NV];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const T* const p = rows + int64_t(at(u + k)) * stride + c;
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[k][i] = load_some<E>(p + i * STEP, d - c - i * STEP);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < E; ++j) v[i][j] += element<T>(raw[k][i], j);
    }
    // this lane's columns, c .. and STEP further, of the rows at(0) .. at(n - 1), AHEAD (up to 8) of them under way
    template <int AHEAD, typename At>
    __device__ __forceinline__ void add(const T* rows, int64_t stride, int c, int d, int n, At&& at)
    {
        int u = 0;
        for (; u + AHEAD <= n; u += AHEAD) add_some<AHEAD>(rows, stride, c, d, u, at);
        if (u + 4 <= n) {
            add_some<4>(rows, stride, c, d, u, at);
            u += 4;
        }
        if (u + 2 <= n) {
            add_some<2>(rows, stride, c, d, u, at);
            u += 2;
        }
        if (u < n) add_some<1>(rows, stride, c, d, u, at);
    }
    // n rows of sums in fp32, d apart
    __device__ __forceinline__ void add_sums(const float* rows, int c, int d, int n)
    {
#pragma unroll 4
        for (int u = 0; u < n; ++u)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int h = 0; h < E; h += 4) {
                    const u32x4 raw = load_piece(rows + size_t(u) * size_t(d) + c + i * STEP + h, d - c - i * STEP - h);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][h + j] += element<float>(raw, j);
                }
    }
    // the sums of all WAVES waves (a power of two), in wave 0: half of the waves give theirs to the others, until one is left.  All threads call it.
    template <int WAVES>
    __device__ __forceinline__ void join(float (*room)[COLS], int wave)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int half = WAVES / 2; half > 0; half >>= 1) {
            __syncthreads();
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int i = 0; i < NV * E; ++i) room[wave - half][i * 64 + lane] = v[i / E][i % E];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int i = 0; i < NV * E; ++i) v[i / E][i % E] += room[wave][i * 64 + lane];
        }
        __syncthreads();
    }
    // a row without uses.  PAST: past the caches, where it is whole pieces
    template <bool PAST, typename TG>
    static __device__ __forceinline__ void store_zeros(TG* row, int c, int d)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = d - c - i * STEP;
            if (PAST && sizeof(TG) * E == 16 && left >= E)
                __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, reinterpret_cast<std::conditional_t<sizeof(TG) == 2, u32x4_at2, u32x4_at4>*>(row + c + i * STEP));
            else {
                const float w[E] = {};
                store_piece<E>(row + c + i * STEP, left, w);
            }
        }
    }
    template <typename TG>
    __device__ __forceinline__ void store(TG* row, int c, int d, float scale)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[E];
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = v[i][j] * scale;
            store_piece<E>(row + c + i * STEP, d - c - i * STEP, w);
        }
    }
};
template <typename T, typename TG> using SumsTo = Sums<T, std::is_same_v<TG, float> ? 4 : PIECE<T>>;

// what this wave's lanes wrote to LDS is there for its other lanes
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int lanes_below(uint64_t who) { return __popcll(who & ((1ull << (threadIdx.x & 63)) - 1)); }

// the first i of [from, n) with is(i), or n: 64 candidates at a time (one by one they took 40 ns each)
template <typename Is>
__device__ __forceinline__ int next_of(int from, int n, Is&& is)
{
    const int lane = threadIdx.x & 63;
    for (; from < n; from += 64) {
        const uint64_t who = __ballot(from + lane < n && is(from + lane));
        if (who) return from + __builtin_ctzll(who);
    }
    return n;
}

// Up to FEW tokens, one launch: every workgroup picks the uses of its rows (up to FEW_ROWS) from all tokens, whose 32 KB it reads in less than the launches of a
// sort would take.
// Tiles of columns are neighbours in the launch, so that workgroups write one part of the table at a time (8192 Zipf tokens, 50021 x 1024 in fp32: 93 us with all
// first tiles ahead of the second, 69 so).  FEW_MANY: uses of a row from which all waves share them (4095 Zipf tokens, 20011 x 512: 1.9 us of 17 less than from 64).
// A row's uses are one workgroup's for a tile of columns, however many there are: 8192 tokens, bf16 into fp32, 1024 wide, take 147 us over 2 rows, and 109 over 50021
// rows with 60 % of them on one token, which the sort of one token more does in 25 and 52.  (Zipf's law over 50021 rows: 41 us, and 54 by the sort.)
constexpr int FEW = 8192, FEW_WAVES = 16, FEW_ROWS = 256, FEW_MANY = 24, FEW_STEPS = FEW / (FEW_WAVES * 64);

template <typename T, typename TG, bool PAST>
__global__ __launch_bounds__(FEW_WAVES * 64, 8) void k_embed_grad_few(const int32_t* __restrict__ tokens, const T* __restrict__ dout, TG* __restrict__ dtable, int n, int V, int d,
                                                                      int64_t dout_stride, float scale, int rows_each, int tiles)
{
    __shared__ uint32_t uses[FEW];                             // place of the token * FEW_ROWS + row, in the tokens' order
    __shared__ int32_t found[FEW_WAVES], count[FEW_ROWS];
    __shared__ uint32_t mine[FEW_WAVES][64];
    using S = SumsTo<T, TG>;
    constexpr int AHEAD = sizeof(T) == 2 ? 6 : 8;              // (what 64 registers hold; two rows more of bfloat16 spilled: 21.5 us for 18.4, 4095 tokens, 20011 x 512)
    __shared__ float room[FEW_WAVES / 2][S::COLS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = int(blockIdx.x % unsigned(tiles)), v0 = int(blockIdx.x / unsigned(tiles)) * rows_each, rows = min(rows_each, V - v0);
    constexpr uint32_t NONE = 0xffffffffu;
    if (threadIdx.x < FEW_ROWS) count[threadIdx.x] = 0;
    // wave w looks through its sixteenth of the tokens
    const int per = (n + FEW_WAVES - 1) / FEW_WAVES, t0 = wave * per, t1 = min(n, t0 + per);
    uint32_t row[FEW_STEPS];
    int total = 0;
#pragma unroll
    for (int i = 0; i < FEW_STEPS; ++i) {
        const int t = t0 + i * 64 + lane;
        row[i] = t < t1 ? uint32_t(tokens[t]) - uint32_t(v0) : NONE;             // (a token below v0 is far above)
        if (row[i] >= uint32_t(rows)) row[i] = NONE;
    }
#pragma unroll
    for (int i = 0; i < FEW_STEPS; ++i) total += __popcll(__ballot(row[i] != NONE));
    if (lane == 0) found[wave] = total;
    __syncthreads();
    int at = 0, all = 0;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) {
        at += w < wave ? found[w] : 0;
        all += found[w];
    }
#pragma unroll
    for (int i = 0; i < FEW_STEPS; ++i) {
        const uint64_t who = __ballot(row[i] != NONE);
        if (row[i] != NONE) {
            uses[at + lanes_below(who)] = uint32_t(t0 + i * 64 + lane) * FEW_ROWS + row[i];
            atomicAdd(&count[row[i]], 1);
        }
        at += __popcll(who);
    }
    __syncthreads();
    // rows with few uses: a wave's each
    for (int r = wave; r < rows; r += FEW_WAVES) {
        const int k = __builtin_amdgcn_readfirstlane(count[r]);
        if (k > FEW_MANY) continue;
        if (k == 0) {
            for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS)
                S::template store_zeros<PAST>(dtable + size_t(v0 + r) * size_t(d), c, d);
            continue;
        }
        for (int u = 0, seen = 0; seen < k; u += 64) {
            const uint32_t use = u + lane < all ? uses[u + lane] : NONE;
            const bool on = u + lane < all && use % FEW_ROWS == uint32_t(r);
            const uint64_t who = __ballot(on);
            if (on) mine[wave][seen + lanes_below(who)] = use / FEW_ROWS;
            seen += __popcll(who);
        }
        wave_sync();
        for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS) {
            S s;
            s.clear();
            s.template add<AHEAD>(dout, dout_stride, c, d, k, [&](int u) { return __builtin_amdgcn_readfirstlane(mine[wave][u]); });
            s.store(dtable + size_t(v0 + r) * size_t(d), c, d, scale);
        }
        wave_sync();
    }
    // rows with many: all waves', a sixteenth of the list each
    const int from = all * wave / FEW_WAVES, to = all * (wave + 1) / FEW_WAVES;
    for (int r = -1;;) {
        r = next_of(r + 1, rows, [&](int i) { return count[i] > FEW_MANY; });
        if (r >= rows) break;
        for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS) {
            S s;
            s.clear();
            for (int u = from; u < to; u += 64) {
                const uint32_t use = u + lane < to ? uses[u + lane] : NONE;
                const bool on = u + lane < to && use % FEW_ROWS == uint32_t(r);
                const uint64_t who = __ballot(on);
                if (on) mine[wave][lanes_below(who)] = use / FEW_ROWS;
                wave_sync();
                s.template add<AHEAD>(dout, dout_stride, c, d, __popcll(who), [&](int i) { return __builtin_amdgcn_readfirstlane(mine[wave][i]); });
                wave_sync();
            }
            s.template join<FEW_WAVES>(room, wave);
            if (wave == 0) s.store(dtable + size_t(v0 + r) * size_t(d), c, d, scale);
        }
    }
}

// More tokens: a stable sort by token, digit by digit (the last digit first), with two launches a digit: how often every digit value comes in every
// block of tokens, and the tokens to their places.  At most SORT_BLOCKS blocks, so that a workgroup can add up what stands ahead of its own by itself; its
// sixteen waves keep the chains of dependent accesses short, of which such launches are made (65536 tokens: 34 us with four, 22 with sixteen).
constexpr int SORT_BITS = 9, SORT_VALUES = 1 << SORT_BITS, SORT_BLOCKS = 128, SORT_WAVES = 16, SORT_STEPS = 2, SORT_STEP = SORT_WAVES * SORT_STEPS * 64;

struct Range { int32_t begin, end; };                          // a row's sorted uses

// the sort's key: the token, or V where it is outside the table
__device__ __forceinline__ uint32_t key_of(const int32_t* tokens, const uint32_t* keys, int i, int V)
{
    if (keys) return keys[i];
    const uint32_t t = uint32_t(tokens[i]);
    return t < uint32_t(V) ? t : uint32_t(V);
}

// (workgroups behind the blocks' clear the rows' ranges)
__global__ __launch_bounds__(1024) void k_sort_count(const int32_t* __restrict__ tokens, const uint32_t* __restrict__ keys, int32_t* __restrict__ counts, int n, int per, int V,
                                                     int shift, int bits, int blocks, Range* __restrict__ ranges)
{
    __shared__ int32_t c[SORT_VALUES];
    if (int(blockIdx.x) >= blocks) {
        for (int v = (int(blockIdx.x) - blocks) * 1024 + int(threadIdx.x); v < V; v += (int(gridDim.x) - blocks) * 1024) ranges[v] = Range{0, 0};
        return;
    }
    const int values = 1 << bits;
    if (int(threadIdx.x) < values) c[threadIdx.x] = 0;
    __syncthreads();
    const int from = int(blockIdx.x) * per, to = min(n, from + per);
#pragma unroll 2
    for (int i = from + int(threadIdx.x); i < to; i += 1024) atomicAdd(&c[key_of(tokens, keys, i, V) >> shift & uint32_t(values - 1)], 1);
    __syncthreads();
    if (int(threadIdx.x) < values) counts[size_t(blockIdx.x) * SORT_VALUES + threadIdx.x] = c[threadIdx.x];
}

__global__ __launch_bounds__(1024) void k_sort_place(const int32_t* __restrict__ tokens, const uint32_t* __restrict__ keys, const int32_t* __restrict__ places,
                                                     const int32_t* __restrict__ counts, uint32_t* __restrict__ keys_out, int32_t* __restrict__ places_out, int n, int per, int V,
                                                     int shift, int bits, int blocks)
{
    __shared__ int32_t base[SORT_VALUES];                      // where the next key with this digit goes
    __shared__ int32_t half[2][SORT_VALUES];                   // all and those ahead, of the second half of the blocks
    __shared__ int32_t seen[SORT_WAVES][SORT_VALUES];          // of this step, by wave; then how many the waves ahead have
    __shared__ int32_t sums[SORT_VALUES / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, values = 1 << bits;
    const int from = int(blockIdx.x) * per, to = min(n, from + per);
    uint32_t key[SORT_STEPS];
    int32_t place[SORT_STEPS], rank[SORT_STEPS];
    auto load = [&](int s0) {
#pragma unroll
        for (int i = 0; i < SORT_STEPS; ++i) {
            const int at = s0 + (wave * SORT_STEPS + i) * 64 + lane;
            key[i] = at < to ? key_of(tokens, keys, at, V) : 0u;
            place[i] = at < to ? (places ? places[at] : at) : 0;
        }
    };
    load(from);
    {
        // half of the blocks a thread: how many of digit value v there are, and how many in the blocks ahead
        const int v = tid & (SORT_VALUES - 1), h = tid / SORT_VALUES;
        int32_t all = 0, ahead = 0;
        if (v < values) {
#pragma unroll 16
            for (int b = h * ((blocks + 1) / 2); b < (h ? blocks : (blocks + 1) / 2); ++b) {
                const int32_t c = counts[size_t(b) * SORT_VALUES + v];
                all += c;
                ahead += b < int(blockIdx.x) ? c : 0;
            }
        }
        if (h) { half[0][v] = all; half[1][v] = ahead; }
        for (int i = tid; i < SORT_WAVES * SORT_VALUES; i += 1024) (&seen[0][0])[i] = 0;
        __syncthreads();
        int32_t sum = 0;
        if (!h) {
            all += half[0][v];
            ahead += half[1][v];
            sum = all;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int32_t u = __shfl_up(sum, o);
                sum += lane >= o ? u : 0;
            }
            if (lane == 63) sums[wave] = sum;
        }
        __syncthreads();
        if (!h) {
            int32_t below = sum - all;
            for (int w = 0; w < wave; ++w) below += sums[w];
            base[v] = below + ahead;
        }
    }
    for (int s0 = from; s0 < to; s0 += SORT_STEP) {
        if (s0 > from) {
            load(s0);
            for (int i = tid; i < SORT_WAVES * SORT_VALUES; i += 1024) (&seen[0][0])[i] = 0;
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < SORT_STEPS; ++i) {
            const bool on = s0 + (wave * SORT_STEPS + i) * 64 + lane < to;
            const uint32_t digit = key[i] >> shift & uint32_t(values - 1);
            uint64_t same = __ballot(on);                      // the lanes with this digit
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(digit >> b & 1);
                same &= digit >> b & 1 ? set : ~set;
            }
            rank[i] = 0;
            if (on) {
                const int below_me = lanes_below(same);
                rank[i] = seen[wave][digit] + below_me;        // (all lanes read ahead of the one that writes)
                wave_sync();
                if (below_me == 0) seen[wave][digit] = rank[i] + __popcll(same);
            }
            wave_sync();
        }
        __syncthreads();
        int32_t sum = 0;
        if (tid < values) {
            int32_t c[SORT_WAVES];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) c[w] = seen[w][tid];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) { seen[w][tid] = sum; sum += c[w]; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SORT_STEPS; ++i)
            if (s0 + (wave * SORT_STEPS + i) * 64 + lane < to) {
                const uint32_t digit = key[i] >> shift & uint32_t(values - 1);
                const int32_t at = base[digit] + seen[wave][digit] + rank[i];
                keys_out[at] = key[i];
                places_out[at] = place[i];
            }
        __syncthreads();
        if (tid < values) base[tid] += sum;
    }
}

// Chunks of CHUNK sorted uses: where a row's begin and end, and of those that are all of one row the sum, for rows with many uses
constexpr int CHUNK = 64;

template <typename T>
__global__ __launch_bounds__(256) void k_embed_chunks(const uint32_t* __restrict__ keys, const int32_t* __restrict__ places, const T* __restrict__ dout, float* __restrict__ sums,
                                                      Range* __restrict__ ranges, int n, int V, int d, int64_t dout_stride)
{
    using S = SumsTo<T, float>;
    __shared__ float room[2][S::COLS];
    const int u0 = int(blockIdx.x) * CHUNK, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int u = u0 + lane;
    const uint32_t key = keys[min(u, n - 1)];
    if (wave == 0 && blockIdx.y == 0 && u < n && key < uint32_t(V)) {
        if (u == 0 || keys[u - 1] != key) ranges[key].begin = u;
        if (u == n - 1 || keys[u + 1] != key) ranges[key].end = u + 1;
    }
    if (u0 + CHUNK > n || key >= uint32_t(V) || __ballot(key == uint32_t(__builtin_amdgcn_readfirstlane(key))) != ~0ull) return;
    const int32_t mine = places[u0 + wave * (CHUNK / 4) + (lane & (CHUNK / 4 - 1))];
    for (int c = int(blockIdx.y) * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += int(gridDim.y) * S::COLS) {
        S s;
        s.clear();
        s.template add<8>(dout, dout_stride, c, d, CHUNK / 4, [&](int i) { return __builtin_amdgcn_readlane(mine, i); });
        s.template join<4>(room, wave);
        if (wave == 0) s.store(sums + size_t(blockIdx.x) * size_t(d), c, d, 1.f);
    }
}

// Tiles of columns are neighbours here, too (65536 tokens: 123 us, 106 so; workgroups of 8 rows: 105, of 4: 110).
constexpr int GRAD_ROWS = 8;                                   // rows of the table of a workgroup
constexpr int MANY = 64;                                       // uses of a row that are one wave's (at least a chunk, so that more of them hold one's border)

template <typename T, typename TG, bool PAST>
__global__ __launch_bounds__(256) void k_embed_grad(const Range* __restrict__ ranges, const int32_t* __restrict__ places, const T* __restrict__ dout,
                                                    const float* __restrict__ sums, TG* __restrict__ dtable, int V, int d, int64_t dout_stride, float scale, int tiles)
{
    using S = SumsTo<T, TG>;
    __shared__ float room[2][S::COLS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (very large tables: blockIdx.y goes on where x ends)
    const int tile = int(blockIdx.x % unsigned(tiles)), v0 = int(blockIdx.y * (gridDim.x / unsigned(tiles)) + blockIdx.x / unsigned(tiles)) * GRAD_ROWS, rows = min(GRAD_ROWS, V - v0);
    if (rows <= 0) return;
    const Range mine = ranges[v0 + min(lane, rows - 1)];
    const int k_mine = mine.end - mine.begin;
    // rows with few uses: neighbours a wave
#pragma unroll
    for (int i = 0; i < GRAD_ROWS / 4; ++i) {
        const int r = wave * (GRAD_ROWS / 4) + i;
        const int from = __builtin_amdgcn_readlane(mine.begin, r), k = __builtin_amdgcn_readlane(k_mine, r);
        if (r >= rows || k > MANY) continue;
        if (k == 0) {
            for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS) S::template store_zeros<PAST>(dtable + size_t(v0 + r) * size_t(d), c, d);
            continue;
        }
        const int32_t use = lane < k ? places[from + lane] : 0;
        for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS) {
            S s;
            s.clear();
            s.template add<8>(dout, dout_stride, c, d, k, [&](int u) { return __builtin_amdgcn_readlane(use, u); });
            s.store(dtable + size_t(v0 + r) * size_t(d), c, d, scale);
        }
    }
    // rows with many: the whole chunks' sums, and the uses ahead of the first and behind the last of them (fewer than 2 * CHUNK), a quarter a wave
    uint64_t many = __ballot(lane < rows && k_mine > MANY);
    for (; many; many &= many - 1) {
        const int r = __builtin_ctzll(many), from = __builtin_amdgcn_readlane(mine.begin, r), to = from + __builtin_amdgcn_readlane(k_mine, r);
        const int c_from = (from + CHUNK - 1) / CHUNK, chunks = to / CHUNK - c_from, ahead = c_from * CHUNK - from, loose = ahead + to % CHUNK;
        const int at = loose * wave / 4, k = loose * (wave + 1) / 4 - at, at_c = int(int64_t(chunks) * wave / 4), k_c = int(int64_t(chunks) * (wave + 1) / 4) - at_c;
        const int i = at + lane;
        const int32_t use = lane < k ? places[i < ahead ? from + i : to - to % CHUNK + i - ahead] : 0;
        for (int c = tile * S::COLS + lane * S::STEP / 64; c - lane * S::STEP / 64 < d; c += tiles * S::COLS) {
            S s;
            s.clear();
            s.add_sums(sums + size_t(c_from + at_c) * size_t(d), c, d, k_c);
            s.template add<8>(dout, dout_stride, c, d, k, [&](int u) { return __builtin_amdgcn_readlane(use, u); });
            s.template join<4>(room, wave);
            if (wave == 0) s.store(dtable + size_t(v0 + r) * size_t(d), c, d, scale);
        }
    }
}

struct SortLayout {
    int per, blocks, passes, bits;                             // tokens of a block, blocks; digits, their bits
    size_t counts, keys[2], places[2], sums, ranges, total;
};

SortLayout sort_layout(const dynb_embed_shape* s)
{
    SortLayout L = {};
    if (s->T <= FEW) { L.total = 256; return L; }
    const int64_t T = s->T, share = (T + SORT_BLOCKS - 1) / SORT_BLOCKS;
    L.per = int((share + SORT_STEP - 1) / SORT_STEP * SORT_STEP);
    L.blocks = int((T + L.per - 1) / L.per);
    int bits = 0;
    while (int64_t(s->V) >> bits) ++bits;                      // (V itself is a key)
    L.passes = (bits + SORT_BITS - 1) / SORT_BITS;
    L.bits = (bits + L.passes - 1) / L.passes;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += (bytes + 255) & ~size_t(255); return at; };
    L.counts = take(size_t(L.blocks) * SORT_VALUES * 4);
    for (int i = 0; i < 2; ++i) {
        L.keys[i] = take(size_t(T) * 4);
        L.places[i] = take(size_t(T) * 4);
    }
    L.sums = take(size_t(T / CHUNK) * size_t(s->d) * 4);
    L.ranges = take(size_t(s->V) * sizeof(Range));
    L.total = o;
    return L;
}

int check(const dynb_embed_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->T < 0 || s->V <= 0 || s->d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_F32 && s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    if (s->T > 1 << 25 || s->V > 1 << 27 || s->d > 1 << 28) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^25 tokens, 2^27 rows or 2^28 columns");   // (a launch has room for 2^32 threads)
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
    auto launch = [&](auto in) {
        using T = decltype(in);
        hipLaunchKernelGGL((k_embed<T>), dim3(unsigned((s->T + 3) / 4)), dim3(256), 0, st, tokens, static_cast<const T*>(table), static_cast<T*>(out), s->T, s->V, s->d, out_stride,
                           s->scale);
    };
    if (s->dtype == DYNB_BF16) launch(bf16_t{});
    else launch(float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_embed: ") + hipGetErrorString(e));
    return DYNB_OK;
}

extern "C" size_t dynb_embed_backward_workspace_bytes(const dynb_embed_shape* s)
{
    if (check(s, "dynb_embed_backward_workspace_bytes") != DYNB_OK) return 0;
    return sort_layout(s).total;
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
    const SortLayout L = sort_layout(s);
    char* const ws = static_cast<char*>(workspace);
    const uint32_t* keys = nullptr;
    const int32_t* places = nullptr;
    Range* const ranges = reinterpret_cast<Range*>(ws + L.ranges);
    for (int i = 0; i < L.passes; ++i) {
        int32_t* const counts = reinterpret_cast<int32_t*>(ws + L.counts);
        uint32_t* const to = reinterpret_cast<uint32_t*>(ws + L.keys[i & 1]);
        int32_t* const places_to = reinterpret_cast<int32_t*>(ws + L.places[i & 1]);
        const unsigned clearing = i == 0 ? unsigned(std::min(s->V / 1024 + 1, 512)) : 0u;
        hipLaunchKernelGGL(k_sort_count, dim3(unsigned(L.blocks) + clearing), dim3(1024), 0, st, tokens, keys, counts, s->T, L.per, s->V, i * L.bits, L.bits, L.blocks, ranges);
        hipLaunchKernelGGL(k_sort_place, dim3(unsigned(L.blocks)), dim3(1024), 0, st, tokens, keys, places, counts, to, places_to, s->T, L.per, s->V, i * L.bits, L.bits, L.blocks);
        keys = to;
        places = places_to;
    }
    auto launch_as = [&](auto in, auto grad, auto past) {
        using T = decltype(in);
        using TG = decltype(grad);
        constexpr bool PAST = decltype(past)::value;
        const T* const from = static_cast<const T*>(dout);
        TG* const to = static_cast<TG*>(dtable);
        const unsigned tiles = unsigned(std::min((s->d - 1) / SumsTo<T, TG>::COLS + 1, 64));
        if (L.passes == 0) {
            // two workgroups a CU, if the rows are not too many for that, nor too few (8192 tokens, 777 x 64: 42 us with 16 rows, 30 with 4; 512 tokens,
            // 2000 x 512: 6.9 with 8)
            const int rows = int(std::min<int64_t>(std::max<int64_t>((int64_t(s->V) * tiles + 511) / 512, 4), FEW_ROWS));
            const unsigned groups = unsigned((s->V + rows - 1) / rows), few_tiles = std::min(tiles, std::max(1u, (1u << 22) / groups));      // (fewer than 2^32 threads)
            hipLaunchKernelGGL((k_embed_grad_few<T, TG, PAST>), dim3(groups * few_tiles), dim3(FEW_WAVES * 64), 0, st, tokens, from, to, s->T, s->V, s->d, dout_stride, s->scale, rows,
                               int(few_tiles));
            return;
        }
        float* const sums = reinterpret_cast<float*>(ws + L.sums);
        hipLaunchKernelGGL((k_embed_chunks<T>), dim3(unsigned((s->T + CHUNK - 1) / CHUNK), tiles), dim3(256), 0, st, keys, places, from, sums, ranges, s->T, s->V, s->d, dout_stride);
        // (an axis of a launch has room for fewer than 2^24 workgroups of 256 threads)
        const unsigned groups = unsigned((s->V + GRAD_ROWS - 1) / GRAD_ROWS), wide = std::min(groups, (1u << 23) / tiles);
        hipLaunchKernelGGL((k_embed_grad<T, TG, PAST>), dim3(wide * tiles, (groups + wide - 1) / wide), dim3(256), 0, st, ranges, places, from, sums, to, s->V, s->d, dout_stride, s->scale,
                           int(tiles));
    };
    // Rows without uses are most of a large table.  Where the gradient is larger than the 256 MB behind the L2s, they are written past the caches, and what is read,
    // or will be, stays (8192 tokens, 128000 rows x 1024 in fp32, with the gradients' norm taken behind it: 406 us through them, 355 past them); a smaller one is
    // left for the norm to find there (50021 rows: 129 us, 138 past them).
    auto launch = [&](auto in, auto grad) {
        if (size_t(s->V) * size_t(s->d) * sizeof(grad) > size_t(256) << 20) launch_as(in, grad, std::true_type{});
        else launch_as(in, grad, std::false_type{});
    };
    if (s->dtype == DYNB_BF16 && grad_dtype == DYNB_BF16) launch(bf16_t{}, bf16_t{});
    else if (s->dtype == DYNB_BF16) launch(bf16_t{}, float{});
    else if (grad_dtype == DYNB_BF16) launch(float{}, bf16_t{});
    else launch(float{}, float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_embed_backward: ") + hipGetErrorString(e));
    return DYNB_OK;
}
