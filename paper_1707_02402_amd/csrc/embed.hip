// Token embeddings: rows of a table by token, scaled, and the table's gradient.
//   out[t] = scale * table[tokens[t]]              dtable[v] = scale * sum over t with tokens[t] = v of dout[t]
// A token outside [0, V) (padding) has a row of zeros and gives no gradient.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "device_utils.h"
#include "plan_internal.h"
#include "rows.h"

using dynb::fail;

namespace {

// a wave a token
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
// order; a row without uses is a row of zeros.  A wave sums a row, 1024 columns at a time (16 a lane), and a workgroup's waves share the uses of
// a row that has many.
constexpr int SUM_LANE = 16, SUM_COLS = 64 * SUM_LANE;
constexpr int MANY = 64;                                       // uses of a row that are one wave's

template <typename T>
struct Sums {
    static constexpr int P = PIECE<T>, NV = SUM_LANE / P;
    float v[NV][P];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) v[i][j] = 0.f;
    }
    // the rows at(0) .. at(n - 1) of `rows`, from column c0 on
    template <int K, typename At>
    __device__ __forceinline__ void add_some(const T* rows, int64_t stride, int c0, int d, int u, At&& at)
    {
        const int c = c0 + int(threadIdx.x & 63) * P;
        u32x4 raw[K][NV];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const T* const p = rows + int64_t(at(u + k)) * stride;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (c0 + i * 64 * P < d) raw[k][i] = load_piece(p + c + i * 64 * P, d - c - i * 64 * P);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (c0 + i * 64 * P < d)
#pragma unroll
                    for (int j = 0; j < P; ++j) v[i][j] += element<T>(raw[k][i], j);
    }
    template <typename At>
    __device__ __forceinline__ void add(const T* rows, int64_t stride, int c0, int d, int n, At&& at)
    {
        int u = 0;
        for (; u + 4 <= n; u += 4) add_some<4>(rows, stride, c0, d, u, at);
        for (; u < n; ++u) add_some<1>(rows, stride, c0, d, u, at);
    }
    // a row of sums in fp32
    __device__ __forceinline__ void add_sums(const float* row, int c0, int d)
    {
        const int c = c0 + int(threadIdx.x & 63) * P;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int h = 0; h < P; h += 4) {
                const u32x4 raw = load_piece(row + c + i * 64 * P + h, d - c - i * 64 * P - h);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][h + j] += element<float>(raw, j);
            }
    }
    // the sums of all WAVES waves (a power of two), in wave 0: halves of the waves give theirs to the others, half of the columns at a time.  All threads call it.
    template <int WAVES>
    __device__ __forceinline__ void join(float (*room)[SUM_COLS / 2], int wave)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int half = WAVES / 2; half > 0; half >>= 1) {
                __syncthreads();
                if (wave >= half && wave < 2 * half)
#pragma unroll
                    for (int i = 0; i < NV / 2; ++i)
#pragma unroll
                        for (int j = 0; j < P; ++j) room[wave - half][(i * P + j) * 64 + lane] = v[h * (NV / 2) + i][j];
                __syncthreads();
                if (wave < half)
#pragma unroll
                    for (int i = 0; i < NV / 2; ++i)
#pragma unroll
                        for (int j = 0; j < P; ++j) v[h * (NV / 2) + i][j] += room[wave][(i * P + j) * 64 + lane];
            }
        __syncthreads();
    }
    template <typename TG>
    __device__ __forceinline__ void store(TG* row, int c0, int d, float scale)
    {
        const int c = c0 + int(threadIdx.x & 63) * P;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[P];
#pragma unroll
            for (int j = 0; j < P; ++j) w[j] = v[i][j] * scale;
            if (c0 + i * 64 * P < d) store_piece<P>(row + c + i * 64 * P, d - c - i * 64 * P, w);
        }
    }
};

// what this wave's lanes wrote to LDS is there for its other lanes
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int lanes_below(uint64_t who) { return __popcll(who & ((1ull << (threadIdx.x & 63)) - 1)); }

// Up to FEW tokens, one launch: every workgroup picks the uses of its 64 rows from all tokens, whose 32 KB it reads in less than the launches of a
// sort would take.
constexpr int FEW = 8192, FEW_WAVES = 16, FEW_ROWS = 64, FEW_STEPS = FEW / (FEW_WAVES * 64);

template <typename T, typename TG>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_embed_grad_few(const int32_t* __restrict__ tokens, const T* __restrict__ dout, TG* __restrict__ dtable, int n, int V, int d,
                                                                   int64_t dout_stride, float scale)
{
    __shared__ uint32_t uses[FEW];                             // place of the token * 64 + row, in the tokens' order
    __shared__ int32_t found[FEW_WAVES], count[FEW_ROWS];
    __shared__ uint32_t mine[FEW_WAVES][MANY];
    __shared__ float room[FEW_WAVES / 2][SUM_COLS / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int v0 = int(blockIdx.x) * FEW_ROWS, rows = min(FEW_ROWS, V - v0);
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
        if (k > MANY) continue;
        for (int u = 0, seen = 0; seen < k; u += 64) {
            const uint32_t use = u + lane < all ? uses[u + lane] : NONE;
            const bool on = u + lane < all && use % FEW_ROWS == uint32_t(r);
            const uint64_t who = __ballot(on);
            if (on) mine[wave][seen + lanes_below(who)] = use / FEW_ROWS;
            seen += __popcll(who);
        }
        wave_sync();
        for (int c0 = 0; c0 < d; c0 += SUM_COLS) {
            Sums<T> s;
            s.clear();
            s.add(dout, dout_stride, c0, d, k, [&](int u) { return __builtin_amdgcn_readfirstlane(mine[wave][u]); });
            s.store(dtable + size_t(v0 + r) * size_t(d), c0, d, scale);
        }
        wave_sync();
    }
    // rows with many: all waves', a sixteenth of the list each
    for (int r = 0; r < rows; ++r) {
        if (count[r] <= MANY) continue;
        const int from = all * wave / FEW_WAVES, to = all * (wave + 1) / FEW_WAVES;
        for (int c0 = 0; c0 < d; c0 += SUM_COLS) {
            Sums<T> s;
            s.clear();
            for (int u = from; u < to; u += 64) {
                const uint32_t use = u + lane < to ? uses[u + lane] : NONE;
                const bool on = u + lane < to && use % FEW_ROWS == uint32_t(r);
                const uint64_t who = __ballot(on);
                if (on) mine[wave][lanes_below(who)] = use / FEW_ROWS;
                wave_sync();
                s.add(dout, dout_stride, c0, d, __popcll(who), [&](int i) { return __builtin_amdgcn_readfirstlane(mine[wave][i]); });
                wave_sync();
            }
            s.template join<FEW_WAVES>(room, wave);
            if (wave == 0) s.store(dtable + size_t(v0 + r) * size_t(d), c0, d, scale);
        }
    }
}

// More tokens: a stable sort by token, digit by digit (the last digit first), with two launches a digit: how often every digit value comes in every
// block of tokens, and the tokens to their places.  At most SORT_BLOCKS blocks, so that a workgroup can add up what stands ahead of its own by itself.
constexpr int SORT_BITS = 9, SORT_VALUES = 1 << SORT_BITS, SORT_BLOCKS = 128, SORT_STEP = 2048;

// the sort's key: the token, or V where it is outside the table
__device__ __forceinline__ uint32_t key_of(const int32_t* tokens, const uint32_t* keys, int i, int V)
{
    if (keys) return keys[i];
    const uint32_t t = uint32_t(tokens[i]);
    return t < uint32_t(V) ? t : uint32_t(V);
}

__global__ __launch_bounds__(256) void k_sort_count(const int32_t* __restrict__ tokens, const uint32_t* __restrict__ keys, int32_t* __restrict__ counts, int n, int per, int V,
                                                    int shift, int bits)
{
    __shared__ int32_t c[SORT_VALUES];
    const int values = 1 << bits;
    for (int i = threadIdx.x; i < values; i += 256) c[i] = 0;
    __syncthreads();
    const int from = int(blockIdx.x) * per, to = min(n, from + per);
#pragma unroll 8
    for (int i = from + int(threadIdx.x); i < to; i += 256) atomicAdd(&c[key_of(tokens, keys, i, V) >> shift & uint32_t(values - 1)], 1);
    __syncthreads();
    for (int i = threadIdx.x; i < values; i += 256) counts[size_t(blockIdx.x) * SORT_VALUES + i] = c[i];
}

__global__ __launch_bounds__(256) void k_sort_place(const int32_t* __restrict__ tokens, const uint32_t* __restrict__ keys, const int32_t* __restrict__ places,
                                                    const int32_t* __restrict__ counts, uint32_t* __restrict__ keys_out, int32_t* __restrict__ places_out, int n, int per, int V,
                                                    int shift, int bits, int blocks)
{
    __shared__ int32_t base[SORT_VALUES];                      // where the next key with this digit goes
    __shared__ int32_t seen[4][SORT_VALUES];                   // of this step, by wave
    __shared__ int32_t sums[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, values = 1 << bits;
    // two digit values a thread: all that is below them, and what is in the blocks ahead
    int32_t all[2] = {0, 0}, ahead[2] = {0, 0};
#pragma unroll 8
    for (int b = 0; b < blocks; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int32_t c = 2 * tid + i < values ? counts[size_t(b) * SORT_VALUES + 2 * tid + i] : 0;
            all[i] += c;
            ahead[i] += b < int(blockIdx.x) ? c : 0;
        }
    int32_t sum = all[0] + all[1];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int32_t v = __shfl_up(sum, o);
        sum += lane >= o ? v : 0;
    }
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int32_t below = sum - all[0] - all[1];
    for (int w = 0; w < wave; ++w) below += sums[w];
    if (2 * tid < values) {
        base[2 * tid] = below + ahead[0];
        base[2 * tid + 1] = below + all[0] + ahead[1];
    }
    const int from = int(blockIdx.x) * per, to = min(n, from + per);
    for (int s0 = from; s0 < to; s0 += SORT_STEP) {
        for (int i = tid; i < 4 * SORT_VALUES; i += 256) (&seen[0][0])[i] = 0;
        __syncthreads();
        uint32_t key[SORT_STEP / 256];
        int32_t place[SORT_STEP / 256], rank[SORT_STEP / 256];
        const int w0 = s0 + wave * (SORT_STEP / 4);
#pragma unroll
        for (int i = 0; i < SORT_STEP / 256; ++i) {
            const int at = w0 + i * 64 + lane;
            key[i] = at < to ? key_of(tokens, keys, at, V) : 0u;
            place[i] = at < to ? (places ? places[at] : at) : 0;
        }
#pragma unroll
        for (int i = 0; i < SORT_STEP / 256; ++i) {
            const bool on = w0 + i * 64 + lane < to;
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
#pragma unroll
        for (int i = 0; i < SORT_STEP / 256; ++i)
            if (w0 + i * 64 + lane < to) {
                const uint32_t digit = key[i] >> shift & uint32_t(values - 1);
                int32_t to_place = base[digit] + rank[i];
                for (int w = 0; w < wave; ++w) to_place += seen[w][digit];
                keys_out[to_place] = key[i];
                places_out[to_place] = place[i];
            }
        __syncthreads();
        for (int i = tid; i < values; i += 256) base[i] += seen[0][i] + seen[1][i] + seen[2][i] + seen[3][i];
        __syncthreads();
    }
}

// Chunks of CHUNK sorted uses that are all of one row: their sums, for rows with many uses
constexpr int CHUNK = 64;

template <typename T>
__global__ __launch_bounds__(256) void k_embed_chunks(const uint32_t* __restrict__ keys, const int32_t* __restrict__ places, const T* __restrict__ dout, float* __restrict__ sums,
                                                      int V, int d, int64_t dout_stride)
{
    __shared__ float room[2][SUM_COLS / 2];
    const size_t u0 = size_t(blockIdx.x) * CHUNK;
    if (keys[u0] != keys[u0 + CHUNK - 1] || keys[u0] >= uint32_t(V)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t mine = places[u0 + size_t(wave) * (CHUNK / 4) + (threadIdx.x & (CHUNK / 4 - 1))];
    for (int c0 = 0; c0 < d; c0 += SUM_COLS) {
        Sums<T> s;
        s.clear();
        s.add(dout, dout_stride, c0, d, CHUNK / 4, [&](int u) { return __builtin_amdgcn_readlane(mine, u); });
        s.template join<4>(room, wave);
        if (wave == 0) s.store(sums + size_t(blockIdx.x) * size_t(d), c0, d, 1.f);
    }
}

// the first sorted use whose key is not below `key`, among lo .. hi
__device__ __forceinline__ int first_use(const uint32_t* keys, int lo, int hi, uint32_t key)
{
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

constexpr int GRAD_ROWS = 32;                                  // rows of the table of a workgroup

template <typename T, typename TG>
__global__ __launch_bounds__(256) void k_embed_grad(const uint32_t* __restrict__ keys, const int32_t* __restrict__ places, const T* __restrict__ dout,
                                                    const float* __restrict__ sums, TG* __restrict__ dtable, int n, int V, int d, int64_t dout_stride, float scale)
{
    __shared__ int32_t first[GRAD_ROWS + 1];
    __shared__ int32_t mine[4][MANY];
    __shared__ float room[2][SUM_COLS / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int v0 = int(blockIdx.x) * GRAD_ROWS, rows = min(GRAD_ROWS, V - v0);
    if (wave == 0) {
        // the rows' uses: 64 places of the list at a time narrow down where they begin, then every lane looks for a row
        int lo = 0, hi = n;
        while (hi - lo > 64) {
            const int step = (hi - lo + 63) / 64, at = lo + lane * step;
            const uint64_t less = __ballot(at < hi && keys[min(at, hi - 1)] < uint32_t(v0));
            if (less == 0) { hi = lo; break; }
            const int last = 63 - __builtin_clzll(less);
            hi = min(hi, lo + (last + 1) * step);
            lo += last * step;
        }
        const int begin = first_use(keys, lo, hi, uint32_t(v0));
        int end = n;                                           // (of lane r's search: doubled until it is behind row v0 + r)
        for (int64_t step = 64; begin + step < n; step *= 2)
            if (keys[begin + step] >= uint32_t(v0 + rows)) { end = int(begin + step); break; }
        if (lane <= rows) first[lane] = first_use(keys, begin, end, uint32_t(v0 + lane));
    }
    __syncthreads();
    for (int r = wave; r < rows; r += 4) {
        const int s0 = __builtin_amdgcn_readfirstlane(first[r]), k = __builtin_amdgcn_readfirstlane(first[r + 1]) - s0;
        if (k > MANY) continue;
        const int32_t use = lane < k ? places[s0 + lane] : 0;
        for (int c0 = 0; c0 < d; c0 += SUM_COLS) {
            Sums<T> s;
            s.clear();
            s.add(dout, dout_stride, c0, d, k, [&](int u) { return __builtin_amdgcn_readlane(use, u); });
            s.store(dtable + size_t(v0 + r) * size_t(d), c0, d, scale);
        }
    }
    for (int r = 0; r < rows; ++r) {
        const int from = __builtin_amdgcn_readfirstlane(first[r]), to = __builtin_amdgcn_readfirstlane(first[r + 1]);
        if (to - from <= MANY) continue;
        // the uses ahead of the first whole chunk (wave 0), the chunks (a quarter each), the uses behind them (wave 3)
        const int c_from = (from + CHUNK - 1) / CHUNK, chunks = to / CHUNK - c_from;
        const int at = wave == 0 ? from : to / CHUNK * CHUNK, k = wave == 0 ? c_from * CHUNK - from : wave == 3 ? to - at : 0;
        const int32_t use = lane < k ? places[at + lane] : 0;
        for (int c0 = 0; c0 < d; c0 += SUM_COLS) {
            Sums<T> s;
            s.clear();
            if (wave == 0) s.add(dout, dout_stride, c0, d, k, [&](int u) { return __builtin_amdgcn_readlane(use, u); });
#pragma unroll 4
            for (int c = int(int64_t(chunks) * wave / 4); c < int(int64_t(chunks) * (wave + 1) / 4); ++c) s.add_sums(sums + size_t(c_from + c) * size_t(d), c0, d);
            if (wave == 3) s.add(dout, dout_stride, c0, d, k, [&](int u) { return __builtin_amdgcn_readlane(use, u); });
            s.template join<4>(room, wave);
            if (wave == 0) s.store(dtable + size_t(v0 + r) * size_t(d), c0, d, scale);
        }
    }
}

struct SortLayout {
    int per, blocks, passes, bits;                             // tokens of a block, blocks; digits, their bits
    size_t counts, keys[2], places[2], sums, total;
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
    L.total = o;
    return L;
}

int check(const dynb_embed_shape* s, const std::string& who)
{
    if (!s) return fail(DYNB_E_INVAL, who + ": NULL shape");
    if (s->T < 0 || s->V <= 0 || s->d <= 0) return fail(DYNB_E_INVAL, who + ": sizes must be positive");
    if (s->dtype != DYNB_F32 && s->dtype != DYNB_BF16) return fail(DYNB_E_UNSUPPORTED, who + ": unknown dtype");
    if (s->T > 1 << 25 || s->V > 1 << 27) return fail(DYNB_E_UNSUPPORTED, who + ": more than 2^25 tokens or 2^27 rows");   // (a launch has room for 2^32 threads)
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
    for (int i = 0; i < L.passes; ++i) {
        int32_t* const counts = reinterpret_cast<int32_t*>(ws + L.counts);
        uint32_t* const to = reinterpret_cast<uint32_t*>(ws + L.keys[i & 1]);
        int32_t* const places_to = reinterpret_cast<int32_t*>(ws + L.places[i & 1]);
        hipLaunchKernelGGL(k_sort_count, dim3(unsigned(L.blocks)), dim3(256), 0, st, tokens, keys, counts, s->T, L.per, s->V, i * L.bits, L.bits);
        hipLaunchKernelGGL(k_sort_place, dim3(unsigned(L.blocks)), dim3(256), 0, st, tokens, keys, places, counts, to, places_to, s->T, L.per, s->V, i * L.bits, L.bits, L.blocks);
        keys = to;
        places = places_to;
    }
    auto launch = [&](auto in, auto grad) {
        using T = decltype(in);
        using TG = decltype(grad);
        const T* const from = static_cast<const T*>(dout);
        TG* const to = static_cast<TG*>(dtable);
        if (L.passes == 0) {
            hipLaunchKernelGGL((k_embed_grad_few<T, TG>), dim3(unsigned((s->V + FEW_ROWS - 1) / FEW_ROWS)), dim3(FEW_WAVES * 64), 0, st, tokens, from, to, s->T, s->V, s->d, dout_stride,
                               s->scale);
            return;
        }
        float* const sums = reinterpret_cast<float*>(ws + L.sums);
        hipLaunchKernelGGL((k_embed_chunks<T>), dim3(unsigned(s->T / CHUNK)), dim3(256), 0, st, keys, places, from, sums, s->V, s->d, dout_stride);
        hipLaunchKernelGGL((k_embed_grad<T, TG>), dim3(unsigned((s->V + GRAD_ROWS - 1) / GRAD_ROWS)), dim3(256), 0, st, keys, places, from, sums, to, s->T, s->V, s->d, dout_stride,
                           s->scale);
    };
    if (s->dtype == DYNB_BF16 && grad_dtype == DYNB_BF16) launch(bf16_t{}, bf16_t{});
    else if (s->dtype == DYNB_BF16) launch(bf16_t{}, float{});
    else if (grad_dtype == DYNB_BF16) launch(float{}, bf16_t{});
    else launch(float{}, float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DYNB_E_HIP, std::string("dynb_embed_backward: ") + hipGetErrorString(e));
    return DYNB_OK;
}
