// Tables of vectors: rows looked up by symbol and scaled, and the table's gradient.
//
// Forward: out[n, :] = scale * table[tokens[n], :].  Bound by memory: every lane moves one 16-byte vector of a row at a time, four
// of them in flight (262144 rows of 1024 floats: 295 us, 3.6 TB/s written).
//
// Backward: row v of the gradient is the sum of the upstream rows whose symbol is v.  Adding rows with atomics would make results depend on
// the order of arrival and a frequent symbol's row a bottleneck, so the symbols are sorted first (stably, least significant digit
// first) together with their places.  What is left is V + count events in one order: "add upstream row n" for every symbol in
// sorted order, and "write row v" after the last symbol v.  Every unit (the lanes that share a row's columns) takes the same number of
// consecutive events, so that neither a frequent symbol nor a stretch of absent ones makes one unit work longer; where a unit
// begins in the sorted symbols is found by a search on the diagonal i + key[i].  A row whose events are spread over several
// units is finished by a second launch from what they hand over, in their order.  Bound by memory as well: 131072 rows of 4096 bfloat16 from 8192
// tokens 215 us (5.3 TB/s), 50257 rows of 1024 floats from 262144 tokens 290 us (4.4 TB/s); the sort takes 20 and 54 us of that call, the joins 13 and 38.
#include <cfloat>
#include <cmath>

#include "st_dev.h"
#include "st_kernels.h"

namespace st {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------------------------------------ forward
// A lane moves U vectors of E entries (16 bytes where a row has as much), all symbols loaded before the first row and all rows before the first
// store: no branch stands between them.  A row's last vector ends with the row, whatever its length: it may write entries of the one before a second
// time, with the same values.
// A: the product's type, double unless the scale is a float (then a float's product, rounded once, is the same number); of 16-bit types float.
// items: fewer than 2^31 vectors (a 32-bit division for each).
template <typename T, typename A, int E, int U>
__global__ __launch_bounds__(kThreads) void embed_fwd_kernel(const void* tokens, int it, const T* table, T* out, int64_t V, int64_t D, A scale,
                                                             uint32_t per_row, uint32_t items)
{
    const uint32_t first = blockIdx.x * (kThreads * U) + threadIdx.x;
    int64_t symbol[U], at[U];
    int64_t col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t item = first + u * kThreads < items ? first + u * kThreads : items - 1;
        const uint32_t row = item / per_row;
        const int64_t c = (int64_t)(item - row * per_row) * E;
        col[u] = c <= D - E ? c : D - E;
        at[u] = (int64_t)row * D + col[u];
        symbol[u] = load_index(tokens, (int64_t)row, it);
    }
    Vec<T, E> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_vec<T, E>(table + (symbol[u] >= 0 && symbol[u] < V ? symbol[u] : 0) * D + col[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool there = symbol[u] >= 0 && symbol[u] < V;
#pragma unroll
        for (int i = 0; i < E; ++i) v[u].v[i] = there ? (T)((A)v[u].v[i] * scale) : T(0);
        if (first + u * kThreads < items) store_vec(out + at[u], v[u]);
    }
}

// (a table without rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void zeros_kernel(T* out, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) out[i] = T(0);
}

template <typename T, typename A, int E>
hipError_t run_fwd(const void* tokens, const T* table, T* out, int64_t count, int64_t V, int64_t D, double scale, int it, hipStream_t st)
{
    const int64_t per_row = (D + E - 1) / E, most = (((int64_t)1 << 31) - 1) / per_row;   // (rows of at most 2^24 entries)
    const A f = (A)scale;
    for (int64_t row = 0; row < count; row += most) {   // a launch has at most 2^32 threads
        const int64_t items = (count - row < most ? count - row : most) * per_row;
        const void* from = static_cast<const char*>(tokens) + row * (it == ST_I32 ? 4 : 8);
        // four vectors per lane; one where that leaves compute units idle
        auto launch = [&](auto kernel, int64_t vectors) {
            kernel<<<(unsigned)((items + vectors - 1) / vectors), kThreads, 0, st>>>(from, it, table, out + row * D, V, D, f, (uint32_t)per_row,
                                                                                  (uint32_t)items);
            return hipGetLastError();
        };
        const hipError_t e = items < (int64_t)kThreads * 2048 ? launch(embed_fwd_kernel<T, A, E, 1>, kThreads) : launch(embed_fwd_kernel<T, A, E, 4>, kThreads * 4);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ------------------------------------------------------------------------------------------------ sort
// A workgroup of 16 waves takes ROWS * 1024 symbols, consecutive ones per wave, in ROWS rows of 64.  Eight rows share the work of counting and
// scanning among most symbols; two rows give more workgroups while there are few (32768 symbols of 1000, one digit: 4 workgroups and 20 us, or 16 and 13 us).
constexpr int kSortThreads = 1024, kSortWaves = 16, kManyRows = 8, kFewRows = 2;
constexpr int kSmall = kSortThreads * kManyRows;   // what one workgroup sorts by itself
constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;   // at most
static_assert(kDigits <= kSortThreads);

__device__ __forceinline__ uint32_t symbol_key(const void* tokens, int64_t i, int it, uint32_t V)
{
    const int64_t s = load_index(tokens, i, it);
    return s >= 0 && s < (int64_t)V ? (uint32_t)s : V;   // symbols outside the table go behind all others
}

// Ranks a wave's symbols by their digit, in order: counts (of the wave, cleared before) ends up with the number of each digit.
template <int ROWS>
__device__ __forceinline__ void rank_wave(const uint32_t (&key)[ROWS], const bool (&live)[ROWS], int shift, int bits, volatile uint32_t* counts,
                                          uint32_t (&rank)[ROWS])
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t digit = key[r] >> shift & ((1u << bits) - 1);
        uint64_t same = __ballot(live[r]);
        for (int b = 0; b < bits; ++b) {
            const bool one = digit >> b & 1;
            const uint64_t ones = __ballot(one);
            same &= one ? ones : ~ones;
        }
        if (live[r]) {
            const uint32_t before = counts[digit];
            rank[r] = before + __popcll(same & below);
            if ((same & below) == 0) counts[digit] = before + __popcll(same);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Exclusive sums over the workgroup's threads; *all: the total.  scratch: kSortWaves words.
__device__ __forceinline__ uint32_t scan_block(uint32_t x, uint32_t* scratch, uint32_t* all)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t t = __shfl_up(s, o);
        if (lane >= o) s += t;
    }
    if (lane == 63) scratch[w] = s;
    __syncthreads();
    uint32_t base = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) {
        const uint32_t t = scratch[i];
        if (i < w) base += t;
        total += t;
    }
    __syncthreads();
    *all = total;
    return base + s - x;
}

// counts[wave][digit] -> where the wave's first symbol of the digit goes, from `begin`(digit) on
template <class Begin>
__device__ __forceinline__ void wave_offsets(uint32_t* counts, uint32_t* scratch, int bits, Begin&& begin)
{
    const int digit = threadIdx.x;
    uint32_t mine = 0;
    if (digit < (1 << bits))
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) mine += counts[(w << bits) + digit];
    uint32_t all;
    const uint32_t local = scan_block(mine, scratch, &all);
    if (digit < (1 << bits)) {
        uint32_t at = begin(digit, local);
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = counts[(w << bits) + digit];
            counts[(w << bits) + digit] = at;
            at += c;
        }
    }
    __syncthreads();
}

// Up to kSmall symbols: all digits in one launch, symbols and places in registers and LDS.
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(const void* tokens, int it, uint32_t n, uint32_t V, int passes, int bits,
                                                                  uint32_t* keys, uint32_t* places, uint32_t* list)
{
    if (threadIdx.x < 2) list[threadIdx.x] = 0;
    __shared__ uint32_t counts[kSortWaves * kDigits];
    __shared__ uint32_t key_at[kSmall], place_at[kSmall];
    __shared__ uint32_t scratch[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[kManyRows], place[kManyRows], rank[kManyRows];
    bool live[kManyRows];
#pragma unroll
    for (int r = 0; r < kManyRows; ++r) {
        const uint32_t i = w * (64 * kManyRows) + r * 64 + lane;
        live[r] = i < n;
        place[r] = i;
        key[r] = live[r] ? symbol_key(tokens, i, it, V) : 0;
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        for (int i = threadIdx.x; i < kSortWaves << bits; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        rank_wave(key, live, shift, bits, counts + (w << bits), rank);
        __syncthreads();
        wave_offsets(counts, scratch, bits, [](int, uint32_t local) { return local; });
#pragma unroll
        for (int r = 0; r < kManyRows; ++r)
            if (live[r]) {
                const uint32_t to = counts[(w << bits) + (key[r] >> shift & ((1u << bits) - 1))] + rank[r];
                key_at[to] = key[r];
                place_at[to] = place[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kManyRows; ++r) {
            const uint32_t i = w * (64 * kManyRows) + r * 64 + lane;
            if (live[r]) {
                key[r] = key_at[i];
                place[r] = place_at[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kManyRows; ++r) {
        const uint32_t i = w * (64 * kManyRows) + r * 64 + lane;
        if (live[r]) {
            keys[i] = key[r];
            places[i] = place[r];
        }
    }
}

// One digit of many symbols: the digits' numbers in every tile, counts[digit][tile], their running sums (by digit, then by tile), and the symbols to
// where they go.  Of at most kAddTiles tiles the last launch adds up the numbers itself, counts[tile][digit], which takes it less than a launch in
// between.  keys_in null: the first digit, from the caller's symbols.
constexpr int kAddTiles = 128;
template <int ROWS>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const void* tokens, int it, const uint32_t* keys_in, uint32_t n, uint32_t V,
                                                                  int shift, int bits, uint32_t* counts, uint32_t* list)
{
    if (blockIdx.x == 0 && threadIdx.x < 2) list[threadIdx.x] = 0;
    __shared__ uint32_t bin[kDigits];
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) bin[i] = 0;
    __syncthreads();
    const uint64_t base = (uint64_t)blockIdx.x * (ROWS * kSortThreads);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint64_t i = base + r * kSortThreads + threadIdx.x;
        if (i < n) {
            const uint32_t key = keys_in ? keys_in[i] : symbol_key(tokens, (int64_t)i, it, V);
            atomicAdd(&bin[key >> shift & ((1u << bits) - 1)], 1u);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (1 << bits); i += kSortThreads)
        counts[gridDim.x <= kAddTiles ? ((size_t)blockIdx.x << bits) + i : (size_t)i * gridDim.x + blockIdx.x] = bin[i];
}

__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(uint32_t* counts, int64_t entries)
{
    __shared__ uint32_t scratch[kSortWaves];
    constexpr int kEach = 8;
    uint32_t before = 0;
    for (int64_t first = 0; first < entries; first += kSortThreads * kEach) {
        const int64_t i = first + threadIdx.x * kEach;
        uint32_t c[kEach], sum = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) c[j] = i + j < entries ? counts[i + j] : 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum += c[j];
        uint32_t all;
        uint32_t at = before + scan_block(sum, scratch, &all);
        before += all;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (i + j < entries) counts[i + j] = at;
            at += c[j];
        }
    }
}

template <int ROWS>
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(const void* tokens, int it, const uint32_t* keys_in, const uint32_t* places_in,
                                                                 uint32_t n, uint32_t V, int shift, int bits, const uint32_t* begin,
                                                                 uint32_t* keys, uint32_t* places)
{
    __shared__ uint32_t counts[kSortWaves * kDigits];
    __shared__ uint32_t scratch[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[ROWS], place[ROWS], rank[ROWS];
    bool live[ROWS];
    for (int i = threadIdx.x; i < kSortWaves << bits; i += kSortThreads) counts[i] = 0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint64_t i = (uint64_t)blockIdx.x * (ROWS * kSortThreads) + w * (64 * ROWS) + r * 64 + lane;
        live[r] = i < n;
        key[r] = !live[r] ? 0 : keys_in ? keys_in[i] : symbol_key(tokens, (int64_t)i, it, V);
        place[r] = !live[r] ? 0 : keys_in ? places_in[i] : (uint32_t)i;
    }
    __syncthreads();
    rank_wave(key, live, shift, bits, counts + (w << bits), rank);
    __syncthreads();
    if (gridDim.x <= kAddTiles) {
        uint32_t before = 0, total = 0, all;
        if (threadIdx.x < 1 << bits)
#pragma unroll 8
            for (uint32_t t = 0; t < gridDim.x; ++t) {
                const uint32_t c = begin[((size_t)t << bits) + threadIdx.x];
                total += c;
                before += t < blockIdx.x ? c : 0;
            }
        before += scan_block(total, scratch, &all);
        wave_offsets(counts, scratch, bits, [&](int, uint32_t) { return before; });
    } else {
        wave_offsets(counts, scratch, bits, [&](int digit, uint32_t) { return begin[(size_t)digit * gridDim.x + blockIdx.x]; });
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (live[r]) {
            const uint32_t to = counts[(w << bits) + (key[r] >> shift & ((1u << bits) - 1))] + rank[r];
            keys[to] = key[r];
            places[to] = place[r];
        }
}

// ------------------------------------------------------------------------------------------------ sums
constexpr uint32_t kWrite = 0xffffffffu, kNothing = 0xfffffffeu;   // events that are no upstream row

// Of the events before `d`, how many are symbols: the first i with key[i] + i >= d.  By a whole wave, 64 probes at a time.
__device__ __forceinline__ uint32_t symbols_before(const uint32_t* keys, int64_t n, int64_t V, int64_t d)
{
    const int lane = threadIdx.x & 63;
    int64_t lo = d > V ? d - V : 0, hi = d < n ? d : n;
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool in = at < hi;
        const uint64_t probes = __ballot(in), yes = __ballot(in && (int64_t)keys[in ? at : lo] + at >= d);
        if (yes == 0) {
            lo += (63 - __clzll(probes)) * step + 1;
        } else {
            const int f = __ffsll((unsigned long long)yes) - 1;
            hi = lo + f * step;
            if (f > 0) lo = hi - step + 1;
        }
    }
    return (uint32_t)lo;
}

// What a unit hands over: the sum of the row it has not finished, and the last part of the row it finished but did not begin.  The units of the
// latter kind are listed with their rows and the symbols before them (in the order they come; what is made of one does not depend on the others),
// those whose row has symbols kLong units before in a list of their own.
constexpr int kLong = 8;
struct Listed {
    uint32_t unit, row, before;
};
template <typename A>
struct Handed {
    A *carry, *head;       // [units][D]
    uint32_t* many;        // entries of both lists, cleared by the sort's first launch
    Listed* list[2];       // short, long
};

// P: the type of a sum's product with the scale.
template <typename T, typename P>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(const T* grad, T* out, const uint32_t* keys, const uint32_t* places, int64_t n,
                                                              int64_t V, int64_t D, int lanes, int events, P scale,
                                                              Handed<sum_t<T>> handed)
{
    constexpr int E = kPer16<T>, kAhead = 8;
    using A = sum_t<T>;
    extern __shared__ uint32_t event[];
    __shared__ uint32_t ends[2];
    __shared__ uint32_t symbols[kThreads];
    const int units = kThreads / lanes, span = units * events;
    const int64_t d0 = (int64_t)blockIdx.x * span, total = n + V, d1 = d0 + span < total ? d0 + span : total;
    const int w = threadIdx.x >> 6;
    if (w < 2) {
        const uint32_t i = symbols_before(keys, n, V, w == 0 ? d0 : d1);
        if ((threadIdx.x & 63) == 0) ends[w] = i;
    }
    for (int i = threadIdx.x; i < span; i += kThreads) event[i] = d0 + i < d1 ? kWrite : kNothing;
    __syncthreads();
    for (uint32_t i = ends[0] + threadIdx.x; i < ends[1]; i += kThreads) {
        const uint32_t key = keys[i];
        event[(int64_t)i + key - d0] = key < V ? places[i] : kNothing;
    }
    __syncthreads();
    const int unit = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    if (threadIdx.x < units) {   // (symbols that are none, behind all rows, count as well)
        uint32_t c = 0;
        for (int i = 0; i < events; ++i) {
            const int at = threadIdx.x * events + i;
            if (event[at] != kWrite && d0 + at < d1) ++c;
        }
        symbols[threadIdx.x] = c;
    }
    __syncthreads();
    for (int o = 1; o < units; o *= 2) {
        uint32_t t = 0;
        if (threadIdx.x < units && threadIdx.x >= o) t = symbols[threadIdx.x - o];
        __syncthreads();
        if (threadIdx.x < units) symbols[threadIdx.x] += t;
        __syncthreads();
    }
    const int64_t mine = d0 + unit * events;
    if (mine >= d1) return;
    const int64_t before = (int64_t)ends[0] + (unit > 0 ? symbols[unit - 1] : 0);
    int64_t row = mine - before;
    const bool begun = before > 0 && row < V && keys[before - 1] == row;
    const int64_t at = (int64_t)blockIdx.x * units + unit;
    const int64_t col = ((int64_t)blockIdx.y * lanes + lane) * E;
    const int width = D - col >= E ? E : D > col ? (int)(D - col) : 0;
    bool wrote = false, some = false;
    const int64_t first_row = row;
    Vec<T, E> zeros;
#pragma unroll
    for (int i = 0; i < E; ++i) zeros.v[i] = T(0);
    T* to = out + row * D + col;
    A sum[E];
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i] = 0;
    for (int e0 = 0; e0 < events; e0 += kAhead) {
        Vec<T, E> v[kAhead];
        uint32_t ev[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            ev[j] = event[unit * events + e0 + j];
            if (ev[j] < kNothing) {
                const T* from = grad + (int64_t)ev[j] * D + col;
                if (width == E) v[j] = load_vec<T, E>(from);
                else if (width > 0) v[j] = load_some<T, E>(from, width);
            }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (ev[j] == kNothing) continue;
            if (ev[j] != kWrite) {
                some = true;
                if (width > 0)
#pragma unroll
                    for (int i = 0; i < E; ++i) sum[i] += (A)v[j].v[i];
                continue;
            }
            if (!wrote && begun) {
                if (width > 0)
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        if (i < width) handed.head[at * D + col + i] = sum[i];
            } else if (!some) {   // (a symbol that does not occur)
                if (width == E) store_vec(to, zeros);
                else if (width > 0) store_some(to, zeros, width);
            } else if (width > 0) {
                Vec<T, E> r;
#pragma unroll
                for (int i = 0; i < E; ++i) r.v[i] = (T)((P)sum[i] * scale);
                if (width == E) store_vec(to, r);
                else store_some(to, r, width);
            }
            if (some || begun)
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] = 0;
            to += D;
            wrote = true;
            some = false;
            ++row;
        }
    }
    const bool carries = some || (!wrote && begun);
    if (carries && width > 0)
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < width) handed.carry[at * D + col + i] = sum[i];
    if (lane == 0 && blockIdx.y == 0 && begun && wrote) {
        const int64_t back = before - 1 - (int64_t)kLong * events;
        const bool is_long = back >= 0 && keys[back] == (uint32_t)first_row;
        // (one atomic addition for all units of the wave)
        const uint64_t longs = __ballot(is_long), shorts = __ballot(!is_long), mine = is_long ? longs : shorts;
        const int self = threadIdx.x & 63, leader = __ffsll((unsigned long long)mine) - 1;
        uint32_t place = 0;
        if (self == leader) place = atomicAdd(handed.many + is_long, (uint32_t)__popcll(mine));
        place = __shfl(place, leader) + __popcll(mine & (((uint64_t)1 << self) - 1));
        handed.list[is_long][place] = {(uint32_t)at, (uint32_t)first_row, (uint32_t)before};
    }
}

// Rows that more than one unit added to: the units' sums in their order, from the one with the row's first symbol on.  Of a frequent symbol's row (of
// thousands of units, it may be) a workgroup takes 64 columns, each wave a quarter of the units; of the others a workgroup takes kShare columns.
constexpr int kJoinWaves = 4, kShare = 512;
template <typename A>
__device__ __forceinline__ A carried(const A* carry, int64_t from, int64_t to, int64_t D, int64_t c)
{
    A sum = 0;
    int64_t i = from;
    for (; i + 8 <= to; i += 8) {
        A part[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) part[j] = carry[(i + j) * D + c];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += part[j];
    }
    for (; i < to; ++i) sum += carry[i * D + c];
    return sum;
}
template <typename T, typename P>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(T* out, const uint32_t* keys, int64_t D, int events, P scale,
                                                                     Handed<sum_t<T>> handed)
{
    using A = sum_t<T>;
    __shared__ A parts[kJoinWaves][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t slices = (uint32_t)((D + 63) / 64);
    const uint32_t shares = (uint32_t)((D + kShare - 1) / kShare);
    const uint64_t few = (uint64_t)handed.many[0] * shares, many = (uint64_t)handed.many[1] * slices;
    for (uint64_t task = blockIdx.x; task < few + many; task += gridDim.x) {
        const bool is_long = task < many;
        const Listed l = is_long ? handed.list[1][task / slices] : handed.list[0][(task - many) / shares];
        // the row's first symbol
        int64_t lo = is_long ? 0 : (int64_t)l.before - 1 - (int64_t)kLong * events, hi = (int64_t)l.before - 1;
        if (lo < 0) lo = 0;
        while (lo < hi) {
            const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
            const bool in = at < hi;
            const uint64_t probes = __ballot(in), yes = __ballot(in && keys[in ? at : lo] >= l.row);
            if (yes == 0) {
                lo += (63 - __clzll(probes)) * step + 1;
            } else {
                const int f = __ffsll((unsigned long long)yes) - 1;
                hi = lo + f * step;
                if (f > 0) lo = hi - step + 1;
            }
        }
        const int64_t u = l.unit, row = l.row, first = (lo + row) / events;
        if (!is_long) {
            const int64_t c0 = (int64_t)((task - many) % shares) * kShare, c1 = c0 + kShare < D ? c0 + kShare : D;
            for (int64_t c = c0 + threadIdx.x; c < c1; c += 64 * kJoinWaves)
                out[row * D + c] = (T)((P)(carried(handed.carry, first, u, D, c) + handed.head[u * D + c]) * scale);
            continue;
        }
        const int64_t c = (int64_t)(task % slices) * 64 + lane;
        parts[w][lane] = c < D ? carried(handed.carry, first + (u - first) * w / kJoinWaves, first + (u - first) * (w + 1) / kJoinWaves, D, c) : (A)0;
        __syncthreads();
        if (w == 0 && c < D) {
            A all = 0;
#pragma unroll
            for (int j = 0; j < kJoinWaves; ++j) all += parts[j][lane];
            out[row * D + c] = (T)((P)(all + handed.head[u * D + c]) * scale);
        }
        __syncthreads();
    }
}

template <typename F>
hipError_t by_type(int dt, F&& f)
{
    switch (dt) {
    case ST_F64: return f(double{});
    case ST_F32: return f(float{});
    case ST_BF16: return f(bf16{});
    default: return f(f16{});
    }
}

// Whether a float holds the scale as well as any other: outside its normal numbers 0 times it may be NaN, and others' products 0.
bool float_scale(double scale) { return scale == 0 || (std::fabs(scale) >= FLT_MIN && std::fabs(scale) <= FLT_MAX); }

}  // namespace

hipError_t embed_fwd(const void* tokens, const void* table, void* out, int64_t count, int64_t V, int64_t D, double scale, int it, int dt,
                     hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        const T* from = static_cast<const T*>(table);
        T* to = static_cast<T*>(out);
        if (V == 0) {
            const int64_t blocks = (count * D + kThreads - 1) / kThreads;
            zeros_kernel<T><<<(unsigned)(blocks < 16384 ? blocks : 16384), kThreads, 0, st>>>(to, count * D);
            return hipGetLastError();
        }
        auto by_width = [&](auto a) {
            using A = decltype(a);
            if (D >= kPer16<T>) return run_fwd<T, A, kPer16<T>>(tokens, from, to, count, V, D, scale, it, st);
            if constexpr (kPer16<T> > 4)
                if (D >= 4) return run_fwd<T, A, 4>(tokens, from, to, count, V, D, scale, it, st);
            if constexpr (kPer16<T> > 2)
                if (D >= 2) return run_fwd<T, A, 2>(tokens, from, to, count, V, D, scale, it, st);
            return run_fwd<T, A, 1>(tokens, from, to, count, V, D, scale, it, st);
        };
        if constexpr (sizeof(T) == 4) {
            if ((double)(float)scale == scale) return by_width(float{});
        } else if constexpr (sizeof(T) == 2) {
            if (float_scale(scale)) return by_width(float{});
        }
        return by_width(double{});
    });
}

EmbedPlan embed_plan(int64_t count, int64_t V, int64_t D, int dt)
{
    EmbedPlan p{};
    p.count = count;
    p.V = V;
    p.D = D;
    const int size = dtype_size(dt), sum_size = size == 2 ? 4 : 8;
    const int64_t vectors = (D * size + 15) / 16;
    p.lanes = 1;
    while (p.lanes < vectors && p.lanes < kThreads) p.lanes *= 2;
    p.slices = (int)((vectors + p.lanes - 1) / p.lanes);
    const int per_group = kThreads / p.lanes;
    // 32 events share the search for their beginning; fewer while there are not two workgroups for every compute unit
    p.events = 32;
    while (p.events > 8 && (count + V) / (p.events * per_group) * p.slices < 512) p.events /= 2;
    p.units = (count + V + p.events - 1) / p.events;
    p.groups = (p.units + per_group - 1) / per_group;
    int bits = 1;
    while (bits < 32 && ((uint64_t)V >> bits) != 0) ++bits;   // the largest key is V
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.rows = count <= 128 * kSortThreads ? kFewRows : kManyRows;
    const int64_t tile = (int64_t)p.rows * kSortThreads;
    p.tiles = count <= kSmall ? 0 : (count + tile - 1) / tile;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    const int halves = p.tiles != 0 && p.passes > 1 ? 2 : 1;
    for (int i = 0; i < 2; ++i) {
        p.off_keys[i] = i < halves ? take((size_t)count * 4) : p.off_keys[0];
        p.off_places[i] = i < halves ? take((size_t)count * 4) : p.off_places[0];
    }
    p.off_counts = take((size_t)p.tiles * 4 << p.bits);
    const int64_t slots = p.groups * per_group;
    p.off_carry = take((size_t)slots * D * sum_size);
    p.off_head = take((size_t)slots * D * sum_size);
    p.off_list = take(256 + (size_t)p.units * 2 * sizeof(Listed));
    p.total = at;
    return p;
}

hipError_t embed_bwd(const EmbedPlan& p, const void* tokens, const void* grad_out, void* grad_table, double scale, int it, int dt, void* ws,
                     hipStream_t st)
{
    unsigned char* base = static_cast<unsigned char*>(ws);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + p.off_keys[0]), reinterpret_cast<uint32_t*>(base + p.off_keys[1])};
    uint32_t* places[2] = {reinterpret_cast<uint32_t*>(base + p.off_places[0]), reinterpret_cast<uint32_t*>(base + p.off_places[1])};
    uint32_t* list = reinterpret_cast<uint32_t*>(base + p.off_list);
    const uint32_t n = (uint32_t)p.count, V = (uint32_t)p.V;
    hipError_t e;
    int from = 0;
    if (n == 0) {
    } else if (p.tiles == 0) {
        sort_small_kernel<<<1, kSortThreads, 0, st>>>(tokens, it, n, V, p.passes, p.bits, keys[0], places[0], list);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
        uint32_t* counts = reinterpret_cast<uint32_t*>(base + p.off_counts);
        for (int i = 0; i < p.passes; ++i) {
            const uint32_t *keys_in = i ? keys[from] : nullptr, *places_in = i ? places[from] : nullptr;
            const int to = i ? 1 - from : 0, shift = i * p.bits;
            const auto count = p.rows == kFewRows ? sort_count_kernel<kFewRows> : sort_count_kernel<kManyRows>;
            count<<<(unsigned)p.tiles, kSortThreads, 0, st>>>(tokens, it, keys_in, n, V, shift, p.bits, counts, list);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (p.tiles > kAddTiles) {
                sort_scan_kernel<<<1, kSortThreads, 0, st>>>(counts, p.tiles << p.bits);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
            const auto move = p.rows == kFewRows ? sort_move_kernel<kFewRows> : sort_move_kernel<kManyRows>;
            move<<<(unsigned)p.tiles, kSortThreads, 0, st>>>(tokens, it, keys_in, places_in, n, V, shift, p.bits, counts, keys[to], places[to]);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            from = to;
        }
    }
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        using A = sum_t<T>;
        const Handed<A> handed{reinterpret_cast<A*>(base + p.off_carry), reinterpret_cast<A*>(base + p.off_head), list,
                               {reinterpret_cast<Listed*>(list + 64), reinterpret_cast<Listed*>(list + 64) + p.units}};
        const size_t lds = (size_t)(kThreads / p.lanes) * p.events * 4;
        auto sums = [&](auto factor) {
            using P = decltype(factor);
            embed_sums_kernel<T, P><<<dim3((unsigned)p.groups, p.slices), kThreads, lds, st>>>(
                static_cast<const T*>(grad_out), static_cast<T*>(grad_table), keys[from], places[from], p.count, p.V, p.D, p.lanes, p.events, factor,
                handed);
            const hipError_t err = hipGetLastError();
            if (err != hipSuccess || p.count == 0) return err;
            // (as many workgroups as run at once take the list in turns)
            const int64_t most = p.units * 2;
            embed_join_kernel<T, P><<<(unsigned)(most < 2048 ? most : 2048), 64 * kJoinWaves, 0, st>>>(static_cast<T*>(grad_table), keys[from], p.D, p.events,
                                                                                                    factor, handed);
            return hipGetLastError();
        };
        if constexpr (sizeof(T) == 2)
            if (float_scale(scale)) return sums((float)scale);
        return sums(scale);
    });
}

}  // namespace st
