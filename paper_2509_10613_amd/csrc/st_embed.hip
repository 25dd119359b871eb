// Tables of vectors: rows looked up by symbol and scaled, and the table's gradient.
//
// Forward: out[n, :] = scale * table[tokens[n], :].  Bound by memory: every lane moves one 16-byte vector of a row at a time, four
// of them in flight.
//
// Backward: row v of the gradient is the sum of the upstream rows whose symbol is v.  Adding rows with atomics would make results depend on
// the order of arrival and a frequent symbol's row a bottleneck, so the symbols are sorted first (stably, least significant digit
// first) together with their places.  What is left is V + count events in one order: "add upstream row n" for every symbol in
// sorted order, and "write row v" after the last symbol v.  Every unit (the lanes that share a row's columns) takes the same number of
// consecutive events, so that neither a frequent symbol nor a stretch of absent ones makes one unit work longer; where a unit
// begins in the sorted symbols is found by a search on the diagonal i + key[i].  A row whose events are spread over several
// units is finished by a second launch from what they hand over, in their order.
#include "st_dev.h"
#include "st_kernels.h"

namespace st {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------------------------------------ forward
// Index: uint32_t where the number of vectors allows (a 32-bit division per vector instead of a 64-bit one).
template <typename T, typename Index>
__global__ __launch_bounds__(kThreads) void embed_fwd_kernel(const void* tokens, int it, const T* table, T* out, int64_t count, int64_t V,
                                                             int64_t D, sum_t<T> scale, Index per_row, Index items)
{
    constexpr int E = kPer16<T>, U = 4;
    const Index stride = (Index)gridDim.x * kThreads;
    for (Index first = (Index)blockIdx.x * kThreads + threadIdx.x; first < items; first += stride * U) {
        Vec<T, E> v[U];
        int n[U];
        T* to[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Index item = first + u * stride;
            n[u] = 0;
            if (item >= items || item < first) continue;   // (the second: the sum passed the type's end)
            const Index row = item / per_row;
            const int64_t col = (int64_t)(item - row * per_row) * E;
            const int64_t symbol = load_index(tokens, (int64_t)row, it);
            n[u] = D - col < E ? (int)(D - col) : E;
            to[u] = out + (int64_t)row * D + col;
            const bool there = symbol >= 0 && symbol < V;
            const T* from = table + (there ? symbol : 0) * D + col;
            if (!there)
#pragma unroll
                for (int i = 0; i < E; ++i) v[u].v[i] = T(0);
            else if (n[u] == E) v[u] = load_vec<T, E>(from);
            else v[u] = load_some<T, E>(from, n[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n[u] == 0) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) v[u].v[i] = (T)((sum_t<T>)v[u].v[i] * scale);
            if (n[u] == E) store_vec(to[u], v[u]);
            else store_some(to[u], v[u], n[u]);
        }
    }
}

// ------------------------------------------------------------------------------------------------ sort
// A workgroup of 16 waves takes kTile symbols, 512 consecutive ones per wave, in 8 rows of 64.
constexpr int kSortThreads = 1024, kSortWaves = 16, kSortRows = 8, kTile = kSortThreads * kSortRows, kDigits = 512;

__device__ __forceinline__ uint32_t symbol_key(const void* tokens, int64_t i, int it, uint32_t V)
{
    const int64_t s = load_index(tokens, i, it);
    return s >= 0 && s < (int64_t)V ? (uint32_t)s : V;   // symbols outside the table go behind all others
}

// Ranks a wave's 512 symbols by their digit, in order: counts (of the wave, cleared before) ends up with the number of each digit.
__device__ __forceinline__ void rank_wave(const uint32_t (&key)[kSortRows], const bool (&live)[kSortRows], int shift, int bits,
                                          volatile uint32_t* counts, uint32_t (&rank)[kSortRows])
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int r = 0; r < kSortRows; ++r) {
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
        for (int w = 0; w < kSortWaves; ++w) mine += counts[w * kDigits + digit];
    uint32_t all;
    const uint32_t local = scan_block(mine, scratch, &all);
    if (digit < (1 << bits)) {
        uint32_t at = begin(digit, local);
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = counts[w * kDigits + digit];
            counts[w * kDigits + digit] = at;
            at += c;
        }
    }
    __syncthreads();
}

// Up to kTile symbols: all digits in one launch, symbols and places in registers and LDS.
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(const void* tokens, int it, uint32_t n, uint32_t V, int passes, int bits,
                                                                  uint32_t* keys, uint32_t* places)
{
    __shared__ uint32_t counts[kSortWaves * kDigits];
    __shared__ uint32_t key_at[kTile], place_at[kTile];
    __shared__ uint32_t scratch[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[kSortRows], place[kSortRows], rank[kSortRows];
    bool live[kSortRows];
#pragma unroll
    for (int r = 0; r < kSortRows; ++r) {
        const uint32_t i = w * (64 * kSortRows) + r * 64 + lane;
        live[r] = i < n;
        place[r] = i;
        key[r] = live[r] ? symbol_key(tokens, i, it, V) : 0;
    }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) counts[i] = 0;
        __syncthreads();
        rank_wave(key, live, shift, bits, counts + w * kDigits, rank);
        __syncthreads();
        wave_offsets(counts, scratch, bits, [](int, uint32_t local) { return local; });
#pragma unroll
        for (int r = 0; r < kSortRows; ++r)
            if (live[r]) {
                const uint32_t to = counts[w * kDigits + (key[r] >> shift & ((1u << bits) - 1))] + rank[r];
                key_at[to] = key[r];
                place_at[to] = place[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSortRows; ++r) {
            const uint32_t i = w * (64 * kSortRows) + r * 64 + lane;
            if (live[r]) {
                key[r] = key_at[i];
                place[r] = place_at[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kSortRows; ++r) {
        const uint32_t i = w * (64 * kSortRows) + r * 64 + lane;
        if (live[r]) {
            keys[i] = key[r];
            places[i] = place[r];
        }
    }
}

// One digit of many symbols, three launches: the digits' numbers in every tile, their running sums (by digit, then by tile),
// and the symbols to where they go.  keys_in null: the first digit, from the caller's symbols.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const void* tokens, int it, const uint32_t* keys_in, uint32_t n, uint32_t V,
                                                                  int shift, int bits, uint32_t* counts)
{
    __shared__ uint32_t bin[kDigits];
    for (int i = threadIdx.x; i < kDigits; i += kSortThreads) bin[i] = 0;
    __syncthreads();
    const uint64_t base = (uint64_t)blockIdx.x * kTile;
#pragma unroll
    for (int r = 0; r < kSortRows; ++r) {
        const uint64_t i = base + r * kSortThreads + threadIdx.x;
        if (i < n) {
            const uint32_t key = keys_in ? keys_in[i] : symbol_key(tokens, (int64_t)i, it, V);
            atomicAdd(&bin[key >> shift & ((1u << bits) - 1)], 1u);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (1 << bits); i += kSortThreads) counts[(size_t)i * gridDim.x + blockIdx.x] = bin[i];
}

__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(uint32_t* counts, int64_t entries)
{
    __shared__ uint32_t scratch[kSortWaves];
    uint32_t before = 0;
    for (int64_t first = 0; first < entries; first += kSortThreads * 4) {
        const int64_t i = first + threadIdx.x * 4;
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c[j] = i + j < entries ? counts[i + j] : 0;
            sum += c[j];
        }
        uint32_t all;
        uint32_t at = before + scan_block(sum, scratch, &all);
        before += all;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i + j < entries) counts[i + j] = at;
            at += c[j];
        }
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(const void* tokens, int it, const uint32_t* keys_in, const uint32_t* places_in,
                                                                 uint32_t n, uint32_t V, int shift, int bits, const uint32_t* begin,
                                                                 uint32_t* keys, uint32_t* places)
{
    __shared__ uint32_t counts[kSortWaves * kDigits];
    __shared__ uint32_t scratch[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[kSortRows], place[kSortRows], rank[kSortRows];
    bool live[kSortRows];
    for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) counts[i] = 0;
#pragma unroll
    for (int r = 0; r < kSortRows; ++r) {
        const uint64_t i = (uint64_t)blockIdx.x * kTile + w * (64 * kSortRows) + r * 64 + lane;
        live[r] = i < n;
        key[r] = !live[r] ? 0 : keys_in ? keys_in[i] : symbol_key(tokens, (int64_t)i, it, V);
        place[r] = !live[r] ? 0 : keys_in ? places_in[i] : (uint32_t)i;
    }
    __syncthreads();
    rank_wave(key, live, shift, bits, counts + w * kDigits, rank);
    __syncthreads();
    wave_offsets(counts, scratch, bits, [&](int digit, uint32_t) { return begin[(size_t)digit * gridDim.x + blockIdx.x]; });
#pragma unroll
    for (int r = 0; r < kSortRows; ++r)
        if (live[r]) {
            const uint32_t to = counts[w * kDigits + (key[r] >> shift & ((1u << bits) - 1))] + rank[r];
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

// What a unit hands over (rows: -1 for nothing): the sum of the row it has not finished, and the last part of the row it finished but
// did not begin.
template <typename A>
struct Handed {
    A *carry, *head;                 // [units][D]
    int64_t *carry_row, *head_row;   // [units]
};

template <typename T>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(const T* grad, T* out, const uint32_t* keys, const uint32_t* places, int64_t n,
                                                              int64_t V, int64_t D, int lanes, int events, sum_t<T> scale,
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
            } else if (width > 0) {
                Vec<T, E> r;
#pragma unroll
                for (int i = 0; i < E; ++i) r.v[i] = (T)(sum[i] * scale);
                if (width == E) store_vec(out + row * D + col, r);
                else store_some(out + row * D + col, r, width);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) sum[i] = 0;
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
    if (lane == 0 && blockIdx.y == 0) {
        handed.carry_row[at] = carries ? row : -1;
        handed.head_row[at] = begun && wrote ? first_row : -1;
    }
}

// Rows that more than one unit added to: the units' sums in their order.
template <typename T>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(T* out, int64_t D, sum_t<T> scale, Handed<sum_t<T>> handed)
{
    using A = sum_t<T>;
    const int64_t u = blockIdx.x, row = handed.head_row[u];
    if (row < 0) return;
    const int lane = threadIdx.x & 63;
    int64_t first = u;   // the first unit that carries this row
    for (;;) {
        const int64_t at = first - 1 - lane;
        const uint64_t other = __ballot(at < 0 || handed.carry_row[at < 0 ? 0 : at] != row);
        if (other) {
            first -= __ffsll((unsigned long long)other) - 1;
            break;
        }
        first -= 64;
    }
    for (int64_t c = (int64_t)blockIdx.y * kThreads + threadIdx.x; c < D; c += (int64_t)gridDim.y * kThreads) {
        A sum = 0;
        int64_t i = first;
        for (; i + 8 <= u; i += 8) {
            A part[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = handed.carry[(i + j) * D + c];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += part[j];
        }
        for (; i < u; ++i) sum += handed.carry[i * D + c];
        out[row * D + c] = (T)((sum + handed.head[u * D + c]) * scale);
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

}  // namespace

hipError_t embed_fwd(const void* tokens, const void* table, void* out, int64_t count, int64_t V, int64_t D, double scale, int it, int dt,
                     hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        const int64_t per_row = (D + kPer16<T> - 1) / kPer16<T>, items = count * per_row;
        int64_t blocks = (items + kThreads * 4 - 1) / (kThreads * 4);
        // few vectors: one per lane, on as many compute units as there are
        if (blocks < 1024) blocks = (items + kThreads - 1) / kThreads < 1024 ? (items + kThreads - 1) / kThreads : 1024;
        if (blocks > 65536) blocks = 65536;
        const T* from = static_cast<const T*>(table);
        T* to = static_cast<T*>(out);
        if (items < (int64_t)1 << 31)
            embed_fwd_kernel<T, uint32_t><<<(unsigned)blocks, kThreads, 0, st>>>(tokens, it, from, to, count, V, D, (sum_t<T>)scale,
                                                                                   (uint32_t)per_row, (uint32_t)items);
        else
            embed_fwd_kernel<T, uint64_t><<<(unsigned)blocks, kThreads, 0, st>>>(tokens, it, from, to, count, V, D, (sum_t<T>)scale,
                                                                                   (uint64_t)per_row, (uint64_t)items);
        return hipGetLastError();
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
    p.events = 32;
    p.units = (count + V + p.events - 1) / p.events;
    const int per_group = kThreads / p.lanes;
    p.groups = (p.units + per_group - 1) / per_group;
    int bits = 1;
    while (bits < 32 && ((uint64_t)V >> bits) != 0) ++bits;   // the largest key is V
    p.passes = (bits + 8) / 9;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = count <= kTile ? 0 : (count + kTile - 1) / kTile;
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
    p.off_rows = take((size_t)slots * 16);
    p.total = at;
    return p;
}

hipError_t embed_bwd(const EmbedPlan& p, const void* tokens, const void* grad_out, void* grad_table, double scale, int it, int dt, void* ws,
                     hipStream_t st)
{
    unsigned char* base = static_cast<unsigned char*>(ws);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + p.off_keys[0]), reinterpret_cast<uint32_t*>(base + p.off_keys[1])};
    uint32_t* places[2] = {reinterpret_cast<uint32_t*>(base + p.off_places[0]), reinterpret_cast<uint32_t*>(base + p.off_places[1])};
    const uint32_t n = (uint32_t)p.count, V = (uint32_t)p.V;
    hipError_t e;
    int from = 0;
    if (n == 0) {
    } else if (p.tiles == 0) {
        sort_small_kernel<<<1, kSortThreads, 0, st>>>(tokens, it, n, V, p.passes, p.bits, keys[0], places[0]);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else {
        uint32_t* counts = reinterpret_cast<uint32_t*>(base + p.off_counts);
        for (int i = 0; i < p.passes; ++i) {
            const uint32_t *keys_in = i ? keys[from] : nullptr, *places_in = i ? places[from] : nullptr;
            const int to = i ? 1 - from : 0, shift = i * p.bits;
            sort_count_kernel<<<(unsigned)p.tiles, kSortThreads, 0, st>>>(tokens, it, keys_in, n, V, shift, p.bits, counts);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            sort_scan_kernel<<<1, kSortThreads, 0, st>>>(counts, p.tiles << p.bits);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            sort_move_kernel<<<(unsigned)p.tiles, kSortThreads, 0, st>>>(tokens, it, keys_in, places_in, n, V, shift, p.bits, counts, keys[to],
                                                                         places[to]);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            from = to;
        }
    }
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        using A = sum_t<T>;
        const int64_t slots = p.groups * (kThreads / p.lanes);
        int64_t* rows = reinterpret_cast<int64_t*>(base + p.off_rows);
        const Handed<A> handed{reinterpret_cast<A*>(base + p.off_carry), reinterpret_cast<A*>(base + p.off_head), rows, rows + slots};
        const size_t lds = (size_t)(kThreads / p.lanes) * p.events * 4;
        embed_sums_kernel<T><<<dim3((unsigned)p.groups, p.slices), kThreads, lds, st>>>(
            static_cast<const T*>(grad_out), static_cast<T*>(grad_table), keys[from], places[from], p.count, p.V, p.D, p.lanes, p.events,
            (A)scale, handed);
        hipError_t err = hipGetLastError();
        if (err != hipSuccess || p.count == 0) return err;
        const int64_t slices = (p.D + kThreads - 1) / kThreads;
        embed_join_kernel<T><<<dim3((unsigned)p.units, (unsigned)(slices < 16 ? slices : 16)), kThreads, 0, st>>>(static_cast<T*>(grad_table), p.D,
                                                                                                                (A)scale, handed);
        return hipGetLastError();
    });
}

}  // namespace st
