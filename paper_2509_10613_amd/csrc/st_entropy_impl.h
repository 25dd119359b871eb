// Softmax cross entropy of a linear read-out, and its gradients, in pieces of the classes.
//
// Forward: the logits z = h w^T are formed tile by tile on the matrix cores and reduced in registers to every row's maximum and sum
// of exponentials over the tile (and the target's logit); no logit is written.  Backward: the logits of a piece of the classes are formed
// again, their gradients G = u (exp(z - lse) - [class = target]) rounded to the arrays' type and written (what of u stays out of them:
// upstream_kernel), and multiplied: grad_h += G w and grad_w = G^T h.  The floor is the products: 2 T V D operations for the loss, 4 T V D for the gradients and, since the logits are not kept, 2 T V D
// once more.  8192 rows, 4096 channels, 131072 classes in bfloat16: 27.7 ms in all, forward 6.8 (1300 TFLOP/s), logits and their gradients 7.7,
// grad_h 6.6, grad_w 6.7 (1320); a large library product reaches 1150 to 1440 on this card.
//
// All products are of one form, C[m, n] = sum_k A[m, k] B[n, k] with rows of A and B in whole steps of 128 bytes, so one main loop serves
// every type: a lane holds 16 consecutive bytes of a row, which are one matrix instruction's operand for 16-bit types and four or two
// instructions' for float and double (the order of k does not matter as long as both sides have the same).  The side whose index the
// result's rows run along is B: a lane then holds results that lie side by side in a row.  Where k runs along the columns of a matrix (grad_h: w;
// grad_w: G and h) 16-bit operands are turned by the reads of LDS, others come from turned copies.
#pragma once
#include <algorithm>
#include <climits>
#include <utility>

#include "st_dev.h"
#include "st_kernels.h"

namespace st {
namespace {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using f64x4 = __attribute__((ext_vector_type(4))) double;
using bf16x8 = __attribute__((ext_vector_type(8))) bf16;
using f16x8 = __attribute__((ext_vector_type(8))) f16;

// c[j] += a b[j]^T; between(j) after the j-th: the other instructions that hide behind the matrix instructions.  Sums of float stay in the
// accumulation registers for as long as the products last: the instructions are written out, since the compiler, left to place 256 sums and the
// operands of two half steps, moves 140 to 250 registers between the two files for every 128 matrix instructions.  What the compiler would wait
// for, `settle` does; operands come from LDS, whose loads it waits for as for any instruction's.
template <typename T>
struct Types;
template <>
struct Types<bf16> {
    using Sum = float;
    using Frag = bf16x8;   // 16 bytes of a row
    using Acc = f32x4;     // a lane's part of a 16 x 16 tile
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    template <int N, class F>
    static __device__ __forceinline__ void products(Frag a, const Frag (&b)[N], Acc (&c)[N], F&& between)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c[j]) : "v"(a), "v"(b[j]));
            between(j);
        }
    }
};
template <>
struct Types<f16> {
    using Sum = float;
    using Frag = f16x8;
    using Acc = f32x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    template <int N, class F>
    static __device__ __forceinline__ void products(Frag a, const Frag (&b)[N], Acc (&c)[N], F&& between)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c[j]) : "v"(a), "v"(b[j]));
            between(j);
        }
    }
};
template <>
struct Types<float> {
    using Sum = float;
    using Frag = f32x4;
    using Acc = f32x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
        return c;
    }
    template <int N, class F>
    static __device__ __forceinline__ void products(Frag a, const Frag (&b)[N], Acc (&c)[N], F&& between)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k)   // (instructions on one sum lie apart)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c[j]) : "v"(a[k]), "v"(b[j][k]));
                if (k == 0) between(j);
            }
    }
};
template <>
struct Types<double> {
    using Sum = double;
    using Frag = __attribute__((ext_vector_type(2))) double;
    using Acc = f64x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) c = __builtin_amdgcn_mfma_f64_16x16x4f64(a[k], b[k], c, 0, 0, 0);
        return c;
    }
    template <int N, class F>
    static __device__ __forceinline__ void products(Frag a, const Frag (&b)[N], Acc (&c)[N], F&& between)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                c[j] = __builtin_amdgcn_mfma_f64_16x16x4f64(a[k], b[j][k], c[j], 0, 0, 0);
                if (k == 0) between(j);
            }
    }
};
// Between instructions that write sums and instructions of other kinds that read or wrote them: more than the 19 cycles the longest of these
// matrix instructions' results take.
template <int M, int N>
__device__ __forceinline__ void settle(f32x4 (&acc)[M][N])
{
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j == 0) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[i][j]));
            else asm volatile("" : "+a"(acc[i][j]));
}
template <int M, int N>
__device__ __forceinline__ void settle(f64x4 (&)[M][N])
{
}
// The row of a 16 x 16 result tile that a lane's r-th number belongs to (its column is lane % 16).
template <typename T>
__device__ __forceinline__ int acc_row(int lane, int r)
{
    return sizeof(T) == 8 ? (lane >> 4) + 4 * r : (lane >> 4) * 4 + r;
}

__device__ __forceinline__ double exp_of(double x, double) { return exp(x); }
__device__ __forceinline__ float exp_of(float x, float) { return expf(x); }
// of logits that are sums of products of 16-bit numbers: the instruction's error is far below theirs
__device__ __forceinline__ float exp_of(float x, bf16) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float exp_of(float x, f16) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ double log_of(double x) { return log(x); }
__device__ __forceinline__ float log_of(float x) { return logf(x); }

template <typename S>
__device__ __forceinline__ S lowest()
{
    return -(S)__builtin_inf();
}
// What is subtracted for a maximum m: exp(x - base(m)) is 0 for every x = -inf also where m is the maximum of nothing else, and NaN for NaN.
template <typename S>
__device__ __forceinline__ S base(S m)
{
    return m == lowest<S>() ? (S)0 : m;
}
template <typename T, typename S>
__device__ __forceinline__ S exp_below(S x, S m)
{
    return exp_of(x - base(m), T{});
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }   // (not a NaN if one is a number)
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

// ------------------------------------------------------------------------------------------------ the products
constexpr int kThreads = 256;   // four waves, two by two

// f(std::integral_constant 0), ... f(N - 1)
template <class F, int... I>
__device__ __forceinline__ void unroll_(F& f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unroll(F&& f)
{
    unroll_(f, std::make_integer_sequence<int, N>{});
}
// what is the same in all lanes, in scalar registers
__device__ __forceinline__ const char* uniform(const char* p)
{
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const char*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

struct Operands {
    const char *a, *b;
    int64_t a_pitch, b_pitch;   // bytes between rows
    int64_t m, n;               // rows
    int64_t steps;              // of kStepBytes along k
    const char* a_tail = nullptr;   // A turned: the last step's rows, if not those behind the others
    const char* a_zero = nullptr;   // A not turned: where 16 zeros are, if its rows end within the last step
    int a_left = 0;                 // ... and how many bytes of that step they have, a multiple of 16
};
using i16x4 = __attribute__((ext_vector_type(4))) short;
using as3_i16x4 = __attribute__((address_space(3))) i16x4;

// A wave's tile is SUB x SUB tiles of 16 x 16 (2, 4 or, of 16-bit types, 8), a workgroup's twice that on either side.  Large tiles read least from LDS
// per product: 128 x 128 per wave (256 x 256 per workgroup) take 1024 of the 2048 cycles a step's matrix instructions last, and 512 for the loads
// that arrive; that is 256 registers of sums, and one workgroup on a compute unit.  Instructions for floats and doubles last eight times as long:
// there two smaller workgroups, whose beginnings and ends hide behind each other's products, are faster (2048 rows, 1024 channels, 32768 classes
// of float, loss and gradients: tiles of 256 4.02 ms, of 128 3.91).
// TURN_A, TURN_B (16-bit types): the operand lies with k along its rows, [k][m], and is turned on its way from LDS to the registers, by the reads that
// hand each of 16 lanes one column of four rows.  Its step is 64 rows of the tile's columns; 32-byte pieces of a row are exchanged by the row's
// number, so that the 16 rows that one read takes from lie in different banks.
template <typename T, int SUB, bool TURN_A = false, bool TURN_B = false>
struct Product {
    using Frag = typename Types<T>::Frag;
    using Acc = typename Types<T>::Acc;
    static constexpr int kWave = SUB * 16, kTile = 2 * kWave;
    static constexpr int kSide = kTile * kStepBytes;           // bytes of one operand's step in LDS
    static constexpr size_t kLds = 4 * kSide;                  // two steps of two operands
    static constexpr int kLoads = kSide / (16 * kThreads);     // 16-byte loads per thread, side and step
    static_assert(kLoads >= 1 && (sizeof(T) == 2 || (SUB <= 4 && !TURN_A && !TURN_B)));
    static constexpr int kRow = kTile * 2, kSlots = kTile / 8;   // a turned row's bytes and 16-byte chunks
    // what a turned row's pieces are exchanged by: different for eight of rows 8 q .. 8 q + 3 (of two q), beyond what their place in the banks is
    static __device__ __forceinline__ int mixed(int k)
    {
        return kTile == 64 ? (k >> 1 & 1) | (k >> 3 & 1) << 1 : (k & 3) | (k >> 3 & 1) << 2;
    }

    Acc acc[SUB][SUB];
    int lane, wm, wn;

    // 64 lanes' 16 bytes (at base + offset) to LDS address to + PAST and behind it, past the registers.  Not counted by the compiler, which would
    // wait for all of them before any read of LDS: the waits below are the kernel's own.
    template <int PAST>
    static __device__ __forceinline__ void load(const char* base, uint32_t offset, uint32_t to)
    {
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3"
                     :
                     : "s"(to), "n"(PAST), "v"(offset), "s"(base)
                     : "memory", "scc", "m0");
    }

    // ... at an address of each lane's own
    template <int PAST>
    static __device__ __forceinline__ void load_at(const char* from, uint32_t to)
    {
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off" : : "s"(to), "n"(PAST), "v"(from) : "memory", "scc", "m0");
    }

    // (the instruction alone does not keep the compiler from moving reads of LDS over it)
    static __device__ __forceinline__ void barrier()
    {
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    // The tile with rows m0.. of A and n0.. of B.  A step's operands lie in LDS as rows of 128 bytes, the 16-byte chunks of a row exchanged by
    // its number modulo 8, so that eight rows' chunks of one column lie in different banks.  Two steps are under way: a wave reads the second half
    // of step s, multiplies the first half, and after the one barrier of a step (everybody has read step s, step s + 1 has arrived) sends for
    // step s + 2, reads the first half of step s + 1 and multiplies the second half of step s.
    __device__ __forceinline__ void run(const Operands& o, int64_t m0, int64_t n0, char* lds)
    {
        lane = threadIdx.x & 63;
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = w >> 1;
        wn = w & 1;
#pragma unroll
        for (int i = 0; i < SUB; ++i)
#pragma unroll
            for (int j = 0; j < SUB; ++j) acc[i][j] = {0, 0, 0, 0};
        // (32 bits: rows of at most 4 000 000 entries, 256 or, of double, 128 of them)
        uint32_t from_a[kLoads], from_b[kLoads];
        const char *pa = uniform(TURN_A ? o.a : o.a + m0 * o.a_pitch), *pb = uniform(TURN_B ? o.b : o.b + n0 * o.b_pitch);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            // (rows, or columns, behind the last are read from the last: their results are dropped)
            const int row = (i * 4 + w) * 8 + (lane >> 3), c = ((lane & 7) ^ (row & 7)) * 16;
            const int slot = (i * 4 + w) * 64 + lane, k = slot / kSlots, at = slot % kSlots, col = ((at >> 1) ^ mixed(k)) * 32 + (at & 1) * 16;
            if constexpr (TURN_A) from_a[i] = (uint32_t)(k * o.a_pitch + (m0 * 2 + col < o.a_pitch ? m0 * 2 + col : o.a_pitch - 16));
            else from_a[i] = (uint32_t)((m0 + row < o.m ? row : o.m - 1 - m0) * o.a_pitch) + c;
            if constexpr (TURN_B) from_b[i] = (uint32_t)(k * o.b_pitch + (n0 * 2 + col < o.b_pitch ? n0 * 2 + col : o.b_pitch - 16));
            else from_b[i] = (uint32_t)((n0 + row < o.n ? row : o.n - 1 - n0) * o.b_pitch) + c;
        }
        const int64_t step_a = TURN_A ? 64 * o.a_pitch : kStepBytes, step_b = TURN_B ? 64 * o.b_pitch : kStepBytes;
        int64_t to_send = o.steps;
        if (TURN_A && to_send == 1 && o.a_tail) pa = uniform(o.a_tail);
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + w * 1024;
        // the i-th of a step's loads, A's and B's in turn
        auto send = [&](int half, auto i) {
            constexpr int k = decltype(i)::value / 2;
            if constexpr (decltype(i)::value % 2 == 0) load<k * 4096>(pa, from_a[k], base + half * 2 * kSide);
            else load<kSide + k * 4096>(pb, from_b[k], base + half * 2 * kSide);
        };
        // ... of the last step where A's rows end within it: zeros behind them (what lies there may be infinite, or nobody's)
        const bool ends = ((lane & 7) ^ (lane >> 3)) * 16 >= o.a_left;
        auto send_end = [&](int half, auto i) {
            constexpr int k = decltype(i)::value / 2;
            if constexpr (decltype(i)::value % 2 == 0) load_at<k * 4096>(ends ? o.a_zero : pa + from_a[k], base + half * 2 * kSide);
            else send(half, i);
        };
        auto sent = [&] {   // a whole step
            pa += step_a;
            pb += step_b;
            if (TURN_A && --to_send == 1 && o.a_tail) pa = uniform(o.a_tail);
        };
        settle(acc);
        Frag fa[2][SUB], fb[2][SUB];
        const int at = (lane & 15) * kStepBytes + (((lane >> 4) ^ (lane & 7)) << 4);
        const char *la = lds + wm * kWave * kStepBytes + at, *lb = lds + kSide + wn * kWave * kStepBytes + at;
        // a turned operand's: lane 16 q + c asks for row 8 q + c / 4 and the four rows behind, columns 4 (c % 4) .., and gets column c of them
        const int k0 = (lane >> 4) * 8 + (lane >> 2 & 3), turned = k0 * kRow + (lane & 3) * 8, mix = mixed(k0) << 5;
        auto turn_read = [&](int side, int which, int kk, int half) {
            const as3_i16x4* from = (const as3_i16x4*)(lds + half * 2 * kSide + side + kk * 32 * kRow + turned + ((which << 5) ^ mix));
            union {
                i16x4 part[2];
                Frag all;
            } f;
            f.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((as3_i16x4*)from);
            f.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((as3_i16x4*)from + kRow / 2);   // (four rows further on)
            return f.all;
        };
        // the i-th of a half step's operands, B's and A's in turn (the second half's chunks are four further on: bit 6 of the address, exchanged
        // or not)
        auto read = [&](int half, int kk, int i) {
            const int to = half * 2 * kSide + i / 2 * 16 * kStepBytes;
            if (i % 2 == 0) {
                if constexpr (TURN_B) fb[kk][i / 2] = turn_read(kSide, wn * SUB + i / 2, kk, half);
                else fb[kk][i / 2] = *reinterpret_cast<const Frag*>(kk ? lds + ((uintptr_t)(lb - lds) ^ 64) + to : lb + to);
            } else {
                if constexpr (TURN_A) fa[kk][i / 2] = turn_read(0, wm * SUB + i / 2, kk, half);
                else fa[kk][i / 2] = *reinterpret_cast<const Frag*>(kk ? lds + ((uintptr_t)(la - lds) ^ 64) + to : la + to);
            }
        };
        // Step s in one half of the LDS, s + 1 in the other; more: 1 if there is a step s + 2, 2 if that is one where A's rows end.  One wave per SIMD has to hide every other instruction
        // behind its matrix instructions: one read of LDS or one load after each of them, as written.
        auto step = [&](int half, auto next, auto more) {
            constexpr bool kNext = decltype(next)::value;
            constexpr int kMore = decltype(more)::value;
            constexpr int kAll = SUB * SUB, kEvery = SUB == 8 ? 2 : 1;
            unroll<SUB>([&](auto i) {
                Types<T>::products(fa[0][i], fb[0], acc[i], [&](int j) {
                    const int at = i * SUB + j;
                    if (at % kEvery == 0 && at / kEvery < 2 * SUB) read(half, 1, at / kEvery);
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            if constexpr (kNext) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
                barrier();
            }
            unroll<SUB>([&](auto i) {
                Types<T>::products(fa[1][i], fb[1], acc[i], [&](int j) {
                    const int at = i * SUB + j;
                    if (kNext && at % kEvery == 0 && at / kEvery < 2 * SUB) read(half ^ 1, 0, at / kEvery);
                    if constexpr (kMore != 0)
                        unroll<2 * kLoads>([&](auto l) {
                            if (at != l * kEvery + kEvery - 1) return;
                            if constexpr (kMore == 2) send_end(half, l);
                            else send(half, l);
                        });
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            static_assert(2 * SUB * kEvery <= kAll && 2 * kLoads * kEvery <= kAll);
            if constexpr (kMore != 0) sent();
        };
        using Yes = std::true_type;
        const bool end = !TURN_A && o.a_zero != nullptr;
        auto send_first = [&](int half) {   // the first step, or the second
            if (end && o.steps == half + 1) {
                if constexpr (!TURN_A) unroll<2 * kLoads>([&](auto i) { send_end(half, i); });
            } else {
                unroll<2 * kLoads>([&](auto i) { send(half, i); });
            }
            sent();
        };
        send_first(0);
        if (o.steps > 1) {
            send_first(1);
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * kLoads) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        }
        barrier();
#pragma unroll
        for (int i = 0; i < 2 * SUB; ++i) read(0, 0, i);
        int half = 0;
        const int64_t whole = o.steps - (end ? 1 : 0);
        for (int64_t s = 2; s < whole; ++s) {
            step(half, Yes{}, std::integral_constant<int, 1>{});
            half ^= 1;
        }
        if constexpr (!TURN_A)
            if (end && o.steps > 2) {
                step(half, Yes{}, std::integral_constant<int, 2>{});
                half ^= 1;
            }
        if (o.steps > 1) {
            step(half, Yes{}, std::integral_constant<int, 0>{});
            half ^= 1;
        }
        step(half, std::false_type{}, std::integral_constant<int, 0>{});
        settle(acc);
        __syncthreads();   // (what follows may use the LDS)
    }
};
// Which tile a workgroup takes.  Workgroups go to the eight dies in turn, and a die's 32 compute units share a cache: a die's
// workgroups get tiles that are neighbours, eight by four.
struct TileOrder {
    uint32_t tiles_m, tiles_n;   // (fewer than 2^31 workgroups: a grid's limit)
    uint32_t parts;              // workgroups per tile, which lie one behind the other
};
__device__ __forceinline__ int tile_of(const TileOrder& t, int64_t& m, int64_t& n)
{
    constexpr uint32_t kDies = 8, kAcross = 4;
    const uint32_t all = t.tiles_m * t.tiles_n * t.parts, die = blockIdx.x % kDies, each = all / kDies, more = all % kDies;
    const uint32_t place = die * each + (die < more ? die : more) + blockIdx.x / kDies, at = place / t.parts;
    const uint32_t group = at / (t.tiles_m * kAcross), left = at - group * t.tiles_m * kAcross;
    const uint32_t across = t.tiles_n - group * kAcross < kAcross ? t.tiles_n - group * kAcross : kAcross;
    m = __builtin_amdgcn_readfirstlane(left / across);
    n = __builtin_amdgcn_readfirstlane(group * kAcross + left % across);
    return __builtin_amdgcn_readfirstlane(place - at * t.parts);
}

// Results of 16 bits leave through LDS, as whole rows of the tile: straight from the registers a store takes 32 bytes each of 16 rows, and the
// logits' gradients took 1.04 ms instead of 1.00 for 8192 rows and 16384 classes.  The tile's rows lie in LDS one behind the other, their 16-byte chunks
// exchanged by the row's number, so that neither direction meets one bank twice.
template <typename T, int TILE>
struct Outbox {
    static_assert(sizeof(T) == 2);
    static constexpr int kChunks = TILE / 8;
    char* lds;
    // four entries from column `col` (a multiple of four) on
    __device__ __forceinline__ void put(int row, int col, const Vec<T, 4>& v) const
    {
        __builtin_memcpy(__builtin_assume_aligned(lds + row * (TILE * 2) + (((col >> 3) ^ (row & (kChunks - 1))) << 4) + (col & 4) * 2, 8), &v, 8);
    }
    // the whole tile, between two barriers; `cols` columns are left in the rows of `out`
    __device__ __forceinline__ void send(T* out, int64_t pitch, int64_t rows, int64_t cols) const
    {
        __syncthreads();
        const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
        constexpr int kRows = 64 / kChunks;   // per wave and store
#pragma unroll 4
        for (int i = 0; i < TILE / (4 * kRows); ++i) {
            const int row = (i * 4 + w) * kRows + lane / kChunks, chunk = lane % kChunks;
            Vec<T, 8> v;
            __builtin_memcpy(&v, __builtin_assume_aligned(lds + row * (TILE * 2) + ((chunk ^ (row & (kChunks - 1))) << 4), 16), 16);
            if (row >= rows) continue;
            T* to = out + row * pitch + chunk * 8;
            const int64_t left = cols - chunk * 8;
            if (left >= 8) store_vec(to, v);
            else if (left > 0) store_some(to, v, (int)left);
        }
        __syncthreads();
    }
};

__device__ __forceinline__ float power(float x, int e) { return ldexpf(x, e); }   // x 2^e
__device__ __forceinline__ double power(double x, int e) { return ldexp(x, e); }

// What is upstream of the rows, as upstream_kernel divides it between the logits' gradients and the other sides of the products.  up: the part in the
// logits' gradients (0: the row is left out).  exps (null: all 0): grad_h's row is 2^exps[t] times its products and *unscale, and the
// row of h that grad_w is made from is 2^(exps[t] + shift) h[t].  largest: of that row's entries' exponents, before the shift, which puts it at 2^15;
// w_unscale: what grad_w's products are multiplied by, written by the kernel that makes the copy of h.
template <typename S>
struct Upstream {
    S* up = nullptr;
    int* exps = nullptr;
    int* largest = nullptr;
    S *unscale = nullptr, *w_unscale = nullptr;

    __device__ __forceinline__ int shift() const
    {
        const int top = *largest;
        return top == INT_MIN ? 0 : 15 - top;   // (no entry counts: any does)
    }
    // (one thread of the launch that makes the copy)
    __device__ __forceinline__ void put_w_unscale() const { *w_unscale = power(*unscale, -shift()); }
    __device__ __forceinline__ int exponent(int64_t row) const { return exps ? exps[row] : 0; }
};
template <typename T, int E, typename S>
__device__ __forceinline__ void times_power(Vec<T, E>& v, S, int e)
{
#pragma unroll
    for (int i = 0; i < E; ++i) v.v[i] = (T)power((S)v.v[i], e);
}

// A result in the arrays' type; a 0 stays one whatever is upstream (rows without a target).
template <typename T, typename S>
__device__ __forceinline__ T scaled(S x, S f)
{
    return (T)(x == 0 ? x : x * f);
}
// ... f 2^e x
template <typename T, typename S>
__device__ __forceinline__ T scaled(S x, S f, int e)
{
    return (T)power(x == 0 ? x : x * f, e);
}
struct NoOutbox {
    char* lds;
};
template <typename T, int TILE>
using OutboxOf = typename std::conditional_t<sizeof(T) == 2, std::enable_if<true, Outbox<std::conditional_t<sizeof(T) == 2, T, bf16>, TILE>>,
                                             std::enable_if<true, NoOutbox>>::type;

// Forward: every row's maximum and sum of exponentials over the tile's classes (A: classes of w, B: rows of h).  (Of 16-bit types with the largest tile
// 24 registers are kept in scratch memory, 52 bytes a lane, besides 256 of each file; no other of these kernels does.)
template <typename T, int SUB>
__global__ __launch_bounds__(kThreads, SUB == 8 ? 1 : 2) void stats_kernel(Operands o, TileOrder order, const void* targets, int it, int64_t first_class, int64_t V,
                                                         typename Types<T>::Sum* part_max, typename Types<T>::Sum* part_sum,
                                                         typename Types<T>::Sum* hit)
{
    using S = typename Types<T>::Sum;
    using P = Product<T, SUB>;
    constexpr int kTile = P::kTile, kWave = P::kWave;
    extern __shared__ __align__(16) char lds[];
    int64_t tile_m, tile_n;
    tile_of(order, tile_m, tile_n);
    const int64_t m0 = tile_m * kTile, n0 = tile_n * kTile;
    P p;
    p.run(o, m0, n0, lds);
    auto& acc = p.acc;
    const int lane = p.lane, wm = p.wm, wn = p.wn;
    S* waves = reinterpret_cast<S*>(lds);   // [2 halves of the classes][2: maximum, sum][kTile]
    if (m0 + kTile > o.m)   // classes behind the last
#pragma unroll
        for (int i = 0; i < SUB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (m0 + wm * kWave + i * 16 + acc_row<T>(lane, r) >= o.m)
#pragma unroll
                    for (int j = 0; j < SUB; ++j) acc[i][j][r] = lowest<S>();
#pragma unroll
    for (int j = 0; j < SUB; ++j) {
        const int64_t row = n0 + wn * kWave + j * 16 + (lane & 15);
        const int64_t target = row < o.n ? load_index(targets, row, it) : -1;
        const int64_t wanted64 = target >= 0 && target < V ? target - first_class - m0 - wm * kWave : -1;
        const int wanted = wanted64 >= 0 && wanted64 < kWave ? (int)wanted64 : -1;   // of this wave's classes
        if (__any(wanted >= 0)) {   // (of few tiles)
            S mine = 0;
#pragma unroll
            for (int i = 0; i < SUB; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) mine = i * 16 + acc_row<T>(lane, r) == wanted ? acc[i][j][r] : mine;
            // (of the four lanes that share the row, the one that holds the class)
            if (wanted >= 0 && (sizeof(T) == 8 ? wanted & 3 : wanted >> 2 & 3) == lane >> 4) hit[row] = mine;
        }
        // NaN passes by the maximum, and through the sum
        S top = lowest<S>();
#pragma unroll
        for (int i = 0; i < SUB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = larger(acc[i][j][r], top);
        top = larger(top, __shfl_xor(top, 16));
        top = larger(top, __shfl_xor(top, 32));
        const S from = base(top);
        S sum = 0;
#pragma unroll
        for (int i = 0; i < SUB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += exp_of(acc[i][j][r] - from, T{});
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) {
            waves[(wm * 2 + 0) * kTile + wn * kWave + j * 16 + lane] = top;
            waves[(wm * 2 + 1) * kTile + wn * kWave + j * 16 + lane] = sum;
        }
    }
    __syncthreads();
    static_assert(kTile <= kThreads);
    const int64_t row = n0 + threadIdx.x;
    if (threadIdx.x < kTile && row < o.n) {
        const S a = waves[threadIdx.x], b = waves[2 * kTile + threadIdx.x];
        const S top = larger(a, b);
        part_max[tile_m * o.n + row] = top;
        part_sum[tile_m * o.n + row] =
            waves[kTile + threadIdx.x] * exp_below<T>(a, top) + waves[3 * kTile + threadIdx.x] * exp_below<T>(b, top);
    }
}

// Forward with at most 16 rows: bound by reading w once.  Every wave takes 16 classes and all of their columns straight from memory in the matrix
// instruction's layout (no row of w is read twice, so LDS would be a detour), eight loads of 1 KiB under way; h comes from the caches.
template <typename T>
__global__ __launch_bounds__(kThreads) void few_stats_kernel(const T* w, const T* h, int64_t classes, int rows, int64_t D, const void* targets, int it,
                                                             int64_t first_class, int64_t V, typename Types<T>::Sum* part_max,
                                                             typename Types<T>::Sum* part_sum, typename Types<T>::Sum* hit)
{
    using S = typename Types<T>::Sum;
    using Frag = typename Types<T>::Frag;
    constexpr int E = kPer16<T>, U = 8;
    __shared__ S waves[4][2][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15;
    const int64_t m0 = (int64_t)blockIdx.x * 64 + wave * 16, cls = m0 + (lane & 15);
    const T* from_w = w + (cls < classes ? cls : classes - 1) * D + (lane >> 4) * E;
    const T* from_h = h + (int64_t)(row < rows ? row : rows - 1) * D + (lane >> 4) * E;
    typename Types<T>::Acc acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = {0, 0, 0, 0};
    auto frag = [](const T* p) {
        Frag f;
        __builtin_memcpy(&f, p, 16);
        return f;
    };
    int64_t k = 0;
    for (; k + U * 4 * E <= D; k += U * 4 * E) {
        Frag a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) a[u] = frag(from_w + k + u * 4 * E);
#pragma unroll
        for (int u = 0; u < U; ++u) b[u] = frag(from_h + k + u * 4 * E);
#pragma unroll
        for (int u = 0; u < U; ++u) acc[u % 4] = Types<T>::product(a[u], b[u], acc[u % 4]);
    }
    for (; k < D; k += 4 * E) {
        const int64_t left = D - k - (lane >> 4) * E;
        const int n = left >= E ? E : left > 0 ? (int)left : 0;
        const Vec<T, E> va = load_some<T, E>(from_w + k, n), vb = load_some<T, E>(from_h + k, n);
        Frag a, b;
        __builtin_memcpy(&a, &va, 16);
        __builtin_memcpy(&b, &vb, 16);
        acc[0] = Types<T>::product(a, b, acc[0]);
    }
    S z[4], top = lowest<S>();
    const int64_t target = row < rows ? load_index(targets, row, it) : -1;
    const int64_t wanted = target >= 0 && target < V ? target - first_class - m0 : -1;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        z[r] = (acc[0][r] + acc[1][r]) + (acc[2][r] + acc[3][r]);
        const int at = acc_row<T>(lane, r);
        if (m0 + at >= classes) z[r] = lowest<S>();
        else if (at == wanted) hit[row] = z[r];
        top = larger(z[r], top);
    }
    top = larger(top, __shfl_xor(top, 16));
    top = larger(top, __shfl_xor(top, 32));
    S sum = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += exp_below<T>(z[r], top);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) {
        waves[wave][0][lane] = top;
        waves[wave][1][lane] = sum;
    }
    __syncthreads();
    if (threadIdx.x >= rows) return;
    S all = lowest<S>(), total = 0;
    for (int i = 0; i < 4; ++i) all = larger(all, waves[i][0][threadIdx.x]);
    for (int i = 0; i < 4; ++i) total += waves[i][1][threadIdx.x] * exp_below<T>(waves[i][0][threadIdx.x], all);
    part_max[(int64_t)blockIdx.x * rows + threadIdx.x] = all;
    part_sum[(int64_t)blockIdx.x * rows + threadIdx.x] = total;
}

// Few tiles of many steps: the products are divided among workgroups, which leave the piece's logits as sums over `parts` of their steps,
// z[part][row][class].  From these, every row's maximum and sum of exponentials over 256 classes, as stats_kernel leaves them.
template <typename T>
__global__ __launch_bounds__(kThreads) void parts_stats_kernel(const typename Types<T>::Sum* z, int parts, int64_t classes, int64_t rows, const void* targets,
                                                               int it, int64_t first_class, int64_t V, typename Types<T>::Sum* part_max,
                                                               typename Types<T>::Sum* part_sum, typename Types<T>::Sum* hit)
{
    using S = typename Types<T>::Sum;
    __shared__ S tops[4], sums[4];
    const int64_t row = blockIdx.y, cls = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t target = load_index(targets, row, it);
    S x = lowest<S>();
    if (cls < classes) {
        x = 0;
        for (int k = 0; k < parts; ++k) x += z[(k * rows + row) * classes + cls];
        if (target >= 0 && target < V && target - first_class == cls) hit[row] = x;
    }
    S top = larger(x, lowest<S>());
#pragma unroll
    for (int o = 32; o > 0; o /= 2) top = larger(top, __shfl_xor(top, o));
    S sum = exp_below<T>(x, top);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) {
        tops[threadIdx.x >> 6] = top;
        sums[threadIdx.x >> 6] = sum;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 0; i < 4; ++i) top = larger(top, tops[i]);
    sum = 0;
    for (int i = 0; i < 4; ++i) sum += sums[i] * exp_below<T>(tops[i], top);
    part_max[blockIdx.x * rows + row] = top;
    part_sum[blockIdx.x * rows + row] = sum;
}

// ... and their gradients, as grads_kernel leaves them.  A workgroup takes 32 rows and 32 classes.
template <typename T>
__global__ __launch_bounds__(kThreads) void parts_grads_kernel(const typename Types<T>::Sum* z, int parts, int64_t classes, int64_t rows, const void* targets,
                                                               int it, int64_t first_class, const typename Types<T>::Sum* lse,
                                                               const typename Types<T>::Sum* up, T* g, int64_t g_pitch, T* gt, int64_t gt_pitch)
{
    using S = typename Types<T>::Sum;
    constexpr int N = 32;
    __shared__ T tile[N][N + 1];
    const int64_t c0 = (int64_t)blockIdx.x * N, r0 = (int64_t)blockIdx.y * N;
    for (int i = threadIdx.x; i < N * N; i += kThreads) {
        const int64_t row = r0 + i / N, cls = c0 + i % N;
        T v = T(0);
        if (row < rows && cls < classes) {
            const S u = up[row];
            S x = 0;
            for (int k = 0; k < parts; ++k) x += z[(k * rows + row) * classes + cls];
            const S p = exp_of(x - lse[row], T{}) - (load_index(targets, row, it) - first_class == cls ? (S)1 : (S)0);
            v = u != 0 ? (T)(u * p) : T(0);
        }
        tile[i / N][i % N] = v;
        if (row < (sizeof(T) == 2 ? gt_pitch : rows) && cls < g_pitch) g[row * g_pitch + cls] = v;
    }
    if constexpr (sizeof(T) == 2) return;
    __syncthreads();
    for (int i = threadIdx.x; i < N * N; i += kThreads) {
        const int64_t row = r0 + i % N, cls = c0 + i / N;
        if (cls < classes && row < gt_pitch) gt[cls * gt_pitch + row] = tile[i % N][i / N];
    }
}

// Backward: the gradients of the piece's logits, g[row][class] with zeros up to whole steps; of 16-bit types also zeros in the rows up to whole steps
// (`gt_pitch` of them), of others gt[class][row], the same turned.
template <typename T, int SUB>
__global__ __launch_bounds__(kThreads, SUB == 8 ? 1 : 2) void grads_kernel(Operands o, TileOrder order, const void* targets, int it, int64_t first_class,
                                                         const typename Types<T>::Sum* lse, const typename Types<T>::Sum* up, T* g,
                                                         int64_t g_pitch, T* gt, int64_t gt_pitch)
{
    using S = typename Types<T>::Sum;
    using P = Product<T, SUB>;
    constexpr int kTile = P::kTile, kWave = P::kWave;
    extern __shared__ __align__(16) char lds[];
    int64_t tile_m, tile_n;
    tile_of(order, tile_m, tile_n);
    const int64_t m0 = tile_m * kTile, n0 = tile_n * kTile;
    P p;
    p.run(o, m0, n0, lds);
    auto& acc = p.acc;
    const int lane = p.lane, wm = p.wm, wn = p.wn;
    const bool inside = m0 + kTile <= o.m;
    const OutboxOf<T, kTile> outbox{lds};
#pragma unroll
    for (int j = 0; j < SUB; ++j) {
        const int64_t row = n0 + wn * kWave + j * 16 + (lane & 15);
        const bool there = row < o.n;
        const int64_t target = there ? load_index(targets, row, it) : -1;
        const int64_t wanted64 = target - first_class - m0 - wm * kWave;
        const int wanted = wanted64 >= 0 && wanted64 < kWave ? (int)wanted64 : -1;
        const S u = there ? up[row] : (S)0, l = there ? lse[row] : (S)0;
        const bool some = u != 0, any = __any(wanted >= 0);
        T* g_at = g + row * g_pitch + m0 + wm * kWave + acc_row<T>(lane, 0);
        T* gt_at = gt + (m0 + wm * kWave + acc_row<T>(lane, 0)) * gt_pitch + row;
#pragma unroll
        for (int i = 0; i < SUB; ++i) {
            const int64_t cls = m0 + wm * kWave + i * 16;
            S x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = u * exp_of(acc[i][j][r] - l, T{});
            if (any)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = i * 16 + acc_row<T>(lane, r) == wanted ? u * (exp_of(acc[i][j][r] - l, T{}) - (S)1) : x[r];
            if (!inside)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = cls + acc_row<T>(lane, r) < o.m ? x[r] : (S)0;
            Vec<T, 4> v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v.v[r] = (T)(some ? x[r] : (S)0);   // rows without a target stay 0 whatever their logits are
            if constexpr (sizeof(T) == 2) {
                outbox.put(wn * kWave + j * 16 + (lane & 15), wm * kWave + i * 16 + acc_row<T>(lane, 0), v);
                continue;
            }
            // (g_pitch is a multiple of 16: the tile is in or out)
            if (there && cls < g_pitch)
#pragma unroll
                for (int r = 0; r < 4; ++r) g_at[i * 16 + acc_row<T>(0, r)] = v.v[r];
            if (row < gt_pitch)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (inside || cls + acc_row<T>(lane, r) < o.m) gt_at[(i * 16 + acc_row<T>(0, r)) * gt_pitch] = v.v[r];
        }
    }
    if constexpr (sizeof(T) == 2) {
        outbox.send(g + n0 * g_pitch + m0, g_pitch, gt_pitch - n0, g_pitch - m0);
    }
}

// out[n][m] (pitch D) = the products times *unscale and, of grad_h (`rows`), the rows' powers of two, rounded; 0 in the rows whose up[n] is 0: 0 times
// an infinity of the read-out is no gradient of a row that has no target; or, with SUMS, sum[part][n][m] = the products over the part's steps, added to
// what is there unless `first`.  parts: the steps are divided among this many workgroups per tile, one step each at least (the main loop multiplies one
// whatever it is told).  A call with fewer parts than the first adds to the first of the sums.
template <typename T, int SUB, bool SUMS, bool TURN_A, bool TURN_B>
__global__ __launch_bounds__(kThreads, SUB == 8 ? 1 : 2) void product_kernel(Operands o, TileOrder order, typename Types<T>::Sum* sum, T* out, int64_t D, bool first,
                                                              const typename Types<T>::Sum* unscale, Upstream<typename Types<T>::Sum> rows)
{
    using S = typename Types<T>::Sum;
    using P = Product<T, SUB, TURN_A, TURN_B>;
    constexpr int kTile = P::kTile, kWave = P::kWave;
    extern __shared__ __align__(16) char lds[];
    int64_t tile_m, tile_n;
    const int part = tile_of(order, tile_m, tile_n);
    const int64_t m0 = tile_m * kTile, n0 = tile_n * kTile;
    if constexpr (SUMS) {
        const int64_t from = o.steps * part / order.parts, to = o.steps * (part + 1) / order.parts;
        o.a += from * (TURN_A ? 64 * o.a_pitch : kStepBytes);
        o.b += from * (TURN_B ? 64 * o.b_pitch : kStepBytes);
        if (to < o.steps) o.a_tail = o.a_zero = nullptr;
        o.steps = to - from;
        sum += part * o.n * D;
    }
    P p;
    p.run(o, m0, n0, lds);
    auto& acc = p.acc;
    const int lane = p.lane, wm = p.wm, wn = p.wn;
    const S f = SUMS ? (S)1 : *unscale;
    const OutboxOf<T, kTile> outbox{lds};
#pragma unroll
    for (int j = 0; j < SUB; ++j) {
        const int64_t n = n0 + wn * kWave + j * 16 + (lane & 15);
        if (n >= o.n) continue;
        const bool none = !SUMS && rows.up && rows.up[n] == 0;
        const int e = SUMS ? 0 : rows.exponent(n);
#pragma unroll
        for (int i = 0; i < SUB; ++i) {
            const int col = wm * kWave + i * 16 + acc_row<T>(lane, 0);
            const int64_t m = m0 + col, at = n * D + m;
            constexpr int kApart = sizeof(T) == 8 ? 4 : 1;   // between the lane's four numbers
            Vec<S, 4> x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x.v[r] = acc[i][j][r];
            if constexpr (SUMS) {
                if (kApart == 1 && m + 3 < o.m) {
                    if (!first) {
                        const Vec<S, 4> before = load_vec<S, 4>(sum + at);
#pragma unroll
                        for (int r = 0; r < 4; ++r) x.v[r] += before.v[r];
                    }
                    store_vec(sum + at, x);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (m + r * kApart < o.m) sum[at + r * kApart] = first ? x.v[r] : sum[at + r * kApart] + x.v[r];
                }
            } else {
                Vec<T, 4> v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v.v[r] = scaled<T>(x.v[r], f);
                if (rows.exps)
#pragma unroll
                    for (int r = 0; r < 4; ++r) v.v[r] = scaled<T>(x.v[r], f, e);
                if (none) v = Vec<T, 4>{};
                if constexpr (sizeof(T) == 2) outbox.put(wn * kWave + j * 16 + (lane & 15), col, v);
                else if (kApart == 1 && m + 3 < o.m) store_vec(out + at, v);
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (m + r * kApart < o.m) out[at + r * kApart] = v.v[r];
            }
        }
    }
    if constexpr (sizeof(T) == 2 && !SUMS) outbox.send(out + n0 * D + m0, D, o.n - n0, o.m - m0);
}

// out = the parts' sums in their order, times *unscale and, of grad_h, the powers of two of its rows of D entries, rounded; 0 in the rows whose up is 0.
template <typename T>
__global__ __launch_bounds__(256) void finish_kernel(const typename Types<T>::Sum* sum, int parts, int64_t entries, const typename Types<T>::Sum* unscale,
                                                     T* out, int64_t D, Upstream<typename Types<T>::Sum> rows)
{
    using S = typename Types<T>::Sum;
    constexpr int E = 16 / sizeof(S);
    const S f = *unscale;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E; i < entries; i += (int64_t)gridDim.x * 256 * E) {
        const int n = entries - i < E ? (int)(entries - i) : E;
        Vec<S, E> x = n == E ? load_vec<S, E>(sum + i) : load_some<S, E>(sum + i, n);
#pragma unroll 8
        for (int k = 1; k < parts; ++k) {
            const S* from = sum + k * entries + i;
            const Vec<S, E> y = n == E ? load_vec<S, E>(from) : load_some<S, E>(from, n);
#pragma unroll
            for (int e = 0; e < E; ++e) x.v[e] += y.v[e];
        }
        Vec<T, E> v;
#pragma unroll
        for (int e = 0; e < E; ++e) v.v[e] = scaled<T>(x.v[e], f);
        if (rows.up) {
            int64_t row = (uint64_t)entries >> 32 ? i / D : (int64_t)((uint32_t)i / (uint32_t)D), left = D - (i - row * D);
            if (left >= E && !rows.exps) {   // one row, as most
                if (rows.up[row] == 0) v = Vec<T, E>{};
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (e < n) v.v[e] = rows.up[row] == 0 ? T(0) : scaled<T>(x.v[e], f, rows.exponent(row));
                    if (--left == 0) {
                        ++row;
                        left = D;
                    }
                }
            }
        }
        if (n == E) store_vec(out + i, v);
        else store_some(out + i, v, n);
    }
}

// ------------------------------------------------------------------------------------------------ few classes
// At most 16 classes and wide rows (features of signatures and a handful of labels): h is what is read, w fits in registers.  Tiles of 64 classes and
// copies of h in whole steps would move h six times in a training step; here it is read for the loss, read again for the logits' gradients and read once
// more while grad_h is written.
constexpr int kFewClasses = 16;

// z[part][row][16]: a wave takes 16 rows and a part of their columns, straight from memory.
template <typename T>
__global__ __launch_bounds__(kThreads) void narrow_logits_kernel(const T* h, const T* w, int64_t rows, int classes, int64_t D, int64_t columns,
                                                                 typename Types<T>::Sum* z)
{
    using Frag = typename Types<T>::Frag;
    constexpr int E = kPer16<T>, U = 8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = ((int64_t)blockIdx.x * 4 + wave) * 16, row = m0 + (lane & 15);
    if (m0 >= rows) return;
    const int64_t first = (int64_t)blockIdx.y * columns, end = first + columns < D ? first + columns : D;
    const T* from_h = h + (row < rows ? row : rows - 1) * D + (lane >> 4) * E;
    const T* from_w = w + (int64_t)((lane & 15) < classes ? lane & 15 : classes - 1) * D + (lane >> 4) * E;
    typename Types<T>::Acc acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = {0, 0, 0, 0};
    auto frag = [](const T* p) {
        Frag f;
        __builtin_memcpy(&f, p, 16);
        return f;
    };
    int64_t k = first;
    for (; k + U * 4 * E <= end; k += U * 4 * E) {
        Frag a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) a[u] = frag(from_h + k + u * 4 * E);
#pragma unroll
        for (int u = 0; u < U; ++u) b[u] = frag(from_w + k + u * 4 * E);
#pragma unroll
        for (int u = 0; u < U; ++u) acc[u % 4] = Types<T>::product(a[u], b[u], acc[u % 4]);
    }
    for (; k < end; k += 4 * E) {
        const int64_t left = end - k - (lane >> 4) * E;
        const int n = left >= E ? E : left > 0 ? (int)left : 0;
        const Vec<T, E> va = load_some<T, E>(from_h + k, n), vb = load_some<T, E>(from_w + k, n);
        Frag a, b;
        __builtin_memcpy(&a, &va, 16);
        __builtin_memcpy(&b, &vb, 16);
        acc[0] = Types<T>::product(a, b, acc[0]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t at = m0 + acc_row<T>(lane, r);
        if (at < rows) z[((int64_t)blockIdx.y * rows + at) * kFewClasses + (lane & 15)] = (acc[0][r] + acc[1][r]) + (acc[2][r] + acc[3][r]);
    }
}

// 16 lanes per row add the parts.  Forward (g null): lse and the row's loss; backward: the logits' gradients g[row][16], not rounded.
template <typename T>
__global__ __launch_bounds__(kThreads) void narrow_rows_kernel(const typename Types<T>::Sum* z, int parts, int64_t rows, int classes, const void* targets,
                                                               int it, typename Types<T>::Sum* lse, typename Types<T>::Sum* losses,
                                                               const typename Types<T>::Sum* up, typename Types<T>::Sum* g)
{
    using S = typename Types<T>::Sum;
    const int lane = threadIdx.x & 15;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const bool there = row < rows;
    const int64_t at = there ? row : rows - 1;
    S x = 0;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) x += z[((int64_t)k * rows + at) * kFewClasses + lane];
    const int64_t target = load_index(targets, at, it);
    if (g) {
        const S u = up[at], p = exp_of(x - lse[at], T{}) - (target == lane ? (S)1 : (S)0);
        if (there) g[row * kFewClasses + lane] = u != 0 && lane < classes ? u * p : (S)0;
        return;
    }
    if (lane >= classes) x = lowest<S>();
    S top = larger(x, lowest<S>());
#pragma unroll
    for (int o = 8; o > 0; o /= 2) top = larger(top, __shfl_xor(top, o));
    S sum = exp_below<T>(x, top);
#pragma unroll
    for (int o = 8; o > 0; o /= 2) sum += __shfl_xor(sum, o);
    const bool has = target >= 0 && target < classes;
    const S hit = __shfl(x, has ? (int)target : 0, 16), l = top + log_of(sum);
    if (there && lane == 0) {
        lse[row] = l;
        losses[row] = has ? l - hit : (S)0;
    }
}

// grad_h[row] = g[row] w, and dw[part] = the sum over the part's rows of g[row]^T h[row]: a lane keeps E columns of w, and of the sums, for all classes.
// Rows whose upstream is 0 are zeros and left out, whatever they and the read-out hold.  E: 16 bytes, 8 of 16-bit types (32 registers of w and as many of sums
// per two columns of double).  CLASSES: 4, 8 or 16, whichever holds them.
template <typename T>
constexpr int kNarrowCols = sizeof(T) == 8 ? 2 : 4;
template <typename T, int CLASSES>
__global__ __launch_bounds__(kThreads) void narrow_grads_kernel(const T* __restrict__ h, const T* __restrict__ w,
                                                                const typename Types<T>::Sum* __restrict__ g,
                                                                const typename Types<T>::Sum* __restrict__ up,
                                                                const typename Types<T>::Sum* __restrict__ scaling, int64_t rows, int64_t rows_each, int classes,
                                                                int64_t D, T* grad_h, typename Types<T>::Sum* dw)
{
    using S = typename Types<T>::Sum;
    constexpr int E = kNarrowCols<T>, U = 8;
    const int64_t col = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * E;
    if (col >= D) return;
    const int width = D - col < E ? (int)(D - col) : E;
    const S f = *scaling;
    S ws[CLASSES][E], sums[CLASSES][E];
#pragma unroll
    for (int v = 0; v < CLASSES; ++v) {
        const Vec<T, E> x = v >= classes ? load_some<T, E>(w, 0) : width == E ? load_vec<T, E>(w + v * D + col) : load_some<T, E>(w + v * D + col, width);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            ws[v][e] = (S)x.v[e];
            sums[v][e] = 0;
        }
    }
    const int64_t first = (int64_t)blockIdx.y * rows_each, end = first + rows_each < rows ? first + rows_each : rows;
    for (int64_t t = first; t < end; t += U) {
        Vec<T, E> x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const T* from = h + (t + i < end ? t + i : t) * D + col;
            if (dw) x[i] = width == E ? load_vec<T, E>(from) : load_some<T, E>(from, width);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (t + i >= end) break;
            const S* gr = g + (t + i) * kFewClasses;
            const bool some = up[t + i] != 0;
            S y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = 0;
            if (some)
#pragma unroll
                for (int v = 0; v < CLASSES; ++v) {
                    const S q = gr[v];
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        y[e] += q * ws[v][e];
                        if (dw) sums[v][e] += q * (S)x[i].v[e];
                    }
                }
            if (grad_h) {
                Vec<T, E> out;
#pragma unroll
                for (int e = 0; e < E; ++e) out.v[e] = scaled<T>(y[e], f);
                if (width == E) store_vec(grad_h + (t + i) * D + col, out);
                else store_some(grad_h + (t + i) * D + col, out, width);
            }
        }
    }
    if (!dw) return;
#pragma unroll
    for (int v = 0; v < CLASSES; ++v)
        if (v < classes)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < width) dw[((int64_t)blockIdx.y * classes + v) * D + col + e] = sums[v][e];
}

// ------------------------------------------------------------------------------------------------ copies
// dst[all][pitch] = src[rows][cols], zeros behind the columns and the rows.  With `u` rows whose up is 0 are zeros, whatever they hold, and others
// have their power of two.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* src, T* dst, int64_t rows, int64_t all, int64_t cols, int64_t pitch,
                                                   Upstream<typename Types<T>::Sum> u)
{
    using S = typename Types<T>::Sum;
    constexpr int E = kPer16<T>;
    if (u.exps && blockIdx.x == 0 && threadIdx.x == 0) u.put_w_unscale();
    const int shift = u.exps ? u.shift() : 0;
    const int64_t per_row = pitch / E, items = all * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row, col = (i - row * per_row) * E;
        int64_t left = row < rows ? cols - col : 0;
        if (u.up && row < rows && u.up[row] == 0) left = 0;
        const T* from = src + row * cols + col;
        Vec<T, E> v = left >= E ? load_vec<T, E>(from) : load_some<T, E>(from, (int)(left > 0 ? left : 0));
        if (u.exps && left > 0) times_power(v, S{}, u.exps[row] + shift);
        store_vec(dst + row * pitch + col, v);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = T(0);
}

// dst[cols][pitch] = src[rows][cols] transposed, zeros behind the rows.  `u`: as in pack_kernel.
// A workgroup turns 64 x 64 entries (32 x 64 of double), moved as 16 bytes either way.  All tiles are the grid's first index: there may be more than 65536
// along either side.
template <typename T>
constexpr int kTurnCols = sizeof(T) == 8 ? 32 : 64;
template <typename T>
__global__ __launch_bounds__(256) void transpose_kernel(const T* src, T* dst, int64_t rows, int64_t cols, int64_t pitch,
                                                        Upstream<typename Types<T>::Sum> u)
{
    using S = typename Types<T>::Sum;
    if (u.exps && blockIdx.x == 0 && threadIdx.x == 0) u.put_w_unscale();
    const int shift = u.exps ? u.shift() : 0;
    constexpr int R = 64, C = kTurnCols<T>, E = kPer16<T>, kPad = 4 / sizeof(T) ? 4 / sizeof(T) : 1;
    __shared__ T tile[C][R + kPad];   // (an odd number of words from column to column, or of double words)
    const uint32_t across = (uint32_t)((pitch + R - 1) / R), down = blockIdx.x / across;
    const int64_t r0 = (int64_t)(blockIdx.x - down * across) * R, c0 = (int64_t)down * C;
    for (int i = threadIdx.x; i < R * C / E; i += 256) {
        const int row = i / (C / E), col = i % (C / E) * E;
        const int64_t r = r0 + row, left = cols - c0 - col;
        const bool there = r < rows && left > 0 && !(u.up && u.up[r] == 0);
        Vec<T, E> v;
        const T* from = src + r * cols + c0 + col;
        if (there && left >= E) v = load_vec<T, E>(from);
        else v = load_some<T, E>(from, there ? (int)left : 0);
        if (u.exps && there) times_power(v, S{}, u.exps[r] + shift);
#pragma unroll
        for (int e = 0; e < E; ++e) tile[col + e][row] = v.v[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < R * C / E; i += 256) {
        const int col = i / (R / E), row = i % (R / E) * E;
        // (the pitch is a multiple of 16 bytes)
        if (c0 + col >= cols || r0 + row >= pitch) continue;
        Vec<T, E> v;
#pragma unroll
        for (int e = 0; e < E; ++e) v.v[e] = tile[col][row + e];
        store_vec(dst + (c0 + col) * pitch + r0 + row, v);
    }
}

// ------------------------------------------------------------------------------------------------ rows
// Joins the tiles' maxima and sums of a piece with the running ones; after the last piece lse and the row's loss.
// A workgroup takes 64 rows, 16 threads each over the tiles.
template <typename T>
__global__ __launch_bounds__(1024) void join_kernel(const typename Types<T>::Sum* part_max, const typename Types<T>::Sum* part_sum, int64_t tiles,
                                                    int64_t rows, bool first, bool last, typename Types<T>::Sum* run_max,
                                                    typename Types<T>::Sum* run_sum, const typename Types<T>::Sum* hit, const void* targets, int it,
                                                    int64_t V, typename Types<T>::Sum* lse, typename Types<T>::Sum* losses)
{
    using S = typename Types<T>::Sum;
    __shared__ S tops[16][64], sums[16][64];
    const int lane = threadIdx.x & 63, seg = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 64 + lane;
    S top = lowest<S>(), sum = 0;
    auto add = [&](S t, S s) {
        const S m = larger(t, top);
        sum = sum * exp_below<T>(top, m) + s * exp_below<T>(t, m);
        top = m;
    };
    if (row < rows) {
        if (seg == 0 && !first) add(run_max[row], run_sum[row]);
        for (int64_t i = seg; i < tiles; i += 16) add(part_max[i * rows + row], part_sum[i * rows + row]);
    }
    tops[seg][lane] = top;
    sums[seg][lane] = sum;
    __syncthreads();
    if (seg != 0 || row >= rows) return;
    for (int i = 1; i < 16; ++i) add(tops[i][lane], sums[i][lane]);
    if (!last) {
        run_max[row] = top;
        run_sum[row] = sum;
        return;
    }
    const S l = top + log_of(sum);
    const int64_t target = load_index(targets, row, it);
    lse[row] = l;
    losses[row] = target >= 0 && target < V ? l - hit[row] : (S)0;
}

// The same, and what reduce_kernel does, for at most 16 rows and one piece: a wave per row, in one launch.
template <typename T>
__global__ __launch_bounds__(1024) void few_join_kernel(const typename Types<T>::Sum* part_max, const typename Types<T>::Sum* part_sum, int64_t tiles,
                                                        int rows, const typename Types<T>::Sum* hit, const void* targets, int it, int64_t V, int reduction,
                                                        typename Types<T>::Sum* lse, typename Types<T>::Sum* loss, double* count)
{
    using S = typename Types<T>::Sum;
    __shared__ double losses[16], counted[16];
    const int lane = threadIdx.x & 63, row = threadIdx.x >> 6;
    if (row < rows) {
        S top = lowest<S>(), sum = 0;
        for (int64_t i = lane; i < tiles; i += 64) top = larger(part_max[i * rows + row], top);
#pragma unroll
        for (int o = 32; o > 0; o /= 2) top = larger(top, __shfl_xor(top, o));
        for (int64_t i = lane; i < tiles; i += 64) sum += part_sum[i * rows + row] * exp_below<T>(part_max[i * rows + row], top);
#pragma unroll
        for (int o = 32; o > 0; o /= 2) sum += __shfl_xor(sum, o);
        const int64_t target = load_index(targets, row, it);
        const bool has = target >= 0 && target < V;
        const S l = top + log_of(sum), x = has ? l - hit[row] : (S)0;
        if (lane == 0) {
            lse[row] = l;
            if (reduction == ST_NONE) loss[row] = x;
            losses[row] = (double)x;
            counted[row] = has ? 1 : 0;
        }
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    double sum = 0, n = 0;
    for (int i = 0; i < rows; ++i) {
        sum += losses[i];
        n += counted[i];
    }
    *count = n;
    if (reduction == ST_SUM) *loss = (S)sum;
    if (reduction == ST_MEAN) *loss = (S)(n > 0 ? sum / n : 0.0);
}

// The rows with a target and, unless reduction is ST_NONE, the sum or mean of their losses.  One workgroup.
template <typename S>
__global__ __launch_bounds__(1024) void reduce_kernel(const S* losses, const void* targets, int it, int64_t rows, int64_t V, int reduction, S* loss,
                                                      double* count)
{
    __shared__ double scratch[32];
    double sum = 0, n = 0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const int64_t t = load_index(targets, i, it);
        if (t >= 0 && t < V) {
            n += 1;
            if (reduction != ST_NONE) sum += (double)losses[i];
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) {
        sum += __shfl_xor(sum, o);
        n += __shfl_xor(n, o);
    }
    if ((threadIdx.x & 63) == 0) {
        scratch[threadIdx.x >> 6] = sum;
        scratch[16 + (threadIdx.x >> 6)] = n;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = n = 0;
    for (int i = 0; i < 16; ++i) {
        sum += scratch[i];
        n += scratch[16 + i];
    }
    *count = n;
    if (reduction == ST_SUM) *loss = (S)sum;
    if (reduction == ST_MEAN) *loss = (S)(n > 0 ? sum / n : 0.0);
}

// What is upstream of every row, divided (Upstream).  The logits' gradients are rounded to T, and a common factor that T does not hold (one over the
// number of rows) would put all of them off by the same part of a step: it stays out of them.  Rows with upstream gradients of their own are divided by
// the largest of them, and of what is left the powers of two stay out as well: float16 holds little more than the probabilities' range, and a
// row's gradient of h is rounded as well as any other's however small the row's upstream is beside the largest.  f16 takes 2^14 times as much, or
// small probabilities would be subnormal.  exps null (few classes: their logits' gradients are not rounded): nothing is divided.  One workgroup.
template <typename T>
__global__ __launch_bounds__(1024) void upstream_kernel(const typename Types<T>::Sum* grad, const void* targets, int it, int64_t rows, int64_t V,
                                                        int reduction, const double* count, Upstream<typename Types<T>::Sum> u)
{
    using S = typename Types<T>::Sum;
    constexpr int kRange = std::is_same_v<T, f16> ? 14 : 0;
    __shared__ S tops[16];
    auto has = [&](int64_t i) {
        const int64_t t = load_index(targets, i, it);
        return t >= 0 && t < V;
    };
    const S inf = (S)__builtin_inf();
    if (reduction != ST_NONE || !u.exps) {
        const S one = u.exps ? power((S)1, kRange) : (S)1;
        for (int64_t i = threadIdx.x; i < rows; i += 1024) u.up[i] = !has(i) ? (S)0 : reduction == ST_NONE ? grad[i] : one;
        if (threadIdx.x == 0)
            *u.unscale = *u.w_unscale = (reduction == ST_MEAN ? (S)((double)grad[0] / *count) : reduction == ST_SUM ? grad[0] : (S)1) / one;
        return;
    }
    S top = 0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const S a = has(i) ? (grad[i] < 0 ? -grad[i] : grad[i]) : (S)0;
        top = a > top && a < inf ? a : top;
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) {
        const S a = __shfl_xor(top, o);
        top = a > top ? a : top;
    }
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int i = 0; i < 16; ++i) top = tops[i] > top ? tops[i] : top;
    if (top == 0) top = 1;
    int top_exp;
    const S part = frexp(top, &top_exp);
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const S x = has(i) ? grad[i] : (S)0;
        int e = top_exp;
        S y = x;   // 0, infinite or NaN
        if (x != 0 && x > -inf && x < inf) y = frexp(x, &e) / part;
        u.up[i] = power(y, kRange);
        u.exps[i] = e - kRange;
    }
    if (threadIdx.x == 0) {
        *u.unscale = part;
        *u.largest = kRange != 0 ? INT_MIN : 15 + top_exp;   // (a shift that takes the largest power of two away, or largest_kernel's)
    }
}

// The largest exponent among the entries of h, each with its row's power of two.  A wave per row, one atomic operation per workgroup.
template <typename T>
__global__ __launch_bounds__(kThreads) void largest_kernel(const T* h, int64_t rows, int64_t D, Upstream<typename Types<T>::Sum> u)
{
    using S = typename Types<T>::Sum;
    constexpr int E = kPer16<T>;
    const int lane = threadIdx.x & 63;
    int largest = INT_MIN;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        const S up = u.up[row];
        if (up == 0 || !(up - up == 0)) continue;   // left out, or infinite
        S top = 0;
        for (int64_t k = lane * E; k < D; k += 64 * E) {
            const Vec<T, E> v = D - k >= E ? load_vec<T, E>(h + row * D + k) : load_some<T, E>(h + row * D + k, (int)(D - k));
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const S a = (S)v.v[i] < 0 ? -(S)v.v[i] : (S)v.v[i];
                top = a > top && a < (S)__builtin_inf() ? a : top;
            }
        }
        int e;
        frexp(top, &e);
        if (top > 0) largest = max(largest, e + u.exps[row]);
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) largest = max(largest, __shfl_xor(largest, o));
    __shared__ int waves[4];
    if (lane == 0) waves[threadIdx.x >> 6] = largest;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < 4; ++i) largest = max(largest, waves[i]);
    if (largest != INT_MIN) atomicMax(u.largest, largest);   // (a whole number: in any order)
}

unsigned blocks_for(int64_t items) { return (unsigned)((items + 255) / 256 < 16384 ? (items + 255) / 256 : 16384); }

#define ST_TRY(call)                               \
    do {                                           \
        (call);                                    \
        const hipError_t err_ = hipGetLastError(); \
        if (err_ != hipSuccess) return err_;       \
    } while (0)

// A matrix with rows in whole steps: the caller's, or a copy, with zeros in the rows up to `all`.  pitch: in whole steps; what comes back may also be the
// caller's with rows of whole 16 bytes (`ends`: the products that read it take zeros for what is behind them).
template <typename T>
hipError_t in_steps(const T* src, int64_t rows, int64_t all, int64_t cols, int64_t* pitch, void* copy, const T** out, bool ends, hipStream_t st)
{
    *out = src;
    if ((cols == *pitch || (ends && cols % kPer16<T> == 0)) && reinterpret_cast<uintptr_t>(src) % 16 == 0) {
        *pitch = cols;
        return hipSuccess;
    }
    *out = static_cast<const T*>(copy);
    ST_TRY((pack_kernel<T><<<blocks_for(all * (*pitch / kPer16<T>)), 256, 0, st>>>(src, static_cast<T*>(copy), rows, all, cols, *pitch, Upstream<typename Types<T>::Sum>{})));
    return hipSuccess;
}
// The logits' operands: classes of w, in rows of `pitch`, and h in whole steps (whose first row, where D is none, has zeros behind it).
template <typename T>
Operands logits_of(const T* w, int64_t pitch, int64_t n, const T* hs, const EntropyPlan& p)
{
    Operands o{reinterpret_cast<const char*>(w), reinterpret_cast<const char*>(hs), pitch * (int64_t)sizeof(T), p.Dp * (int64_t)sizeof(T), n, p.T,
               p.Dp * (int64_t)sizeof(T) / kStepBytes};
    if (pitch != p.Dp) {
        o.a_zero = reinterpret_cast<const char*>(hs + p.D);
        o.a_left = (int)(p.D * (int64_t)sizeof(T) % kStepBytes);
    }
    return o;
}

template <typename T>
Operands operands(const T* a, int64_t a_cols, int64_t m, const T* b, int64_t b_cols, int64_t n, int64_t k)
{
    return {reinterpret_cast<const char*>(a), reinterpret_cast<const char*>(b), a_cols * (int64_t)sizeof(T), b_cols * (int64_t)sizeof(T), m, n,
            k * (int64_t)sizeof(T) / kStepBytes};
}
// f(std::integral_constant of the wave's 16 x 16 tiles on a side)
template <typename T, class F>
hipError_t with_sub(int sub, F&& f)
{
    if constexpr (sizeof(T) == 2)
        if (sub == 8) return f(std::integral_constant<int, 8>{});
    if (sub == 4) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 2>{});
}
// A products' kernel for every tile of m rows of A and n of B.  (More than 64 KiB of LDS have to be asked for, on every device.)
template <typename T, int SUB, typename K, typename... Args>
hipError_t launch_product(K kernel, const Operands& o, int parts, hipStream_t st, const Args&... args)
{
    using P = Product<T, SUB>;
    const TileOrder t{(uint32_t)((o.m + P::kTile - 1) / P::kTile), (uint32_t)((o.n + P::kTile - 1) / P::kTile), (uint32_t)parts};
    if (P::kLds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)P::kLds);
        if (e != hipSuccess) return e;
    }
    kernel<<<t.tiles_m * t.tiles_n * t.parts, kThreads, P::kLds, st>>>(o, t, args...);
    return hipGetLastError();
}
template <typename T, bool TURN_A = false, bool TURN_B = false>
hipError_t launch_sums(const Operands& o, Tiling t, typename Types<T>::Sum* sum, int64_t pitch, bool first, hipStream_t st)
{
    return with_sub<T>(t.sub, [&](auto sub) {
        constexpr int SUB = decltype(sub)::value;
        return launch_product<T, SUB>(product_kernel<T, SUB, true, TURN_A, TURN_B>, o, parts_of(t, o.steps), st, sum, (T*)nullptr, pitch, first,
                                      (const typename Types<T>::Sum*)nullptr, Upstream<typename Types<T>::Sum>{});
    });
}

}  // namespace

template <typename T>
hipError_t entropy_run_fwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, void* loss, void* lse, double* rows, int reduction, int it,
                           unsigned char* ws, hipStream_t st)
{
    using S = typename Types<T>::Sum;
    if (p.T == 0) {
        ST_TRY((reduce_kernel<S><<<1, 1024, 0, st>>>(nullptr, nullptr, it, 0, p.V, reduction, static_cast<S*>(loss), rows)));
        return hipSuccess;
    }
    S *run_max = reinterpret_cast<S*>(ws + p.off_max), *run_sum = reinterpret_cast<S*>(ws + p.off_sum), *hit = reinterpret_cast<S*>(ws + p.off_hit);
    if (p.narrow) {
        S* z = reinterpret_cast<S*>(ws + p.off_z);
        S* losses = reduction == ST_NONE ? static_cast<S*>(loss) : run_max;
        ST_TRY((narrow_logits_kernel<T><<<dim3((unsigned)((p.T + 63) / 64), (unsigned)p.narrow_parts), kThreads, 0, st>>>(h, w, p.T, (int)p.V, p.D,
                                                                                                                        p.narrow_columns, z)));
        ST_TRY((narrow_rows_kernel<T><<<(unsigned)((p.T + 15) / 16), kThreads, 0, st>>>(z, p.narrow_parts, p.T, (int)p.V, targets, it, static_cast<S*>(lse),
                                                                                       losses, nullptr, nullptr)));
        ST_TRY((reduce_kernel<S><<<1, 1024, 0, st>>>(losses, targets, it, p.T, p.V, reduction, static_cast<S*>(loss), rows)));
        return hipSuccess;
    }
    const int64_t most = (p.piece + p.part_classes - 1) / p.part_classes;
    S *part_max = reinterpret_cast<S*>(ws + p.off_part), *part_sum = part_max + most * p.T;
    const T* hs = h;
    hipError_t e = hipSuccess;
    int64_t h_pitch = p.Dp;
    if (!p.few && (e = in_steps(h, p.T, p.T, p.D, &h_pitch, ws + p.off_h, &hs, false, st)) != hipSuccess) return e;
    // (the running maxima are dead where the losses of the rows are written: a thread reads its own first)
    S* losses = reduction == ST_NONE ? static_cast<S*>(loss) : run_max;
    for (int64_t i = 0; i < p.pieces; ++i) {
        const int64_t first = i * p.piece, n = p.V - first < p.piece ? p.V - first : p.piece, tiles = (n + p.part_classes - 1) / p.part_classes;
        if (p.few) {
            ST_TRY((few_stats_kernel<T><<<(unsigned)tiles, kThreads, 0, st>>>(w + first * p.D, h, n, (int)p.T, p.D, targets, it, first, p.V, part_max,
                                                                            part_sum, hit)));
        } else {
            const T* wsrc;
            int64_t pitch = p.Dp;
            if ((e = in_steps(w + first * p.D, n, n, p.D, &pitch, ws + p.off_w, &wsrc, true, st)) != hipSuccess) return e;
            const Operands o = logits_of(wsrc, pitch, n, hs, p);
            if (p.logits.parts > 1) {
                S* z = reinterpret_cast<S*>(ws + p.off_z);
                if ((e = launch_sums<T>(o, p.logits, z, n, true, st)) != hipSuccess) return e;
                ST_TRY((parts_stats_kernel<T><<<dim3((unsigned)tiles, (unsigned)p.T), kThreads, 0, st>>>(z, p.logits.parts, n, p.T, targets, it, first,
                                                                                                       p.V, part_max, part_sum, hit)));
            } else {
                e = with_sub<T>(p.logits.sub, [&](auto sub) {
                    constexpr int SUB = decltype(sub)::value;
                    return launch_product<T, SUB>(stats_kernel<T, SUB>, o, 1, st, targets, it, first, p.V, part_max, part_sum, hit);
                });
                if (e != hipSuccess) return e;
            }
        }
        if (p.T <= 16 && p.pieces == 1) {
            ST_TRY((few_join_kernel<T><<<1, 1024, 0, st>>>(part_max, part_sum, tiles, (int)p.T, hit, targets, it, p.V, reduction, static_cast<S*>(lse),
                                                         static_cast<S*>(loss), rows)));
            return hipSuccess;
        }
        ST_TRY((join_kernel<T><<<(unsigned)((p.T + 63) / 64), 1024, 0, st>>>(part_max, part_sum, tiles, p.T, i == 0, i + 1 == p.pieces, run_max, run_sum,
                                                                            hit, targets, it, p.V, static_cast<S*>(lse), losses)));
    }
    ST_TRY((reduce_kernel<S><<<1, 1024, 0, st>>>(losses, targets, it, p.T, p.V, reduction, static_cast<S*>(loss), rows)));
    return hipSuccess;
}

template <typename T>
hipError_t entropy_run_bwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, const void* lse, const double* rows, const void* grad,
                           T* grad_h, T* grad_w, int reduction, int it, unsigned char* ws, hipStream_t st)
{
    using S = typename Types<T>::Sum;
    if (p.T == 0) {
        if (grad_w) ST_TRY((zero_kernel<T><<<blocks_for(p.V * p.D), 256, 0, st>>>(grad_w, p.V * p.D)));
        return hipSuccess;
    }
    S *up = reinterpret_cast<S*>(ws + p.off_up), *scaling = up + p.T, *dh = reinterpret_cast<S*>(ws + p.off_dh);
    int* exps = reinterpret_cast<int*>(ws + p.off_exps);
    Upstream<S> rows_up{up, p.narrow ? nullptr : exps, exps + p.T, scaling, scaling + 1};
    // 16-bit types: g, w and h are turned on their way to the registers; others: copies of them are
    constexpr bool kTurned = sizeof(T) == 2;
    T *ht = reinterpret_cast<T*>(ws + p.off_ht), *wt = reinterpret_cast<T*>(ws + p.off_wt);
    T *g = reinterpret_cast<T*>(ws + p.off_g), *gt = reinterpret_cast<T*>(ws + p.off_gt);
    ST_TRY((upstream_kernel<T><<<1, 1024, 0, st>>>(static_cast<const S*>(grad), targets, it, p.T, p.V, reduction, rows, rows_up)));
    if (reduction != ST_NONE) rows_up.exps = nullptr;   // (one factor for all rows)
    const Upstream<S> all{};
    if (p.narrow) {
        S *z = reinterpret_cast<S*>(ws + p.off_z), *gs = reinterpret_cast<S*>(ws + p.off_g), *dw = reinterpret_cast<S*>(ws + p.off_dw);
        ST_TRY((narrow_logits_kernel<T><<<dim3((unsigned)((p.T + 63) / 64), (unsigned)p.narrow_parts), kThreads, 0, st>>>(h, w, p.T, (int)p.V, p.D,
                                                                                                                        p.narrow_columns, z)));
        ST_TRY((narrow_rows_kernel<T><<<(unsigned)((p.T + 15) / 16), kThreads, 0, st>>>(z, p.narrow_parts, p.T, (int)p.V, targets, it,
                                                                                       static_cast<S*>(const_cast<void*>(lse)), nullptr, up, gs)));
        const int64_t per = kThreads * kNarrowCols<T>;
        const auto grads = p.V <= 4 ? narrow_grads_kernel<T, 4> : p.V <= 8 ? narrow_grads_kernel<T, 8> : narrow_grads_kernel<T, kFewClasses>;
        ST_TRY((grads<<<dim3((unsigned)((p.D + per - 1) / per), (unsigned)p.narrow_ranges), kThreads, 0, st>>>(
            h, w, gs, up, scaling, p.T, p.narrow_rows, (int)p.V, p.D, grad_h, grad_w ? dw : nullptr)));
        if (grad_w)
            ST_TRY((finish_kernel<T><<<blocks_for((p.V * p.D + 3) / 4), 256, 0, st>>>(dw, p.narrow_ranges, p.V * p.D, scaling, grad_w, p.D,
                                                                                     all)));
        return hipSuccess;
    }
    const T* hs;
    int64_t h_pitch = p.Dp;
    hipError_t e = in_steps(h, p.T, p.T, p.D, &h_pitch, ws + p.off_h, &hs, false, st);
    if (e != hipSuccess) return e;
    auto turn = [&](const T* src, T* dst, int64_t r, int64_t pitch, Upstream<S> u) -> hipError_t {
        const int64_t tiles = (pitch + 63) / 64 * ((p.D + kTurnCols<T> - 1) / kTurnCols<T>);
        ST_TRY((transpose_kernel<T><<<(unsigned)tiles, 256, 0, st>>>(src, dst, r, p.D, pitch, u)));
        return hipSuccess;
    };
    if (grad_w && std::is_same_v<T, f16> && rows_up.exps)
        ST_TRY((largest_kernel<T><<<(unsigned)std::min<int64_t>((p.T + 3) / 4, 256), kThreads, 0, st>>>(h, p.T, p.D, rows_up)));
    if (grad_w && !kTurned && (e = turn(h, ht, p.T, p.Tp, rows_up)) != hipSuccess) return e;
    if (grad_w && kTurned)
        ST_TRY((pack_kernel<T><<<blocks_for(p.Tp * (p.Dp / kPer16<T>)), 256, 0, st>>>(h, ht, p.T, p.Tp, p.D, p.Dp, rows_up)));
    for (int64_t i = 0; i < p.pieces; ++i) {
        const int64_t first = i * p.piece, n = p.V - first < p.piece ? p.V - first : p.piece;
        const int64_t per = kStepBytes / (int64_t)sizeof(T), np = (n + per - 1) / per * per;
        const T* wsrc;
        int64_t pitch = p.Dp;
        if ((e = in_steps(w + first * p.D, n, kTurned ? np : n, p.D, &pitch, ws + p.off_w, &wsrc, true, st)) != hipSuccess) return e;
        const Operands logits = logits_of(wsrc, pitch, n, hs, p);
        if (p.logits.parts > 1) {
            S* z = reinterpret_cast<S*>(ws + p.off_z);
            if ((e = launch_sums<T>(logits, p.logits, z, n, true, st)) != hipSuccess) return e;
            const dim3 grid((unsigned)((np + 31) / 32), (unsigned)((p.Tp + 31) / 32));
            ST_TRY((parts_grads_kernel<T><<<grid, kThreads, 0, st>>>(z, p.logits.parts, n, p.T, targets, it, first, static_cast<const S*>(lse), up, g, np,
                                                                   gt, p.Tp)));
        } else {
            e = with_sub<T>(p.logits.sub, [&](auto sub) {
                constexpr int SUB = decltype(sub)::value;
                return launch_product<T, SUB>(grads_kernel<T, SUB>, logits, 1, st, targets, it, first, static_cast<const S*>(lse), up, g, np, gt, p.Tp);
            });
            if (e != hipSuccess) return e;
        }
        if (grad_h) {
            Operands o;
            if constexpr (kTurned) {
                o = operands(wsrc, pitch, p.D, g, np, p.T, np);
                if (wsrc == w + first * p.D && n != np) {   // (behind the caller's last row nothing may be read)
                    o.a_tail = reinterpret_cast<const char*>(wt);
                    const int64_t whole = np - per;
                    ST_TRY((pack_kernel<T><<<blocks_for(per * (pitch / kPer16<T>)), 256, 0, st>>>(wsrc + whole * pitch, wt, n - whole, per, p.D, pitch, all)));
                }
            } else {
                if ((e = turn(w + first * p.D, wt, n, np, all)) != hipSuccess) return e;
                o = operands(wt, np, p.D, g, np, p.T, np);
            }
            if (p.sums) e = launch_sums<T, kTurned, false>(o, p.by_h, dh, p.D, i == 0, st);
            else
                e = with_sub<T>(p.by_h.sub, [&](auto sub) {
                    constexpr int SUB = decltype(sub)::value;
                    return launch_product<T, SUB>(product_kernel<T, SUB, false, kTurned, false>, o, 1, st, (S*)nullptr, grad_h, p.D, true, (const S*)scaling,
                                                   rows_up);
                });
            if (e != hipSuccess) return e;
        }
        if (grad_w) {
            const Operands o = kTurned ? operands(ht, p.Dp, p.D, g, np, n, p.Tp) : operands(ht, p.Tp, p.D, gt, p.Tp, n, p.Tp);
            if (p.by_w.parts > 1) {
                S* dw = reinterpret_cast<S*>(ws + p.off_dw);
                if ((e = launch_sums<T, kTurned, kTurned>(o, p.by_w, dw, p.D, true, st)) != hipSuccess) return e;
                ST_TRY((finish_kernel<T><<<blocks_for((n * p.D + 3) / 4), 256, 0, st>>>(dw, p.by_w.parts, n * p.D, scaling + 1, grad_w + first * p.D,
                                                                                            p.D, all)));
                continue;
            }
            e = with_sub<T>(p.by_w.sub, [&](auto sub) {
                constexpr int SUB = decltype(sub)::value;
                return launch_product<T, SUB>(product_kernel<T, SUB, false, kTurned, kTurned>, o, 1, st, (S*)nullptr, grad_w + first * p.D, p.D, true,
                                              (const S*)scaling + 1, all);
            });
            if (e != hipSuccess) return e;
        }
    }
    if (grad_h && p.sums)
        ST_TRY((finish_kernel<T><<<blocks_for((p.T * p.D + 3) / 4), 256, 0, st>>>(dh, p.by_h.parts, p.T * p.D, scaling, grad_h, p.D, rows_up)));
    return hipSuccess;
}

#define ST_ENTROPY(T)                                                                                                                                   \
    template hipError_t entropy_run_fwd<T>(const EntropyPlan&, const T*, const T*, const void*, void*, void*, double*, int, int, unsigned char*,        \
                                           hipStream_t);                                                                                                \
    template hipError_t entropy_run_bwd<T>(const EntropyPlan&, const T*, const T*, const void*, const void*, const double*, const void*, T*, T*, int,   \
                                           int, unsigned char*, hipStream_t);

}  // namespace st
