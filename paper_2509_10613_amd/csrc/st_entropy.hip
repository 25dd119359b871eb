// Cross entropy of a linear read-out: the pieces, tiles and scratch of a call (the kernels: st_entropy_impl.h, compiled for each type).
#include <algorithm>

#include "st_dev.h"
#include "st_kernels.h"

namespace st {

template <typename T>
hipError_t entropy_run_fwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, void* loss, void* lse, double* rows, int reduction, int it,
                           unsigned char* ws, hipStream_t st);
template <typename T>
hipError_t entropy_run_bwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, const void* lse, const double* rows, const void* grad,
                           T* grad_h, T* grad_w, int reduction, int it, unsigned char* ws, hipStream_t st);

namespace {

// The tiles of a product of m by n results over `steps`, on 256 compute units: of the sizes there are, divided among up to most_parts workgroups
// each (which leave sums, to be added by another launch), those that take the fewest cycles by this estimate.
// A step of a tile of 32 sub by 32 sub takes 32 sub^2 cycles of matrix instructions (16-bit types; 1.35 times that as measured; float and double
// eight times as many), or what arrives at 40 bytes a cycle, and with one workgroup on a compute unit no less than the way to memory and back.
Tiling choose_tiling(int size, int64_t m, int64_t n, int64_t steps, int64_t most_parts, int sum_size)
{
    Tiling best{};
    double least = 1e300;
    for (int sub = size == 2 ? 8 : 4; sub >= 2; sub /= 2) {
        const int64_t tile = 32 * sub, tiles = ((m + tile - 1) / tile) * ((n + tile - 1) / tile);
        const double busy = sub * sub * (size == 2 ? 43.0 : 270.0), fed = sub * 205.0 + 100.0;
        for (int64_t parts = 1; parts <= most_parts && (parts == 1 || steps / parts >= 8); parts *= 2) {
            const int64_t groups = tiles * parts, rounds = (groups + 255) / 256;
            double step = std::max(busy, fed);
            if (rounds == 1) step = std::max(step, 1000.0);
            double cost = (double)rounds * ((double)((steps + parts - 1) / parts) * step + 6000.0);
            if (parts > 1) cost += 8000.0 + 2.0 * (double)(parts * m * n * sum_size) / 2000.0;
            if (cost < least) {
                least = cost;
                best = {sub, (int)parts};
            }
        }
    }
    return best;
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

EntropyPlan entropy_plan(bool backward, int64_t T, int64_t V, int64_t D, int dt, bool least, size_t ws_bytes)
{
    EntropyPlan p{};
    p.T = T;
    p.V = V;
    p.D = D;
    p.size = dtype_size(dt);
    p.sum_size = dt == ST_F64 ? 8 : 4;
    const int64_t per = kStepBytes / p.size;
    auto steps = [&](int64_t n) { return (n + per - 1) / per * per; };
    p.Dp = steps(D);
    p.Tp = steps(T);
    bool parts = !least;   // (the least workspace has no place for parts)
    auto lay = [&](int64_t piece) {
        p.piece = piece;
        p.pieces = (V + piece - 1) / piece;
        const int64_t classes = std::min(piece, V);
        size_t at = 0;
        auto take = [&](int64_t entries, int size) {
            const size_t here = at;
            at += round_up((size_t)entries * size, 256);
            return here;
        };
        p.few = !backward && T <= 16;
        // (where the logits are few their parts are small)
        p.logits = choose_tiling(p.size, classes, T, p.Dp / per, p.few || !parts || T > 65535 || classes * T > (1 << 22) ? 1 : 16, p.sum_size);
        p.off_h = take(p.few ? 0 : T * p.Dp, p.size);
        p.off_w = take(p.few ? 0 : piece * p.Dp, p.size);
        p.off_z = take(p.logits.parts > 1 ? p.logits.parts * T * classes : 0, p.sum_size);
        if (!backward) {
            p.part_classes = p.few ? 64 : p.logits.parts > 1 ? 256 : 32 * p.logits.sub;
            p.off_max = take(T, p.sum_size);
            p.off_sum = take(T, p.sum_size);
            p.off_hit = take(T, p.sum_size);
            p.off_part = take(2 * T * ((piece + p.part_classes - 1) / p.part_classes), p.sum_size);
        } else {
            p.by_h = choose_tiling(p.size, D, T, (classes + per - 1) / per, parts ? 64 : 1, p.sum_size);
            p.by_w = choose_tiling(p.size, D, classes, p.Tp / per, parts && classes * D <= 1 << 24 ? 16 : 1, p.sum_size);
            p.sums = p.pieces > 1 || p.by_h.parts > 1;
            p.off_up = take(T + 2, p.sum_size);
            p.off_exps = take(T + 1, 4);
            const bool turned = p.size == 2;   // (the products turn what others need turned copies of)
            p.off_ht = take(turned ? p.Tp * p.Dp : D * p.Tp, p.size);
            p.off_wt = take(turned ? per * p.Dp : D * piece, p.size);
            p.off_g = take((turned ? p.Tp : T) * piece, p.size);
            p.off_gt = take(turned ? 0 : piece * p.Tp, p.size);
            p.off_dh = take(p.sums ? p.by_h.parts * T * D : 0, p.sum_size);
            p.off_dw = take(p.by_w.parts > 1 ? p.by_w.parts * classes * D : 0, p.sum_size);
        }
        p.total = std::max<size_t>(at, 256);
    };
    const int64_t all = (V + kTileRows - 1) / kTileRows * kTileRows;
    // Few classes of wide rows.  By tiles and like this, loss and gradients, ten classes: 1000 rows of 37449 floats 458 and 222 us (loss 105 and 41), of 5461
    // doubles 161 and 98, of 512 floats 97 and 87 (256 floats: 92 and 89, most lanes of the gradients' kernel idle; the other way for 4000 rows of 2000
    // bfloat16 and 16 classes, 103 and 124).  The loss of at most 16 rows goes to the kernel for those, whose workgroups are the classes' alone: of ten classes that
    // is one, 195 to 259 us for 1 to 16 rows of 37449 floats where this would take 25 (1000 floats: 23 and 25).  Ranges of 48 rows at least: their sums
    // of grad_w are added up by one launch.
    if (V <= 16 && D >= 512 && (backward || T > 16)) {
        p.narrow = true;
        p.piece = all;
        p.pieces = 1;
        const int64_t groups = std::max<int64_t>((T + 63) / 64, 1), each = 64 * 16 / p.size;   // of rows; columns that a wave takes at least
        const int64_t cols = (D + each - 1) / each, blocks = (D * p.size + 4095) / 4096;
        p.narrow_parts = (int)(parts ? std::max<int64_t>(1, std::min(1024 / groups, cols)) : 1);
        p.narrow_columns = (cols + p.narrow_parts - 1) / p.narrow_parts * each;
        p.narrow_parts = (int)((D + p.narrow_columns - 1) / p.narrow_columns);
        p.narrow_ranges = (int)(parts ? std::max<int64_t>(1, std::min<int64_t>({1024 / blocks, (T + 47) / 48, ((int64_t)64 << 20) / (V * D * p.sum_size)})) : 1);
        p.narrow_rows = std::max<int64_t>((T + p.narrow_ranges - 1) / p.narrow_ranges, 1);
        size_t at = 0;
        auto take = [&](int64_t entries, int size) {
            const size_t here = at;
            at += round_up((size_t)entries * size, 256);
            return here;
        };
        p.off_z = take(p.narrow_parts * T * 16, p.sum_size);
        p.off_max = p.off_up = take(T + 2, p.sum_size);
        if (backward) {
            p.off_g = take(T * 16, p.sum_size);
            p.off_dw = take(p.narrow_ranges * V * D, p.sum_size);
        }
        p.total = std::max<size_t>(at, 256);
        if (ws_bytes != 0 && p.total > ws_bytes && !least) return entropy_plan(backward, T, V, D, dt, true, 0);
        return p;
    }
    if (least) {   // the smallest pieces, or a single one: then grad_h needs no sums
        lay(all);
        const size_t single = p.total;
        lay(kTileRows);
        if (single < p.total) lay(all);
        const EntropyPlan best = entropy_plan(backward, T, V, D, dt, false, 0);   // (a few classes: it may take less)
        return best.total < p.total ? best : p;
    }
    // Pieces of at most 1 GiB of what a class takes, and of those the size for which the compute units' rounds of tiles, over all pieces and products, are
    // fewest: 8192 rows and 4096 channels in pieces of 10240 classes have 640 tiles of grad_w, two and a half rounds that take three.
    const int64_t each = backward ? (p.size == 2 ? 1 : 2) * (p.Tp + p.Dp) * p.size : (T <= 16 ? 0 : p.Dp * p.size) + 2 * T * p.sum_size / 64 + 1;
    int64_t most = ((int64_t)1 << 30) / each / kTileRows;
    if (most < 1) most = 1;
    if (most > (1 << 14)) most = 1 << 14;   // (2^22 classes: a tile's 128 rows of that many doubles lie within 32-bit offsets)
    if (most > all / kTileRows) most = all / kTileRows;
    auto fits = [&](int64_t rows) {
        lay(rows * kTileRows);
        return ws_bytes == 0 || p.total <= ws_bytes;
    };
    if (!fits(most)) {   // the largest that does, between one that does and one that does not
        int64_t yes = 1, no = most;
        while (no - yes > 1) {
            const int64_t mid = (yes + no) / 2;
            (fits(mid) ? yes : no) = mid;
        }
        most = yes;
    }
    int64_t best = most;
    if (backward && most < all / kTileRows) {
        const int64_t tile = p.size == 2 ? 256 : 128, units = 256, per_row = kTileRows / tile;
        const int64_t tt = (T + tile - 1) / tile, td = (D + tile - 1) / tile;
        auto rounds = [&](int64_t tiles) { return (double)((tiles + units - 1) / units); };
        double least_cost = 1e300;
        for (int64_t rows = most; rows > most / 2 && rows > most - 64; --rows) {
            // a round of logits takes D steps, of grad_w T and of grad_h the piece's classes
            const double one = rounds(rows * per_row * tt) * (double)D + rounds(rows * per_row * td) * (double)T + rounds(tt * td) * (double)(rows * kTileRows);
            const double cost = one * (double)((all / kTileRows + rows - 1) / rows);
            if (cost < least_cost * 0.999 && fits(rows)) {
                least_cost = cost;
                best = rows;
            }
        }
    }
    if (!backward) {   // of about the same size
        const int64_t count = (all / kTileRows + most - 1) / most;
        best = (all / kTileRows + count - 1) / count;
        if (!fits(best)) best = most;
    }
    if (!fits(best)) return entropy_plan(backward, T, V, D, dt, true, 0);
    return p;
}

hipError_t entropy_fwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, void* loss, void* lse, double* rows,
                       int reduction, int it, int dt, void* ws, hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        return entropy_run_fwd<T>(p, static_cast<const T*>(h), static_cast<const T*>(w), targets, loss, lse, rows, reduction, it,
                          static_cast<unsigned char*>(ws), st);
    });
}

hipError_t entropy_bwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, const void* lse, const double* rows,
                       const void* grad, void* grad_h, void* grad_w, int reduction, int it, int dt, void* ws, hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        return entropy_run_bwd<T>(p, static_cast<const T*>(h), static_cast<const T*>(w), targets, lse, rows, grad, static_cast<T*>(grad_h),
                          static_cast<T*>(grad_w), reduction, it, static_cast<unsigned char*>(ws), st);
    });
}

}  // namespace st
