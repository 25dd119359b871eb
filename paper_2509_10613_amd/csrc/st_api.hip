// C-ABI entry points of include/sigtrain.h: argument checks, workspaces and the launches of st_embed.hip, st_entropy.hip and
// st_clip.hip.  Host code only.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "sigtrain.h"
#include "sk_error.h"
#include "st_kernels.h"

namespace {

int fail(int code, const char* fmt, ...)
{
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    return sk::set_error(code, text);
}

int done(hipError_t e, const char* what)
{
    return e == hipSuccess ? SK_OK : fail(SK_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool known_type(int dt) { return dt == ST_F32 || dt == ST_F64 || dt == ST_BF16 || dt == ST_F16; }

int check_types(int it, int dt)
{
    if (!known_type(dt)) return fail(SK_ERR_DTYPE, "dtype %d is none of ST_F32, ST_F64, ST_BF16, ST_F16", dt);
    if (it != ST_I32 && it != ST_I64) return fail(SK_ERR_DTYPE, "index type %d is neither ST_I32 nor ST_I64", it);
    return SK_OK;
}

int check_workspace(const void* ws, size_t have, size_t need)
{
    if (need == 0) return SK_OK;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255)) return fail(SK_ERR_WORKSPACE, "workspace pointer is NULL or not 256-byte aligned");
    if (have < need) return fail(SK_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
    return SK_OK;
}

// addresses of elements
int check_aligned(int dt, std::initializer_list<const void*> pointers)
{
    for (const void* p : pointers)
        if (reinterpret_cast<uintptr_t>(p) % (size_t)st::dtype_size(dt)) return fail(SK_ERR_NULL, "a pointer is not aligned to its elements");
    return SK_OK;
}

constexpr int64_t kMostIndex = ((int64_t)1 << 31) - 2, kMostColumns = (int64_t)1 << 24, kMostRows = 4000000;

int check_embed(int64_t count, int64_t V, int64_t D, double scale, int it, int dt)
{
    int rc = check_types(it, dt);
    if (rc != SK_OK) return rc;
    if (count < 0 || V < 0 || D < 1 || D > kMostColumns)
        return fail(SK_ERR_SHAPE, "need count >= 0, V >= 0 and 1 <= D <= 2^24 (got %lld, %lld, %lld)", (long long)count, (long long)V, (long long)D);
    if (V > kMostIndex || count > (int64_t)1 << 40) return fail(SK_ERR_SHAPE, "V must stay below 2^31 - 1, count below 2^40");
    if (count > 0 && D > ((int64_t)1 << 41) / count) return fail(SK_ERR_SHAPE, "more than 2^41 entries");
    if (!std::isfinite(scale)) return fail(SK_ERR_SHAPE, "scale is not finite");
    return SK_OK;
}

int check_entropy(int64_t T, int64_t V, int64_t D, int reduction, int it, int dt)
{
    int rc = check_types(it, dt);
    if (rc != SK_OK) return rc;
    if (reduction != ST_NONE && reduction != ST_MEAN && reduction != ST_SUM) return fail(SK_ERR_SHAPE, "unknown reduction %d", reduction);
    if (T < 0 || T > kMostRows || V < 1 || V > kMostIndex || D < 1 || D > kMostRows)
        return fail(SK_ERR_SHAPE, "need 0 <= T <= 4000000, 1 <= V < 2^31 - 1 and 1 <= D <= 4000000 (got %lld, %lld, %lld)", (long long)T, (long long)V,
                    (long long)D);
    return SK_OK;
}

}  // namespace

extern "C" {

int sigtrain_embed_fwd(const void* tokens, const void* table, void* out, int64_t count, int64_t V, int64_t D, double scale, st_itype it,
                       st_dtype dt, void* stream)
{
    int rc = check_embed(count, V, D, scale, it, dt);
    if (rc != SK_OK || count == 0) return rc;
    if (!tokens || !out || (!table && V > 0)) return fail(SK_ERR_NULL, "tokens, table or out is NULL");
    if ((rc = check_aligned(dt, {table, out})) != SK_OK) return rc;
    return done(st::embed_fwd(tokens, table, out, count, V, D, scale, it, dt, static_cast<hipStream_t>(stream)), "embed_fwd");
}

size_t sigtrain_embed_bwd_workspace_bytes(int64_t count, int64_t V, int64_t D, st_dtype dt)
{
    if (check_embed(count, V, D, 1.0, ST_I64, dt) != SK_OK || count > kMostIndex) return 0;
    return st::embed_plan(count, V, D, dt).total;
}

int sigtrain_embed_bwd(const void* tokens, const void* grad_out, void* grad_table, int64_t count, int64_t V, int64_t D, double scale,
                       st_itype it, st_dtype dt, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_embed(count, V, D, scale, it, dt);
    if (rc != SK_OK) return rc;
    if (count > kMostIndex) return fail(SK_ERR_SHAPE, "count must stay below 2^31 - 1");
    if (V == 0) return SK_OK;
    if (!grad_table || (count > 0 && (!tokens || !grad_out))) return fail(SK_ERR_NULL, "tokens, grad_out or grad_table is NULL");
    if ((rc = check_aligned(dt, {grad_out, grad_table})) != SK_OK) return rc;
    const st::EmbedPlan p = st::embed_plan(count, V, D, dt);
    if ((rc = check_workspace(ws, ws_bytes, p.total)) != SK_OK) return rc;
    return done(st::embed_bwd(p, tokens, grad_out, grad_table, scale, it, dt, ws, static_cast<hipStream_t>(stream)), "embed_bwd");
}

size_t sigtrain_entropy_workspace_bytes(int backward, int64_t T, int64_t V, int64_t D, st_dtype dt, int least)
{
    if (check_entropy(T, V, D, ST_NONE, ST_I64, dt) != SK_OK) return 0;
    return st::entropy_plan(backward != 0, T, V, D, dt, least != 0, 0).total;
}

int sigtrain_entropy_fwd(const void* h, const void* w, const void* targets, void* loss, void* lse, double* rows, int64_t T, int64_t V, int64_t D,
                         int reduction, st_itype it, st_dtype dt, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_entropy(T, V, D, reduction, it, dt);
    if (rc != SK_OK) return rc;
    if (!rows || (!loss && (T > 0 || reduction != ST_NONE)) || (T > 0 && (!h || !w || !targets || !lse)))
        return fail(SK_ERR_NULL, "h, w, targets, loss, lse or rows is NULL");
    if ((rc = check_aligned(dt, {h, w})) != SK_OK) return rc;
    const st::EntropyPlan least = st::entropy_plan(false, T, V, D, dt, true, 0);
    if (T > 0 && (rc = check_workspace(ws, ws_bytes, least.total)) != SK_OK) return rc;
    const st::EntropyPlan p = st::entropy_plan(false, T, V, D, dt, false, ws_bytes);
    return done(st::entropy_fwd(p, h, w, targets, loss, lse, rows, reduction, it, dt, ws, static_cast<hipStream_t>(stream)), "entropy_fwd");
}

int sigtrain_entropy_bwd(const void* h, const void* w, const void* targets, const void* lse, const double* rows, const void* grad, void* grad_h,
                         void* grad_w, int64_t T, int64_t V, int64_t D, int reduction, st_itype it, st_dtype dt, void* ws, size_t ws_bytes,
                         void* stream)
{
    int rc = check_entropy(T, V, D, reduction, it, dt);
    if (rc != SK_OK) return rc;
    if (!grad_h && !grad_w) return SK_OK;
    if (T > 0 && (!h || !w || !targets || !lse || !rows || !grad)) return fail(SK_ERR_NULL, "h, w, targets, lse, rows or grad is NULL");
    if ((rc = check_aligned(dt, {h, w, grad_h, grad_w})) != SK_OK) return rc;
    const st::EntropyPlan least = st::entropy_plan(true, T, V, D, dt, true, 0);
    if (T > 0 && (rc = check_workspace(ws, ws_bytes, least.total)) != SK_OK) return rc;
    const st::EntropyPlan p = st::entropy_plan(true, T, V, D, dt, false, ws_bytes);
    return done(st::entropy_bwd(p, h, w, targets, lse, rows, grad, grad_h, grad_w, reduction, it, dt, ws, static_cast<hipStream_t>(stream)),
                "entropy_bwd");
}

size_t sigtrain_clip_workspace_bytes(int64_t n) { return n < 0 || n > kMostIndex ? 0 : st::clip_workspace(n); }

static int check_clip(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n,
                      const double* norm)
{
    if (n < 0 || n > kMostIndex) return fail(SK_ERR_SHAPE, "the number of arrays is negative or too large");
    if (!norm || (n > 0 && (!grads || !counts || !dts))) return fail(SK_ERR_NULL, "grads, counts, dts or norm is NULL");
    for (int64_t i = 0; i < n; ++i) {
        if (!known_type(dts[i]) || (out_dts && !known_type(out_dts[i]))) return fail(SK_ERR_DTYPE, "array %lld has an unknown dtype", (long long)i);
        if (counts[i] < 0 || counts[i] > (int64_t)1 << 40) return fail(SK_ERR_SHAPE, "array %lld has %lld entries", (long long)i, (long long)counts[i]);
        if (counts[i] == 0) continue;
        if (!grads[i] || (out && !out[i])) return fail(SK_ERR_NULL, "array %lld is NULL", (long long)i);
        int rc = check_aligned(dts[i], {grads[i]});
        if (rc == SK_OK && out) rc = check_aligned(out_dts[i], {out[i]});
        if (rc != SK_OK) return rc;
        if (out && out[i] == grads[i] && out_dts[i] != dts[i])
            return fail(SK_ERR_DTYPE, "array %lld is scaled in place but its types differ", (long long)i);
    }
    return SK_OK;
}

// No output may overlap another output, or an input other than its own.
static int check_overlap(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n)
{
    struct Range {
        uintptr_t from, to;
        int64_t array;
        bool written;
    };
    std::vector<Range> ranges;
    try {
        ranges.reserve(2 * (size_t)n);
    } catch (const std::bad_alloc&) {
        return fail(SK_ERR_SHAPE, "no host memory to check %lld arrays", (long long)n);
    }
    for (int64_t i = 0; i < n; ++i) {
        if (counts[i] == 0) continue;
        const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]), o = reinterpret_cast<uintptr_t>(out[i]);
        if (g != o) ranges.push_back({g, g + (uintptr_t)counts[i] * (uintptr_t)st::dtype_size(dts[i]), i, false});
        ranges.push_back({o, o + (uintptr_t)counts[i] * (uintptr_t)st::dtype_size(out_dts[i]), i, true});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t read_to = 0, written_to = 0;   // ends of what lies before
    for (const Range& r : ranges) {
        if (r.from < written_to || (r.written && r.from < read_to))
            return fail(SK_ERR_SHAPE, "the output of array %lld overlaps another array, or the other way round", (long long)r.array);
        (r.written ? written_to : read_to) = std::max(r.written ? written_to : read_to, r.to);
    }
    return SK_OK;
}

int sigtrain_grad_norm(const void* const* grads, const int64_t* counts, const int* dts, int64_t n, double* norm, void* ws, size_t ws_bytes,
                       void* stream)
{
    int rc = check_clip(grads, nullptr, counts, dts, nullptr, n, norm);
    if (rc != SK_OK) return rc;
    if ((rc = check_workspace(ws, ws_bytes, st::clip_workspace(n))) != SK_OK) return rc;
    return done(st::clip(grads, nullptr, counts, dts, nullptr, n, 0.0, norm, ws, static_cast<hipStream_t>(stream)), "grad_norm");
}

int sigtrain_clip(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n,
                  double max_norm, double* norm, void* ws, size_t ws_bytes, void* stream)
{
    if (n > 0 && (!out || !out_dts)) return fail(SK_ERR_NULL, "out or out_dts is NULL");
    int rc = check_clip(grads, out, counts, dts, out_dts, n, norm);
    if (rc != SK_OK) return rc;
    if (!(max_norm >= 0)) return fail(SK_ERR_SHAPE, "max_norm must not be negative or NaN");
    if ((rc = check_overlap(grads, out, counts, dts, out_dts, n)) != SK_OK) return rc;
    if ((rc = check_workspace(ws, ws_bytes, st::clip_workspace(n))) != SK_OK) return rc;
    return done(st::clip(grads, out, counts, dts, out_dts, n, max_norm, norm, ws, static_cast<hipStream_t>(stream)), "clip");
}

int sigtrain_describe(int op, int64_t n, int64_t V, int64_t D, st_dtype dt, size_t ws_bytes, char* out, size_t out_bytes)
{
    if (!out || out_bytes == 0) return fail(SK_ERR_NULL, "out is NULL or empty");
    if (op < 0 || op > 3) return fail(SK_ERR_SHAPE, "unknown operation %d", op);
    const int rc = op < 2 ? check_embed(n, V, D, 1.0, ST_I64, dt) : check_entropy(n, V, D, ST_NONE, ST_I64, dt);
    if (rc != SK_OK) return rc;
    if (op == 0) {
        snprintf(out, out_bytes, "embed_fwd vectors_per_row=%lld", (long long)((D * st::dtype_size(dt) + 15) / 16));
    } else if (op == 1) {
        if (n > kMostIndex) return fail(SK_ERR_SHAPE, "count must stay below 2^31 - 1");
        const st::EmbedPlan p = st::embed_plan(n, V, D, dt);
        snprintf(out, out_bytes, "embed_bwd sort_tiles=%lld digits=%d bits=%d lanes=%d slices=%d units=%lld groups=%lld ws=%zu", (long long)p.tiles,
                 p.passes, p.bits, p.lanes, p.slices, (long long)p.units, (long long)p.groups, p.total);
    } else {
        const st::EntropyPlan p = st::entropy_plan(op == 3, n, V, D, dt, false, ws_bytes);
        const int used = snprintf(out, out_bytes, "%s piece=%lld pieces=%lld ws=%zu", op == 3 ? "entropy_bwd" : "entropy_fwd", (long long)p.piece,
                                  (long long)p.pieces, p.total);
        if (op == 3 && !p.narrow && used > 0 && (size_t)used < out_bytes) {
            const int64_t per = st::kStepBytes / p.size, last = V - (p.pieces - 1) * p.piece, whole = p.piece < V ? p.piece : V;
            const int64_t steps = (whole + per - 1) / per, last_steps = (last + per - 1) / per;
            snprintf(out + used, out_bytes - used, " grad_h_steps=%lld parts=%d last_steps=%lld last_parts=%d", (long long)steps,
                     st::parts_of(p.by_h, steps), (long long)last_steps, st::parts_of(p.by_h, last_steps));
        }
    }
    return SK_OK;
}

}  // extern "C"
