// Launchers of the kernels of sigtrain.h.  They enqueue on `st` and return the launch's error; arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "sigtrain.h"

namespace st {

inline int dtype_size(int dt) { return dt == ST_F64 ? 8 : dt == ST_F32 ? 4 : 2; }
inline size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// ---------------------------------------------------------------- tables (st_embed.hip)
hipError_t embed_fwd(const void* tokens, const void* table, void* out, int64_t count, int64_t V, int64_t D, double scale, int it, int dt,
                     hipStream_t st);

// The gradient's scratch: sorted symbols with their places, the sort's other half and counts, and what units of the sums hand over.
struct EmbedPlan {
    int64_t count, V, D;
    int lanes;            // lanes that share a row's columns (a power of two), one vector each
    int slices;           // ... times this many slices of the columns
    int events;           // tokens added and rows written per unit
    int64_t units, groups;   // units; workgroups of them
    int passes, bits;     // of the sort: digits, bits per digit
    int rows;             // ... rows of 64 symbols per wave
    int64_t tiles;        // ... and workgroups (0: one workgroup sorts everything)
    size_t off_keys[2], off_places[2], off_counts, off_carry, off_head, off_list, total;
};
EmbedPlan embed_plan(int64_t count, int64_t V, int64_t D, int dt);
hipError_t embed_bwd(const EmbedPlan& p, const void* tokens, const void* grad_out, void* grad_table, double scale, int it, int dt, void* ws,
                     hipStream_t st);

// ---------------------------------------------------------------- cross entropy (st_entropy.hip)
// One call's pieces of the classes and scratch.  Everything that is multiplied has rows of whole steps (kStepBytes), zeros behind the last entry:
// the caller's arrays where they have that form, copies elsewhere.
constexpr int kStepBytes = 128;   // of a row, taken at a time by the products
constexpr int kTileRows = 256;    // pieces of the classes are multiples of this
struct Tiling {
    int sub = 2, parts = 1;       // 16 x 16 tiles on a side of a wave's, and workgroups that divide a tile's steps
};
// The workgroups that divide `steps`: each takes one step at least.  (Parts are chosen for a whole piece of the classes; the last may have fewer steps.)
inline int parts_of(const Tiling& t, int64_t steps) { return steps < t.parts ? (int)steps : t.parts; }
struct EntropyPlan {
    int64_t T, V, D;
    int size, sum_size;        // bytes of an element and of a sum
    int64_t Dp, Tp;            // D and T in whole steps
    int64_t piece, pieces;     // classes per piece (a multiple of kTileRows)
    bool few;                  // forward, of at most 16 rows: w is read straight from memory
    bool narrow;               // at most 16 classes and wide rows: h is read straight from memory
    int narrow_parts, narrow_ranges;             // ... in parts of its columns for the logits, in ranges of its rows for grad_w
    int64_t narrow_columns, narrow_rows;         // ... of so many
    int64_t part_classes;      // forward: classes whose maximum and sum are formed together
    Tiling logits, by_h, by_w; // the products of the logits and of both gradients
    bool sums;                 // whether grad_h is summed over pieces or parts
    size_t off_h, off_w;       // copies of h and of a piece of w with rows of Dp (used where the caller's do not fit)
    size_t off_z;              // the logits as sums over parts, where they are divided
    size_t off_max, off_sum, off_hit;   // forward: running maximum and sum, and the target's logit, of every row
    size_t off_part;           // ... and those of the piece's tiles
    size_t off_up;             // backward: every row's upstream gradient (and behind them the scaling, two numbers)
    size_t off_exps;           // ... and the powers of two that stay out of it (and behind them the largest of h's)
    size_t off_ht, off_wt;     // ... h and a piece of w transposed; 16-bit types: h without rows that have no target, and w's last step
    size_t off_g, off_gt;      // ... the piece's gradients of the logits, as they are and (not of 16-bit types) transposed
    size_t off_dh, off_dw;     // ... the sums of grad_h, and of a piece's grad_w, one per part
    size_t total;
};
// ws_bytes 0: as fast as it gets; otherwise pieces that fit it.  least: the smallest pieces.
EntropyPlan entropy_plan(bool backward, int64_t T, int64_t V, int64_t D, int dt, bool least, size_t ws_bytes);
hipError_t entropy_fwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, void* loss, void* lse, double* rows,
                       int reduction, int it, int dt, void* ws, hipStream_t st);
hipError_t entropy_bwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, const void* lse, const double* rows,
                       const void* grad, void* grad_h, void* grad_w, int reduction, int it, int dt, void* ws, hipStream_t st);

// ---------------------------------------------------------------- norm and clipping (st_clip.hip)
constexpr int kClipBatch = 96;          // arrays per launch: their table travels as a kernel argument
constexpr int kClipBlocks = 2048;       // workgroups of a call's norm, all launches together (a few more with many launches)
size_t clip_workspace(int64_t n);
// out: null for the norm alone
hipError_t clip(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n,
                double max_norm, double* norm, void* ws, hipStream_t st);

}  // namespace st
