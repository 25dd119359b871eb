/*
 * sigtrain.h - C ABI of the operators at both ends of a model that is trained around signatures; part of libsigkernel.
 *
 *  - Tables of vectors that turn sequences of symbols into paths, and their gradient (sigtrain_embed_*).
 *  - The softmax cross entropy of a linear read-out over many classes, and its gradients, in pieces of the classes: the
 *    logits of all classes never exist at once (sigtrain_entropy_*).
 *  - The norm of all gradients of a step, and clipping by it (sigtrain_grad_norm, sigtrain_clip).
 *
 * Conventions are those of sigkernel.h: device pointers to dense row-major arrays owned by the caller (aligned to their
 * elements, no more), outputs overwritten, caller-owned 256-byte aligned workspace of at least the bytes the query says,
 * calls only enqueue kernels on `stream` (they can be captured into a HIP graph), return value SK_OK or a negative
 * SK_ERR_* code with a message in sigkernel_last_error(), nothing enqueued on an argument error.  Calls that share a workspace must be ordered.
 * Results do not depend on the order in which workgroups run: the same call gives the same bits.
 */
#ifndef SIGKERNEL_SIGTRAIN_H
#define SIGKERNEL_SIGTRAIN_H

#include "sigkernel.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of this header's arrays.  Sums and softmax statistics are held in double for ST_F64, otherwise in float or double. */
typedef enum { ST_F32 = SK_F32, ST_F64 = SK_F64, ST_BF16 = 2, ST_F16 = 3 } st_dtype;
/* Types of symbols and targets. */
typedef enum { ST_I32 = 0, ST_I64 = 1 } st_itype;

/*
 * out[n, :] = scale * table[tokens[n], :] for tokens[count], table[V, D], out[count, D].  A token outside 0 .. V - 1 stands for
 * no symbol (padding): its row is 0, and it takes no part in the gradient.  The product is formed in float (double for ST_F32, ST_F64
 * and scales that are no normal float) and rounded once.
 */
int sigtrain_embed_fwd(const void* tokens, const void* table, void* out, int64_t count, int64_t V, int64_t D, double scale,
                       st_itype it, st_dtype dt, void* stream);

/*
 * grad_table[v, :] = scale * sum over the n with tokens[n] = v of grad_out[n, :], every row written (0 for symbols that do not
 * occur).  The tokens are sorted (stably), and every row is summed in a fixed order, in float (ST_BF16, ST_F16) or double.
 * count and V below 2^31 - 1.
 */
size_t sigtrain_embed_bwd_workspace_bytes(int64_t count, int64_t V, int64_t D, st_dtype dt);
int sigtrain_embed_bwd(const void* tokens, const void* grad_out, void* grad_table, int64_t count, int64_t V, int64_t D, double scale,
                       st_itype it, st_dtype dt, void* ws, size_t ws_bytes, void* stream);

/* What becomes of the rows' losses. */
enum { ST_NONE = 0, ST_MEAN = 1, ST_SUM = 2 };

/*
 * Softmax cross entropy of the linear read-out z = h w^T, h[T, D], w[V, D]:
 *     lse[t] = log sum_v exp z[t, v],   row t's loss = lse[t] - z[t, targets[t]].
 * A row whose target is outside 0 .. V - 1 has no target (padding, a prompt): its loss is 0, its gradient is 0 (whatever the read-out
 * holds), it is not counted and what its row of h holds reaches neither the loss nor grad_w.
 * reduction ST_NONE: loss[T]; ST_SUM: loss[1]; ST_MEAN: loss[1], the sum divided by the number of rows with a target (0 if there are none).
 * loss and lse are arrays of float (double for ST_F64); rows with a target, as a double: *rows.
 * Products are summed in float (double for ST_F64), and logits are never rounded to fewer bits.
 *
 * Backward: `grad` is dF/dloss, shaped and typed as `loss`; lse and rows are the forward call's.  grad_h[T, D] and grad_w[V, D]
 * (either may be NULL).  With ST_NONE a row whose upstream gradient is 0 is left out as one without a target.  The logits' gradients
 * u_t (exp(z - lse) - [v = target]) of a piece of the classes are rounded to the arrays' type before they are multiplied by w and h (except of at
 * most 16 classes of wide rows): without the mean's and the sum's common factor, or, with ST_NONE, divided by the largest finite |u_t| and by the
 * power of two that this leaves of their own row, none of which 16-bit types need hold; for ST_F16 times 2^14, so that small probabilities stay in its range.  The
 * products are multiplied by all of that again, in the sums' type; the rows of h that grad_w is made from have the powers of two beforehand.
 *
 * The workspace query gives what the call is fastest with; with `least` set, what it takes (smaller pieces).
 */
size_t sigtrain_entropy_workspace_bytes(int backward, int64_t T, int64_t V, int64_t D, st_dtype dt, int least);
int sigtrain_entropy_fwd(const void* h, const void* w, const void* targets, void* loss, void* lse, double* rows, int64_t T, int64_t V,
                         int64_t D, int reduction, st_itype it, st_dtype dt, void* ws, size_t ws_bytes, void* stream);
int sigtrain_entropy_bwd(const void* h, const void* w, const void* targets, const void* lse, const double* rows, const void* grad,
                         void* grad_h, void* grad_w, int64_t T, int64_t V, int64_t D, int reduction, st_itype it, st_dtype dt, void* ws,
                         size_t ws_bytes, void* stream);

/*
 * *norm = sqrt(sum of the squares of all entries of `n` arrays): grads[i] (device) of counts[i] entries of type dts[i]; the three
 * lists are host memory and free again when the call returns.  Squares and sums are in double (doubles beyond 1e154 have an infinite norm).
 *
 * sigtrain_clip also writes out[i] = grads[i] * min(1, max_norm / *norm), rounded once to out_dts[i] from a product in double (in float where
 * neither side has more than 32 bits, the entries have 16 and the factor is a normal float).  out[i] may be grads[i]
 * (then out_dts[i] = dts[i]); otherwise no output may overlap an input or another output (SK_ERR_SHAPE).  If the norm is
 * infinite or NaN the entries are passed on as they are: *norm says so.  max_norm >= 0.
 */
size_t sigtrain_clip_workspace_bytes(int64_t n);
int sigtrain_grad_norm(const void* const* grads, const int64_t* counts, const int* dts, int64_t n, double* norm, void* ws,
                       size_t ws_bytes, void* stream);
int sigtrain_clip(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n,
                  double max_norm, double* norm, void* ws, size_t ws_bytes, void* stream);

/* Diagnostics: human-readable launch plan of a call, as sigkernel_describe.  op: 0 embed_fwd, 1 embed_bwd, 2 entropy_fwd, 3 entropy_bwd;
 * n: count or T. */
int sigtrain_describe(int op, int64_t n, int64_t V, int64_t D, st_dtype dt, size_t ws_bytes, char* out, size_t out_bytes);

#ifdef __cplusplus
}
#endif
#endif /* SIGKERNEL_SIGTRAIN_H */
