/*
 * hwr_ops.h -- operators that follow a routing decision (libhwr, GB300).
 *
 * hwr_route_batch (hwr.h) answers with one deployment per query: chosen[Q],
 * -1 where a query has none.  Where the deployments share the GPU -- experts
 * with weights of their own, or low-rank adapters of one base model -- these
 * calls carry the answer out, and train what it chose:
 *   hwr_dispatch            the rows of each choice together (a plan)
 *   hwr_grouped_forward     y[t] = W[c] x[t],   c = the choice of row t
 *   hwr_grouped_backward    dx[t] = W[c]^T dy[t],  dW[g] = sum dy[t] x[t]^T
 *   hwr_adapter_forward     y[t] = W x[t] + scale[c] B[c] (A[c] x[t])
 *   hwr_adapter_backward    dx, dA, dB of the same (W is left as it is)
 *   hwr_clip_gradients      global norm of many tensors, and clipping
 *   hwr_gradients_clip      the same over a list that is laid out once
 *
 * Conventions (those of hwr.h, and)
 *   - A context of its own (hwr_ops): one CUDA stream, one workspace.  Calls
 *     are queued on the stream and return without synchronising it; they are
 *     not thread-safe on one context.
 *   - Every array is device memory unless said otherwise.  A call neither
 *     keeps nor changes its inputs.  Outputs may not overlap inputs, except
 *     where hwr_clip_gradients says so.
 *   - Rows are row-major with a leading dimension in elements: row t of x
 *     begins at x + t * x_ld.  Weights are [out][in], group g at w + g *
 *     w_group, row n at + n * w_ld.  Any pointer aligned to its element and any
 *     leading dimension >= the row's length is accepted.  A weight that is not
 *     on a 16-byte boundary, or whose strides are not whole 16-byte units, is
 *     first copied to the workspace with padded rows (an extra read and write of
 *     it, and that much workspace).  The rows of x and dy are copied there by
 *     group where that is cheaper than picking each by its index, in backward
 *     calls with weight gradients, and where they are not so aligned.
 *   - Sums run in fp32 on the tensor cores; each output is rounded once.
 *   - Results do not depend on timing: the same call gives the same bits.
 *   - The workspace grows (cudaMalloc) when a call needs more than any call
 *     before; hwr_ops_reserve does that ahead of time.  No call needs more bytes
 *     than, with P = rows + 15 min(rows, groups), n_in + n_out = S, rank r,
 *       hwr_dispatch   5 (rows / 4,096 + 16) (groups + 1)
 *       hwr_grouped_*  16,384 + 4 groups + 2 P (S + 18)
 *                      + 2 groups n_out (n_in + 8)
 *       hwr_adapter_*  16,384 + 12 groups + 2 P (S + 18) + 12 P (r + 63)
 *                      + 2 n_out (n_in + 8) + 6 groups (r + 63) (S + 16)
 *       hwr_clip_gradients  8 bytes for each 1,024 of the gradients' bytes and 32
 *                      for each gradient
 *     (weights that are read in place are the terms with n_out (n_in + 8) less).
 *   - Stream capture: calls can be captured into graphs.  A call that would have
 *     to grow the workspace then is refused (UNSUPPORTED, nothing is queued, the
 *     context stays usable): make a call of the same sizes before, or reserve.
 *     So are hwr_ops_synchronize and hwr_gradients_create.  Workspace and lists of
 *     gradients that a captured call uses are kept until hwr_ops_destroy, also when
 *     a later call takes a larger block; the context outlives its graphs.  A replay
 *     uses the context's workspace, partial sums and counters as an eager call
 *     does: order it with the context's other work (the same stream, or
 *     hwr_ops_after / hwr_ops_before); two of them at a time spoil each other.
 *   - After HWR_ERR_CUDA or HWR_ERR_TIMEOUT the context is broken (hwr.h).
 */
#ifndef HWR_OPS_H
#define HWR_OPS_H

#include "hwr.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HWR_OPS_MAX_GROUPS 1024 /* groups of one plan */
#define HWR_OPS_MAX_RANK 256    /* rank of an adapter */

typedef struct hwr_ops hwr_ops;

/* Create a context on cuda_stream (NULL: a non-blocking stream of its own) of
 * the current device, which must be current at every later call (another one:
 * INVALID_ARG, and the context stays usable).
 * Errors: INVALID_ARG, OOM, CUDA. */
hwr_status hwr_ops_create(void *cuda_stream, hwr_ops **out);
hwr_status hwr_ops_destroy(hwr_ops *ops);          /* synchronises; NULL is fine */
hwr_status hwr_ops_synchronize(hwr_ops *ops);      /* reports asynchronous failures */
const char *hwr_ops_last_error(const hwr_ops *ops); /* NULL: of hwr_ops_create */
/* Order the context's later work after what is queued on another stream now, and
 * another stream's later work after what the context has queued (for calls whose
 * arrays belong to that stream; 1 is the legacy default stream).  A context on
 * the default stream cannot follow a stream that is being captured (UNSUPPORTED).
 * hwr_ops_before orders what a context has queued that is broken by now, too.
 * Errors: INVALID_ARG, UNSUPPORTED, STATE, CUDA. */
hwr_status hwr_ops_after(hwr_ops *ops, void *cuda_stream);
hwr_status hwr_ops_before(hwr_ops *ops, void *cuda_stream);
/* Make the workspace at least `bytes` large.  Errors: INVALID_ARG, STATE, OOM, CUDA. */
hwr_status hwr_ops_reserve(hwr_ops *ops, uint64_t bytes);

/*
 * Bring the rows of each choice together.
 *   choice   [rows] int32; a value outside [0, groups) is a row without a choice
 *   offsets  [groups + 1] out: rows order[offsets[g] .. offsets[g + 1]) chose g
 *   order    [rows] out: row indices, ascending within a group; the rows
 *            without a choice follow, ascending, from offsets[groups] on
 * offsets and order are the plan of the calls below.  They read it as it is on
 * the device; a plan that did not come from this call gives wrong results, but
 * no access outside the arrays.
 * Limits: 1 <= groups <= HWR_OPS_MAX_GROUPS.  Errors: INVALID_ARG, UNSUPPORTED,
 * STATE, OOM, CUDA.
 */
hwr_status hwr_dispatch(hwr_ops *ops, int32_t rows, int32_t groups, const int32_t *choice,
                        int32_t *offsets, int32_t *order);

/* A plan and the shape of the products over it. */
typedef struct {
    int32_t rows, groups;     /* T, G */
    int32_t n_in, n_out;      /* K, N: widths of x and y */
    hwr_dtype dtype;          /* HWR_BF16 or HWR_F16: every operand and output */
    const int32_t *offsets, *order;
    const void *x;            /* [T][K] */
    int64_t x_ld;
    const void *w;            /* grouped: [G][N][K]; adapter: [N][K] */
    int64_t w_ld, w_group;    /* (w_group: grouped only) */
} hwr_rows;

/* y [T][N]; rows without a choice get zeros. */
hwr_status hwr_grouped_forward(hwr_ops *ops, const hwr_rows *r, void *y, int64_t y_ld);

/* From dy [T][N]: dx [T][K] (rows without a choice get zeros) and dw, which is
 * laid out as w (a group without rows gets zeros).  dx or dw may be NULL; x is
 * read for dw only, w for dx only. */
hwr_status hwr_grouped_backward(hwr_ops *ops, const hwr_rows *r, const void *dy, int64_t dy_ld,
                                void *dx, int64_t dx_ld, void *dw);

/* Low-rank adapters beside the shared projection r->w, contiguous:
 * a [G][rank][K], b [G][N][rank] in the rows' type, scale [G] fp32. */
typedef struct {
    int32_t rank;             /* 1 .. HWR_OPS_MAX_RANK */
    const void *a, *b;
    const float *scale;
} hwr_adapters;

/* y [T][N]; a row without a choice gets the shared projection alone.  The inner
 * product scale A x is summed in fp32 and enters the second product as two bf16
 * terms (within 2^-16, at any magnitude); of up to 16 aligned rows in fp32. */
hwr_status hwr_adapter_forward(hwr_ops *ops, const hwr_rows *r, const hwr_adapters *ad, void *y,
                               int64_t y_ld);

/* From dy [T][N]: dx [T][K], da [G][rank][K], db [G][N][rank] (contiguous; zeros
 * for an adapter without rows).  Each may be NULL.  Inner products as above; in da
 * and db two terms of the rows' type, in fp16 scaled by a power of two of each
 * adapter's own (within 2^-22 of the value, 2^-38 of the adapter's largest). */
hwr_status hwr_adapter_backward(hwr_ops *ops, const hwr_rows *r, const hwr_adapters *ad,
                                const void *dy, int64_t dy_ld, void *dx, int64_t dx_ld, void *da,
                                void *db);

/* One gradient: n elements at `in`, the clipped ones at `out` (in == out: in
 * place).  dtype HWR_F32, HWR_BF16 or HWR_F16. */
typedef struct {
    const void *in;
    void *out;
    int64_t n;
    hwr_dtype dtype;
} hwr_gradient;

/*
 * norm = sqrt(sum of squares over all tensors);
 * out = in * min(1, max_norm / (norm + 1e-6)).
 *   grads     host array of n >= 0 entries
 *   max_norm  > 0, may be +inf (nothing is scaled)
 *   norm      device, one float: the norm before clipping
 * A NaN among the gradients gives norm = NaN and NaN gradients; an infinity
 * norm = inf, zeros for the finite values and NaN for the infinite ones.
 * Squares beyond fp32's range do not overflow the norm.
 */
hwr_status hwr_clip_gradients(hwr_ops *ops, int32_t n, const hwr_gradient *grads, float max_norm,
                              float *norm);

/*
 * The same for gradients that stay where they are from step to step: create
 * lays their table out in device memory once (synchronises the stream); clip
 * reads and writes the arrays as they are at the call, which must still be
 * there.  destroy synchronises; NULL is fine.  A list goes with its context
 * (hwr_ops_destroy), if not before.
 */
typedef struct hwr_gradients hwr_gradients;
hwr_status hwr_gradients_create(hwr_ops *ops, int32_t n, const hwr_gradient *grads,
                                hwr_gradients **out);
hwr_status hwr_gradients_clip(hwr_ops *ops, const hwr_gradients *list, float max_norm, float *norm);
hwr_status hwr_gradients_destroy(hwr_ops *ops, hwr_gradients *list);

#ifdef __cplusplus
}
#endif

#endif /* HWR_OPS_H */
