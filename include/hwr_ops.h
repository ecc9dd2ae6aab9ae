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
 *   hwr_adamw_step          the optimizer's step over many tensors at once
 *   hwr_expert_layer        a whole layer of experts for the few rows of a decode step
 *   hwr_token_logprobs      log probabilities, entropies and best alternatives of the
 *                           tokens of an answer, and (_backward) their gradient
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
 *     (weights that are read in place are the terms with n_out (n_in + 8) less),
 *       hwr_expert_layer  4,096 + 8 rows top (hidden + 9 + 8 n_out)
 *       hwr_token_logprobs  2,176 for each of the device's SMs
 *     and the other calls none.
 *   - Stream capture: calls can be captured into graphs.  A call that would have
 *     to grow the workspace then is refused (UNSUPPORTED, nothing is queued, the
 *     context stays usable): make a call of the same sizes before, or reserve.
 *     So are hwr_ops_synchronize, hwr_gradients_create and hwr_adamw_create.  Workspace,
 *     lists of gradients and optimizers' tables that a captured call uses are kept until
 *     hwr_ops_destroy, also when
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
#define HWR_EXPERTS_MAX_ROWS 128    /* rows of a layer of experts (beyond: dispatch and grouped products) */
#define HWR_EXPERTS_MAX_TOP 16      /* choices of a row */
#define HWR_EXPERTS_MAX_OUT 65536   /* width of its result, */
#define HWR_EXPERTS_MAX_WIDTH 262144    /* of its input and of the experts' hidden layer */
#define HWR_TOKENS_MAX_TOP 32       /* alternatives of a token */
#define HWR_ADAMW_BLOCK 256         /* elements that share a scale where moments have 8 bits */

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

/*
 * One AdamW step over many tensors.  With g the gradients (times min(1, max_norm /
 * (norm + 1e-6)) where a norm is given), t the step's number, from 1:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   param -= lr (weight_decay param + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
 * Parameters are fp32; `copy`, where it is set, gets them rounded to copy_dtype (HWR_BF16
 * or HWR_F16), for the products.  Moments are fp32, or (bits 8) m and sqrt(v) as e4m3
 * values times a power of two of each HWR_ADAMW_BLOCK elements in m_scale and v_scale
 * [(n + HWR_ADAMW_BLOCK - 1) / HWR_ADAMW_BLOCK].  They are rounded up or down by 16 bits
 * of a hash of seed, t, the tensor's number and the element's: their expectation is the
 * value, down to 2^-17 of their block's largest; the same call gives the same bits.  A
 * positive sqrt(v) does not become 0.  A moment that is not finite makes its block NaN.
 * All zeros (and scale 0) is the state before the first step.
 */
typedef struct {
    float *param;             /* [n] */
    void *copy;               /* [n], may be NULL */
    hwr_dtype copy_dtype;
    void *m, *v;              /* [n] fp32, or bytes */
    float *m_scale, *v_scale; /* bits 8 only */
    int64_t n;
} hwr_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    const float *lr_device;   /* device, one float in lr's place; may be NULL */
    const float *norm;        /* device, one float (of hwr_clip_gradients, max_norm +inf); may be NULL */
    float max_norm;           /* with norm: > 0 */
    uint32_t seed;
} hwr_adamw_options;

/* An optimizer over tensors that stay where they are (its table is laid out in device
 * memory once; synchronises the stream).  `step`, device, one int32: the number of steps
 * done, which each step counts up, so that captured steps go on counting.  It and the
 * tensors are the caller's, to be saved and restored; they go on existing as long as the
 * optimizer, and none of them overlaps another (INVALID_ARG).  An optimizer goes with its context, if not before. */
typedef struct hwr_adamw hwr_adamw;
hwr_status hwr_adamw_create(hwr_ops *ops, int32_t n, const hwr_adamw_tensor *tensors, int32_t bits,
                            int32_t *step, hwr_adamw **out);
/* grads, dtypes: host arrays of a device pointer (NULL: that tensor is left as it is) and
 * a type (any of hwr_dtype) for each tensor.  A step whose norm is not finite changes
 * nothing, and does not count. */
hwr_status hwr_adamw_step(hwr_ops *ops, const hwr_adamw *optimizer, const hwr_adamw_options *options,
                          const void *const *grads, const hwr_dtype *dtypes);
hwr_status hwr_adamw_destroy(hwr_ops *ops, hwr_adamw *optimizer); /* synchronises; NULL is fine */

/*
 * A layer of experts for a few rows:
 *   y[t] = sum over j < top of p[t][j] W_out[e] h,   e = the j-th choice of row t,
 *   h = act(W_in[e] x[t])                                       (gated = 0), or
 *   h = act(W_in[e][0 .. hidden) x[t]) * (W_in[e][hidden ..) x[t])   (gated)
 * With scores [rows][groups], the choices are the `top` largest scores of a row (ties to
 * the lowest index; NaN and -inf are never chosen), and p the softmax over them, or
 * (over_all) over all of the row's scores, NaN where one of those is.  Without, they are
 * choice and gates [rows][top]; a choice outside [0, groups) is none, the same one may come
 * twice.  A row without a choice gets zeros.  Experts that no row chooses are not read.
 * h is summed in fp32 and enters the second product whole, as three bf16 terms (from
 * 2^-110 on; in fp16 layers as two, within 2^-20 of it, at any magnitude); y is rounded once.
 */
typedef enum { HWR_ACT_SILU = 0, HWR_ACT_GELU = 1 /* u Phi(u) */, HWR_ACT_RELU = 2 } hwr_activation;
typedef struct {
    int32_t rows, groups, top;
    int32_t n_in, hidden, n_out;
    hwr_dtype dtype;          /* HWR_BF16 or HWR_F16: x, weights and y */
    hwr_activation activation;
    int32_t gated, over_all;
    const void *x;            /* [rows][n_in] */
    int64_t x_ld;
    const void *w_in;         /* [groups][gated ? 2 hidden : hidden][n_in] */
    int64_t w_in_ld, w_in_group;
    const void *w_out;        /* [groups][n_out][hidden] */
    int64_t w_out_ld, w_out_group;
    const float *scores;      /* may be NULL */
    int64_t scores_ld;
    const int32_t *choice;
    const float *gates;
} hwr_experts;
hwr_status hwr_expert_layer(hwr_ops *ops, const hwr_experts *layer, void *y, int64_t y_ld);

/*
 * Rows of logits z and a token of each; with q = softmax(z):
 *   logprob [rows]   log q[token]; 0 for a token outside [0, vocab) or no tokens at all
 *   entropy [rows]   -sum of q log q
 *   stats [rows][2]  the largest logit, and the log of the sum of exp(z - largest)
 *   top_token, top_logprob [rows][top]  the most probable tokens (ties to the lowest
 *                    index, NaN last) and their log probabilities
 * A logit of -inf has probability 0 and adds nothing.  A row of nothing else has
 * probabilities 0: log probabilities -inf, entropy 0.  A NaN or +inf makes its row's
 * results NaN (top_token apart).
 */
typedef struct {
    int32_t rows, vocab;
    hwr_dtype dtype;          /* HWR_F32, HWR_BF16 or HWR_F16 */
    const void *logits;
    int64_t ld;
    const int32_t *token;     /* [rows], may be NULL */
} hwr_logits;
hwr_status hwr_token_logprobs(hwr_ops *ops, const hwr_logits *logits, int32_t top, float *logprob,
                              float *entropy, float *stats, int32_t *top_token, float *top_logprob);
/* The gradient of sum over rows of dlogprob logprob + dentropy entropy (either may be
 * NULL: zeros) with respect to the logits, in their type: with a and b a row's two,
 *   dz[v] = a (1[v = token] - q[v]) - b q[v] (log q[v] + entropy),
 * a = 0 for a row without a token; zeros for a row of -inf.  entropy and stats: of
 * hwr_token_logprobs.  dlogits may be the logits themselves. */
hwr_status hwr_token_logprobs_backward(hwr_ops *ops, const hwr_logits *logits, const float *entropy,
                                       const float *stats, const float *dlogprob, const float *dentropy,
                                       void *dlogits, int64_t dlogits_ld);

#ifdef __cplusplus
}
#endif

#endif /* HWR_OPS_H */
