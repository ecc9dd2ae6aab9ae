// C-ABI host code of the operators around the products of routed rows: the layer of
// experts for a few rows, log probabilities of tokens and their gradient, the AdamW
// step (declarations in include/hwr_ops.h).
#include <math.h>

#include <algorithm>

#include "ops_context.cuh"

// ---- a layer of experts ----------------------------------------------------------

static hwr_status check_experts(hwr_ops *c, const hwr_experts *e, const void *y, int64_t y_ld) {
    if (!e) return fail(c, HWR_ERR_INVALID_ARG, "NULL layer");
    if (e->rows < 0 || e->groups < 1 || e->top < 1 || e->n_in < 1 || e->hidden < 1 || e->n_out < 1)
        return fail(c, HWR_ERR_INVALID_ARG, "rows %d, groups %d, top %d, widths %d, %d, %d", e->rows, e->groups, e->top,
                    e->n_in, e->hidden, e->n_out);
    if (e->dtype != HWR_BF16 && e->dtype != HWR_F16) return fail(c, HWR_ERR_DTYPE, "dtype %d", (int)e->dtype);
    if (e->activation != HWR_ACT_SILU && e->activation != HWR_ACT_GELU && e->activation != HWR_ACT_RELU)
        return fail(c, HWR_ERR_INVALID_ARG, "activation %d", (int)e->activation);
    if (e->rows > EXPERTS_MAX_ROWS || e->groups > OPS_MAX_GROUPS || e->top > EXPERTS_MAX_TOP || e->n_out > EXPERTS_MAX_OUT ||
        e->n_in > EXPERTS_MAX_WIDTH || e->hidden > EXPERTS_MAX_WIDTH)
        return fail(c, HWR_ERR_UNSUPPORTED, "rows %d (at most %d), groups %d (%d), top %d (%d), widths %d, %d (%d), %d (%d)",
                    e->rows, EXPERTS_MAX_ROWS, e->groups, OPS_MAX_GROUPS, e->top, EXPERTS_MAX_TOP, e->n_in, e->hidden,
                    EXPERTS_MAX_WIDTH, e->n_out, EXPERTS_MAX_OUT);
    if (e->rows == 0) return HWR_OK;
    if (!e->x || !e->w_in || !e->w_out || !y) return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    if (e->scores) {
        if (e->top > e->groups) return fail(c, HWR_ERR_INVALID_ARG, "top %d of %d groups", e->top, e->groups);
        if (e->scores_ld < e->groups)
            return fail(c, HWR_ERR_INVALID_ARG, "scores_ld %lld < %d", (long long)e->scores_ld, e->groups);
    } else if (!e->choice || !e->gates) {
        return fail(c, HWR_ERR_INVALID_ARG, "neither scores nor choice and gates");
    }
    if (((uintptr_t)e->x | (uintptr_t)e->w_in | (uintptr_t)e->w_out | (uintptr_t)y) & 1)
        return fail(c, HWR_ERR_INVALID_ARG, "an array is not aligned to its elements");
    if (((uintptr_t)e->scores | (uintptr_t)e->choice | (uintptr_t)e->gates) & 3)
        return fail(c, HWR_ERR_INVALID_ARG, "scores, choice or gates are not aligned to their elements");
    const int64_t wide = e->gated ? 2 * (int64_t)e->hidden : e->hidden;
    if (e->x_ld < e->n_in || e->w_in_ld < e->n_in || e->w_out_ld < e->hidden || y_ld < e->n_out)
        return fail(c, HWR_ERR_INVALID_ARG, "a leading dimension is shorter than its rows");
    if (e->groups > 1 && (e->w_in_group < (wide - 1) * e->w_in_ld + e->n_in ||
                          e->w_out_group < (e->n_out - 1) * e->w_out_ld + e->hidden))
        return fail(c, HWR_ERR_INVALID_ARG, "groups of weights overlap");
    return HWR_OK;
}

// Matrices [groups][rows][width] in boxes of 64 columns x 8 rows, cols / 64 of them side by
// side; false where they cannot be mapped so.
static bool map_weights(WeightMaps *m, bool f16, const void *w, int64_t ld, int64_t z, int64_t rows, int width, int groups,
                        int cols) {
    memset(m, 0, sizeof *m);
    if (((uintptr_t)w & 15) || ld % 8 || (groups > 1 && z % 8)) return false;
    const int whole = width / 64, steps = (width + cols - 1) / cols, last = whole - (steps - 1) * (cols / 64);
    const auto map = [&](CUtensorMap *to, int inner, int blocks, int of_box) {
        const cuuint64_t dims[4] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)blocks, (cuuint64_t)groups};
        const cuuint64_t strides[3] = {(cuuint64_t)ld * 2, 128, (cuuint64_t)(groups > 1 ? z : ld * rows) * 2};
        const cuuint32_t box[4] = {64, 8, (cuuint32_t)of_box, 1}, one[4] = {1, 1, 1, 1};
        return g_encode(to, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(w),
                        dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (width % 64 == 0) return map(&m->whole, 64, whole, cols / 64);
    // (a map that no step uses is left out)
    return (steps == 1 || map(&m->whole, 64, whole, cols / 64)) && (last == 0 || map(&m->last, 64, whole, last)) &&
           map(&m->tail, width, 1, 1);
}

extern "C" hwr_status hwr_expert_layer(hwr_ops *c, const hwr_experts *e, void *y, int64_t y_ld) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_expert_layer");
    OK(ready(c));
    OK(check_experts(c, e, y, y_ld));
    if (e->rows == 0) return HWR_OK;
    Experts p;
    p.rows = e->rows;
    p.groups = e->groups;
    p.top = e->top;
    p.n_in = e->n_in;
    p.hidden = e->hidden;
    p.n_out = e->n_out;
    p.gated = e->gated != 0;
    p.act = e->activation;
    p.over_all = e->over_all != 0;
    p.x = (const uint16_t *)e->x;
    p.x_ld = e->x_ld;
    p.w_in = (const uint16_t *)e->w_in;
    p.w_in_ld = e->w_in_ld;
    p.w_in_z = e->w_in_group;
    p.w_out = (const uint16_t *)e->w_out;
    p.w_out_ld = e->w_out_ld;
    p.w_out_z = e->w_out_group;
    p.scores = e->scores;
    p.scores_ld = e->scores_ld;
    p.choice = e->choice;
    p.gates = e->gates;
    p.y = (uint16_t *)y;
    p.y_ld = y_ld;
    p.h_ld = (e->hidden + 7) / 8 * 8;
    p.splits = expert_splits(e->hidden);
    const bool whole = e->top == 1 && p.splits == 1;
    const size_t pairs = (size_t)e->rows * e->top, term = e->dtype == HWR_F16 ? 4 : 2;
    const size_t h = (pairs * p.h_ld * expert_terms(e->dtype == HWR_F16) * term + 1023) / 1024 * 1024;
    const size_t used = (expert_tables(e->rows, e->top) + 16 + 1023) / 1024 * 1024;
    OK(reserve(c, h + used + (whole ? 0 : pairs * p.splits * p.n_out * 4)));
    p.h = c->ws;
    p.used_splits = (int32_t *)(c->ws + h);
    p.tables = c->ws + h + 16;
    p.part = (float *)(c->ws + h + used);
    p.status = c->status_d;
    p.test_stall = c->test_stall;
    const bool f16 = e->dtype == HWR_F16;
    ExpertMaps m;
    expert_plan(p, f16, &m);
    // (rows of x are not filled up behind their last eight columns, those of h are with zeros)
    m.in_boxes = e->n_in % 8 == 0 && map_weights(&m.in, f16, e->w_in, e->w_in_ld, e->w_in_group,
                                                 e->gated ? 2 * (int64_t)e->hidden : e->hidden, e->n_in, e->groups, m.in_cols);
    m.out_boxes = map_weights(&m.out, f16, e->w_out, e->w_out_ld, e->w_out_group, e->n_out, e->hidden, e->groups, m.out_cols);
    CK(c, launch_experts(p, m, f16, c->nsm, c->stream), "expert kernels");
    return HWR_OK;
}

// ---- rows of logits -------------------------------------------------------------------

static hwr_status check_logits(hwr_ops *c, const hwr_logits *l) {
    if (!l) return fail(c, HWR_ERR_INVALID_ARG, "NULL logits");
    if (l->rows < 0 || l->vocab < 1) return fail(c, HWR_ERR_INVALID_ARG, "rows %d, vocab %d", l->rows, l->vocab);
    if (l->dtype != HWR_F32 && l->dtype != HWR_BF16 && l->dtype != HWR_F16)
        return fail(c, HWR_ERR_DTYPE, "dtype %d", (int)l->dtype);
    if (l->rows == 0) return HWR_OK;
    if (!l->logits) return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    if (l->ld < l->vocab) return fail(c, HWR_ERR_INVALID_ARG, "ld %lld < %d", (long long)l->ld, l->vocab);
    if ((uintptr_t)l->logits & (l->dtype == HWR_F32 ? 3 : 1) || (uintptr_t)l->token & 3)
        return fail(c, HWR_ERR_INVALID_ARG, "logits or token are not aligned to their elements");
    return HWR_OK;
}

extern "C" hwr_status hwr_token_logprobs(hwr_ops *c, const hwr_logits *l, int32_t top, float *logprob, float *entropy,
                                         float *stats, int32_t *top_token, float *top_logprob) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_token_logprobs");
    OK(ready(c));
    OK(check_logits(c, l));
    if (top < 0 || top > l->vocab) return fail(c, HWR_ERR_INVALID_ARG, "top %d of %d", top, l->vocab);
    if (top > TOKENS_MAX_TOP) return fail(c, HWR_ERR_UNSUPPORTED, "top %d > %d", top, TOKENS_MAX_TOP);
    if (l->rows == 0) return HWR_OK;
    if (!logprob || !entropy || !stats || (top && (!top_token || !top_logprob)))
        return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    TokenRows p;
    p.rows = l->rows;
    p.vocab = l->vocab;
    p.top = top;
    p.logits = l->logits;
    p.ld = l->ld;
    p.token = l->token;
    p.logprob = logprob;
    p.entropy = entropy;
    p.stats = stats;
    p.top_token = top_token;
    p.top_logprob = top_logprob;
    p.splits = token_splits(l->rows, l->vocab, l->dtype, top > 0, c->nsm);
    if (l->rows > ARRIVALS_STEP - ARRIVALS_ROWS) p.splits = 1;
    if (p.splits > 1) OK(reserve(c, (size_t)l->rows * p.splits * sizeof(TokenPart)));
    p.part = (TokenPart *)c->ws;
    p.arrivals = c->arrivals + ARRIVALS_ROWS;
    CK(c, launch_token_rows(p, l->dtype, c->nsm, c->stream), "token kernel");
    return HWR_OK;
}

extern "C" hwr_status hwr_token_logprobs_backward(hwr_ops *c, const hwr_logits *l, const float *entropy,
                                                  const float *stats, const float *dlogprob, const float *dentropy,
                                                  void *dlogits, int64_t dlogits_ld) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_token_logprobs_backward");
    OK(ready(c));
    OK(check_logits(c, l));
    if (l->rows == 0) return HWR_OK;
    if (!entropy || !stats || !dlogits) return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    if (dlogits_ld < l->vocab) return fail(c, HWR_ERR_INVALID_ARG, "dlogits_ld %lld < %d", (long long)dlogits_ld, l->vocab);
    if ((uintptr_t)dlogits & (l->dtype == HWR_F32 ? 3 : 1))
        return fail(c, HWR_ERR_INVALID_ARG, "dlogits is not aligned to its elements");
    if (dlogits == l->logits && dlogits_ld != l->ld)
        return fail(c, HWR_ERR_INVALID_ARG, "dlogits in the logits' place with another leading dimension");
    TokenGrad p;
    p.rows = l->rows;
    p.vocab = l->vocab;
    p.splits = 1;
    p.logits = l->logits;
    p.ld = l->ld;
    p.token = l->token;
    p.stats = stats;
    p.entropy = entropy;
    p.da = dlogprob;
    p.db = dentropy;
    p.out = dlogits;
    p.out_ld = dlogits_ld;
    CK(c, launch_token_grad(p, l->dtype, c->nsm, c->stream), "token gradient kernel");
    return HWR_OK;
}

// ---- the optimizer's step ----------------------------------------------------------------

// What a step writes has to lie nowhere twice: blocks take their elements in any order.
static hwr_status check_apart(hwr_ops *c, int32_t n, const hwr_adamw_tensor *tensors, int32_t bits, const int32_t *step) {
    struct Range {
        uintptr_t begin, end;
    };
    Range *all = new (std::nothrow) Range[6 * (size_t)n + 1];
    if (!all) return fail(c, HWR_ERR_OOM, "host allocation failed");
    size_t k = 0;
    const auto add = [&](const void *p, int64_t bytes) {
        if (p && bytes) all[k++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes};
    };
    add(step, 4);
    for (int i = 0; i < n; ++i) {
        const hwr_adamw_tensor &t = tensors[i];
        add(t.param, t.n * 4);
        add(t.copy, t.n * 2);
        add(t.m, t.n * (bits / 8));
        add(t.v, t.n * (bits / 8));
        if (bits == 32) continue;
        add(t.m_scale, (t.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK * 4);
        add(t.v_scale, (t.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK * 4);
    }
    std::sort(all, all + k, [](const Range &a, const Range &b) { return a.begin < b.begin; });
    bool apart = true;
    for (size_t i = 1; i < k; ++i) apart = apart && all[i - 1].end <= all[i].begin;
    delete[] all;
    return apart ? HWR_OK : fail(c, HWR_ERR_INVALID_ARG, "tensors overlap");
}

extern "C" hwr_status hwr_adamw_create(hwr_ops *c, int32_t n, const hwr_adamw_tensor *tensors, int32_t bits,
                                       int32_t *step, hwr_adamw **out) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_adamw_create");
    if (!out) return fail(c, HWR_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    OK(ready(c));
    bool captured;
    OK(capturing(c, &captured));
    if (captured) return fail(c, HWR_ERR_UNSUPPORTED, "an optimizer cannot be made during a stream capture");
    if (n < 0 || (n && !tensors) || !step || (uintptr_t)step & 3)
        return fail(c, HWR_ERR_INVALID_ARG, "n %d, or a NULL or unaligned array", n);
    if (bits != 8 && bits != 32) return fail(c, HWR_ERR_INVALID_ARG, "moments of %d bits", bits);
    int64_t chunks = 0;
    for (int i = 0; i < n; ++i) {
        const hwr_adamw_tensor &t = tensors[i];
        if (t.n < 0 || (t.n && (!t.param || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale)))))
            return fail(c, HWR_ERR_INVALID_ARG, "tensor %d: n %lld or a NULL array", i, (long long)t.n);
        if (t.copy && t.copy_dtype != HWR_BF16 && t.copy_dtype != HWR_F16)
            return fail(c, HWR_ERR_DTYPE, "tensor %d: copy of dtype %d", i, (int)t.copy_dtype);
        const uintptr_t words = (uintptr_t)t.param | (uintptr_t)t.m_scale | (uintptr_t)t.v_scale |
                                (bits == 32 ? (uintptr_t)t.m | (uintptr_t)t.v : 0);
        if (words & 3 || (uintptr_t)t.copy & 1)
            return fail(c, HWR_ERR_INVALID_ARG, "tensor %d is not aligned to its elements", i);
        chunks += t.n > INT64_MAX / 2 ? INT32_MAX : (t.n + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
        if (chunks >= INT32_MAX) return fail(c, HWR_ERR_UNSUPPORTED, "too many elements");
    }
    OK(check_apart(c, n, tensors, bits, step));
    hwr_adamw *o = new (std::nothrow) hwr_adamw;
    const size_t bytes = n * sizeof(AdamWTensor) + (chunks ? chunks : 1) * sizeof(AdamWChunk);
    char *host = new (std::nothrow) char[bytes];
    if (o) o->chunk0 = new (std::nothrow) int[n + 1];
    hwr_status s = o && host && o->chunk0 ? HWR_OK : fail(c, HWR_ERR_OOM, "host allocation failed");
    char *device = nullptr;
    if (s == HWR_OK) s = alloc(c, &device, bytes);
    if (s == HWR_OK) {
        o->tensors = (AdamWTensor *)device;
        o->table = (AdamWChunk *)(device + n * sizeof(AdamWTensor));
        o->n = n;
        o->bits = bits;
        o->step = step;
        int at = 0;
        for (int i = 0; i < n; ++i) {
            const hwr_adamw_tensor &t = tensors[i];
            AdamWTensor d;
            d.param = (float *)t.param;
            d.copy = t.copy;
            d.m = t.m;
            d.v = t.v;
            d.m_scale = t.m_scale;
            d.v_scale = t.v_scale;
            d.n = t.n;
            d.copy_dtype = t.copy_dtype;
            d.aligned = (((uintptr_t)t.param | (uintptr_t)t.copy | (uintptr_t)t.m | (uintptr_t)t.v) & 15) == 0;
            memcpy(host + i * sizeof d, &d, sizeof d);
            o->chunk0[i] = at;
            for (int64_t k = 0; k * ADAMW_CHUNK < t.n; ++k, ++at) {
                const AdamWChunk chunk = {i, (int32_t)k};
                memcpy(host + n * sizeof d + at * sizeof chunk, &chunk, sizeof chunk);
            }
        }
        o->chunk0[n] = at;
        cudaError_t e = cudaMemcpyAsync(device, host, bytes, cudaMemcpyHostToDevice, c->stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize(c->stream);
        if (e != cudaSuccess) s = cuda_fail(c, e, "optimizer table");
    }
    delete[] host;
    if (s != HWR_OK) {
        const Unwatched memory;
        cudaFree(device);
        if (o) delete[] o->chunk0;
        delete o;
        return s;
    }
    o->next = c->optimizers;
    c->optimizers = o;
    *out = o;
    return HWR_OK;
}

// Whether an optimizer is one of the context's.
static bool owned(const hwr_ops *c, const hwr_adamw *o) {
    const hwr_adamw *at = c->optimizers;
    while (at && at != o) at = at->next;
    return at;
}

extern "C" hwr_status hwr_adamw_step(hwr_ops *c, const hwr_adamw *o, const hwr_adamw_options *a,
                                     const void *const *grads, const hwr_dtype *dtypes) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_adamw_step");
    OK(ready(c));
    if (!o || !a) return fail(c, HWR_ERR_INVALID_ARG, "NULL argument");
    if (!owned(c, o)) return fail(c, HWR_ERR_INVALID_ARG, "not an optimizer of this context");
    if (o->n && (!grads || !dtypes)) return fail(c, HWR_ERR_INVALID_ARG, "NULL argument");
    if (!(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1))
        return fail(c, HWR_ERR_INVALID_ARG, "betas %g, %g", a->beta1, a->beta2);
    if (!(a->eps >= 0) || !(a->weight_decay >= 0) || (!a->lr_device && !(a->lr >= 0)))
        return fail(c, HWR_ERR_INVALID_ARG, "lr %g, eps %g, weight decay %g", a->lr, a->eps, a->weight_decay);
    if (a->norm && !(a->max_norm > 0)) return fail(c, HWR_ERR_INVALID_ARG, "max_norm %g", a->max_norm);
    if (((uintptr_t)a->norm | (uintptr_t)a->lr_device) & 3)
        return fail(c, HWR_ERR_INVALID_ARG, "norm or lr is not aligned to its elements");
    for (int i = 0; i < o->n; ++i) {
        if (!grads[i]) continue;
        if (dtypes[i] != HWR_F32 && dtypes[i] != HWR_BF16 && dtypes[i] != HWR_F16)
            return fail(c, HWR_ERR_DTYPE, "gradient %d: dtype %d", i, (int)dtypes[i]);
        if ((uintptr_t)grads[i] & (dtypes[i] == HWR_F32 ? 3 : 1))
            return fail(c, HWR_ERR_INVALID_ARG, "gradient %d is not aligned to its elements", i);
    }
    bool captured;
    OK(capturing(c, &captured));
    o->held = o->held || captured;
    AdamWStep p;
    p.arrivals = c->arrivals + ARRIVALS_STEP;
    p.step = o->step;
    p.lr = a->lr_device;
    p.norm = a->norm;
    p.rate = (float)a->lr;
    p.max_norm = a->norm ? a->max_norm : 1.f;
    p.b1 = (float)a->beta1;
    p.b2 = (float)a->beta2;
    p.one_b1 = (float)(1 - a->beta1);
    p.one_b2 = (float)(1 - a->beta2);
    p.log_b1 = (float)log(a->beta1);           // (-inf for 0: no correction)
    p.log_b2 = (float)log(a->beta2);
    p.eps = (float)a->eps;
    p.decay = (float)a->weight_decay;
    p.seed = a->seed;
    const int launches = (o->n + ADAMW_TABLE - 1) / ADAMW_TABLE;
    p.blocks = 0;
    for (int k = 0; k < launches || k == 0; ++k) {
        const int t0 = k * ADAMW_TABLE, t1 = o->n < t0 + ADAMW_TABLE ? o->n : t0 + ADAMW_TABLE;
        p.blocks += adamw_grid(o->chunk0[t1] - o->chunk0[t0], o->bits, c->nsm);
    }
    for (int k = 0; k < launches || k == 0; ++k) {
        const int t0 = k * ADAMW_TABLE, t1 = o->n < t0 + ADAMW_TABLE ? o->n : t0 + ADAMW_TABLE;
        p.tensors = o->tensors;
        p.table = o->table + o->chunk0[t0];
        p.chunks = o->chunk0[t1] - o->chunk0[t0];
        p.tensor0 = t0;
        for (int i = t0; i < t1; ++i) {
            p.grad[i - t0] = grads[i];
            p.dtype[i - t0] = (uint8_t)dtypes[i];
        }
        const cudaError_t e = c->fail_launch > 0 && ++c->launches == c->fail_launch
                                  ? cudaErrorMemoryAllocation
                                  : launch_adamw(p, o->bits, adamw_grid(p.chunks, o->bits, c->nsm), c->stream);
        // (whatever the reason: some tensors have made the step and others not, and the blocks'
        // count is left between)
        if (e != cudaSuccess && k > 0)
            return fail(c, HWR_ERR_CUDA, "optimizer kernel, after others of the step: %s", cudaGetErrorString(e));
        CK(c, e, "optimizer kernel");
    }
    return HWR_OK;
}

extern "C" hwr_status hwr_adamw_destroy(hwr_ops *c, hwr_adamw *o) {
    if (!o) return HWR_OK;
    if (!c) return HWR_ERR_INVALID_ARG;
    if (!owned(c, o)) return fail(c, HWR_ERR_INVALID_ARG, "not an optimizer of this context");
    bool captured;
    OK(capturing(c, &captured));
    if (captured || o->held) {          // (during a capture nothing is waited for or freed)
        OK(retire(c, o->tensors));
    } else {
        const Unwatched memory;
        cudaStreamSynchronize(c->stream);
        cudaFree(o->tensors);
        cudaGetLastError();
    }
    hwr_adamw **at = &c->optimizers;
    while (*at != o) at = &(*at)->next;
    *at = o->next;
    delete[] o->chunk0;
    delete o;
    return HWR_OK;
}
