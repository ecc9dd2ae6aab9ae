// C-ABI host code of the operators that follow a routing decision
// (declarations in include/hwr_ops.h): argument checks, the workspace, tensor
// maps, and the launches of each call on the context's stream.
#include <math.h>

#include "ops_context.cuh"

using namespace hwr;

extern "C" hwr_status hwr_ops_create(void *cuda_stream, hwr_ops **out) {
    if (!out) return fail(nullptr, HWR_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    hwr_ops *c = new (std::nothrow) hwr_ops;
    if (!c) return fail(nullptr, HWR_ERR_OOM, "host allocation failed");
    if (const char *e = getenv("HWR_TEST_FAIL_ALLOC")) c->fail_at = atol(e);
    if (const char *e = getenv("HWR_TEST_FAIL_LAUNCH")) c->fail_launch = atol(e);
    if (const char *e = getenv("HWR_TEST_STALL")) c->test_stall = atoi(e) != 0;
    if (const char *e = getenv("HWR_TEST_DEVICE")) c->test_device = atoi(e);
    const Unwatched memory;
    auto body = [&]() -> hwr_status {
        CK(c, cudaGetDevice(&c->device), "cudaGetDevice");
        const int dev = c->device;
        CK(c, cudaDeviceGetAttribute(&c->nsm, cudaDevAttrMultiProcessorCount, dev), "device attribute");
        if (!g_encode) {
            void *fn = nullptr;
            cudaDriverEntryPointQueryResult qr;
            CK(c, cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &qr),
               "cuTensorMapEncodeTiled");
            if (qr != cudaDriverEntryPointSuccess || !fn)
                return fail(c, HWR_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
            g_encode = (PFN_cuTensorMapEncodeTiled_v12000)fn;
        }
        CK(c, group_prepare(c->nsm, &c->ctas), "kernel attributes");
        CK(c, ops_prepare(&c->cluster), "kernel attributes");
        CK(c, experts_prepare(), "kernel attributes");
        if (getenv("HWR_TEST_SMALL_CLUSTERS")) c->cluster = 8;
        if (cuda_stream) {
            c->stream = (cudaStream_t)cuda_stream;
        } else {
            CK(c, cudaStreamCreateWithFlags(&c->stream, cudaStreamNonBlocking), "stream");
            c->own_stream = true;
        }
        CK(c, cudaEventCreateWithFlags(&c->event, cudaEventDisableTiming), "event");
        CK(c, cudaHostAlloc((void **)&c->status_h, 64, cudaHostAllocMapped), "status word");
        memset(c->status_h, 0, 64);
        CK(c, cudaHostGetDevicePointer((void **)&c->status_d, c->status_h, 0), "status word");
        OK(alloc(c, &c->part, group_part_floats(c->ctas)));
        OK(alloc(c, &c->count, c->ctas));
        OK(alloc(c, &c->sums, clip_blocks(INT64_MAX, c->nsm) + 1));
        CK(c, cudaMemsetAsync(c->sums, 0, (clip_blocks(INT64_MAX, c->nsm) + 1) * sizeof(double), c->stream), "memset");
        CK(c, cudaMemsetAsync(c->count, 0, c->ctas * sizeof(uint32_t), c->stream), "memset");
        OK(alloc(c, &c->arrivals, ARRIVALS));
        CK(c, cudaMemsetAsync(c->arrivals, 0, ARRIVALS * sizeof(uint32_t), c->stream), "memset");
        return HWR_OK;
    };
    const hwr_status s = body();
    if (s != HWR_OK) {
        g_create_error = c->err;
        hwr_ops_destroy(c);
        return s;
    }
    *out = c;
    return HWR_OK;
}

extern "C" hwr_status hwr_ops_destroy(hwr_ops *c) {
    if (!c) return HWR_OK;
    const Unwatched memory;
    if (c->stream) cudaStreamSynchronize(c->stream);
    cudaFree(c->ws);
    while (hwr_gradients *l = c->lists) {
        c->lists = l->next;
        cudaFree(l->table);
        delete l;
    }
    while (hwr_adamw *o = c->optimizers) {
        c->optimizers = o->next;
        cudaFree(o->tensors);
        delete[] o->chunk0;
        delete o;
    }
    while (Retired *r = c->retired) {
        c->retired = r->next;
        cudaFree(r->p);
        delete r;
    }
    cudaFree(c->part);
    cudaFree(c->count);
    cudaFree(c->sums);
    cudaFree(c->arrivals);
    if (c->status_h) cudaFreeHost(c->status_h);
    if (c->event) cudaEventDestroy(c->event);
    if (c->own_stream) cudaStreamDestroy(c->stream);
    cudaGetLastError();
    delete c;
    return HWR_OK;
}

extern "C" hwr_status hwr_ops_synchronize(hwr_ops *c) {
    if (!c) return HWR_ERR_INVALID_ARG;
    if (c->broken) return fail(c, HWR_ERR_STATE, "context unusable after an earlier failure");
    bool captured;
    OK(capturing(c, &captured));
    if (captured) return fail(c, HWR_ERR_UNSUPPORTED, "the stream is being captured");
    CK(c, cudaStreamSynchronize(c->stream), "synchronize");
    return alive(c);
}

extern "C" const char *hwr_ops_last_error(const hwr_ops *c) {
    return c ? c->err.c_str() : g_create_error.c_str();
}

static hwr_status order_streams(hwr_ops *c, cudaStream_t first, cudaStream_t then) {
    CK(c, cudaEventRecord(c->event, first), "event record");
    CK(c, cudaStreamWaitEvent(then, c->event, 0), "stream wait");
    return HWR_OK;
}

extern "C" hwr_status hwr_ops_after(hwr_ops *c, void *stream) {
    if (!c) return HWR_ERR_INVALID_ARG;
    OK(alive(c));
    if (!stream) return fail(c, HWR_ERR_INVALID_ARG, "NULL stream");
    if (c->stream == cudaStreamLegacy) {
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        CK(c, cudaStreamIsCapturing((cudaStream_t)stream, &capture), "capture status");
        if (capture != cudaStreamCaptureStatusNone)
            return fail(c, HWR_ERR_UNSUPPORTED, "a context on the default stream cannot take part in a stream capture");
    }
    return order_streams(c, (cudaStream_t)stream, c->stream);
}

extern "C" hwr_status hwr_ops_before(hwr_ops *c, void *stream) {
    if (!c) return HWR_ERR_INVALID_ARG;
    if (!stream) return fail(c, HWR_ERR_INVALID_ARG, "NULL stream");
    // (a broken context's work may still be running)
    const hwr_status s = alive(c), o = order_streams(c, c->stream, (cudaStream_t)stream);
    return s != HWR_OK ? s : o;
}

extern "C" hwr_status hwr_ops_reserve(hwr_ops *c, uint64_t bytes) {
    if (!c) return HWR_ERR_INVALID_ARG;
    OK(ready(c));
    return reserve(c, bytes);
}

// ---------------------------------------------------------------------------

extern "C" hwr_status hwr_dispatch(hwr_ops *c, int32_t rows, int32_t groups, const int32_t *choice,
                                   int32_t *offsets, int32_t *order) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_dispatch");
    OK(ready(c));
    if (rows < 0 || groups < 1) return fail(c, HWR_ERR_INVALID_ARG, "rows %d, groups %d", rows, groups);
    if (groups > OPS_MAX_GROUPS)
        return fail(c, HWR_ERR_UNSUPPORTED, "groups %d > %d", groups, OPS_MAX_GROUPS);
    if (!offsets || (rows && (!choice || !order))) return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    const size_t ints = dispatch_scratch_ints(rows, groups, c->nsm, c->cluster);
    OK(reserve(c, ints * 4));
    CK(c, launch_dispatch(rows, groups, choice, offsets, order, (int32_t *)c->ws, c->nsm, c->cluster, c->stream),
       "dispatch kernel");
    return HWR_OK;
}

// ---------------------------------------------------------------------------
// Operands of the products: nz matrices of rows x cols 16-bit elements.

namespace {

struct Operand {
    const void *p = nullptr;
    int64_t ld = 0, z = 0, nz = 1, rows = 0;
    int cols = 0;
    bool pad = false;
    size_t off = 0;      // of the padded copy in the workspace
};

int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
bool on16(const void *p, int64_t ld, int64_t z, int64_t nz) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && (nz == 1 || z % 8 == 0);
}

// What a call takes from the workspace, in the order it is asked for.
struct Carver {
    size_t at = 0;
    size_t take(size_t bytes) {
        const size_t o = at;
        at = (size_t)up((int64_t)(at + bytes), 1024);
        return o;
    }
    // an operand that TMA cannot read in place gets a padded copy
    Operand operand(const void *p, int64_t ld, int64_t rows, int cols, int64_t z = 0, int64_t nz = 1) {
        Operand o;
        o.p = p;
        o.ld = ld;
        o.rows = rows;
        o.cols = cols;
        o.nz = nz;
        o.z = nz > 1 ? z : 0;
        o.pad = !on16(p, ld, z, nz);
        if (o.pad) o.off = take((size_t)(nz * rows * up(cols, 8) * 2));
        return o;
    }
};

}  // namespace

static hwr_status settle(hwr_ops *c, Operand *o) {
    if (!o->pad) {
        if (o->nz == 1) o->z = up(o->ld * o->rows, 8);
        return HWR_OK;
    }
    const int64_t ld = up(o->cols, 8);
    CK(c, launch_pad(c->ws + o->off, ld, o->p, o->ld, o->z, o->nz, o->rows, o->cols, c->nsm, c->stream),
       "padding copy");
    o->p = c->ws + o->off;
    o->ld = ld;
    o->z = ld * o->rows;
    return HWR_OK;
}

// A map over nz matrices: boxes of box0 columns (64, 32 or 16: swizzled over their
// 128, 64 or 32 bytes) x box1 rows.
static hwr_status encode(hwr_ops *c, CUtensorMap *m, bool f16, const Operand &o, int box0, int box1) {
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.nz};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.z * 2};
    const cuuint32_t box[3] = {(cuuint32_t)box0, (cuuint32_t)box1, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = g_encode(
        m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(o.p),
        dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
        box0 == 64   ? CU_TENSOR_MAP_SWIZZLE_128B
        : box0 == 32 ? CU_TENSOR_MAP_SWIZZLE_64B
                     : CU_TENSOR_MAP_SWIZZLE_32B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(c, HWR_ERR_INVALID_ARG, "operand of %lld x %lld x %d (stride %lld) cannot be mapped",
                    (long long)o.nz, (long long)o.rows, o.cols, (long long)o.ld);
    return HWR_OK;
}

// Values of the widest store that the rows of the result are aligned to.
static int vec_of(const void *p, int64_t ld, int64_t z) {
    for (int v = 8; v > 1; v /= 2)
        if ((uintptr_t)p % (2 * v) == 0 && ld % v == 0 && z % v == 0) return v;
    return 1;
}

// What the products of a call share: the plan and the rows of its inputs, by
// place (copied to the workspace) or where the caller has them.
struct Rows {
    GroupPlan plan;
    bool sorted = false;
    Operand x, dy;
    size_t offsets_off = 0, order_off = 0;     // padded plan
    size_t peak_off = 0;                       // words that are zeroed beside the copy
    int peaks = 0;
};

// Whether a product picks its rows by index, or they are copied by place first.
// Picking saves the copy (its start and the rows' bytes, in and out) and costs each
// tile: four of the eight epilogue warps pick, and where rows are a shared product's
// A side, all pairs' loads.  Fitted on 130 shapes timed either way, this function
// returning the one or the other throughout.  In us, each with its dispatch: 10,188 rows
// of 3,136 columns to 512 over 12 experts, 59 picked, 77 copied; 10,013 of 512 to 6,528,
// 122 and 95; 65,536 of 1,024 to 2,048 over 64, 258 and 259; through 5 adapters of rank 16
// 950 of 4,608 to 1,984, 63 and 66; through 8 7,354 of 4,352 to 4,544, 242 and 235.
// Four warps write a tile whose results are aligned to less than 16 bytes (vec: values
// of a store) slowly: 1,000 rows of 512 columns to 1,028 over 4 experts 29 us picked, 24
// copied.  (Where the two are near, the rule may miss: 300 of these rows are picked, 23
// and 21; so are 512 rows beside 4,096 x 4,096 with 12 fp16 adapters of rank 64, 79 and 71.)
static bool picks_rows(const hwr_ops *c, const hwr_rows *r, int k, int n, bool shared, int vec) {
    const float rows = (float)r->rows, pairs = c->ctas / 2, copy = rows * k * 4e-6f / 6;
    const float tiles = rows * ((n + GP_TILE - 1) / GP_TILE) / (GP_TILE * pairs);      // a pair
    if (!shared) {
        if (vec == 8) return 2.6f * tiles <= 0.8f + 1.4f * copy;
        const float full = rows / r->groups / GP_TILE;                                  // of a tile's columns
        return 12 * (tiles > 1 ? tiles : full < 1 ? full : 1) <= 3.5f + 1.4f * copy;
    }
    const float write = (vec == 8 ? 0.f : vec == 4 ? 1.f : vec == 2 ? 4.f : 7.f) * (rows < GP_TILE ? rows / GP_TILE : 1);
    return 3.3f * tiles + (tiles > 1 ? 0.25f / GP_BK * k * tiles : 0) + write <= 3 + 1.4f * copy;
}

// The shared product of one tile's picked rows takes narrower tiles: more pairs have a
// tile of their own, and a tile has fewer pieces to join.  (3,778 rows: 79 us, 62 with
// whole tiles.)
constexpr int FEW_BN = 128;
// So do those of up to three eighths as many tiles as pairs: 171 rows through
// 4,992 x 576 43 -> 39 us, 263 through 3,712 x 832 46 -> 39.  (With three quarters 336
// rows of 46 adapters take 78 us for 57; with 32 columns 35 of 57 take 41 for 36.)
constexpr int LEAST_BN = 64;
// Inner products without tensor cores: values of the adapters that are read, and
// blocks (a row and four ranks each).  With either twice as many the tensor cores
// are faster, at 8 to 128 ranks and 256 to 4,096 columns (4,096 rows of rank 8 and
// 1,024 columns: 41 us against 36; 2,048 rows: 31 against 35).
constexpr int64_t LOW_FEW_VALUES = 64 << 20, LOW_FEW_BLOCKS = 4096;

// contracted: a gradient contracts over the rows, which takes the padded plan.
static Rows plan_rows(Carver &cv, const hwr_rows *r, const void *dy, int64_t dy_ld, bool need_x, bool contracted,
                      bool pick) {
    Rows s;
    s.plan.rows = s.plan.places = r->rows;
    s.plan.groups = r->groups;
    s.plan.offsets = r->offsets;
    s.plan.order = r->order;
    auto operand = [&](const void *p, int64_t ld, int cols) {
        Operand o;
        o.p = p;
        o.ld = ld;
        o.rows = r->rows;
        o.cols = cols;
        return o;
    };
    if (need_x) s.x = operand(r->x, r->x_ld, r->n_in);
    if (dy) s.dy = operand(dy, dy_ld, r->n_out);
    s.sorted = contracted || !pick || (need_x && !on16(r->x, r->x_ld, 0, 1)) ||
               (dy && !on16(dy, dy_ld, 0, 1));
    if (!s.sorted) return s;
    if (contracted) {
        s.plan.padded = 1;
        s.plan.places = r->rows + 15 * (r->rows < r->groups ? r->rows : r->groups);
        s.offsets_off = cv.take((size_t)(r->groups + 2) * 4);
        s.order_off = cv.take((size_t)s.plan.places * 4);
    }
    if (need_x) s.x.off = cv.take((size_t)s.plan.places * up(r->n_in, 8) * 2);
    if (dy) s.dy.off = cv.take((size_t)s.plan.places * up(r->n_out, 8) * 2);
    return s;
}

static hwr_status sort_rows(hwr_ops *c, Rows *s) {
    if (!s->sorted) return HWR_OK;
    SortRows m;
    for (Operand *o : {&s->x, &s->dy}) {
        if (!o->p) continue;
        m.src[m.n] = (const uint16_t *)o->p;
        m.src_ld[m.n] = o->ld;
        m.cols[m.n] = o->cols;
        o->p = c->ws + o->off;
        o->ld = up(o->cols, 8);
        o->rows = s->plan.places;
        m.dst[m.n] = (uint16_t *)(c->ws + o->off);
        m.dst_ld[m.n++] = o->ld;
    }
    int32_t *offsets = s->plan.padded ? (int32_t *)(c->ws + s->offsets_off) : nullptr;
    int32_t *order = s->plan.padded ? (int32_t *)(c->ws + s->order_off) : nullptr;
    m.zero = (uint32_t *)(c->ws + s->peak_off);
    m.nzero = s->peaks;
    CK(c, launch_sort_rows(s->plan, m, s->plan.places, offsets, order, c->nsm, c->stream), "row copy");
    if (s->plan.padded) {
        s->plan.offsets = offsets;
        s->plan.order = order;
    }
    for (Operand *o : {&s->x, &s->dy}) o->z = up(o->ld * o->rows, 8);
    return HWR_OK;
}

static GroupProduct product(hwr_ops *c, const hwr_rows *r, const Rows &s) {
    GroupProduct p;
    p.plan = s.plan;
    p.sorted = s.sorted;
    p.f16 = r->dtype == HWR_F16;
    p.part = c->part;
    p.count = c->count;
    p.status = c->status_d;
    p.test_stall = c->test_stall;
    return p;
}

// Columns of a tile: n in as few tiles of at most `most` as it takes, evenly.
static int even_tiles(int n, int most) {
    const int tiles = (n + most - 1) / most;
    return (int)up((n + tiles - 1) / tiles, 16);
}

// Columns of a tile whose A side are rows.
static int tile_columns(const hwr_ops *c, const GroupProduct &p, int n) {
    int most = p.sorted || !p.shared || p.plan.places > GP_TILE ? GP_TILE : FEW_BN;
    const int64_t mtiles = (p.plan.places + GP_TILE - 1) / GP_TILE;
    while (p.shared && !p.dense_mn && most > LEAST_BN && mtiles * ((n + most / 2 - 1) / (most / 2)) * 16 <= 3 * c->ctas)
        most /= 2;
    return most;
}

static hwr_status check_tiles(hwr_ops *c, const GroupProduct &p) {
    if (((int64_t)p.plan.places / GP_TILE + 1) * p.plan.groups * p.ntiles > INT32_MAX)
        return fail(c, HWR_ERR_UNSUPPORTED, "rows %d x groups %d x columns %d is too large", p.plan.rows, p.plan.groups,
                    p.n);
    return HWR_OK;
}

static hwr_status launch(hwr_ops *c, GroupCall *calls, int n = 1, double share = 1) {
    CK(c, launch_group(calls, n, share, c->ctas, c->stream), "product kernel");
    return HWR_OK;
}

// out[t] = W[g(t)] x[t] (w K-major: [out][in]) or W[g(t)]^T x[t] (w_mn), to be launched.
static hwr_status rows_product(hwr_ops *c, GroupProduct p, const Operand &x, const Operand &w, bool w_mn, int n,
                               const Operand *u, const Operand *eb, GroupCall *call) {
    p.k = x.cols;
    p.n = n;
    p.dense_mn = w_mn;
    if (!p.sorted) {
        p.x = (const uint16_t *)x.p;
        p.x_ld = x.ld;
    }
    if (p.mode == GP_GROUPED) p.bn = (int)up(p.plan.places < GP_TILE ? p.plan.places : GP_TILE, 16);
    else p.bn = even_tiles(n, tile_columns(c, p, n));
    group_plan(&p);
    OK(check_tiles(c, p));
    call->p = p;
    GroupMaps &m = call->maps;
    memset(&m, 0, sizeof m);
    if (p.sorted) {
        OK(encode(c, &m.x, p.f16, x, 64, GP_ROW_BOX));
        OK(encode(c, &m.xx, p.f16, x, 64, 128));
    }
    OK(encode(c, &m.w, p.f16, w, 64, w_mn ? 64 : p.mode == GP_GROUPED ? 128 : p.bn / 2));
    if (u) {         // (bf16 terms whatever the rows' type)
        OK(encode(c, &m.u, false, *u, 64, GP_ROW_BOX));
        OK(w_mn ? encode(c, &m.eb, false, *eb, 64, GP_RC)
                : encode(c, &m.eb, false, *eb, p.rank <= 16 ? 16 : GP_RC, p.bn / 2));
    }
    return HWR_OK;
}

// out[g] = sum over the rows of g of l[t] r[t]^T, to be launched.
static hwr_status grad_product(hwr_ops *c, GroupProduct p, const Operand &l, const Operand &r, GroupCall *call) {
    p.mode = GP_WGRAD;
    p.m = l.cols;
    p.n = r.cols;
    p.bn = p.out_kind == GP_OUT_GROUP ? even_tiles(p.n, GP_TILE) : p.n < GP_TILE ? p.n : GP_TILE;
    group_plan(&p);
    if ((int64_t)p.plan.groups * p.mtiles * p.ntiles > INT32_MAX)
        return fail(c, HWR_ERR_UNSUPPORTED, "groups %d x %d x %d is too large", p.plan.groups, p.m, p.n);
    call->p = p;
    GroupMaps &m = call->maps;
    memset(&m, 0, sizeof m);
    OK(encode(c, &m.x, p.f16, l, 64, GP_BK));
    OK(encode(c, &m.w, p.f16, r, 64, GP_BK));
    return HWR_OK;
}

static hwr_status check_rows(hwr_ops *c, const hwr_rows *r, bool need_x, bool need_w, bool grouped) {
    if (!r) return fail(c, HWR_ERR_INVALID_ARG, "NULL rows");
    if (r->rows < 0 || r->groups < 1 || r->n_in < 1 || r->n_out < 1)
        return fail(c, HWR_ERR_INVALID_ARG, "rows %d, groups %d, n_in %d, n_out %d", r->rows, r->groups, r->n_in,
                    r->n_out);
    if (r->groups > OPS_MAX_GROUPS) return fail(c, HWR_ERR_UNSUPPORTED, "groups %d > %d", r->groups, OPS_MAX_GROUPS);
    if (r->rows > INT32_MAX - 32 * OPS_MAX_GROUPS) return fail(c, HWR_ERR_UNSUPPORTED, "rows %d", r->rows);
    if (r->dtype != HWR_BF16 && r->dtype != HWR_F16)
        return fail(c, HWR_ERR_DTYPE, "dtype %d: products take bf16 or fp16", (int)r->dtype);
    if (r->rows && (!r->offsets || !r->order || (need_x && !r->x) || (need_w && !r->w)))
        return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    if (need_x && r->x_ld < r->n_in) return fail(c, HWR_ERR_INVALID_ARG, "x_ld %lld < n_in", (long long)r->x_ld);
    if (r->w_ld < r->n_in) return fail(c, HWR_ERR_INVALID_ARG, "w_ld %lld < n_in", (long long)r->w_ld);
    if (grouped && r->groups > 1 && r->w_group < r->w_ld * (r->n_out - 1) + r->n_in)
        return fail(c, HWR_ERR_INVALID_ARG, "w_group %lld: groups overlap", (long long)r->w_group);
    return HWR_OK;
}

static hwr_status check_out(hwr_ops *c, const hwr_rows *r, const void *p, int64_t ld, int width, const char *name) {
    if (r->rows && !p) return fail(c, HWR_ERR_INVALID_ARG, "%s is NULL", name);
    if (ld < width) return fail(c, HWR_ERR_INVALID_ARG, "%s_ld %lld < %d", name, (long long)ld, width);
    return HWR_OK;
}

extern "C" hwr_status hwr_grouped_forward(hwr_ops *c, const hwr_rows *r, void *y, int64_t y_ld) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_grouped_forward");
    OK(ready(c));
    OK(check_rows(c, r, true, true, true));
    OK(check_out(c, r, y, y_ld, r->n_out, "y"));
    if (r->rows == 0) return HWR_OK;
    Carver cv;
    Rows rows = plan_rows(cv, r, nullptr, 0, true, false, picks_rows(c, r, r->n_in, r->n_out, false, vec_of(y, y_ld, 0)));
    Operand w = cv.operand(r->w, r->w_ld, r->n_out, r->n_in, r->w_group, r->groups);
    OK(reserve(c, cv.at));
    OK(sort_rows(c, &rows));
    OK(settle(c, &w));
    GroupProduct p = product(c, r, rows);
    p.mode = GP_GROUPED;
    p.out_kind = GP_OUT_ROWS;
    p.out = y;
    p.ld = y_ld;
    p.vec = vec_of(y, y_ld, 0);
    GroupCall call;
    OK(rows_product(c, p, rows.x, w, false, r->n_out, nullptr, nullptr, &call));
    return launch(c, &call);
}

extern "C" hwr_status hwr_grouped_backward(hwr_ops *c, const hwr_rows *r, const void *dy, int64_t dy_ld, void *dx,
                                           int64_t dx_ld, void *dw) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_grouped_backward");
    OK(ready(c));
    OK(check_rows(c, r, dw != nullptr, dx != nullptr, true));
    OK(check_out(c, r, dy, dy_ld, r->n_out, "dy"));
    if (dx) OK(check_out(c, r, dx, dx_ld, r->n_in, "dx"));
    if (r->rows == 0) {
        for (int g = 0; dw && g < r->groups; ++g)
            CK(c, cudaMemset2DAsync((uint16_t *)dw + g * (r->groups > 1 ? r->w_group : 0), r->w_ld * 2, 0,
                                    (size_t)r->n_in * 2, r->n_out, c->stream), "memset");
        return HWR_OK;
    }
    if (!dx && !dw) return HWR_OK;
    Carver cv;
    Rows rows = plan_rows(cv, r, dy, dy_ld, dw != nullptr, dw != nullptr, picks_rows(c, r, r->n_out, r->n_in, false, vec_of(dx, dx_ld, 0)));
    Operand w;
    if (dx) w = cv.operand(r->w, r->w_ld, r->n_out, r->n_in, r->w_group, r->groups);
    OK(reserve(c, cv.at));
    OK(sort_rows(c, &rows));
    GroupCall call;
    if (dx) {
        OK(settle(c, &w));
        GroupProduct p = product(c, r, rows);
        p.mode = GP_GROUPED;
        p.out_kind = GP_OUT_ROWS;
        p.out = dx;
        p.ld = dx_ld;
        p.vec = vec_of(dx, dx_ld, 0);
        OK(rows_product(c, p, rows.dy, w, true, r->n_in, nullptr, nullptr, &call));
        OK(launch(c, &call));
    }
    if (dw) {
        GroupProduct p = product(c, r, rows);
        p.out_kind = GP_OUT_GROUP;
        p.out = dw;
        p.ld = r->w_ld;
        p.gstride = r->groups > 1 ? r->w_group : 0;
        p.vec = vec_of(dw, r->w_ld, p.gstride);
        OK(grad_product(c, p, rows.dy, rows.x, &call));
        OK(launch(c, &call));
    }
    return HWR_OK;
}

static hwr_status check_adapters(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad) {
    if (!ad) return fail(c, HWR_ERR_INVALID_ARG, "NULL adapters");
    if (ad->rank < 1) return fail(c, HWR_ERR_INVALID_ARG, "rank %d", ad->rank);
    if (ad->rank > OPS_MAX_RANK) return fail(c, HWR_ERR_UNSUPPORTED, "rank %d > %d", ad->rank, OPS_MAX_RANK);
    if (r->rows && (!ad->a || !ad->b || !ad->scale)) return fail(c, HWR_ERR_INVALID_ARG, "NULL array");
    return HWR_OK;
}

// scale[g] M[g] x[t] (or M[g]^T x[t]) by place, as two bf16 terms: [places]
// [32-rank chunks][high, low], an even number of chunks; or, with the groups' peaks,
// in fp32 in the same room.
static hwr_status low_rank(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad, const Rows &rows, const Operand &x,
                           const Operand &m, bool m_mn, const Operand &u, uint32_t *peak, GroupCall *call) {
    GroupProduct p = product(c, r, rows);
    p.mode = GP_ROWS;
    p.out_kind = peak ? GP_OUT_WIDE : GP_OUT_PACK;
    p.peak = peak;
    p.out = const_cast<void *>(u.p);
    p.ld = u.ld;
    p.scale = ad->scale;
    return rows_product(c, p, x, m, m_mn, ad->rank, nullptr, nullptr, call);
}

// The same of picked rows without tensor cores, or (wide) as fp32 [places][rank]:
// a row reads its adapter's matrix once, and so few bytes need none (64 rows, rank
// 16, 4,096 columns: 27 us on them, 5 us without).
static hwr_status low_rank_few(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad, const Rows &rows,
                               const Operand &a, const Operand &u, bool wide) {
    LowFew f;
    f.plan = rows.plan;
    f.k = rows.x.cols;
    f.rank = ad->rank;
    f.x = (const uint16_t *)rows.x.p;
    f.a = (const uint16_t *)a.p;
    f.x_ld = rows.x.ld;
    f.a_ld = a.ld;
    f.a_z = a.z;
    f.scale = ad->scale;
    f.u = (uint16_t *)const_cast<void *>(u.p);
    f.u_ld = u.ld;
    f.by_place = rows.sorted;
    f.wide = wide ? (float *)const_cast<void *>(u.p) : nullptr;
    CK(c, launch_low_few(f, r->dtype == HWR_F16, c->stream), "low-rank kernel");
    return HWR_OK;
}

// The packed inner products' place in the workspace.
static Operand packed(Carver &cv, const Rows &rows, const hwr_adapters *ad) {
    Operand u;
    u.cols = (int)up(ad->rank, 2 * GP_RC) * 2;
    u.ld = u.cols;
    u.rows = rows.plan.places;
    u.z = up(u.ld * u.rows, 8);
    u.off = cv.take((size_t)u.rows * u.ld * 2);
    return u;
}

// The adapters' matrices as the extension takes them: as they are in bf16, as two bf16
// terms of fp16 ones.
static Operand ext_operand(Carver &cv, const hwr_rows *r, const void *m, int rows, int rank, bool mn) {
    const int G = r->groups;
    if (r->dtype == HWR_BF16)
        return mn ? cv.operand(m, rows, rank, rows, (int64_t)rank * rows, G)
                  : cv.operand(m, rank, rows, rank, (int64_t)rows * rank, G);
    Operand o;
    o.p = m;
    o.nz = G;
    o.rows = mn ? ext_terms_ranks(rank, mn) : rows;
    o.cols = mn ? rows : ext_terms_ranks(rank, mn);
    o.off = cv.take((size_t)G * o.rows * up(o.cols, 8) * 2);
    return o;
}

static hwr_status settle_ext(hwr_ops *c, const hwr_rows *r, Operand *o, int rank, bool mn) {
    if (r->dtype == HWR_BF16) return settle(c, o);
    const uint16_t *src = (const uint16_t *)o->p;
    o->p = c->ws + o->off;
    o->ld = up(o->cols, 8);
    o->z = o->ld * o->rows;
    CK(c, launch_ext_terms((uint16_t *)(c->ws + o->off), o->ld, src, r->groups, (int)(mn ? o->cols : o->rows), rank, mn,
                           c->nsm, c->stream),
       "adapters' terms");
    return HWR_OK;
}

// W x[t] (or W^T x[t]) and the extension of t's group.
static hwr_status shared_product(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad, const Rows &rows,
                                 const Operand &x, const Operand &w, bool w_mn, const Operand &u, const Operand &eb,
                                 void *out, int64_t ld, int n) {
    GroupCall call;
    GroupProduct p = product(c, r, rows);
    p.mode = GP_ROWS;
    p.shared = 1;
    p.rank = ad->rank;
    p.out_kind = GP_OUT_ROWS;
    p.out = out;
    p.ld = ld;
    p.vec = vec_of(out, ld, 0);
    OK(rows_product(c, p, x, w, w_mn, n, &u, &eb, &call));
    return launch(c, &call);
}

extern "C" hwr_status hwr_adapter_forward(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad, void *y,
                                          int64_t y_ld) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_adapter_forward");
    OK(ready(c));
    OK(check_rows(c, r, true, true, false));
    OK(check_adapters(c, r, ad));
    OK(check_out(c, r, y, y_ld, r->n_out, "y"));
    if (r->rows == 0) return HWR_OK;
    const int K = r->n_in, N = r->n_out, R = ad->rank, G = r->groups;
    Carver cv;
    Rows rows = plan_rows(cv, r, nullptr, 0, true, false, picks_rows(c, r, K, N, true, vec_of(y, y_ld, 0)));
    Operand w = cv.operand(r->w, r->w_ld, N, K);
    Operand a = cv.operand(ad->a, K, R, K, (int64_t)R * K, G);
    const bool few = !rows.sorted && r->rows <= FEW_ROWS;
    Operand b;
    if (!few) b = ext_operand(cv, r, ad->b, N, R, false);
    Operand u = packed(cv, rows, ad);
    OK(reserve(c, cv.at));
    u.p = c->ws + u.off;
    OK(sort_rows(c, &rows));
    OK(settle(c, &a));
    OK(settle(c, &w));
    if (few) {
        FewRows f;
        f.plan = rows.plan;
        f.k = K;
        f.n = N;
        f.x = (const uint16_t *)rows.x.p;
        f.x_ld = rows.x.ld;
        f.w = (const uint16_t *)w.p;
        f.w_ld = w.ld;
        f.out = (uint16_t *)y;
        f.ld = y_ld;
        f.rank = R;
        f.u = (const float *)u.p;       // (a row of two 16-bit terms has room for it)
        f.b = (const uint16_t *)ad->b;
        f.b_ld = R;
        f.b_z = (int64_t)N * R;
        OK(low_rank_few(c, r, ad, rows, a, u, true));
        CK(c, launch_few_rows(f, r->dtype == HWR_F16, c->stream), "few-rows kernel");
        return HWR_OK;
    }
    OK(settle_ext(c, r, &b, R, false));
    if ((int64_t)r->rows * R * K <= LOW_FEW_VALUES && (int64_t)r->rows * ((R + 3) / 4) <= LOW_FEW_BLOCKS) {
        OK(low_rank_few(c, r, ad, rows, a, u, false));
    } else {
        GroupCall call;
        OK(low_rank(c, r, ad, rows, rows.x, a, false, u, nullptr, &call));
        OK(launch(c, &call));
    }
    return shared_product(c, r, ad, rows, rows.x, w, false, u, b, y, y_ld, N);
}

extern "C" hwr_status hwr_adapter_backward(hwr_ops *c, const hwr_rows *r, const hwr_adapters *ad, const void *dy,
                                           int64_t dy_ld, void *dx, int64_t dx_ld, void *da, void *db) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_adapter_backward");
    OK(ready(c));
    OK(check_rows(c, r, da || db, dx != nullptr, false));
    OK(check_adapters(c, r, ad));
    OK(check_out(c, r, dy, dy_ld, r->n_out, "dy"));
    if (dx) OK(check_out(c, r, dx, dx_ld, r->n_in, "dx"));
    const int K = r->n_in, N = r->n_out, R = ad->rank, G = r->groups;
    if (r->rows == 0) {
        if (da) CK(c, cudaMemsetAsync(da, 0, (size_t)G * R * K * 2, c->stream), "memset");
        if (db) CK(c, cudaMemsetAsync(db, 0, (size_t)G * N * R * 2, c->stream), "memset");
        return HWR_OK;
    }
    if (!dx && !da && !db) return HWR_OK;
    Carver cv;
    Rows rows = plan_rows(cv, r, dy, dy_ld, da || db, da || db, picks_rows(c, r, N, K, true, vec_of(dx, dx_ld, 0)));
    // In fp16 the gradients take the inner products as fp16 terms that are scaled by
    // each group's peak: they are made in fp32 and split in a pass of their own
    const bool split = r->dtype == HWR_F16;
    Operand w, a, b, ea, u, v, ev;
    if (dx) w = cv.operand(r->w, r->w_ld, N, K);
    if (db) a = cv.operand(ad->a, K, R, K, (int64_t)R * K, G);
    const bool one = db && r->dtype == HWR_BF16;       // (dx and dB take the same A)
    if (dx && !one) ea = ext_operand(cv, r, ad->a, K, R, true);
    if (dx || da) {
        b = cv.operand(ad->b, R, N, R, (int64_t)N * R, G);
        v = packed(cv, rows, ad);
    }
    if (db) u = packed(cv, rows, ad);
    if (split && dx && da) ev = packed(cv, rows, ad);
    if (split && (da || db)) {
        rows.peaks = 2 * G;
        rows.peak_off = cv.take((size_t)rows.peaks * 4);
    }
    OK(reserve(c, cv.at));
    u.p = c->ws + u.off;
    v.p = c->ws + v.off;
    ev.p = c->ws + ev.off;
    uint32_t *const upeak = split && db ? (uint32_t *)(c->ws + rows.peak_off) : nullptr;
    uint32_t *const vpeak = split && da ? (uint32_t *)(c->ws + rows.peak_off) + G : nullptr;
    OK(sort_rows(c, &rows));
    if (dx) OK(settle(c, &w));
    if (db) OK(settle(c, &a));
    if (dx && one) ea = a;
    if (dx && !one) OK(settle_ext(c, r, &ea, R, true));
    // v and u are independent of each other, and so are da and db: two in a launch,
    // on shares of the SMs by what they read (a launch of its own takes 10 us)
    GroupCall calls[2];
    SplitLow splits[2];
    int n = 0, nsplit = 0;
    if (dx || da) {
        OK(settle(c, &b));
        OK(low_rank(c, r, ad, rows, rows.dy, b, true, v, vpeak, &calls[n++]));
        if (vpeak) splits[nsplit++] = {(uint16_t *)(c->ws + v.off), dx ? (uint16_t *)(c->ws + ev.off) : nullptr, vpeak};
    }
    if (db) {
        OK(low_rank(c, r, ad, rows, rows.x, a, false, u, upeak, &calls[n++]));
        if (upeak) splits[nsplit++] = {(uint16_t *)(c->ws + u.off), nullptr, upeak};
    }
    const double by_n = (double)N / ((double)N + K);
    OK(launch(c, calls, n, by_n));
    if (nsplit)
        CK(c, launch_split_low(rows.plan, R, 2 * up(R, 2 * GP_RC), splits, nsplit, c->nsm, c->stream), "terms");
    if (dx) OK(shared_product(c, r, ad, rows, rows.dy, w, true, vpeak ? ev : v, ea, dx, dx_ld, K));
    n = 0;
    if (da) {
        GroupProduct p = product(c, r, rows);
        p.out_kind = GP_OUT_LOW_T;
        p.peak = vpeak;
        p.out = da;
        p.ld = K;
        p.gstride = (int64_t)R * K;
        p.rank_out = R;
        p.vec = vec_of(da, K, p.gstride);
        OK(grad_product(c, p, rows.x, v, &calls[n++]));
    }
    if (db) {
        GroupProduct p = product(c, r, rows);
        p.out_kind = GP_OUT_LOW;
        p.peak = upeak;
        p.out = db;
        p.ld = R;
        p.gstride = (int64_t)N * R;
        p.rank_out = R;
        p.vec = vec_of(db, R, p.gstride);
        OK(grad_product(c, p, rows.dy, u, &calls[n++]));
    }
    return n ? launch(c, calls, n, 1 - by_n) : HWR_OK;
}

// ---------------------------------------------------------------------------

// Checks a list, and says into how many chunks of which size it is cut.
static hwr_status check_gradients(hwr_ops *c, int32_t n, const hwr_gradient *grads, int64_t *chunks, int *per) {
    if (n < 0 || (n && !grads)) return fail(c, HWR_ERR_INVALID_ARG, "n %d or a NULL array", n);
    *chunks = 0;
    int64_t all = 0;
    for (int i = 0; i < n; ++i)
        if (grads[i].n > 0 && all <= CLIP_SMALL) all += grads[i].n > CLIP_SMALL ? CLIP_SMALL + 1 : grads[i].n;
    *per = all <= CLIP_SMALL ? 1 : CLIP_PER;
    for (int i = 0; i < n; ++i) {
        const hwr_gradient &g = grads[i];
        if (g.n < 0 || (g.n && (!g.in || !g.out)))
            return fail(c, HWR_ERR_INVALID_ARG, "gradient %d: n %lld or a NULL array", i, (long long)g.n);
        if (g.dtype != HWR_F32 && g.dtype != HWR_BF16 && g.dtype != HWR_F16)
            return fail(c, HWR_ERR_DTYPE, "gradient %d: dtype %d", i, (int)g.dtype);
        const uintptr_t mask = g.dtype == HWR_F32 ? 3 : 1;
        if (((uintptr_t)g.in | (uintptr_t)g.out) & mask)
            return fail(c, HWR_ERR_INVALID_ARG, "gradient %d is not aligned to its elements", i);
        *chunks += g.n > INT64_MAX / 8 ? INT32_MAX : clip_chunks(g.n, g.dtype, *per);
        if (*chunks >= INT32_MAX) return fail(c, HWR_ERR_UNSUPPORTED, "too many elements");
    }
    return HWR_OK;
}

static ClipSums clip_sums(const hwr_ops *c) {
    ClipSums s;
    s.part = c->sums;
    s.count = (uint32_t *)(c->sums + clip_blocks(INT64_MAX, c->nsm));
    s.factor = (float *)(s.count + 1);
    return s;
}

static hwr_status check_norm(hwr_ops *c, float max_norm, const float *norm) {
    if (!norm) return fail(c, HWR_ERR_INVALID_ARG, "norm is NULL");
    if (!(max_norm > 0.f)) return fail(c, HWR_ERR_INVALID_ARG, "max_norm %g", max_norm);
    return HWR_OK;
}

extern "C" hwr_status hwr_clip_gradients(hwr_ops *c, int32_t n, const hwr_gradient *grads, float max_norm,
                                         float *norm) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_clip_gradients");
    OK(ready(c));
    int64_t chunks;
    int per;
    OK(check_gradients(c, n, grads, &chunks, &per));
    OK(check_norm(c, max_norm, norm));
    OK(reserve(c, (size_t)chunks * sizeof(ClipChunk)));
    ClipChunk *table = (ClipChunk *)c->ws;
    ClipTable t;
    t.n = t.at = 0;
    t.per = per;
    t.chunk0[0] = 0;
    for (int i = 0; i < n; ++i) {
        const hwr_gradient &g = grads[i];
        t.in[t.n] = g.in;
        t.out[t.n] = g.out;
        t.count[t.n] = g.n;
        t.dtype[t.n] = (uint8_t)g.dtype;
        t.chunk0[t.n + 1] = t.chunk0[t.n] + (int32_t)clip_chunks(g.n, g.dtype, per);
        if (++t.n < CLIP_TABLE && i + 1 < n) continue;
        CK(c, launch_clip_table(t, table, c->stream), "gradient table kernel");
        t.at += t.chunk0[t.n];
        t.n = 0;
    }
    CK(c, launch_clip(table, (int)chunks, per, c->nsm, clip_sums(c), max_norm, norm, c->stream), "clip kernel");
    return HWR_OK;
}

extern "C" hwr_status hwr_gradients_create(hwr_ops *c, int32_t n, const hwr_gradient *grads, hwr_gradients **out) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_gradients_create");
    if (!out) return fail(c, HWR_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    OK(ready(c));
    bool captured;
    OK(capturing(c, &captured));
    if (captured) return fail(c, HWR_ERR_UNSUPPORTED, "a list of gradients cannot be made during a stream capture");
    int64_t chunks;
    int per;
    OK(check_gradients(c, n, grads, &chunks, &per));
    hwr_gradients *l = new (std::nothrow) hwr_gradients;
    ClipChunk *host = new (std::nothrow) ClipChunk[chunks ? chunks : 1];
    hwr_status s = l && host ? HWR_OK : fail(c, HWR_ERR_OOM, "host allocation failed");
    if (s == HWR_OK) s = alloc(c, &l->table, chunks ? chunks : 1);
    if (s == HWR_OK) {
        l->per = per;
        for (int i = 0; i < n; ++i)
            for (int64_t k = 0, m = clip_chunks(grads[i].n, grads[i].dtype, per); k < m; ++k)
                host[l->chunks++] = clip_chunk(grads[i].in, grads[i].out, grads[i].n, grads[i].dtype, per, k);
        cudaError_t e = cudaMemcpyAsync(l->table, host, chunks * sizeof(ClipChunk), cudaMemcpyHostToDevice, c->stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize(c->stream);
        if (e != cudaSuccess) s = cuda_fail(c, e, "gradient table");
    }
    delete[] host;
    if (s != HWR_OK) {
        const Unwatched memory;
        if (l) cudaFree(l->table);
        delete l;
        return s;
    }
    l->next = c->lists;
    c->lists = l;
    *out = l;
    return HWR_OK;
}

extern "C" hwr_status hwr_gradients_clip(hwr_ops *c, const hwr_gradients *l, float max_norm, float *norm) {
    if (!c) return HWR_ERR_INVALID_ARG;
    ApiRange range("hwr_gradients_clip");
    OK(ready(c));
    if (!l) return fail(c, HWR_ERR_INVALID_ARG, "NULL list");
    OK(check_norm(c, max_norm, norm));
    bool captured;
    OK(capturing(c, &captured));
    l->held = l->held || captured;
    CK(c, launch_clip(l->table, l->chunks, l->per, c->nsm, clip_sums(c), max_norm, norm, c->stream), "clip kernel");
    return HWR_OK;
}

extern "C" hwr_status hwr_gradients_destroy(hwr_ops *c, hwr_gradients *l) {
    if (!l) return HWR_OK;
    if (!c) return HWR_ERR_INVALID_ARG;
    hwr_gradients **at = &c->lists;
    while (*at && *at != l) at = &(*at)->next;
    if (!*at) return fail(c, HWR_ERR_INVALID_ARG, "not a list of this context");
    bool captured;
    OK(capturing(c, &captured));
    if (captured || l->held) {          // (during a capture nothing is waited for or freed)
        OK(retire(c, l->table));
    } else {
        const Unwatched memory;
        cudaStreamSynchronize(c->stream);
        cudaFree(l->table);
        cudaGetLastError();
    }
    *at = l->next;
    delete l;
    return HWR_OK;
}
