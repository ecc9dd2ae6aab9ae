// A layer of experts for a few rows (decode steps): routing, both products, the
// activation between them and the sum over a row's choices, in two or three launches.
//
//   k_experts_in    h[t, j] = act(W_gate[e] x[t]) * (W_up[e] x[t])  (or act(W_in[e] x[t]))
//   k_experts_out   z[t, j] = W_out[e] h[t, j]
//   k_experts_sum   y[t] = sum over j of p[t, j] z[t, j]
//
// (the last where a row has several choices, or the second product's contraction is cut).
// Bound by HBM: of each expert that a row chooses the weights are read once (by up to 8
// of its rows at a time, a job, or 16 where experts have many; an expert of more rows is
// read again from L2), everything else stays in L2.  Every block finds the choices and the experts' rows by
// itself from the scores (a few KB), which costs less than a launch between.  A unit of
// work is 16 rows of a weight matrix (in the first product 8 gate rows and the 8 up rows
// that they meet, so that the activation finds both) and a job.  A block walks a run of
// consecutive units.  Two of its warps copy the weights into a ring in shared memory,
// some steps of up to 512 columns ahead and across the ends of units.  Two teams of eight
// warps take the steps in turn; a team's warps share a step's columns, 32 at a time, and
// load their part of the job's rows of x (or h) from L2 a step ahead.  Two more warps add
// up the teams' sums of a unit, in a fixed order, and write its results.  (A unit a warp,
// each with copies of its own, read 512-byte pieces all over the matrices: 4.4 TB/s.  With
// the rows of x and h copied into the ring too the copying warp was the bound, some 50
// cycles a copy; with one team, its latency from step to step.)
//
// The multiplications are warp-level MMAs: 16 rows of weights, 8 rows of x.  The
// contraction's order is free, so a lane takes eight consecutive columns of a weight's
// row in one 16-byte load, and the same of x.  h is summed in fp32 and enters the second
// product whole: beside bf16 weights as three bf16 terms.  (As two, 16 bits of it, one
// bf16 result in 220 differed from that of fp32 hidden values, with three one in 1,070, as
// many as another order of fp32 sums moves; 16 rows with 6 of 64 experts of 2,048 -> 2 x 1,408
// took 128.5 us for 133, 64 rows with 4 of 24 of 1,024 -> 2 x 2,048 84 for 88.5.)  Beside fp16
// weights, whose range is too small for it, as two tf32 values, within 2^-20 of it, the
// weights widened to tf32 exactly: fp16 results are rounded to 2^-11, and a third would be
// half as many multiplications again.
#include "ops_internal.cuh"
#include "umma.cuh"
#include "values.cuh"

namespace hwr {
namespace {

using umma::bulk_g2s;
using umma::mbar_arrive;
using umma::mbar_arrive_expect_tx;
using umma::mbar_init;
using umma::mbar_wait;

constexpr int EX_TEAM = 8, EX_MMA = 2 * EX_TEAM, EX_COPY = 2, EX_ADD = 2;      // warps that multiply, copy, add up
constexpr int EX_WARPS = EX_MMA + EX_COPY + EX_ADD, EX_THREADS = EX_WARPS * 32;
constexpr int EX_SUMS = 2;                 // units whose sums are under way
constexpr int EX_STRIDE = EX_TEAM * 32;    // columns of a step that a team takes at a time
constexpr int EX_PAIRS = EXPERTS_MAX_ROWS * EXPERTS_MAX_TOP;
constexpr int EX_DEPTH = 6;                // steps of the ring, at most
constexpr int EX_UNIT_COST = 128;          // of a unit, in columns of its weights
// Columns of a step, at most (of the second product in fp16: half).  One row of 4,096 ->
// 2 x 8,192 over 2 of 8 experts: 76 us with 1,024, 73 with 512 (75 since h has three terms).
constexpr int EX_COLS = 512;
constexpr int SUM_THREADS = 128;
// Shared memory of the tables and the ring, at most; what the ring leaves is the L1 that keeps
// x and h.  With 4, 6 and 8 steps 16 rows with 6 of 64 experts of 2,048 -> 2 x 1,408 (evenly spread
// scores) take 168, 160 and 159 us, one row with 2 of 12 of 1,024 -> 2 x 4,096 21.5, 21.5 and 22.1,
// 64 rows with 4 of 24 of 1,024 -> 2 x 2,048 87.6, 88.5 and 90.3, with 2 of 64 of 1,024 -> 2 x 4,096
// in fp16 (a listed case) 227.8, 210.2 and 209.1.
constexpr int EX_RING = 140 * 1024;
constexpr int EX_GROUPS = OPS_MAX_GROUPS, EX_EACH = (EX_GROUPS + EX_THREADS - 1) / EX_THREADS;      // groups a thread
constexpr uint32_t ALL = 0xffffffffu;

template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
    if (F16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma8_tf32(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The first n of eight 16-bit elements, zeros after them.
__device__ __forceinline__ uint4 first(uint4 v, int n) {
    const uint32_t odd = n & 1 ? 0xffffu : 0u;
    const int w = n >> 1;
    v.x &= w > 0 ? ALL : w == 0 ? odd : 0u;
    v.y &= w > 1 ? ALL : w == 1 ? odd : 0u;
    v.z &= w > 2 ? ALL : w == 2 ? odd : 0u;
    v.w &= w > 3 ? ALL : w == 3 ? odd : 0u;
    return v;
}

// The 16 bytes that begin s (even) bytes into a, followed by b.
__device__ __forceinline__ uint4 shifted(const uint4 &a, const uint4 &b, int s) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (s & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    if (s & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    const int h = (s & 2) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], h), __funnelshift_r(w[1], w[2], h), __funnelshift_r(w[2], w[3], h),
                      __funnelshift_r(w[3], w[4], h));
}

// Eight 16-bit elements of a row in shared memory, whose first lies s bytes behind a
// 16-byte boundary.
__device__ __forceinline__ uint4 taken(const char *at, int s) {
    return shifted(*(const uint4 *)at, *(const uint4 *)(at + 16), s);
}

// Eight 16-bit elements of a row of n in global memory from column c on, zeros for no row
// and from the row's end on, but for those of the last eight, which hold anything there
// (masked where they are used: a mask here would wait for the load).  A row that does not
// begin on a 16-byte boundary gives the two aligned units around them, those that hold an
// element of the row.
template <bool ALIGNED>
__device__ __forceinline__ void eight(uint4 (&v)[ALIGNED ? 1 : 2], const uint16_t *row, int c, int n) {
#pragma unroll
    for (int i = 0; i < (ALIGNED ? 1 : 2); ++i) v[i] = make_uint4(0, 0, 0, 0);
    if (!row || c >= n) return;
    if (ALIGNED) {
        v[0] = *(const uint4 *)(row + c);
    } else {
        const uint4 *u = (const uint4 *)((uintptr_t)(row + c) & ~(uintptr_t)15);
        v[0] = u[0];
        if ((const uint16_t *)(u + 1) < row + n) v[1] = u[1];
    }
}

// A lane's row of a step's copies: the 16-byte units that hold its columns [c, c + cols)
// of n (any alignment; a unit holds an element of the row, so none is out of bounds).
struct Piece {
    const char *from;
    uint32_t bytes;
};
__device__ __forceinline__ Piece piece_of(const void *row, int size, int c, int cols, int n) {
    Piece p = {nullptr, 0};
    const int left = n - c < cols ? n - c : cols;
    if (!row || left <= 0) return p;
    const uintptr_t begin = (uintptr_t)row + (int64_t)c * size, end = begin + (int64_t)left * size;
    p.from = (const char *)(begin & ~(uintptr_t)15);
    p.bytes = (uint32_t)(((end + 15) & ~(uintptr_t)15) - (begin & ~(uintptr_t)15));
    return p;
}

// How the weights' rows come.  BOXES: in boxes of 64 columns x 8 rows by tensor copies, one
// for all of a step's columns, and at the end of rows that are not whole 64 columns one for
// those before the last 64 and one for what is left; matrices whose rows begin on 16-byte
// boundaries.  Else: as bulk copies of rows, sixteen a step of any start and length (8 rows
// over 4 of 32 experts, 2,056 -> 2 x 2,816, bf16, in boxes and by rows: 134 and 221 us).

// The map of a unit's first copy (one that is filled in).
__device__ __forceinline__ const CUtensorMap *first_map(const WeightMaps &m, int n, int cols) {
    return n % 64 == 0 || n >= cols ? &m.whole : &m.tail;
}

// The weights' row that stands in row g of an MMA's eight: a quarter of a warp's 16-byte
// loads reads 64 bytes of two rows, which lie four rows apart, so that they are 64 bytes
// apart in the banks.
__device__ __forceinline__ int row_of(int g) { return g >> 1 | (g & 1) << 2; }

// Eight of a step's columns from k + 8 q on of a weight's row (of the first or the second
// eight): boxes are swizzled (the 16-byte units of row i exchanged by i), rows padded by 16.
template <bool BOXES>
__device__ __forceinline__ uint4 weights(const char *at, int row, int q, bool second, int k, int cols, int s) {
    if (BOXES)
        return *(const uint4 *)(at + (second ? cols * 16 : 0) + (k >> 6) * 1024 + row * 128 + (((k >> 5 & 1) * 4 + q) ^ row) * 16);
    return taken(at + (row + (second ? 8 : 0)) * (cols * 2 + 16) + (k + q * 8) * 2, s);
}

// A block's ring: `depth` steps of 16 rows of weights.
struct Ring {
    char *base;
    uint64_t *full, *empty;               // [depth]
    int step, depth;                      // bytes of a step
    int slot;
    uint32_t phase;
    bool ok;
    __device__ __forceinline__ void next() {
        if (++slot == depth) {
            slot = 0;
            phase ^= 1;
        }
    }
    // Where a wait gives up, the block goes on without waiting (or copying), and the call's
    // results are worth nothing.
    __device__ __forceinline__ const char *wait_full(volatile int *abort_flag, int32_t *status) {
        ok = ok && mbar_wait(full + slot, phase, abort_flag, status);
        return base + slot * step;
    }
    __device__ __forceinline__ void release() {
        __syncwarp();                     // (read by all lanes)
        if ((threadIdx.x & 31) == 0) mbar_arrive(empty + slot);
        next();
        next();                           // (the other team's)
    }
    // A step's copies: lane i's row of weights, or (boxes) both of its eight rows by lanes 0
    // and 1.  False where the wait for the slot gave up.
    template <bool BOXES>
    __device__ __forceinline__ bool copy(const WeightMaps &map, int y, int e, const uint16_t *row, int s, int cols, int n,
                                         volatile int *abort_flag, int32_t *status, bool stall) {
        const int lane = threadIdx.x & 31;
        ok = ok && mbar_wait(empty + slot, phase ^ 1, abort_flag, status);
        if (!BOXES) ok = __all_sync(ALL, ok);
        if (!ok) return false;
        char *to = base + slot * step;
        if (BOXES) {
            if (lane < 2 && !stall) {
                to += lane * cols * 16;
                const int box = s * cols / 64, whole = n / 64;
                if (n % 64 == 0 || box + cols / 64 <= whole) {
                    mbar_arrive_expect_tx(full + slot, cols * 16);
                    umma::tma_load_4d(to, &map.whole, full + slot, 0, y, box, e);
                } else {
                    mbar_arrive_expect_tx(full + slot, (whole - box + 1) * 1024);
                    if (box < whole) umma::tma_load_4d(to, &map.last, full + slot, 0, y, box, e);
                    umma::tma_load_4d(to + (whole - box) * 1024, &map.tail, full + slot, whole * 64, y, 0, e);
                }
            }
        } else {
            const Piece p = lane < 16 ? piece_of(row, 2, s * cols, cols, n) : Piece{nullptr, 0};
            const uint32_t bytes = __reduce_add_sync(ALL, p.bytes);
            if (lane < 2 && !stall) mbar_arrive_expect_tx(full + slot, lane ? 0 : bytes);
            __syncwarp();
            if (p.bytes && !stall) bulk_g2s(to + lane * (cols * 2 + 16), p.from, p.bytes, full + slot);
        }
        next();
        next();                           // (the other copying warp's)
        return true;
    }
};

// ---- routing --------------------------------------------------------------------

// Which rows meet which expert: pairs (row t, choice j) at t * top + j, the pairs of an
// expert side by side in `list`, in jobs of at most 8 or 16 of them.  The first product's blocks
// each make the tables, and one of them leaves them in memory for the launches after it.
struct Routing {
    int *jobs;
    float *gate;                          // [pairs]
    int *count;                           // [groups]
    int16_t *choice;                      // [pairs] -1: none
    uint16_t *list, *begin, *expert;      // [pairs] (jobs: begin, expert)
    uint8_t *n;                           // [jobs]
    __device__ __forceinline__ Routing(const Experts &p, char *at) {
        const int pairs = (p.rows * p.top + 7) & ~7;
        jobs = (int *)at;
        choice = (int16_t *)(at + 16);    // (16-byte aligned, read by eights)
        gate = (float *)(choice + pairs);
        list = (uint16_t *)(gate + pairs);
        begin = list + pairs;
        expert = begin + pairs;
        n = (uint8_t *)(expert + pairs);
        count = (int *)(n + pairs);
    }
};
// (the counts are not needed after the routing)
inline __host__ __device__ size_t tables_bytes(const Experts &p) {
    return 16 + (size_t)((p.rows * p.top + 7) & ~7) * (2 + 4 + 6 + 1);      // (whole words)
}
inline size_t routing_bytes(const Experts &p) { return (tables_bytes(p) + 16 + p.groups * 4 + 1023) / 1024 * 1024; }

// Order of a score among the choices: larger ones above; 0 for one that is never chosen
// (-inf, NaN).
__device__ __forceinline__ uint32_t score_order(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return v > -INFINITY ? u ^ (u >> 31 ? 0xffffffffu : 0x80000000u) : 0u;
}
__device__ __forceinline__ float score_of(uint32_t order) {
    return __uint_as_float(order >> 31 ? order ^ 0x80000000u : ~order);
}

__device__ __forceinline__ float warp_sum(float v) {
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(ALL, v, d);
    return v;
}

// A row's choices by a warp: lane j gets the j-th (-1: none) and its p.  LANE: scores that
// a lane holds (rows of at most 32 LANE of them).
template <int LANE>
__device__ __forceinline__ void choose(const float *s, int E, int top, bool over_all, int &choice, float &gate) {
    const int lane = threadIdx.x & 31;
    uint32_t order[LANE];
    float largest = 0.f, mine = 0.f, total = 0.f;
#pragma unroll
    for (int i = 0; i < LANE; ++i) {
        const float v = lane + i * 32 < E ? __ldg(s + lane + i * 32) : -INFINITY;
        order[i] = score_order(v);
        if (v != v) total = v;            // (never chosen, but part of the sum over all)
    }
    choice = -1;
    for (int j = 0; j < top; ++j) {
        uint32_t best = 0;
        int at = 0;
#pragma unroll
        for (int i = 0; i < LANE; ++i)
            if (order[i] > best) {
                best = order[i];
                at = i;
            }
        const uint32_t most = __reduce_max_sync(ALL, best);
        if (!most) break;
        const uint32_t e = __reduce_min_sync(ALL, best == most ? (uint32_t)(lane + at * 32) : ~0u);
        const float v = score_of(most);
        if (j == 0) {
            largest = v;
            if (over_all)
#pragma unroll
                for (int i = 0; i < LANE; ++i) total += order[i] ? expf(score_of(order[i]) - largest) : 0.f;
        }
        if (lane == j) {
            choice = (int)e;
            mine = v;
        }
#pragma unroll
        for (int i = 0; i < LANE; ++i)
            if (e == (uint32_t)(lane + i * 32)) order[i] = 0;
    }
    const float w = choice >= 0 ? expf(mine - largest) : 0.f;
    total = warp_sum(over_all ? total : w);
    gate = choice >= 0 ? w / total : 0.f;
}

template <int LANE>
__device__ __forceinline__ void choose_all(const Experts &p, Routing &r) {
    const int lane = threadIdx.x & 31;
    for (int t = threadIdx.x >> 5; t < p.rows; t += EX_WARPS) {
        int choice;
        float gate;
        choose<LANE>(p.scores + t * p.scores_ld, p.groups, p.top, p.over_all, choice, gate);
        if (lane < p.top) {
            r.choice[t * p.top + lane] = (int16_t)choice;
            r.gate[t * p.top + lane] = gate;
        }
    }
}

// Up to 32 pairs, by one warp: a stable sort by expert.
template <int JOB>
__device__ __forceinline__ void deal_few(const Routing &r, int pairs) {
    const int lane = threadIdx.x & 31;
    const int mine = lane < pairs ? r.choice[lane] : -1;
    int place = 0, rank = 0;              // among all, and among my expert's
    for (int i = 0; i < pairs; ++i) {
        const int c = __shfl_sync(ALL, mine, i);
        const bool before = c == mine && i < lane;
        rank += before;
        place += before || (c >= 0 && c < mine);
    }
    const bool lead = mine >= 0 && rank % JOB == 0;
    const uint32_t same = __match_any_sync(ALL, mine);
    int job = 0;
    for (int i = 0; i < pairs; ++i) {
        const int at = __shfl_sync(ALL, lead ? place : 64, i);
        job += at < place;
    }
    if (mine >= 0) r.list[place] = (uint16_t)lane;
    if (lead) {
        const int left = __popc(same) - rank;
        r.expert[job] = (uint16_t)mine;
        r.begin[job] = (uint16_t)place;
        r.n[job] = (uint8_t)(left < JOB ? left : JOB);
    }
    const uint32_t leads = __ballot_sync(ALL, lead);
    if (lane == 0) *r.jobs = __popc(leads);
}

// Any number, by the block.
template <int JOB>
__device__ __forceinline__ void deal(const Routing &r, int pairs, int E) {
    __shared__ int warp_jobs[EX_WARPS], warp_pairs[EX_WARPS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int i = tid; i < pairs; i += EX_THREADS)
        if (r.choice[i] >= 0) atomicAdd(&r.count[r.choice[i]], 1);
    __syncthreads();
    // some experts a thread: where their pairs and jobs begin
    int jobs = 0, all = 0, n[EX_EACH];
    bool several = false;
#pragma unroll
    for (int k = 0; k < EX_EACH; ++k) {
        n[k] = tid * EX_EACH + k < E ? r.count[tid * EX_EACH + k] : 0;
        several |= n[k] > JOB;
        jobs += (n[k] + JOB - 1) / JOB;
        all += n[k];
    }
    int j = jobs, a = all;
    for (int d = 1; d < 32; d *= 2) {
        const int oj = __shfl_up_sync(ALL, j, d), oa = __shfl_up_sync(ALL, a, d);
        if (lane >= d) {
            j += oj;
            a += oa;
        }
    }
    if (lane == 31) {
        warp_jobs[warp] = j;
        warp_pairs[warp] = a;
    }
    __syncthreads();
    j -= jobs;
    a -= all;
    for (int w = 0; w < warp; ++w) {
        j += warp_jobs[w];
        a += warp_pairs[w];
    }
    if (tid == EX_THREADS - 1) *r.jobs = j + jobs;
#pragma unroll
    for (int k = 0; k < EX_EACH; ++k) {
        if (n[k]) r.count[tid * EX_EACH + k] = a;
        for (int b = 0; b < n[k]; b += JOB, ++j) {
            r.expert[j] = (uint16_t)(tid * EX_EACH + k);
            r.begin[j] = (uint16_t)(a + b);
            r.n[j] = (uint8_t)(n[k] - b < JOB ? n[k] - b : JOB);
        }
        a += n[k];
    }
    // Within a job pairs may lie in any order (a pair's results do not depend on its column
    // of the MMA); where an expert has several jobs, they lie in their own order, so that
    // every block deals them out alike.
    several = __syncthreads_or(several);
    for (int i = tid; i < pairs; i += EX_THREADS) {
        const int e = r.choice[i];
        if (e < 0) continue;
        if (!several) {
            r.list[atomicAdd(&r.count[e], 1)] = (uint16_t)i;
            continue;
        }
        const uint32_t two = (uint32_t)e << 16 | e;
        const uint4 *c = (const uint4 *)r.choice;
        uint32_t before = 0;              // (both halves: of even and of odd places)
        for (int j = 0; j < i / 8; ++j)
            before += __vseteq2(c[j].x, two) + __vseteq2(c[j].y, two) + __vseteq2(c[j].z, two) + __vseteq2(c[j].w, two);
        int at = (int)(before & 0xffff) + (int)(before >> 16);
        for (int j = i & ~7; j < i; ++j) at += r.choice[j] == e;
        r.list[r.count[e] + at] = (uint16_t)i;
    }
}

// The tables, of every block; block 0 leaves them in memory.  (Made in each launch instead
// of read there: one token 24.7 us for 20.8.)
template <int JOB>
__device__ __forceinline__ void route(const Experts &p, Routing &r, char *smem) {
    const int tid = threadIdx.x, pairs = p.rows * p.top, E = p.groups;
    if (pairs > 32)
        for (int i = tid; i < E; i += EX_THREADS) r.count[i] = 0;
    if (!p.scores) {
        for (int i = tid; i < pairs; i += EX_THREADS) {
            const int c = p.choice[i];
            r.choice[i] = (int16_t)((uint32_t)c < (uint32_t)E ? c : -1);
            r.gate[i] = p.gates[i];
        }
    } else if (E <= 32) {
        choose_all<1>(p, r);
    } else if (E <= 128) {
        choose_all<4>(p, r);
    } else {
        choose_all<32>(p, r);
    }
    __syncthreads();
    if (pairs > 32) deal<JOB>(r, pairs, E);
    else if (tid < 32) deal_few<JOB>(r, pairs);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int i = tid; i < (int)tables_bytes(p) / 4; i += EX_THREADS) ((uint32_t *)p.tables)[i] = ((const uint32_t *)smem)[i];
}

// The tables that the first product has left.
__device__ __forceinline__ void load_routing(const Experts &p, char *smem) {
    for (int i = threadIdx.x; i < (int)tables_bytes(p) / 4; i += EX_THREADS)
        ((uint32_t *)smem)[i] = __ldcg((const uint32_t *)p.tables + i);
    __syncthreads();
}

// A block's run of units: by job, piece of the contraction and tile of 16 rows.
struct Walk {
    int u, end, job, split, tile, splits, tiles;
    __device__ __forceinline__ Walk(int jobs, int splits, int tiles) : splits(splits), tiles(tiles) {
        const int units = jobs * splits * tiles;
        u = (int)((int64_t)units * blockIdx.x / gridDim.x);
        end = (int)((int64_t)units * (blockIdx.x + 1) / gridDim.x);
        tile = u % tiles;
        split = u / tiles % splits;
        job = u / tiles / splits;
    }
    __device__ __forceinline__ bool more() const { return u < end; }
    __device__ __forceinline__ void next() {
        ++u;
        if (++tile < tiles) return;
        tile = 0;
        if (++split < splits) return;
        split = 0;
        ++job;
    }
};

// The steps of a run, `per` (the last piece: what is left of `all`) of each unit.
struct Steps {
    Walk w;
    int s, end, per, all;
    __device__ __forceinline__ Steps(const Walk &w, int per, int all) : w(w), per(per), all(all) { begin(); }
    __device__ __forceinline__ void begin() {
        s = w.split * per;
        end = min(s + per, all);
    }
    __device__ __forceinline__ bool more() const { return w.more(); }
    __device__ __forceinline__ void next() {
        if (++s < end) return;
        w.next();
        begin();
    }
};

// (1 + erf would cancel where u is negative.  Out of line: in line its code costs layers of
// other activations too, one token 22.5 us for 22.0.)
__device__ __noinline__ float gelu(float u) { return 0.5f * u * erfcf(-0.70710678f * u); }

__device__ __forceinline__ float activated(float u, int act) {
    if (act == HWR_ACT_RELU) return u < 0.f ? 0.f : u;
    if (act == HWR_ACT_SILU) return u / (1.f + expf(-u));
    return gelu(u);
}

// A value as two bf16 terms, or two of tf32 (the high one cut off strictly below the
// value, as in bf16_terms).
__device__ __forceinline__ void tf32_terms(float v, float &high, float &low) {
    const uint32_t u = __float_as_uint(v), m = u & 0x7fffffffu;
    high = __uint_as_float(m - 1 < 0x7f7fffffu ? (u - 1) & 0xffffe000u : u);
    low = m < 0x7f800000u ? v - high : v;
}

// The high bf16 term of a value, cut off as in bf16_terms, and what it leaves: two more
// terms take the rest exactly (16 bits at most).
__device__ __forceinline__ float bf16_cut(float v, uint16_t &high) {
    const uint32_t u = __float_as_uint(v), m = u & 0x7fffffffu;
    high = (uint16_t)((m - 1 < 0x7f7fffffu ? u - 1 : u) >> 16);
    return m < 0x7f800000u ? v - __uint_as_float((uint32_t)high << 16) : v;
}

// What the block shares beside the routing's tables and the ring.
template <int NB>
struct Shared {
    float4 sums[EX_SUMS][EX_MMA][NB][32];
    uint64_t full[EX_DEPTH], empty[EX_DEPTH], added[EX_SUMS], taken[EX_SUMS];
    int abort_flag;
};

template <int NB>
__device__ __forceinline__ Ring ring_of(const Experts &p, char *smem, Shared<NB> &sh) {
    Ring r;
    r.depth = p.depth;
    r.step = p.step;
    r.base = smem + p.ring_at;
    r.full = sh.full;
    r.empty = sh.empty;
    r.slot = 0;
    r.phase = 0;
    r.ok = true;
    return r;
}
// (before the routing's barriers; both: teams take part in a unit)
template <int NB>
__device__ __forceinline__ void init(Shared<NB> &sh, bool both) {
    if (threadIdx.x < EX_DEPTH) {
        mbar_init(sh.full + threadIdx.x, 2);
        mbar_init(sh.empty + threadIdx.x, EX_TEAM);
    }
    if (threadIdx.x < EX_SUMS) {
        mbar_init(sh.added + threadIdx.x, both ? EX_MMA : EX_TEAM);
        mbar_init(sh.taken + threadIdx.x, 1);
    }
    if (threadIdx.x == 0) sh.abort_flag = 0;
    umma::fence_mbar_init();
}

// A warp's sums of a unit (the turn-th of the block's) go to the warps that add up ...
template <int NB>
__device__ __forceinline__ void give(Shared<NB> &sh, float (&c)[NB][2][4], int turn, int place, bool &ok, int32_t *status) {
    const int b = turn % EX_SUMS, lane = threadIdx.x & 31;
    ok = ok && mbar_wait(sh.taken + b, (turn / EX_SUMS & 1) ^ 1, &sh.abort_flag, status);
#pragma unroll
    for (int j = 0; j < NB; ++j)
        sh.sums[b][place][j][lane] = make_float4(c[j][0][0] + c[j][1][0], c[j][0][1] + c[j][1][1],
                                                 c[j][0][2] + c[j][1][2], c[j][0][3] + c[j][1][3]);
    __syncwarp();
    if (lane == 0) mbar_arrive(sh.added + b);
#pragma unroll
    for (int i = 0; i < NB * 8; ++i) c[i / 8][i / 4 % 2][i % 4] = 0.f;
}
// ... which take them in the warps' order (from one team, where units have one step, or both).
template <int NB>
__device__ __forceinline__ bool take(Shared<NB> &sh, float (&c)[NB][4], int turn, bool both, int32_t *status) {
    const int b = turn % EX_SUMS, lane = threadIdx.x & 31;
    if (!mbar_wait(sh.added + b, turn / EX_SUMS & 1, &sh.abort_flag, status)) return false;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        float4 v = sh.sums[b][0][j][lane];
#pragma unroll
        for (int w = 1; w < EX_MMA; ++w) {
            if (w == EX_TEAM && !both) break;
            const float4 o = sh.sums[b][w][j][lane];
            v.x += o.x;
            v.y += o.y;
            v.z += o.z;
            v.w += o.w;
        }
        c[j][0] = v.x;
        c[j][1] = v.y;
        c[j][2] = v.z;
        c[j][3] = v.w;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(sh.taken + b);
    return true;
}

// ---- the first product --------------------------------------------------------------

template <bool F16, bool BOXES, bool X_ALIGNED, int NB>
__global__ void __launch_bounds__(EX_THREADS)
k_experts_in(const __grid_constant__ Experts p, const __grid_constant__ WeightMaps map) {
    extern __shared__ __align__(1024) char smem[];
    __shared__ Shared<NB> sh;
    constexpr int CH = EX_COLS / EX_STRIDE, XU = X_ALIGNED ? 1 : 2;
    constexpr bool TWICE = NB == 1 && BOXES && X_ALIGNED;      // registers for two steps of x
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q = lane & 3, wr = row_of(g8);
    const int cols = p.cols, steps = (p.n_in + cols - 1) / cols;
    const bool both = steps > 1;
    if (BOXES && tid == 0) umma::tma_prefetch_desc(first_map(map, p.n_in, cols));
    init(sh, both);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Routing r(p, smem);
    route<NB * 8>(p, r, smem);
    Ring ring = ring_of(p, smem, sh);
    const int wide = p.gated ? 8 : 16;
    Walk w(*r.jobs, 1, (p.hidden + wide - 1) / wide);
    const int u0 = w.u;
    const auto weights_row = [&](const Walk &w, int i) -> const uint16_t * {
        const int f = w.tile * wide + (p.gated ? i & 7 : i);
        const int64_t at = p.gated && i >= 8 ? p.hidden + f : f;
        return f < p.hidden ? p.w_in + r.expert[w.job] * p.w_in_z + at * p.w_in_ld : nullptr;
    };
    if (warp >= EX_MMA && warp < EX_MMA + EX_COPY) {
        Steps at(w, steps, steps);
        if (warp > EX_MMA) {
            at.next();
            ring.next();
        }
        while (at.more()) {
            const uint16_t *row = !BOXES && lane < 16 ? weights_row(at.w, lane) : nullptr;
            const int f0 = at.w.tile * wide, y = lane == 0 ? f0 : p.gated ? p.hidden + f0 : f0 + 8;
            if (!ring.copy<BOXES>(map, y, r.expert[at.w.job], row, at.s, cols, p.n_in, &sh.abort_flag, p.status, p.test_stall)) return;
            at.next();
            if (at.more()) at.next();
        }
        return;
    }
    if (warp >= EX_MMA) {
        for (; w.more(); w.next()) {
            const int turn = w.u - u0;
            if (turn % EX_ADD != warp - EX_MMA - EX_COPY) continue;
            const int n = r.n[w.job], begin = r.begin[w.job];
            float c[NB][4];
            if (!take(sh, c, turn, both, p.status)) return;
            // rows wr and wr + 8 of columns 2 q and 2 q + 1
#pragma unroll
            for (int k = 0; k < NB * 4; ++k) {
                const int i = k % 4, column = k / 4 * 8 + 2 * q + (i & 1), f = w.tile * wide + wr + (i & 2) * 4;
                if (column >= n || (p.gated && (i & 2)) || f >= p.h_ld) continue;
                float v = activated(c[k / 4][i], p.act);
                if (p.gated) v *= c[k / 4][i | 2];
                if (f >= p.hidden) v = 0.f;              // (the second product reads whole 16 bytes)
                const int64_t to = (int64_t)r.list[begin + column] * expert_terms(F16) * p.h_ld + f;
                if (F16) {
                    float *h = (float *)p.h + to;
                    tf32_terms(v, h[0], h[p.h_ld]);
                } else {
                    uint16_t *h = (uint16_t *)p.h + to;
                    bf16_terms(bf16_cut(v, h[0]), h[p.h_ld], h[2 * p.h_ld]);
                }
            }
            __syncwarp();
        }
        return;
    }
    const int team = warp / EX_TEAM, member = warp % EX_TEAM;
    // My part of x: of the job's rows g8 (and g8 + 8).  It is loaded a step ahead; where that
    // would not fit the registers, after the step before it (the other team's step is between:
    // 7 unaligned rows 30.1 us for 27.3 so), unless it is the same again.
    const uint16_t *row[NB] = {};
    int row_job = -1, row_step = -1, n = 0;
    const auto fetch = [&](uint4(&x)[CH][NB][XU], const Steps &at) {
        if (!TWICE && at.w.job == row_job && at.s == row_step) return;
        row_step = at.s;
        if (at.w.job != row_job) {
            row_job = at.w.job;
            n = r.n[row_job];
#pragma unroll
            for (int j = 0; j < NB; ++j)
                row[j] = g8 + j * 8 < n ? p.x + r.list[r.begin[row_job] + g8 + j * 8] / p.top * p.x_ld : nullptr;
        }
        const int to = min((at.s + 1) * cols, p.n_in);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) eight<X_ALIGNED>(x[i][j], row[j], at.s * cols + member * 32 + i * EX_STRIDE + q * 8, to);
    };
    Steps ahead(w, steps, steps);         // the next step of this team, whose x is under way
    if (team) {
        ahead.next();
        ring.next();
    }
    int given = u0;
    float c[NB][2][4] = {};
    const auto give_up_to = [&](int u) {
        for (; given < u; ++given) give(sh, c, given - u0, warp, ring.ok, p.status);
    };
    if (both) give_up_to(min(ahead.w.u, w.end));
    if (!ahead.more()) return;
    const auto take_step = [&](uint4(&x)[CH][NB][XU], uint4(&next)[CH][NB][XU]) {
        const Steps at = ahead;
        int sx[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) sx[j] = (int)((uintptr_t)row[j] & 15);
        ahead.next();
        if (ahead.more()) ahead.next();
        if (TWICE && ahead.more()) fetch(next, ahead);
        int sa = 0, sb = 0;
        if (!BOXES) {
            sa = (int)((uintptr_t)weights_row(at.w, wr) & 15);
            sb = (int)((uintptr_t)weights_row(at.w, wr + 8) & 15);
        }
        const char *from = ring.wait_full(&sh.abort_flag, p.status);
        const int left = min(cols, p.n_in - at.s * cols);
        // (all loads before the first multiplication: what is beyond the row is zero)
        uint4 a[CH], d[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int k = member * 32 + i * EX_STRIDE;
            a[i] = d[i] = make_uint4(0, 0, 0, 0);
            if (k < left) {
                a[i] = weights<BOXES>(from, wr, q, false, k, cols, sa);
                d[i] = weights<BOXES>(from, wr, q, true, k, cols, sb);
            }
            if (!BOXES && k + 32 > left) {
                const int e = max(0, min(8, left - k - q * 8));
                a[i] = first(a[i], e);
                d[i] = first(d[i], e);
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (j && n <= j * 8) break;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int k = member * 32 + i * EX_STRIDE;
                uint4 v = X_ALIGNED ? x[i][j][0] : shifted(x[i][j][0], x[i][j][XU - 1], sx[j]);
                if (!BOXES && k + 32 > left) v = first(v, max(0, min(8, left - k - q * 8)));
                mma16<F16>(c[j][0], a[i].x, d[i].x, a[i].y, d[i].y, v.x, v.y);
                mma16<F16>(c[j][1], a[i].z, d[i].z, a[i].w, d[i].w, v.z, v.w);
            }
        }
        ring.release();
        if (!TWICE && ahead.more()) fetch(next, ahead);
        if (both) give_up_to(min(ahead.w.u, w.end));
        else give(sh, c, at.w.u - u0, member, ring.ok, p.status);
        return ahead.more();
    };
    if constexpr (TWICE) {
        uint4 one[CH][NB][XU], two[CH][NB][XU];
        fetch(one, ahead);
        while (take_step(one, two) && take_step(two, one)) {
        }
    } else {
        uint4 x[CH][NB][XU];
        fetch(x, ahead);
        while (take_step(x, x)) {
        }
    }
}

// ---- the second product -----------------------------------------------------------

template <bool F16>
__device__ __forceinline__ void store(const Experts &p, int t, int n, float v) {
    uint16_t *y = p.y + t * p.y_ld + n;
    if (F16) *(__half *)y = __float2half_rn(v);
    else *(__nv_bfloat16 *)y = __float2bfloat16_rn(v);
}

__device__ __forceinline__ uint4 widened(uint32_t lo, uint32_t hi) {
    const float2 a = __half22float2(*(const __half2 *)&lo), b = __half22float2(*(const __half2 *)&hi);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
}

template <bool F16, bool BOXES, int NB>
__global__ void __launch_bounds__(EX_THREADS)
k_experts_out(const __grid_constant__ Experts p, const __grid_constant__ WeightMaps map) {
    extern __shared__ __align__(1024) char smem[];
    __shared__ Shared<NB> sh;
    // a lane's eight columns of 32: h's terms, in 16-byte loads
    constexpr int CH = EX_COLS / (F16 ? 2 : 1) / EX_STRIDE, TERM = F16 ? 2 : 1, TERMS = expert_terms(F16), HU = TERMS * TERM;
    // (registers: no room for two steps of three terms, 149 us for 133 so; and beside two
    // columns of h weights are loaded as they are used)
    constexpr bool TWICE = NB == 1 && BOXES && F16, EARLY = NB == 1 || F16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q = lane & 3, wr = row_of(g8);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (BOXES && tid == 0) umma::tma_prefetch_desc(first_map(map, p.hidden, p.cols));
    init(sh, true);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    Routing r(p, smem);
    load_routing(p, smem);
    Ring ring = ring_of(p, smem, sh);
    // pieces of the contraction, that the busiest block has the least to do
    const int cols = p.cols, tiles = (p.n_out + 15) / 16, all = *r.jobs * tiles, all_steps = (p.hidden + cols - 1) / cols;
    int splits = 1;
    int64_t least = INT64_MAX;
    for (int s = 1; s <= p.splits && s <= all_steps; s *= 2) {
        const int64_t cost = (int64_t)((all * s + gridDim.x - 1) / gridDim.x) * ((all_steps + s - 1) / s * cols + EX_UNIT_COST);
        if (cost < least) {
            least = cost;
            splits = s;
        }
    }
    // Beside several columns of h, pieces of two steps, one a team, whose h stays in the
    // registers from tile to tile (64 rows, 4 of 16 experts each, 1,024 -> 2 x 2,048, bf16:
    // 109 us without, 90 with; in fp16, whose steps are half as wide, 90.7 and 93.5).
    if (NB > 1 && !F16)
        while (splits < p.splits && splits * 2 < all_steps) splits *= 2;
    const int per = (all_steps + splits - 1) / splits;       // steps of a piece, and pieces with any
    splits = (all_steps + per - 1) / per;
    // one choice a row, taken whole: its result is the row's, and rows without one get zeros
    const bool whole = p.top == 1 && p.splits == 1;
    Walk w(*r.jobs, splits, tiles);
    const int u0 = w.u;
    if (warp >= EX_MMA && warp < EX_MMA + EX_COPY) {
        Steps at(w, per, all_steps);
        if (warp > EX_MMA) {
            at.next();
            ring.next();
        }
        while (at.more()) {
            const int o = at.w.tile * 16, e = r.expert[at.w.job];
            const uint16_t *row = nullptr;
            if (!BOXES && lane < 16 && o + lane < p.n_out) row = p.w_out + e * p.w_out_z + (int64_t)(o + lane) * p.w_out_ld;
            if (!ring.copy<BOXES>(map, o + lane * 8, e, row, at.s, cols, p.hidden, &sh.abort_flag, p.status, p.test_stall)) return;
            at.next();
            if (at.more()) at.next();
        }
        return;
    }
    if (warp >= EX_MMA) {
        const int i0 = tid - (EX_MMA + EX_COPY) * 32;
        if (whole) {
            for (int t = blockIdx.x; t < p.rows; t += gridDim.x)
                if (r.choice[t] < 0)
                    for (int o = i0; o < p.n_out; o += EX_ADD * 32) store<F16>(p, t, o, 0.f);
        } else if (blockIdx.x == 0 && i0 == 0) {
            *p.used_splits = splits;
        }
        for (; w.more(); w.next()) {
            const int turn = w.u - u0;
            if (turn % EX_ADD != warp - EX_MMA - EX_COPY) continue;
            const int n = r.n[w.job], begin = r.begin[w.job];
            float c[NB][4];
            if (!take(sh, c, turn, true, p.status)) return;
#pragma unroll
            for (int k = 0; k < NB * 4; ++k) {
                const int i = k % 4, column = k / 4 * 8 + 2 * q + (i & 1), o = w.tile * 16 + wr + (i & 2) * 4;
                if (column >= n || o >= p.n_out) continue;
                const int pair = r.list[begin + column];
                if (whole) store<F16>(p, pair, o, r.gate[pair] * c[k / 4][i]);
                else p.part[((int64_t)pair * splits + w.split) * p.n_out + o] = c[k / 4][i];
            }
            __syncwarp();
        }
        return;
    }
    const int team = warp / EX_TEAM, member = warp % EX_TEAM;
    const int64_t next_term = p.h_ld * (F16 ? 4 : 2) / 16;
    const uint4 *row[NB] = {};
    int row_job = -1, row_step = -1, n = 0;
    const auto fetch = [&](uint4(&h)[CH][NB][HU], const Steps &at) {
        if (!TWICE && at.w.job == row_job && at.s == row_step) return;
        row_step = at.s;
        if (at.w.job != row_job) {
            row_job = at.w.job;
            n = r.n[row_job];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                row[b] = nullptr;
                if (g8 + b * 8 < n)
                    row[b] = (const uint4 *)((const char *)p.h +
                                             (int64_t)r.list[r.begin[row_job] + g8 + b * 8] * TERMS * p.h_ld * (F16 ? 4 : 2));
            }
        }
        const int to = min((at.s + 1) * cols, p.hidden);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = at.s * cols + member * 32 + i * EX_STRIDE + q * 8;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bool in = row[b] && c < to;
#pragma unroll
                for (int j = 0; j < HU; ++j) {
                    h[i][b][j] = make_uint4(0, 0, 0, 0);
                    if (in) h[i][b][j] = row[b][j / TERM * next_term + c / 8 * TERM + j % TERM];
                }
            }
        }
    };
    Steps ahead(w, per, all_steps);       // the next step of this team, whose h is under way
    if (team) {
        ahead.next();
        ring.next();
    }
    int given = u0;
    float c[NB][2][4] = {};
    const auto give_up_to = [&](int u) {
        for (; given < u; ++given) give(sh, c, given - u0, warp, ring.ok, p.status);
    };
    give_up_to(min(ahead.w.u, w.end));
    if (!ahead.more()) return;
    const auto take_step = [&](uint4(&h)[CH][NB][HU], uint4(&next)[CH][NB][HU]) {
        const Steps at = ahead;
        ahead.next();
        if (ahead.more()) ahead.next();
        if (TWICE && ahead.more()) fetch(next, ahead);
        int sa = 0, sb = 0;
        if (!BOXES) {
            const uint16_t *w = p.w_out + r.expert[at.w.job] * p.w_out_z + (int64_t)(at.w.tile * 16 + wr) * p.w_out_ld;
            sa = (int)((uintptr_t)w & 15);
            sb = (int)((uintptr_t)(w + 8 * p.w_out_ld) & 15);
        }
        const char *from = ring.wait_full(&sh.abort_flag, p.status);
        const int left = min(cols, p.hidden - at.s * cols);
        // (EARLY: all loads before the first multiplication; what is beyond the row is zero)
        uint4 a[CH], d[CH];
        const auto load = [&](int i) {
            const int k = member * 32 + i * EX_STRIDE;
            a[i] = d[i] = make_uint4(0, 0, 0, 0);
            if (k < left) {
                a[i] = weights<BOXES>(from, wr, q, false, k, cols, sa);
                d[i] = weights<BOXES>(from, wr, q, true, k, cols, sb);
            }
            if (!BOXES && k + 32 > left) {
                const int e = max(0, min(8, left - k - q * 8));
                a[i] = first(a[i], e);
                d[i] = first(d[i], e);
            }
        };
        if (EARLY)
#pragma unroll
            for (int i = 0; i < CH; ++i) load(i);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (!EARLY) load(i);
            uint4 a0, a1, d0, d1;
            if (F16) {
                a0 = widened(a[i].x, a[i].y), a1 = widened(a[i].z, a[i].w);
                d0 = widened(d[i].x, d[i].y), d1 = widened(d[i].z, d[i].w);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b && n <= b * 8) break;
                if (F16) {
#pragma unroll
                    for (int j = 0; j < HU; j += TERM) {
                        const uint4 v = h[i][b][j], w = h[i][b][j + TERM - 1];
                        mma8_tf32(c[b][0], a0.x, d0.x, a0.y, d0.y, v.x, v.y);
                        mma8_tf32(c[b][1], a0.z, d0.z, a0.w, d0.w, v.z, v.w);
                        mma8_tf32(c[b][0], a1.x, d1.x, a1.y, d1.y, w.x, w.y);
                        mma8_tf32(c[b][1], a1.z, d1.z, a1.w, d1.w, w.z, w.w);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < HU; ++j) {
                        mma16<false>(c[b][0], a[i].x, d[i].x, a[i].y, d[i].y, h[i][b][j].x, h[i][b][j].y);
                        mma16<false>(c[b][1], a[i].z, d[i].z, a[i].w, d[i].w, h[i][b][j].z, h[i][b][j].w);
                    }
                }
            }
        }
        if (!TWICE && ahead.more()) fetch(next, ahead);
        ring.release();
        give_up_to(min(ahead.w.u, w.end));
        return ahead.more();
    };
    if constexpr (TWICE) {
        uint4 one[CH][NB][HU], two[CH][NB][HU];
        fetch(one, ahead);
        while (take_step(one, two) && take_step(two, one)) {
        }
    } else {
        uint4 h[CH][NB][HU];
        fetch(h, ahead);
        while (take_step(h, h)) {
        }
    }
}

// y: what each row's choices gave, added up in their order (and the pieces of each).
template <bool F16>
__global__ void __launch_bounds__(SUM_THREADS)
k_experts_sum(const __grid_constant__ Experts p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int o = blockIdx.x * SUM_THREADS + threadIdx.x, t = blockIdx.y, splits = *p.used_splits;
    if (o >= p.n_out) return;
    const Routing r(p, p.tables);
    float y = 0.f;
    for (int j = 0; j < p.top; ++j) {
        const float gate = r.gate[t * p.top + j];
        if (r.choice[t * p.top + j] < 0) continue;
        const float *part = p.part + (int64_t)(t * p.top + j) * splits * p.n_out + o;
        float v = 0.f;
#pragma unroll 4
        for (int i = 0; i < splits; ++i) v += part[(int64_t)i * p.n_out];
        y = fmaf(gate, v, y);
    }
    store<F16>(p, t, o, y);
}

cudaLaunchConfig_t early(dim3 grid, int threads, size_t smem, cudaStream_t s, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

typedef void (*Kernel)(Experts, WeightMaps);

// Columns of a step: as even as it gets for this width, in whole boxes.
int even_columns(int width, int most) {
    const int steps = (width + most - 1) / most;
    return ((width + steps - 1) / steps + 63) & ~63;
}

constexpr int step_bytes(int cols) { return (16 * (cols * 2 + 16) + 1023) & ~1023; }
static_assert(2 * step_bytes(EX_COLS) + 16 + EX_PAIRS * 13 + 16 + EX_GROUPS * 4 + 1023 <= EX_RING, "tables and two steps");

cudaError_t launch(Kernel kernel, Experts p, const WeightMaps &map, int cols, int nsm, cudaStream_t s) {
    p.cols = cols;
    p.step = step_bytes(cols);
    p.ring_at = (int)routing_bytes(p);
    // (an even number of slots, each of which belongs to one team: another team's use of it,
    // one phase of its barriers later, could not be told from the one before)
    const int depth = (EX_RING - p.ring_at) / p.step & ~1;
    p.depth = depth > EX_DEPTH ? EX_DEPTH : depth;
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early(dim3((unsigned)nsm), EX_THREADS, (size_t)p.ring_at + p.depth * p.step, s, at);
    return cudaLaunchKernelEx(&cfg, kernel, p, map);
}

bool whole16(const void *p, int64_t ld) { return (((uintptr_t)p & 15) | (ld & 7)) == 0; }

template <bool F16, int NB>
Kernel kernel_in(bool boxes, bool x_aligned) {
    return boxes ? x_aligned ? k_experts_in<F16, true, true, NB> : k_experts_in<F16, true, false, NB>
                 : x_aligned ? k_experts_in<F16, false, true, NB> : k_experts_in<F16, false, false, NB>;
}

template <bool F16, int NB>
Kernel kernel_out(bool boxes) {
    return boxes ? k_experts_out<F16, true, NB> : k_experts_out<F16, false, NB>;
}

template <bool F16>
cudaError_t both(const Experts &p, const ExpertMaps &m, int nsm, cudaStream_t s) {
    const bool in = m.in_boxes, out = m.out_boxes;
    // Jobs of 16 pairs where experts have more than 8 on average (64 rows, 4 experts each,
    // 1,024 -> 2 x 2,048, bf16, jobs of 8 and 16: over 24 experts 106 and 89 us, over 28 109 and
    // 98; over 32 106 and 109, for what fewer rows have their registers hold half the loads
    // under way).
    const bool x = whole16(p.x, p.x_ld), two = p.rows * p.top > 8 * p.groups;
    cudaError_t e = launch(two ? kernel_in<F16, 2>(in, x) : kernel_in<F16, 1>(in, x), p, m.in, m.in_cols, nsm, s);
    if (e != cudaSuccess) return e;
    e = launch(two ? kernel_out<F16, 2>(out) : kernel_out<F16, 1>(out), p, m.out, m.out_cols, nsm, s);
    if (e != cudaSuccess || (p.top == 1 && p.splits == 1)) return e;
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg =
        early(dim3((unsigned)((p.n_out + SUM_THREADS - 1) / SUM_THREADS), (unsigned)p.rows), SUM_THREADS, 0, s, at);
    return cudaLaunchKernelEx(&cfg, k_experts_sum<F16>, p);
}

}  // namespace

// The most pieces of the second product's contraction: none under 512 columns.
int expert_splits(int hidden) {
    int n = 1;
    while (n < 16 && n * 2 * 512 <= hidden) n *= 2;
    return n;
}

size_t expert_tables(int rows, int top) {
    Experts p;
    p.rows = rows;
    p.top = top;
    return tables_bytes(p);
}

// Columns of each product's steps.
void expert_plan(const Experts &p, bool f16, ExpertMaps *m) {
    m->in_cols = even_columns(p.n_in, EX_COLS);
    m->out_cols = even_columns(p.hidden, f16 ? EX_COLS / 2 : EX_COLS);
}

template <bool F16>
static cudaError_t prepare() {
    cudaError_t e = cudaSuccess;
    const auto set = [&](Kernel kernel) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, EX_RING);
    };
    for (const bool w : {true, false}) {
        for (const bool x : {true, false}) {
            set(kernel_in<F16, 1>(w, x));
            set(kernel_in<F16, 2>(w, x));
        }
        set(kernel_out<F16, 1>(w));
        set(kernel_out<F16, 2>(w));
    }
    return e;
}

cudaError_t experts_prepare() {
    const cudaError_t e = prepare<true>();
    return e == cudaSuccess ? prepare<false>() : e;
}

cudaError_t launch_experts(const Experts &p, const ExpertMaps &m, bool f16, int nsm, cudaStream_t s) {
    return f16 ? both<true>(p, m, nsm, s) : both<false>(p, m, nsm, s);
}

}  // namespace hwr
