// A layer of experts for a few rows (decode steps): routing, both products, the
// activation between them and the sum over a row's choices, in two launches.
//
//   k_experts_in    h[t, j] = act(W_gate[e] x[t]) * (W_up[e] x[t])  (or act(W_in[e] x[t]))
//   k_experts_out   y[t] = sum over j of p[t, j] W_out[e] h[t, j]
//
// Bound by HBM: of each expert that a row chooses the weights are read once (by up to
// 8 x NB of its rows at a time), everything else stays in L2.  Every block finds the
// choices and the experts' rows by itself from the scores (a few KB), which costs less
// than a launch between.  A unit of work is 16 rows of a weight matrix, whole (in the
// first product 8 gate rows and the 8 up rows that they meet, so that the activation
// finds both in one block); the eight warps of a block share its contraction, 32
// columns in turn, and add their sums up through shared memory.  A block walks a run
// of consecutive units, always one step of loads ahead (32 or 64 bytes a lane of each
// operand, across the ends of units), and the second launch begins under the first's
// end with routing and its first weights.
//
// The multiplications are warp-level MMAs: 16 rows of weights, 8 rows of x.  The
// contraction's order is free, so a lane takes eight consecutive columns of a weight's
// row in one 16-byte load, and the same of x.  h is summed in fp32 and enters the second
// product as two terms that give 16 bits of it or more at any magnitude: two bf16 values
// beside bf16 weights; beside fp16 weights, whose range is too small for it, two tf32
// values, the weights widened to tf32 exactly.
#include "ops_internal.cuh"
#include "values.cuh"

namespace hwr {
namespace {

constexpr int EX_THREADS = 256, EX_WARPS = EX_THREADS / 32;
constexpr int EX_STEP = 4;                 // blocks of 32 columns that a warp loads ahead
constexpr int EX_PAIRS = EXPERTS_MAX_ROWS * EXPERTS_MAX_TOP;
constexpr int EX_GROUPS = OPS_MAX_GROUPS;
constexpr uint32_t ALL = 0xffffffffu;
static_assert(EX_GROUPS == 4 * EX_THREADS, "four groups a thread");

template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma8_tf32(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 zeros() { return make_uint4(0, 0, 0, 0); }

// Read once: not kept in L1, which is x's and h's.
__device__ __forceinline__ uint4 stream16(const void *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
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

// Eight elements of a row of n from column c on, zeros beyond it and for no row.  A row
// that does not begin on a 16-byte boundary takes the two aligned units around them,
// those that hold an element of the row, shifted into place.
template <bool ALIGNED, bool STREAM>
__device__ __forceinline__ uint4 eight(const uint16_t *row, int c, int n) {
    if (!row || c >= n) return zeros();
    const uint16_t *p = row + c;
    uint4 v;
    if (ALIGNED) {
        v = STREAM ? stream16(p) : __ldg((const uint4 *)p);
    } else {
        const int s = (int)((uintptr_t)p & 15);
        const uint16_t *q = (const uint16_t *)((uintptr_t)p - s);
        const uint4 a = __ldg((const uint4 *)q);
        const uint4 b = s && q + 8 < row + n ? __ldg((const uint4 *)q + 1) : zeros();
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (s & 8)
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        if (s & 4)
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        const int h = (s & 2) * 8;
        v = make_uint4(__funnelshift_r(w[0], w[1], h), __funnelshift_r(w[1], w[2], h), __funnelshift_r(w[2], w[3], h),
                       __funnelshift_r(w[3], w[4], h));
    }
    return c + 8 <= n ? v : first(v, n - c);
}

// ---- routing --------------------------------------------------------------------

// Which rows meet which expert: pairs (row t, choice j) at t * top + j, the pairs of an
// expert side by side in `list`, in jobs of at most 8 NB of them.
struct Routing {
    float gate[EX_PAIRS];
    int count[EX_GROUPS];
    alignas(16) int16_t choice[EX_PAIRS + 8];             // -1: none
    uint16_t list[EX_PAIRS], begin[EX_PAIRS], expert[EX_PAIRS];      // (jobs: begin, expert)
    uint8_t n[EX_PAIRS];
    int jobs, warp_jobs[EX_WARPS], warp_pairs[EX_WARPS];
};

// Order of a score among the choices: larger ones above, then lower indices; 0 for one
// that is never chosen (-inf, NaN).
__device__ __forceinline__ uint64_t score_key(float v, int e) {
    if (!(v > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(v + 0.f);
    return (uint64_t)(u ^ (u >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | (uint32_t)~e;
}

__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
    for (int d = 16; d; d /= 2) {
        const uint64_t o = __shfl_xor_sync(ALL, k, d);
        k = k > o ? k : o;
    }
    return k;
}
__device__ __forceinline__ float warp_sum(float v) {
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(ALL, v, d);
    return v;
}

template <int NB>
__device__ __forceinline__ void route(const Experts &p, Routing &r) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, pairs = p.rows * p.top, E = p.groups;
    for (int i = tid; i < E; i += EX_THREADS) r.count[i] = 0;
    if (p.scores) {
        for (int t = warp; t < p.rows; t += EX_WARPS) {
            const float *s = p.scores + t * p.scores_ld;
            uint64_t last = ~0ull;
            float mine = -INFINITY, top = 0.f;
            int choice = -1;
            for (int j = 0; j < p.top; ++j) {
                uint64_t best = 0;
                for (int e = lane; e < E; e += 32) {
                    const uint64_t k = score_key(s[e], e);
                    if (k < last && k > best) best = k;
                }
                last = warp_max(best);
                if (!last) break;
                const int e = (int)~(uint32_t)last;
                const float v = s[e];
                if (j == 0) top = v;
                if (lane == j) {
                    mine = v;
                    choice = e;
                }
            }
            const float w = choice >= 0 ? expf(mine - top) : 0.f;
            float total = w;
            if (p.over_all) {
                total = 0.f;
                for (int e = lane; e < E; e += 32) total += s[e] > -INFINITY ? expf(s[e] - top) : 0.f;
            }
            total = warp_sum(total);
            if (lane < p.top) {
                r.choice[t * p.top + lane] = (int16_t)choice;
                r.gate[t * p.top + lane] = choice >= 0 ? w / total : 0.f;
            }
        }
    } else {
        for (int i = tid; i < pairs; i += EX_THREADS) {
            const int c = p.choice[i];
            r.choice[i] = (int16_t)((uint32_t)c < (uint32_t)E ? c : -1);
            r.gate[i] = p.gates[i];
        }
    }
    __syncthreads();
    for (int i = tid; i < pairs; i += EX_THREADS)
        if (r.choice[i] >= 0) atomicAdd(&r.count[r.choice[i]], 1);
    __syncthreads();
    // four experts a thread: where their pairs and jobs begin
    int jobs = 0, all = 0, n[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        n[k] = tid * 4 + k < E ? r.count[tid * 4 + k] : 0;
        jobs += (n[k] + 8 * NB - 1) / (8 * NB);
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
        r.warp_jobs[warp] = j;
        r.warp_pairs[warp] = a;
    }
    __syncthreads();
    j -= jobs;
    a -= all;
    for (int w = 0; w < warp; ++w) {
        j += r.warp_jobs[w];
        a += r.warp_pairs[w];
    }
    if (tid == EX_THREADS - 1) r.jobs = j + jobs;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (n[k]) r.count[tid * 4 + k] = a;
        for (int b = 0; b < n[k]; b += 8 * NB, ++j) {
            r.expert[j] = (uint16_t)(tid * 4 + k);
            r.begin[j] = (uint16_t)(a + b);
            r.n[j] = (uint8_t)(n[k] - b < 8 * NB ? n[k] - b : 8 * NB);
        }
        a += n[k];
    }
    // Within a job pairs may lie in any order (a pair's results do not depend on its column
    // of the MMA); where an expert has several, they lie in their own order, so that every
    // block deals them out alike.
    bool several = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) several |= n[k] > 8 * NB;
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
    __syncthreads();
}

// A block's run of units.
__device__ __forceinline__ void run_of(int units, int &u, int &end) {
    u = (int)((int64_t)units * blockIdx.x / gridDim.x);
    end = (int)((int64_t)units * (blockIdx.x + 1) / gridDim.x);
}

// Weights of a step: rows g8 and g8 + 8 of the unit.
struct Step {
    uint4 a[EX_STEP], d[EX_STEP];
};

template <bool ALIGNED>
__device__ __forceinline__ void load(Step &s, const uint16_t *ra, const uint16_t *rb, int block, int end, int q, int n) {
#pragma unroll
    for (int i = 0; i < EX_STEP; ++i) {
        const int b = block + i * EX_WARPS, c = b * 32 + q * 8;
        s.a[i] = b < end ? eight<ALIGNED, true>(ra, c, n) : zeros();
        s.d[i] = b < end ? eight<ALIGNED, true>(rb, c, n) : zeros();
    }
}

__device__ __forceinline__ float activated(float u, int act) {
    if (act == HWR_ACT_RELU) return u < 0.f ? 0.f : u;
    if (act == HWR_ACT_SILU) return u / (1.f + expf(-u));
    return 0.5f * u * (1.f + erff(u * 0.70710678f));
}

// A value as two bf16 terms, or two of tf32 (the high one cut off strictly below the
// value, as in bf16_terms).
__device__ __forceinline__ void tf32_terms(float v, float &high, float &low) {
    const uint32_t u = __float_as_uint(v), m = u & 0x7fffffffu;
    high = __uint_as_float(m - 1 < 0x7f7fffffu ? (u - 1) & 0xffffe000u : u);
    low = m < 0x7f800000u ? v - high : v;
}

// ---- the first product --------------------------------------------------------------

template <bool F16, bool ALIGNED, int NB>
__global__ void __launch_bounds__(EX_THREADS, 2)
k_experts_in(const __grid_constant__ Experts p) {
    __shared__ Routing r;
    __shared__ float sums[EX_WARPS][16][8 * NB + 1];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q = lane & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    route<NB>(p, r);
    const int wide = p.gated ? 8 : 16, tiles = (p.hidden + wide - 1) / wide, blocks = (p.n_in + 31) / 32;
    const bool x_aligned = (((uintptr_t)p.x & 15) | (p.x_ld & 7)) == 0;
    int u, end;
    run_of(r.jobs * tiles, u, end);
    if (u >= end) return;
    const uint16_t *ra, *rb;
    auto rows = [&](int unit) {
        const int job = unit / tiles, f = (unit - job * tiles) * wide + g8;
        const uint16_t *w = p.w_in + r.expert[job] * p.w_in_z;
        const int up = p.gated ? p.hidden + f : f + 8;
        ra = f < p.hidden ? w + f * p.w_in_ld : nullptr;
        rb = up < (p.gated ? 2 * p.hidden : p.hidden) ? w + up * p.w_in_ld : nullptr;
    };
    Step now, next;
    rows(u);
    load<ALIGNED>(now, ra, rb, warp, blocks, q, p.n_in);
    for (; u < end; ++u) {
        const int job = u / tiles, n = r.n[job], begin = r.begin[job];
        const uint16_t *x[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int at = b * 8 + g8;
            x[b] = at < n ? p.x + r.list[begin + at] / p.top * p.x_ld : nullptr;
        }
        float c[NB][4] = {};
        for (int b0 = 0; b0 < blocks; b0 += EX_STEP * EX_WARPS) {
            const int more = b0 + EX_STEP * EX_WARPS;
            if (more < blocks) {
                load<ALIGNED>(next, ra, rb, more + warp, blocks, q, p.n_in);
            } else if (u + 1 < end) {
                rows(u + 1);
                load<ALIGNED>(next, ra, rb, warp, blocks, q, p.n_in);
            }
#pragma unroll
            for (int i = 0; i < EX_STEP; ++i) {
                const int k = b0 + warp + i * EX_WARPS;
                if (k >= blocks) break;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (b * 8 >= n) break;
                    const uint4 v = x_aligned ? eight<true, false>(x[b], k * 32 + q * 8, p.n_in)
                                              : eight<false, false>(x[b], k * 32 + q * 8, p.n_in);
                    mma16<F16>(c[b], now.a[i].x, now.d[i].x, now.a[i].y, now.d[i].y, v.x, v.y);
                    mma16<F16>(c[b], now.a[i].z, now.d[i].z, now.a[i].w, now.d[i].w, v.z, v.w);
                }
            }
            now = next;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][g8 + (i >> 1) * 8][b * 8 + 2 * q + (i & 1)] = c[b][i];
        __syncthreads();
        const int f0 = (u - job * tiles) * wide;
        for (int i = tid; i < wide * 8 * NB; i += EX_THREADS) {
            const int f = i % wide, at = i / wide;
            if (at >= n) break;
            float v = 0.f, up = 0.f;
#pragma unroll
            for (int w = 0; w < EX_WARPS; ++w) {
                v += sums[w][f][at];
                if (p.gated) up += sums[w][f + 8][at];
            }
            v = activated(v, p.act);
            if (p.gated) v *= up;
            // (groups of eight: those of the last rows are filled up with zeros)
            const int64_t group = (int64_t)r.list[begin + at] * p.h_groups + (f0 + f) / 8;
            if (f0 + f >= p.h_groups * 8) continue;
            if (F16) {
                float *h = (float *)p.h + group * 16 + (f & 7);
                tf32_terms(v, h[0], h[8]);
            } else {
                uint16_t *h = (uint16_t *)p.h + group * 16 + (f & 7);
                bf16_terms(v, h[0], h[8]);
            }
        }
        __syncthreads();
    }
}

// ---- the second product -----------------------------------------------------------

// Rows without a choice, where no row has one.
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

template <bool F16, bool ALIGNED, int NB>
__global__ void __launch_bounds__(EX_THREADS, 2)
k_experts_out(const __grid_constant__ Experts p) {
    __shared__ Routing r;
    __shared__ float sums[EX_WARPS][16][8 * NB + 1];
    __shared__ bool last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // (what this kernel reads before it waits was there before the first one began)
    route<NB>(p, r);
    const int tiles = (p.n_out + 15) / 16, per_tile = r.jobs * p.splits;
    const int blocks = (p.hidden + 31) / 32, per_split = (blocks + p.splits - 1) / p.splits;
    int u, end;
    run_of(tiles * per_tile, u, end);
    const uint16_t *ra = nullptr, *rb = nullptr;
    int k0 = 0, k1 = 0;
    auto rows = [&](int unit) {
        const int tile = unit / per_tile, at = unit - tile * per_tile, job = at / p.splits;
        const int o = tile * 16 + g8;
        const uint16_t *w = p.w_out + r.expert[job] * p.w_out_z;
        ra = o < p.n_out ? w + o * p.w_out_ld : nullptr;
        rb = o + 8 < p.n_out ? w + (o + 8) * p.w_out_ld : nullptr;
        k0 = (at - job * p.splits) * per_split;
        k1 = min(k0 + per_split, blocks);
    };
    Step now, next;
    if (u < end) {
        rows(u);
        load<ALIGNED>(now, ra, rb, k0 + warp, k1, q, p.hidden);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (r.jobs == 0) {
        for (int i = blockIdx.x * EX_THREADS + tid; i < p.rows * p.n_out; i += gridDim.x * EX_THREADS)
            store<F16>(p, i / p.n_out, i % p.n_out, 0.f);
        return;
    }
    int done = 0;                         // units of this tile
    for (; u < end; ++u) {
        const int tile = u / per_tile, at0 = u - tile * per_tile, job = at0 / p.splits, split = at0 - job * p.splits;
        const int n = r.n[job], begin = r.begin[job];
        const uint4 *h[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int at = b * 8 + g8;
            h[b] = at < n ? (const uint4 *)p.h + (int64_t)r.list[begin + at] * p.h_groups * (F16 ? 4 : 2) : nullptr;
        }
        float c[NB][4] = {};
        const int from = k0, to = k1;
        int b0 = from;
        do {
            const int more = b0 + EX_STEP * EX_WARPS;
            if (more < to) {
                load<ALIGNED>(next, ra, rb, more + warp, to, q, p.hidden);
            } else if (u + 1 < end) {
                rows(u + 1);
                load<ALIGNED>(next, ra, rb, k0 + warp, k1, q, p.hidden);
            }
#pragma unroll
            for (int i = 0; i < EX_STEP; ++i) {
                const int k = b0 + warp + i * EX_WARPS;
                if (k >= to) break;
                const bool in = k * 32 + q * 8 < p.hidden;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (b * 8 >= n) break;
                    const bool mine = in && h[b];
                    if (F16) {
                        const uint4 *v = h[b] + (k * 4 + q) * 4;
                        const uint4 h0 = mine ? __ldcg(v) : zeros(), h1 = mine ? __ldcg(v + 1) : zeros();
                        const uint4 l0 = mine ? __ldcg(v + 2) : zeros(), l1 = mine ? __ldcg(v + 3) : zeros();
                        const uint4 a0 = widened(now.a[i].x, now.a[i].y), a1 = widened(now.a[i].z, now.a[i].w);
                        const uint4 d0 = widened(now.d[i].x, now.d[i].y), d1 = widened(now.d[i].z, now.d[i].w);
                        mma8_tf32(c[b], a0.x, d0.x, a0.y, d0.y, h0.x, h0.y);
                        mma8_tf32(c[b], a0.z, d0.z, a0.w, d0.w, h0.z, h0.w);
                        mma8_tf32(c[b], a1.x, d1.x, a1.y, d1.y, h1.x, h1.y);
                        mma8_tf32(c[b], a1.z, d1.z, a1.w, d1.w, h1.z, h1.w);
                        mma8_tf32(c[b], a0.x, d0.x, a0.y, d0.y, l0.x, l0.y);
                        mma8_tf32(c[b], a0.z, d0.z, a0.w, d0.w, l0.z, l0.w);
                        mma8_tf32(c[b], a1.x, d1.x, a1.y, d1.y, l1.x, l1.y);
                        mma8_tf32(c[b], a1.z, d1.z, a1.w, d1.w, l1.z, l1.w);
                    } else {
                        const uint4 *v = h[b] + (k * 4 + q) * 2;
                        const uint4 hi = mine ? __ldcg(v) : zeros(), lo = mine ? __ldcg(v + 1) : zeros();
                        mma16<false>(c[b], now.a[i].x, now.d[i].x, now.a[i].y, now.d[i].y, hi.x, hi.y);
                        mma16<false>(c[b], now.a[i].z, now.d[i].z, now.a[i].w, now.d[i].w, hi.z, hi.w);
                        mma16<false>(c[b], now.a[i].x, now.d[i].x, now.a[i].y, now.d[i].y, lo.x, lo.y);
                        mma16<false>(c[b], now.a[i].z, now.d[i].z, now.a[i].w, now.d[i].w, lo.z, lo.w);
                    }
                }
            }
            now = next;
            b0 = more;
        } while (b0 < to);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][g8 + (i >> 1) * 8][b * 8 + 2 * q + (i & 1)] = c[b][i];
        __syncthreads();
        for (int i = tid; i < 16 * 8 * NB; i += EX_THREADS) {
            const int o = i & 15, at = i >> 4;
            if (at >= n) break;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < EX_WARPS; ++w) v += sums[w][o][at];
            if (tile * 16 + o < p.n_out)
                p.part[((int64_t)r.list[begin + at] * p.splits + split) * p.n_out + tile * 16 + o] = v;
        }
        __syncthreads();
        ++done;
        if (u + 1 < end && (u + 1) / per_tile == tile) continue;
        // the block that brings a tile's last units adds up what each row's choices gave,
        // in their order
        if (tid == 0) {
            __threadfence();
            last = atomicAdd(p.arrivals + tile, (uint32_t)done) + done == (uint32_t)per_tile;
            if (last) p.arrivals[tile] = 0;
            __threadfence();
        }
        done = 0;
        __syncthreads();
        if (!last) continue;
        for (int i = tid; i < p.rows * 16; i += EX_THREADS) {
            const int o = tile * 16 + (i & 15), t = i >> 4;
            if (o >= p.n_out) continue;
            float y = 0.f;
            for (int j = 0; j < p.top; ++j) {
                const int pair = t * p.top + j;
                if (r.choice[pair] < 0) continue;
                const float *part = p.part + (int64_t)pair * p.splits * p.n_out + o;
                float v = 0.f;
                for (int s = 0; s < p.splits; ++s) v += __ldcg(part + (int64_t)s * p.n_out);
                y = fmaf(r.gate[pair], v, y);
            }
            store<F16>(p, t, o, y);
        }
    }
}

cudaLaunchConfig_t early(int grid, cudaStream_t s, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(EX_THREADS);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

template <bool F16, int NB>
cudaError_t both(const Experts &p, int nsm, bool in_aligned, bool out_aligned, cudaStream_t s) {
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early(2 * nsm, s, at);
    const cudaError_t e = in_aligned ? cudaLaunchKernelEx(&cfg, k_experts_in<F16, true, NB>, p)
                                     : cudaLaunchKernelEx(&cfg, k_experts_in<F16, false, NB>, p);
    if (e != cudaSuccess) return e;
    return out_aligned ? cudaLaunchKernelEx(&cfg, k_experts_out<F16, true, NB>, p)
                       : cudaLaunchKernelEx(&cfg, k_experts_out<F16, false, NB>, p);
}

template <bool F16>
cudaError_t by_rows(const Experts &p, int nsm, bool in_aligned, bool out_aligned, cudaStream_t s) {
    if (p.rows <= 8) return both<F16, 1>(p, nsm, in_aligned, out_aligned, s);
    if (p.rows <= 16) return both<F16, 2>(p, nsm, in_aligned, out_aligned, s);
    return both<F16, 4>(p, nsm, in_aligned, out_aligned, s);
}

}  // namespace

// Pieces of the second product's contraction: enough units for the GPU's blocks where
// tiles and experts are few, none under two steps of 32 columns a warp.
int expert_splits(int rows, int groups, int top, int hidden, int n_out, int nsm) {
    const int64_t pairs = (int64_t)rows * top, jobs = pairs < groups ? pairs : groups;
    const int64_t units = jobs * ((n_out + 15) / 16), most = ((hidden + 31) / 32) / (2 * EX_WARPS);
    int64_t n = (4 * nsm + units - 1) / (units < 1 ? 1 : units);
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n > 16 ? 16 : n);
}

cudaError_t launch_experts(const Experts &p, bool f16, int nsm, cudaStream_t s) {
    const bool in = (((uintptr_t)p.w_in & 15) | (p.w_in_ld & 7) | (p.groups > 1 ? p.w_in_z & 7 : 0)) == 0;
    const bool out = (((uintptr_t)p.w_out & 15) | (p.w_out_ld & 7) | (p.groups > 1 ? p.w_out_z & 7 : 0)) == 0;
    return f16 ? by_rows<true>(p, nsm, in, out, s) : by_rows<false>(p, nsm, in, out, s);
}

}  // namespace hwr
