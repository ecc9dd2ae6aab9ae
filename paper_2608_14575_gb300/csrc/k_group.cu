// Products with ragged groups of rows on the tensor cores (TMA + tcgen05), fp32
// accumulation in TMEM.  One kernel serves
//   rows products   out[t] = W[g(t)] x[t] (W K-major) or W[g(t)]^T x[t] (W
//                   MN-major): a tile is up to 128 rows of one group, gathered
//                   by their indices, times bn columns;
//   weight gradients  out[g] = sum over the group's rows of l[t] r[t]^T: both
//                   operands are gathered rows, MN-major, and the contraction
//                   runs over the group's rows.
// A rows product may carry a low-rank extension: after the contraction, for
// each group g with rows in the tile, the tile's rows of u (two 16-bit terms
// a value) times the group's [n][rank] matrix, accumulated only into the
// lanes of that group's rows (the MMA's lane mask), so that no value of one
// group's matrix ever meets another group's rows.
//
// The iterations (64-deep stages of the contraction) of all tiles are dealt
// evenly: whole tiles first, one to a CTA a round, then the tiles of the last
// rounds as one line of iterations cut into equal pieces.  The pieces of a tile
// leave fp32 partials; the last to arrive adds them in the order of the
// contraction, so the result does not depend on who that is.
#include "ops_internal.cuh"
#include "umma.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hwr {
namespace {

using namespace umma;

constexpr int THREADS = 192;       // warps 0-3 epilogue, 4 TMA producer, 5 MMA issuer
constexpr int A_BYTES = GP_BM * GP_BK * 2;
constexpr int MAX_STAGES = 12;
constexpr int SMEM_MAX = 227 * 1024;
constexpr int MIN_PIECE = 4;       // iterations of the smallest piece of a cut tile

struct Tables {
    int64_t iter0[OPS_MAX_GROUPS + 1];   // first iteration of each group (weight gradients)
    int32_t offs[OPS_MAX_GROUPS + 1];    // first row of each group, clamped
    int32_t eoffs[OPS_MAX_GROUPS + 1];   // the same of the extension's groups
    int32_t tile0[OPS_MAX_GROUPS + 1];   // first tile of each group
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], accf[2], acce[2], done;
    uint32_t tmem;
    int abort_f;
    int last;
};

constexpr int STAGE_ROOM = SMEM_MAX - 1024 - (int)((sizeof(Tables) + 1023) / 1024 * 1024);

// Waits of the unwinding (copies in flight, MMAs issued): bounded, no flags.
__device__ __forceinline__ void drain(uint64_t *bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity))
        if (clock64() - t0 > WAIT_CYCLES) return;
}

struct Work {
    int g, mt, nt;        // group, row tile (or result-row tile) and column tile within it
    int k0, k1, ki;       // iterations of this piece, and of the tile
    int c0, c1;           // first and last CTA with a piece of the tile
};

// The pieces of this CTA, in order.
struct Walk {
    const GroupProduct &p;
    const Tables &t;
    int tiles, dp, kiters, ctas;
    int next_tile;
    int64_t rest, pos, end;

    __device__ Walk(const GroupProduct &p_, const Tables &t_) : p(p_), t(t_) {
        tiles = t.tile0[p.groups];
        kiters = (p.k + GP_BK - 1) / GP_BK;
        const int P = gridDim.x;
        dp = 0;
        if (!p.wgrad && tiles >= 2 * P) dp = (tiles / P - 1) * P;
        rest = p.wgrad ? t.iter0[p.groups] : (int64_t)(tiles - dp) * kiters;
        const int64_t most = rest / MIN_PIECE;
        ctas = most < 1 ? 1 : most < P ? (int)most : P;
        next_tile = blockIdx.x;
        pos = end = 0;
        if ((int)blockIdx.x < ctas) {
            pos = first(blockIdx.x);
            end = first(blockIdx.x + 1);
        }
    }
    __device__ int64_t first(int c) const { return rest * c / ctas; }
    // the CTA whose piece holds iteration i
    __device__ int owner(int64_t i) const { return (int)(((i + 1) * ctas - 1) / rest); }

    __device__ static int find(const int32_t *v, int n, int x) {   // last g with v[g] <= x
        int lo = 0, hi = n - 1;
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (v[m] <= x) lo = m;
            else hi = m - 1;
        }
        return lo;
    }
    __device__ void place(Work &w, int tile) const {
        w.g = find(t.tile0, p.groups, tile);
        const int local = tile - t.tile0[w.g];
        const int mts = (t.tile0[w.g + 1] - t.tile0[w.g]) / p.ntiles;
        // bands of 64 row tiles, column by column: the CTAs at work share
        // columns of W and the band's rows stay in L2
        const int band = local / (64 * p.ntiles), in = local - band * 64 * p.ntiles;
        const int h = min(64, mts - band * 64);
        w.nt = in / h;
        w.mt = band * 64 + (in - w.nt * h);
    }
    __device__ bool next(Work &w) {
        if (next_tile < dp) {
            place(w, next_tile);
            next_tile += gridDim.x;
            w.k0 = 0;
            w.k1 = w.ki = kiters;
            w.c0 = w.c1 = blockIdx.x;
            return true;
        }
        if (pos >= end) return false;
        int64_t start;
        if (p.wgrad) {
            int lo = 0, hi = p.groups - 1;
            while (lo < hi) {
                const int m = (lo + hi + 1) >> 1;
                if (t.iter0[m] <= pos) lo = m;
                else hi = m - 1;
            }
            w.g = lo;
            const int per = t.tile0[lo + 1] - t.tile0[lo];
            w.ki = (int)((t.iter0[lo + 1] - t.iter0[lo]) / per);
            const int local = (int)((pos - t.iter0[lo]) / w.ki);
            start = t.iter0[lo] + (int64_t)local * w.ki;
            w.nt = local / p.mtiles;
            w.mt = local - w.nt * p.mtiles;
        } else {
            const int i = (int)(pos / kiters);
            w.ki = kiters;
            start = (int64_t)i * kiters;
            place(w, dp + i);
        }
        w.k0 = (int)(pos - start);
        const int64_t stop = start + w.ki < end ? start + w.ki : end;
        w.k1 = (int)(stop - start);
        w.c0 = owner(start);
        w.c1 = owner(start + w.ki - 1);
        pos = stop;
        return true;
    }
};

// The extension's stages of a tile: for each group with rows in the tile, the
// rank in steps of GP_RC.
struct Ext {
    const GroupProduct &p;
    const Tables &t;
    int p0, p1, g, r0, a, b;
    __device__ Ext(const GroupProduct &p_, const Tables &t_, int first, int last)
        : p(p_), t(t_), p0(first), p1(last) {
        g = Walk::find(t.eoffs, p.ext_groups, first);   // eoffs[g] <= first, or g = 0
        r0 = 0;
        settle();
    }
    __device__ void settle() {
        for (; g < p.ext_groups; ++g) {
            a = max(t.eoffs[g], p0);
            b = min(t.eoffs[g + 1], p1);
            if (a < b) return;
            if (t.eoffs[g] >= p1) break;
        }
        g = p.ext_groups;
    }
    __device__ bool more() const { return g < p.ext_groups; }
    __device__ void step() {
        r0 += GP_RC;
        if (r0 >= p.rank) {
            r0 = 0;
            ++g;
            settle();
        }
    }
};

template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if (F16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *(const uint32_t *)&h;
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&h;
}

template <bool F16>
__device__ __forceinline__ float widen(uint16_t v) {
    if (F16) return __half2float(__ushort_as_half(v));
    return __uint_as_float((uint32_t)v << 16);
}

// n consecutive 16-bit values of v (32 at most) to dst.
template <bool F16>
__device__ __forceinline__ void store_row(uint16_t *dst, const float (&v)[32], int n, bool vec) {
    if (vec && n == 32) {
#pragma unroll
        for (int j = 0; j < 32; j += 8)
            *(uint4 *)(dst + j) = make_uint4(pack2<F16>(v[j], v[j + 1]), pack2<F16>(v[j + 2], v[j + 3]),
                                             pack2<F16>(v[j + 4], v[j + 5]), pack2<F16>(v[j + 6], v[j + 7]));
        return;
    }
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
        if (vec && j + 8 <= n)
            *(uint4 *)(dst + j) = make_uint4(pack2<F16>(v[j], v[j + 1]), pack2<F16>(v[j + 2], v[j + 3]),
                                             pack2<F16>(v[j + 4], v[j + 5]), pack2<F16>(v[j + 6], v[j + 7]));
        else
#pragma unroll
            for (int i = j; i < j + 8; ++i)
                if (i < n) dst[i] = (uint16_t)pack2<F16>(v[i], 0.f);
    }
}

template <bool F16>
__global__ void __launch_bounds__(THREADS, 1)
k_group(const __grid_constant__ GroupMaps maps, const __grid_constant__ GroupProduct p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Tables &t = *(Tables *)(sm + (size_t)p.stages * p.stage_bytes);
    volatile int *abort_f = &t.abort_f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // Group tables.  Offsets are the caller's: clamped here, so that no value
    // of theirs reads or writes outside the arrays.
    {
        const int ng = p.shared ? p.ext_groups : p.groups;
        int32_t *dst = p.shared ? t.eoffs : t.offs;
        for (int i = threadIdx.x; i <= ng; i += THREADS) {
            const int v = p.offsets[i];
            dst[i] = v < 0 ? 0 : v > p.rows ? p.rows : v;
        }
        if (p.shared && threadIdx.x == 0) {
            t.offs[0] = 0;
            t.offs[1] = p.rows;
        }
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&t.full[s], 1);
            mbar_init(&t.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&t.accf[b], 1);
            mbar_init(&t.acce[b], 128);
        }
        mbar_init(&t.done, 1);
        t.abort_f = 0;
        fence_mbar_init();
    }
    const uint32_t cs = (p.bn + 31) & ~31;      // TMEM columns of one of the two accumulators
    uint32_t tcols = 64;
    while (tcols < 2 * cs) tcols *= 2;
    if (warp == 5) {
        tmem_alloc(&t.tmem, tcols);
        tmem_relinquish();
    }
    __syncthreads();
    if (warp == 0) {
        // first tile (and iteration) of each group: a running sum over 32 groups at a time
        int tile = 0;
        int64_t iter = 0;
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            const int g = g0 + lane;
            int nt = 0, ki = 0;
            if (g < p.groups) {
                const int n = max(0, t.offs[g + 1] - t.offs[g]);
                if (p.wgrad) {
                    nt = p.mtiles * p.ntiles;
                    ki = max(1, (n + GP_BK - 1) / GP_BK);   // an empty group's zeros are written too
                } else {
                    nt = (n + GP_BM - 1) / GP_BM * p.ntiles;
                }
            }
            int st = nt;
            int64_t si = (int64_t)nt * ki;
            for (int d = 1; d < 32; d *= 2) {
                const int a = __shfl_up_sync(0xffffffffu, st, d);
                const int64_t b = __shfl_up_sync(0xffffffffu, si, d);
                if (lane >= d) {
                    st += a;
                    si += b;
                }
            }
            if (g < p.groups) {
                t.tile0[g + 1] = tile + st;
                t.iter0[g + 1] = iter + si;
            }
            tile += __shfl_sync(0xffffffffu, st, 31);
            iter += __shfl_sync(0xffffffffu, si, 31);
        }
        if (lane == 0) {
            t.tile0[0] = 0;
            t.iter0[0] = 0;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = t.tmem;
    const int bblocks = (p.bn + 63) / 64;
    const uint32_t b_bytes = p.wgrad || p.b_mn ? bblocks * 8192 : p.bn * 128;

    if (warp == 4) {
        // producer: gathers 4 rows a lane, one lane loads the W tiles
        uint32_t n = 0;
        bool ok = true;
        Walk walk(p, t);
        Work w;
        while (ok && walk.next(w)) {
            if (p.wgrad) {
                const int first = t.offs[w.g], last = t.offs[w.g + 1];
                // 16 lanes hold the rows of the stage; each gathers its four
                // rows into every block of 64 columns, shared between the two halves
                const int mblocks = min(2, (p.m - w.mt * GP_BM + 63) / 64);
                const int nb = min(bblocks, (p.n - w.nt * p.bn + 63) / 64);
                const uint32_t bytes = (uint32_t)(mblocks + nb) * 8192;
                int next[4];
                auto rows_of = [&](int kb) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int pos = first + kb * GP_BK + 4 * (lane & 15) + j;
                        int r = p.rows;
                        if (kb < w.k1 && pos < last) r = p.order ? p.order[pos] : pos;
                        next[j] = (uint32_t)r < (uint32_t)p.rows ? r : p.rows;
                    }
                };
                rows_of(w.k0);
                for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
                    int idx[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) idx[j] = next[j];
                    rows_of(kb + 1);
                    const int s = n % p.stages;
                    ok = mbar_wait(&t.empty[s], ((n / p.stages) & 1) ^ 1, abort_f, p.status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    uint8_t *st = sm + (size_t)s * p.stage_bytes + (lane & 15) * 512;
                    if (lane == 0) mbar_arrive_expect_tx(&t.full[s], bytes);
                    __syncwarp();
                    for (int b = lane >> 4; b < mblocks + nb; b += 2)
                        if (b < mblocks)
                            tma_gather4(st + b * 8192, &maps.a, &t.full[s], w.mt * GP_BM + b * 64, idx);
                        else
                            tma_gather4(st + A_BYTES + (b - mblocks) * 8192, &maps.b, &t.full[s],
                                        w.nt * p.bn + (b - mblocks) * 64, idx);
                }
            } else {
                const int first = t.offs[w.g] + w.mt * GP_BM;
                const int last = min(first + GP_BM, t.offs[w.g + 1]);
                const int na = (last - first + 3) / 4;     // lanes with rows
                int idx[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int pos = first + 4 * lane + j;
                    int r = p.rows;
                    if (pos < last) r = p.order ? p.order[pos] : pos;
                    idx[j] = (uint32_t)r < (uint32_t)p.rows ? r : p.rows;
                }
                const int n0 = w.nt * p.bn;
                const int nb = min(bblocks, (p.n - n0 + 63) / 64);
                const uint32_t bytes = (p.b_mn ? nb * 8192 : b_bytes) + na * 512;
                for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
                    const int s = n % p.stages;
                    ok = mbar_wait(&t.empty[s], ((n / p.stages) & 1) ^ 1, abort_f, p.status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    uint8_t *st = sm + (size_t)s * p.stage_bytes;
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&t.full[s], bytes);
                        if (p.b_mn)
                            for (int b = 0; b < nb; ++b)
                                tma_load_3d(st + A_BYTES + b * 8192, &maps.b, &t.full[s], n0 + b * 64,
                                            kb * GP_BK, w.g);
                        else
                            tma_load_3d(st + A_BYTES, &maps.b, &t.full[s], kb * GP_BK, n0, w.g);
                    }
                    __syncwarp();
                    if (lane < na) tma_gather4(st + lane * 512, &maps.a, &t.full[s], kb * GP_BK, idx);
                }
                if (ok && p.rank && w.k1 == w.ki) {
                    const uint32_t ebytes =
                        (p.ext_b_mn ? nb * 4096 : p.bn * 64) + na * 512;
                    for (Ext e(p, t, first, last); e.more(); e.step(), ++n) {
                        const int s = n % p.stages;
                        ok = mbar_wait(&t.empty[s], ((n / p.stages) & 1) ^ 1, abort_f, p.status);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        uint8_t *st = sm + (size_t)s * p.stage_bytes;
                        if (lane == 0) {
                            mbar_arrive_expect_tx(&t.full[s], ebytes);
                            if (p.ext_b_mn)
                                for (int b = 0; b < nb; ++b)
                                    tma_load_3d(st + A_BYTES + b * 4096, &maps.eb, &t.full[s],
                                                n0 + b * 64, e.r0, e.g);
                            else
                                tma_load_3d(st + A_BYTES, &maps.eb, &t.full[s], e.r0, n0, e.g);
                        }
                        __syncwarp();
                        if (lane < na) tma_gather4(st + lane * 512, &maps.u, &t.full[s], e.r0 * 2, idx);
                    }
                }
            }
        }
        // the loads still in flight land before the CTA can exit
        const uint32_t f = n > (uint32_t)p.stages ? n - p.stages : 0;
        if (lane == 0)
            for (uint32_t j = f; j < n; ++j) drain(&t.full[j % p.stages], (j / p.stages) & 1);
        __syncwarp();
    } else if (warp == 5) {
        if (lane == 0) {
            uint32_t n = 0, lt = 0;
            bool ok = true;
            Walk walk(p, t);
            Work w;
            const uint32_t idesc = idesc_16bit(GP_BM, p.mma_n, F16, p.wgrad, p.wgrad || p.b_mn);
            const uint32_t eidesc = idesc_16bit(GP_BM, p.mma_n, F16, false, p.ext_b_mn);
            // per 16-deep MMA: two rows of 8 K indices further (MN-major) or 32 bytes (K-major)
            const uint32_t astep = p.wgrad ? 2048 >> 4 : 2, bstep = p.wgrad || p.b_mn ? 2048 >> 4 : 2;
            for (; ok && walk.next(w); ++lt) {
                const int b = lt & 1;
                const uint32_t d = tmem + b * cs;
                ok = mbar_wait(&t.acce[b], ((lt >> 1) & 1) ^ 1, abort_f, p.status);
                if (!ok) break;
                tc_fence_after();
                for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
                    const int s = n % p.stages;
                    ok = mbar_wait(&t.full[s], (n / p.stages) & 1, abort_f, p.status);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t st = smem_u32(sm + (size_t)s * p.stage_bytes);
                    const uint64_t ad = sdesc(st, 8192, 1024, 2), bd = sdesc(st + A_BYTES, 8192, 1024, 2);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_bf16(d, ad + astep * k, bd + bstep * k, idesc, (kb > w.k0) | k);
                    mma_commit(&t.empty[s]);
                }
                if (!ok) break;
                if (p.rank && w.k1 == w.ki) {
                    const int first = t.offs[w.g] + w.mt * GP_BM;
                    const int last = min(first + GP_BM, t.offs[w.g + 1]);
                    for (Ext e(p, t, first, last); e.more(); e.step(), ++n) {
                        uint32_t off[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int a = min(max(e.a - first - 32 * i, 0), 32);
                            const int z = min(max(e.b - first - 32 * i, 0), 32);
                            // lanes [a, z) of this word take part
                            const uint32_t below = a == 32 ? 0xffffffffu : (1u << a) - 1;
                            const uint32_t upto = z == 32 ? 0xffffffffu : (1u << z) - 1;
                            off[i] = ~(upto & ~below);
                        }
                        const int s = n % p.stages;
                        ok = mbar_wait(&t.full[s], (n / p.stages) & 1, abort_f, p.status);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t st = smem_u32(sm + (size_t)s * p.stage_bytes);
                        const uint64_t ad = sdesc(st, 0, 1024, 2);
                        const uint64_t bd = p.ext_b_mn ? sdesc(st + A_BYTES, 4096, 1024, 2)
                                                       : sdesc(st + A_BYTES, 0, 512, 4);
                        const int steps = min(GP_RC, p.rank - e.r0) > 16 ? 2 : 1;
                        const uint32_t eb = p.ext_b_mn ? 2048 >> 4 : 2;
                        for (int k = 0; k < steps; ++k) {
                            mma_16bit_lanes(d, ad + 2 * k, bd + eb * k, eidesc, off, 1);
                            mma_16bit_lanes(d, ad + 4 + 2 * k, bd + eb * k, eidesc, off, 1);
                        }
                        mma_commit(&t.empty[s]);
                    }
                    if (!ok) break;
                }
                mma_commit(&t.accf[b]);
            }
            mma_commit(&t.done);
            drain(&t.done, 0);
        }
        __syncwarp();
    } else {
        // epilogue: thread = TMEM lane = row of the tile
        const int row = threadIdx.x;
        const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
        const int P = gridDim.x;
        if (p.out_kind == GP_OUT_ROWS && !p.shared) {
            // rows without a group: zeros
            for (int64_t pos = (int64_t)t.offs[p.groups] + blockIdx.x * 4 + warp; pos < p.rows;
                 pos += (int64_t)P * 4) {
                const int r = p.order ? p.order[pos] : (int)pos;
                if ((uint32_t)r >= (uint32_t)p.rows) continue;
                uint16_t *dst = (uint16_t *)p.out + (int64_t)r * p.ld;
                if (p.vec)
                    for (int j = lane * 8; j + 8 <= p.n; j += 256) *(uint4 *)(dst + j) = make_uint4(0, 0, 0, 0);
                for (int j = (p.vec ? p.n & ~7 : 0) + lane; j < p.n; j += 32) dst[j] = 0;
            }
        }
        uint32_t lt = 0;
        bool ok = true;
        Walk walk(p, t);
        Work w;
        for (; walk.next(w); ++lt) {
            const int b = lt & 1;
            int64_t orow = -1;     // this lane's row of the output
            int nrows = GP_BM;
            float sc = 1.f;
            if (p.wgrad) {
                nrows = min(GP_BM, p.m - w.mt * GP_BM);
                orow = w.mt * GP_BM + row;
            } else {
                const int first = t.offs[w.g] + w.mt * GP_BM;
                nrows = min(GP_BM, t.offs[w.g + 1] - first);
                if (row < nrows) orow = p.order ? p.order[first + row] : first + row;
                if (p.scale) sc = p.scale[w.g];
            }
            const bool mine = row < nrows && (p.wgrad || (uint64_t)orow < (uint64_t)p.rows);
            ok = mbar_wait(&t.accf[b], (lt >> 1) & 1, abort_f, p.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const bool cut = w.c0 != w.c1;
            bool write = true;
            const int cols = (p.mma_n + 31) & ~31;
            const uint32_t acc = tmem + lane_base + b * cs;
            if (cut) {
                // leave this piece's sums (slot 1: the tile's first piece, which
                // ends its CTA's line; slot 0: a later one, which begins it); the
                // last of the tile's pieces to arrive adds them all
                const int slot = 2 * blockIdx.x + (w.k0 == 0);
                float4 *dst = (float4 *)(p.part + (size_t)slot * GP_BM * GP_MAX_BN) + row;
                for (int c = 0; c < cols; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(acc + c, v);
                    tmem_wait_ld32(v);
                    if (row < nrows)
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            __stcg(dst + (c + j) / 4 * GP_BM,
                                   make_float4(__uint_as_float(v[j]), __uint_as_float(v[j + 1]),
                                               __uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])));
                }
                __threadfence();
                named_bar_sync(1, 128);
                if (threadIdx.x == 0) {
                    const uint32_t before = atomicAdd(&p.count[w.c0], 1u);
                    t.last = before == (uint32_t)(w.c1 - w.c0);
                    if (t.last) p.count[w.c0] = 0;
                    __threadfence();
                }
                named_bar_sync(1, 128);
                write = *(volatile int *)&t.last != 0;
            }
            // 32 columns of the tile from column c on: from TMEM, or the pieces' sum
            auto values = [&](int c, float (&v)[32]) {
                if (!cut) {
                    uint32_t u[32];
                    tmem_ld32(acc + c, u);
                    tmem_wait_ld32(u);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
                    return;
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0.f;
                if (row >= nrows) return;
                for (int o = w.c0; o <= w.c1; ++o) {
                    const int slot = 2 * o + (o == w.c0);
                    const float4 *src = (const float4 *)(p.part + (size_t)slot * GP_BM * GP_MAX_BN) + row;
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 x = __ldcg(src + (c + j) / 4 * GP_BM);
                        v[j] += x.x;
                        v[j + 1] += x.y;
                        v[j + 2] += x.z;
                        v[j + 3] += x.w;
                    }
                }
            };
            if (write) {
                const int n0 = w.nt * p.bn;
                uint16_t *out = (uint16_t *)p.out;
                if (p.out_kind == GP_OUT_ROWS || p.out_kind == GP_OUT_GROUP) {
                    if (p.out_kind == GP_OUT_GROUP) out += w.g * p.gstride;
                    const int width = min(p.bn, p.n - n0);
                    for (int c = 0; c < width; c += 32) {
                        float v[32];
                        values(c, v);
                        if (mine) store_row<F16>(out + orow * p.ld + n0 + c, v, min(32, width - c), p.vec);
                    }
                } else if (p.out_kind == GP_OUT_PACK) {
                    // value = high + low, to about twice the type's precision; an
                    // infinite high term takes a zero low one (not inf - inf)
                    for (int c = 0; c < cols && n0 + c < p.n; c += 32) {
                        float v[32], lo[32];
                        values(c, v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            v[j] = n0 + c + j < p.n ? v[j] * sc : 0.f;
                            const float hi = widen<F16>((uint16_t)pack2<F16>(v[j], 0.f));
                            lo[j] = isinf(hi) ? 0.f : v[j] - hi;
                        }
                        if (mine) {
                            store_row<F16>(out + orow * p.ld + (n0 + c) * 2, v, 32, true);
                            store_row<F16>(out + orow * p.ld + (n0 + c) * 2 + 32, lo, 32, true);
                        }
                    }
                } else {
                    // blocks of 64 columns: the products with the high terms of 32
                    // ranks, then those with the low terms
                    out += w.g * p.gstride;
                    for (int c = 0; c < cols; c += 64) {
                        const int r = (n0 + c) / 2, left = p.rank_out - r;
                        if (left <= 0) break;
                        float v[32], lo[32];
                        values(c, v);
                        values(c + 32, lo);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += lo[j];
                        if (!mine) continue;
                        if (p.out_kind == GP_OUT_LOW)
                            store_row<F16>(out + orow * p.ld + r, v, min(32, left), p.vec);
                        else
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < left) out[(r + j) * p.ld + orow] = (uint16_t)pack2<F16>(v[j], 0.f);
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(&t.acce[b]);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, tcols);
    }
}

}  // namespace

cudaError_t group_prepare() {
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaFuncSetAttribute(k_group<false>, attr, SMEM_MAX);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_group<true>, attr, SMEM_MAX);
    return e;
}

size_t group_part_floats(int nsm) { return (size_t)nsm * 2 * GP_BM * GP_MAX_BN; }

void group_plan(GroupProduct *p) {
    const int bb = p->wgrad || p->b_mn ? (p->bn + 63) / 64 * 8192 : p->bn * 128;
    // an extension stage holds bn x 32 ranks: never more than an ordinary one
    p->stage_bytes = A_BYTES + bb;
    const int fit = STAGE_ROOM / p->stage_bytes;
    p->stages = fit < MAX_STAGES ? fit : MAX_STAGES;
    p->ntiles = (p->n + p->bn - 1) / p->bn;
    p->mtiles = (p->m + GP_BM - 1) / GP_BM;
}

cudaError_t launch_group(const GroupProduct &p, const GroupMaps &maps, int nsm, cudaStream_t s) {
    const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + sizeof(Tables);
    if (p.f16) k_group<true><<<nsm, THREADS, smem, s>>>(maps, p);
    else k_group<false><<<nsm, THREADS, smem, s>>>(maps, p);
    return cudaGetLastError();
}

}  // namespace hwr
