// Dispatch (stable grouping of rows by choice), gradient clipping and padding
// copies: the memory-bound kernels beside the grouped products.
#include "ops_internal.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hwr {
namespace {

// ---------------------------------------------------------------------------
// Dispatch: a stable counting sort of the rows by choice.
//
// A block takes a run of consecutive rows in rounds of DP_ROWS; in a round each
// warp holds DP_PER x 32 consecutive rows in registers.  The rows of a warp
// that share a key find each other by votes over the warp, so a row's place
// is its key's first place (over the blocks, rounds and warps before it) plus
// the peers in lower lanes: no atomics decide an order.  What the blocks before
// hold of each key comes from shared memory within a cluster (up to its blocks,
// one launch) or from a counting pass before (more).  All of it is
// bound by latency: 4 MB of choices are read and written in 1.2 us.

constexpr int DP_THREADS = 512, DP_WARPS = DP_THREADS / 32;
constexpr int DP_PER = 8;
constexpr int DP_ROWS = DP_THREADS * DP_PER;
// Blocks of a cluster: 16, the non-portable size, where the device can place so many
// (of a part of a GPU it may not), else 8.
constexpr int DP_CLUSTER = 16, DP_CLUSTER_LEAST = 8;
constexpr int DP_FEW = 256;      // rows whose places are counted row against row

__device__ __forceinline__ void pdl_begin() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ int key_of(const int32_t *choice, int64_t row, int64_t end, int G) {
    if (row >= end) return G + 1;            // no row
    const int c = choice[row];
    return (uint32_t)c < (uint32_t)G ? c : G;
}

// Lanes of the warp with the same key (of nbits bits): a vote per bit.  (A match
// over the warp takes a step per distinct key.)
__device__ __forceinline__ uint32_t peers_of(int key, int nbits) {
    uint32_t peers = 0xffffffffu;
    for (int b = 0; b < nbits; ++b) {
        const bool on = (key >> b) & 1;
        const uint32_t v = __ballot_sync(0xffffffffu, on);
        peers &= on ? v : ~v;
    }
    return peers;
}

// A few rows: a row's place is the number of rows that come before it.
__global__ void __launch_bounds__(DP_FEW)
k_dispatch_few(int rows, int G, const int32_t *choice, int32_t *offsets, int32_t *order) {
    __shared__ __align__(16) int32_t key[DP_FEW];
    const int tid = threadIdx.x, n4 = (rows + 3) / 4;
    pdl_begin();
    key[tid] = tid < rows ? key_of(choice, tid, rows, G) : G + 1;
    __syncthreads();
    const int4 *k4 = (const int4 *)key;
    if (tid < rows) {
        const int k = key[tid];
        int place = 0;
        for (int j = 0; j < n4; ++j) {
            const int4 v = k4[j];
            place += (v.x < k) + (v.y < k) + (v.z < k) + (v.w < k);
            place += (v.x == k && 4 * j < tid) + (v.y == k && 4 * j + 1 < tid) + (v.z == k && 4 * j + 2 < tid) +
                     (v.w == k && 4 * j + 3 < tid);
        }
        order[place] = tid;
    }
    for (int g = tid; g <= G; g += DP_FEW) {
        int n = 0;
        for (int j = 0; j < n4; ++j) {
            const int4 v = k4[j];
            n += (v.x < g) + (v.y < g) + (v.z < g) + (v.w < g);
        }
        offsets[g] = n;
    }
}

__device__ __forceinline__ int remote_int(const int32_t *p, int rank) {
    uint32_t a;
    int v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Rows of each key in the blocks of a cluster before each of its blocks: hist
// [blocks][G + 1]; then those of each whole cluster: [clusters][G + 1].
template <int CLUSTER>
__global__ void __launch_bounds__(DP_THREADS)
k_dispatch_count(int rows, int G, int64_t per_block, const int32_t *choice, int32_t *hist) {
    extern __shared__ int32_t sh[];
    const int tid = threadIdx.x, lane = tid & 31, nbits = 32 - __clz(G + 1), G1 = G + 1;
    for (int i = tid; i < G1; i += DP_THREADS) sh[i] = 0;
    pdl_begin();
    __syncthreads();
    const int64_t begin = blockIdx.x * per_block;
    const int64_t end = begin + per_block < rows ? begin + per_block : rows;
    for (int64_t r0 = begin; r0 < end; r0 += DP_ROWS) {
        int key[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) key[i] = key_of(choice, r0 + i * DP_THREADS + tid, end, G);
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) {
            const uint32_t peers = peers_of(key[i], nbits);
            if (key[i] <= G && lane == __ffs(peers) - 1) atomicAdd(&sh[key[i]], __popc(peers));
        }
    }
    cluster_barrier();
    const int rank = blockIdx.x % CLUSTER;
    for (int g = tid; g < G1; g += DP_THREADS) {
        int before = 0, all = 0;
#pragma unroll
        for (int b = 0; b < CLUSTER; ++b) {
            const int c = remote_int(&sh[g], b);
            before += b < rank ? c : 0;
            all += c;
        }
        hist[(int64_t)blockIdx.x * G1 + g] = before;
        if (rank == 0) hist[((int64_t)gridDim.x + blockIdx.x / CLUSTER) * G1 + g] = all;
    }
    cluster_barrier();       // the others may still read this block's counts
}

// hist: from k_dispatch_count, of `counted` blocks in clusters of `cluster`; null with
// one block, or with one cluster of blocks of a round each.
__global__ void __launch_bounds__(DP_THREADS)
k_dispatch_place(int rows, int G, int64_t per_block, const int32_t *choice, const int32_t *hist, int counted,
                 int cluster, int32_t *offsets, int32_t *order) {
    extern __shared__ int32_t sh[];
    const int G1 = G + 1, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nb = gridDim.x;
    const int nbits = 32 - __clz(G + 1);
    int32_t *wh = sh;                        // [DP_WARPS][G1] counts, then first places
    int32_t *base = sh + DP_WARPS * G1;      // [G1] next place of each key
    int32_t *total = base + G1;              // [G1] rows of each key in all
    int32_t *round = total + G1;             // [G1] rows of each key in this round
    __shared__ int32_t wsum[DP_WARPS];
    const int64_t begin = blockIdx.x * per_block;
    const int64_t end = begin + per_block < rows ? begin + per_block : rows;

    for (int i = tid; i < G1; i += DP_THREADS) base[i] = total[i] = 0;
    // after the counting pass the choices are known to be there, its counts are not
    if (!hist) pdl_begin();
    for (int64_t r0 = begin; r0 < end || r0 == begin; r0 += DP_ROWS) {
        int key[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i)
            key[i] = key_of(choice, r0 + (warp * DP_PER + i) * 32 + lane, end, G);
        for (int i = tid; i < DP_WARPS * G1; i += DP_THREADS) wh[i] = 0;
        __syncthreads();
        // counts of each warp's rows
        int rank[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) {
            const uint32_t peers = peers_of(key[i], nbits);
            const int leader = __ffs(peers) - 1;
            int c = 0;
            if (key[i] <= G && lane == leader) {
                c = wh[warp * G1 + key[i]];
                wh[warp * G1 + key[i]] = c + __popc(peers);
            }
            c = __shfl_sync(0xffffffffu, c, leader);
            rank[i] = c + __popc(peers & ((1u << lane) - 1));
            __syncwarp();
        }
        if (hist && r0 == begin) {
            // rows of each key in the blocks before this one, and in all
            pdl_begin();
            const int clusters = counted / cluster, mine = blockIdx.x / cluster;
            for (int g = tid; g < G1; g += DP_THREADS) {
                int before = hist[(int64_t)blockIdx.x * G1 + g], all = 0;
#pragma unroll 8
                for (int c = 0; c < clusters; ++c) {
                    const int v = hist[((int64_t)counted + c) * G1 + g];
                    all += v;
                    before += c < mine ? v : 0;
                }
                base[g] = before;
                total[g] = all;
            }
        }
        __syncthreads();
        // over the warps: counts become first places within the round
        for (int g = tid; g < G1; g += DP_THREADS) {
            int sum = 0;
#pragma unroll
            for (int w = 0; w < DP_WARPS; ++w) {
                const int c = wh[w * G1 + g];
                wh[w * G1 + g] = sum;
                sum += c;
            }
            round[g] = sum;
            if (!hist && nb == 1) total[g] = sum;
        }
        if (!hist && nb > 1) {
            cluster_barrier();
            for (int g = tid; g < G1; g += DP_THREADS) {
                int before = 0, all = 0;
                for (int b = 0; b < nb; ++b) {
                    const int c = remote_int(&round[g], b);
                    all += c;
                    before += b < (int)blockIdx.x ? c : 0;
                }
                base[g] = before;
                total[g] = all;
            }
        }
        __syncthreads();
        if (r0 == begin) {
            // first place of each key: a running sum of the totals, two keys a thread
            const int a = 2 * tid < G ? total[2 * tid] : 0, b = 2 * tid + 1 < G ? total[2 * tid + 1] : 0;
            int s = a + b;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int o = __shfl_up_sync(0xffffffffu, s, d);
                if (lane >= d) s += o;
            }
            if (lane == 31) wsum[warp] = s;
            __syncthreads();
            int before = 0, all = 0;
#pragma unroll
            for (int w = 0; w < DP_WARPS; ++w) {
                before += w < warp ? wsum[w] : 0;
                all += wsum[w];
            }
            const int upto = before + s;
            if (2 * tid < G) base[2 * tid] += upto - a - b;
            if (2 * tid + 1 < G) base[2 * tid + 1] += upto - b;
            if (tid == 0) base[G] += all;
            if (blockIdx.x == 0) {
                if (2 * tid < G) offsets[2 * tid + 1] = upto - b;
                if (2 * tid + 1 < G) offsets[2 * tid + 2] = upto;
                if (tid == 0) offsets[0] = 0;
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < DP_PER; ++i)
            if (key[i] <= G)
                order[base[key[i]] + wh[warp * G1 + key[i]] + rank[i]] =
                    (int32_t)(r0 + (warp * DP_PER + i) * 32 + lane);
        __syncthreads();
        for (int g = tid; g < G1; g += DP_THREADS) base[g] += round[g];
    }
    if (!hist && nb > 1) cluster_barrier();      // the others may still read this block's counts
}

size_t place_smem(int G) { return (size_t)(DP_WARPS + 3) * (G + 1) * 4; }

// ---------------------------------------------------------------------------
// Eight values from column 8 i on of a row of `cols` that begins anywhere: two
// aligned loads inside the row, shifted; at its ends value by value, zeros beyond.
__device__ __forceinline__ uint4 unit_of(const uint16_t *src, int i, int cols) {
    const uint16_t *a = src + (int64_t)i * 8;
    const uint32_t off = (uint32_t)(uintptr_t)a & 15;
    const uint4 *w = (const uint4 *)((uintptr_t)a - off);
    if (off == 0 && i * 8 + 8 <= cols) return __ldg(w);
    if (i > 0 && i * 8 + 16 <= cols) {       // (the loads reach 7 values back and 15 on)
        const uint4 lo = __ldg(w), hi = __ldg(w + 1);
        uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        if (off & 8)
#pragma unroll
            for (int j = 0; j < 6; ++j) x[j] = x[j + 2];
        if (off & 4)
#pragma unroll
            for (int j = 0; j < 5; ++j) x[j] = x[j + 1];
        const uint32_t bits = (off & 2) * 8;
        return make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits),
                          __funnelshift_r(x[2], x[3], bits), __funnelshift_r(x[3], x[4], bits));
    }
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i * 8 + j < cols ? a[j] : 0;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// Rows by place: a warp copies a row, or with few rows a slice of one (reads and
// writes of 512 bytes at a time; gridDim.y slices).

constexpr int SR_THREADS = 256;

__global__ void __launch_bounds__(SR_THREADS)
k_sort_rows(const __grid_constant__ GroupPlan plan, const __grid_constant__ SortRows m, int places,
            int32_t *padded_offsets, int32_t *padded_order) {
    extern __shared__ int32_t sh[];
    const int G = plan.groups, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int32_t *offs = sh, *pad = sh + G + 1;       // first place of each group, in either plan
    int total = plan.rows;
    pdl_begin();
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < m.nzero; i += SR_THREADS) m.zero[i] = 0;
    if (padded_offsets) {
        for (int i = threadIdx.x; i <= G; i += SR_THREADS) {
            const int v = plan.offsets[i];
            offs[i] = v < 0 ? 0 : v > plan.rows ? plan.rows : v;
        }
        __syncthreads();
        if (warp == 0) {
            int run = 0;
            for (int g0 = 0; g0 < G; g0 += 32) {
                const int g = g0 + lane;
                int v = g < G ? (max(0, offs[g + 1] - offs[g]) + 15) & ~15 : 0;
                const int own = v;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int o = __shfl_up_sync(0xffffffffu, v, d);
                    if (lane >= d) v += o;
                }
                if (g < G) pad[g] = run + v - own;
                run += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) pad[G] = run;
        }
        __syncthreads();
        total = min(pad[G] + plan.rows - offs[G], places);
        if (blockIdx.x == 0 && blockIdx.y == 0) {
            for (int i = threadIdx.x; i <= G; i += SR_THREADS) padded_offsets[i] = pad[i];
            if (threadIdx.x == 0) padded_offsets[G + 1] = total;
        }
    }
    for (int64_t at = blockIdx.x * (SR_THREADS / 32) + warp; at < total; at += (int64_t)gridDim.x * (SR_THREADS / 32)) {
        int place = (int)at;
        if (padded_offsets) {
            int lo = 0, hi = G;
            while (lo < hi) {                    // last group that begins at or before the place
                const int mid = (lo + hi + 1) >> 1;
                if (pad[mid] <= at) lo = mid;
                else hi = mid - 1;
            }
            place = offs[lo] + (int)(at - pad[lo]);
            if (lo < G && place >= offs[lo + 1]) place = -1;
        }
        int r = place >= 0 && place < plan.rows ? plan.order[place] : -1;
        if ((uint32_t)r >= (uint32_t)plan.rows) r = -1;
        if (padded_offsets && lane == 0 && blockIdx.y == 0) padded_order[at] = r;
        for (int k = 0; k < m.n; ++k) {
            uint4 *dst = (uint4 *)(m.dst[k] + at * m.dst_ld[k]);
            const int units = (int)(m.dst_ld[k] / 8), cols = m.cols[k];
            const uint16_t *src = r < 0 ? nullptr : m.src[k] + r * m.src_ld[k];
            const int first = blockIdx.y * 32 + lane, step = gridDim.y * 32;
            if (!src) {
                for (int i = first; i < units; i += step) dst[i] = make_uint4(0, 0, 0, 0);
            } else if (((uintptr_t)src & 15) == 0 && cols % 8 == 0) {
#pragma unroll 4
                for (int i = first; i < units; i += step) dst[i] = __ldg((const uint4 *)src + i);
            } else {
#pragma unroll 2
                for (int i = first; i < units; i += step) dst[i] = unit_of(src, i, cols);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Low-rank inner products of a few rows: u[place] = scale[g] A[g] x[order[place]]
// as two bf16 terms a value, in the layout of the tensor-core kernel.  A few
// rows read all of A once and compute little: a block takes a row and four
// ranks, its eight warps an eighth of the columns each, so that every load of
// the call is in flight at once.

constexpr int LF_THREADS = 256, LF_WARPS = LF_THREADS / 32, LF_RANKS = 4;

template <bool F16>
__device__ __forceinline__ void widen8(const uint4 &u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (F16) {
            const float2 v = __half22float2(*(const __half2 *)&w[i]);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        } else {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

// Eight elements from column c on of a row of n, zeros beyond it.
__device__ __forceinline__ uint4 row8(const uint16_t *row, int c, int n) {
    if (c + 8 <= n) return __ldg((const uint4 *)(row + c));
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < n ? row[c + j] : 0;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

template <bool F16>
__global__ void __launch_bounds__(LF_THREADS)
k_low_few(const __grid_constant__ LowFew p) {
    __shared__ float part[LF_WARPS][LF_RANKS];
    __shared__ int group;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int place = blockIdx.x, r0 = blockIdx.y * LF_RANKS;
    pdl_begin();
    const int row = p.by_place ? place : p.plan.order[place];
    if (warp == 0) {
        // the place's group: how many groups end at or before it
        int n = 0;
        for (int g = lane; g < p.plan.groups; g += 32) n += p.plan.offsets[g + 1] <= place;
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) group = n;
    }
    __syncthreads();
    const int g = group, ranks = min(LF_RANKS, p.rank - r0);
    float acc[LF_RANKS] = {};
    if (g < p.plan.groups && (uint32_t)row < (uint32_t)p.plan.rows && ranks > 0) {
        const uint16_t *x = p.x + row * p.x_ld;
        const uint16_t *a = p.a + g * p.a_z + (int64_t)r0 * p.a_ld;
#pragma unroll 2
        for (int c = (warp * 32 + lane) * 8; c < p.k; c += LF_THREADS * 8) {
            const uint4 xv = row8(x, c, p.k);
            uint4 av[LF_RANKS];
#pragma unroll
            for (int r = 0; r < LF_RANKS; ++r)
                av[r] = r < ranks ? row8(a + r * p.a_ld, c, p.k) : make_uint4(0, 0, 0, 0);
            float xf[8];
            widen8<F16>(xv, xf);
#pragma unroll
            for (int r = 0; r < LF_RANKS; ++r) {
                float af[8];
                widen8<F16>(av[r], af);
                if (r < ranks)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[r] = fmaf(xf[j], af[j], acc[r]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < LF_RANKS; ++r) {
        for (int d = 16; d; d /= 2) acc[r] += __shfl_down_sync(0xffffffffu, acc[r], d);
        if (lane == 0) part[warp][r] = acc[r];
    }
    __syncthreads();
    // (the last block of a row writes the zeros up to whole 64s of ranks too)
    const int end = blockIdx.y + 1 < gridDim.y || p.wide ? LF_RANKS : (p.rank + 63) / 64 * 64 - r0;
    if (threadIdx.x < end) {
        const int r = r0 + threadIdx.x;
        float v = 0.f;
        if (threadIdx.x < LF_RANKS)
            for (int w = 0; w < LF_WARPS; ++w) v += part[w][threadIdx.x];
        v = r < p.rank && g < p.plan.groups ? v * p.scale[g] : 0.f;
        if (p.wide) {
            if (r < p.rank) p.wide[(int64_t)place * p.rank + r] = v;
            return;
        }
        uint16_t *u = p.u + (int64_t)place * p.u_ld + r / GP_RC * (2 * GP_RC) + r % GP_RC;
        bf16_terms(v, u[0], u[GP_RC]);
    }
}

// ---------------------------------------------------------------------------
// Terms of inner products and of adapters (see SplitLow and launch_ext_terms).  Both
// pass a few MB, and are bound by their launch.

constexpr int SP_THREADS = 256;

struct Split {
    SplitLow of[2];
};

// A warp takes a place: 32 ranks (128 bytes) at a time.
__global__ void __launch_bounds__(SP_THREADS)
k_split_low(const __grid_constant__ GroupPlan plan, const __grid_constant__ Split split, int rank, int64_t ld) {
    extern __shared__ int32_t offs[];
    const SplitLow &s = split.of[blockIdx.y];
    const int G = plan.groups, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_begin();
    for (int i = threadIdx.x; i <= G; i += SP_THREADS) offs[i] = plan.offsets[i];
    __syncthreads();
    const int end = min(offs[G], plan.places);
    for (int64_t at = blockIdx.x * (SP_THREADS / 32) + warp; at < end; at += (int64_t)gridDim.x * (SP_THREADS / 32)) {
        int lo = 0, hi = G - 1;                  // last group that begins at or before the place
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (offs[mid] <= at) lo = mid;
            else hi = mid - 1;
        }
        const float scale = peak_scale(s.peak[lo]);
        for (int64_t c = at * ld; c < at * ld + (rank + 31) / 32 * 64; c += 64) {
            const float v = ((const float *)(s.u + c))[lane];
            __syncwarp();                        // (the terms take the values' place)
            // (a high term is zero only where the value is: what becomes of infinities is
            // taken from the high terms alone)
            const float f = v * scale;
            __half h = __float2half_rn(f);
            if (v != 0.f && __half2float(h) == 0.f) h = __ushort_as_half(v < 0.f ? 0x8001 : 1);
            s.u[c + lane] = __half_as_ushort(h);
            s.u[c + 32 + lane] = __half_as_ushort(__float2half_rn(isfinite(f) ? f - __half2float(h) : 0.f));
            if (s.ext) bf16_terms(v, s.ext[c + lane], s.ext[c + 32 + lane]);
        }
    }
}

// As bf16_terms, of a value that one or two terms hold exactly: a value that the first
// one holds keeps it, beside 2^-126 of its sign, which no sum of finite values notices.
__device__ __forceinline__ void matrix_terms(float v, uint16_t &high, uint16_t &low) {
    const uint32_t u = __float_as_uint(v), h = u & 0xffff0000u, m = u & 0x7fffffffu;
    uint32_t l = __float_as_uint(v - __uint_as_float(h));        // (exact: its lower half is 0)
    if (m >= 0x7f800000u) l = u;
    else if (u == h) l = m ? (u & 0x80000000u) | 0x00800000u : u;
    high = (uint16_t)(h >> 16);
    low = (uint16_t)(l >> 16);
}

// A thread takes eight values: of a row's ranks, or (MN) along the rows of one rank; 32-bit
// divisions where they do.
template <bool MN>
__global__ void __launch_bounds__(SP_THREADS)
k_ext_terms(uint16_t *dst, int64_t dst_ld, const uint16_t *src, int groups, int rows, int rank) {
    const int wide = !MN && rank <= 16 ? 16 : GP_RC, ranks = (rank + wide - 1) / wide * wide;
    const int units = MN ? (int)(dst_ld / 8) : ranks / 8;
    const int64_t lines = (int64_t)groups * (MN ? ranks : rows), all = lines * units;
    pdl_begin();
#pragma unroll 2
    for (int64_t i = blockIdx.x * (int64_t)SP_THREADS + threadIdx.x; i < all; i += (int64_t)gridDim.x * SP_THREADS) {
        const int64_t line = all <= INT32_MAX ? (uint32_t)i / (uint32_t)units : i / units;
        const int unit = (int)(i - line * units);
        const int64_t group = !MN ? 0 : all <= INT32_MAX ? (uint32_t)line / (uint32_t)ranks : line / ranks;
        const int r = MN ? (int)(line - group * ranks) : unit * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rank)
            v = MN ? unit_of(src + (group * rank + r) * rows, unit, rows) : unit_of(src + line * rank, unit, rank);
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
        uint32_t high[4], low[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*(const __half2 *)&x[k]);
            uint16_t h0, l0, h1, l1;
            matrix_terms(f.x, h0, l0);
            matrix_terms(f.y, h1, l1);
            high[k] = h0 | (uint32_t)h1 << 16;
            low[k] = l0 | (uint32_t)l1 << 16;
        }
        const int at = r / wide * (2 * wide) + r % wide;         // of the high terms
        uint16_t *to = MN ? dst + (group * (2 * ranks) + at) * dst_ld + unit * 8 : dst + line * dst_ld + at;
        *(uint4 *)to = make_uint4(high[0], high[1], high[2], high[3]);
        *(uint4 *)(to + (MN ? wide * dst_ld : wide)) = make_uint4(low[0], low[1], low[2], low[3]);
    }
}

// ---------------------------------------------------------------------------
// Padding copy of 16-bit elements.

__global__ void __launch_bounds__(256)
k_pad(uint16_t *dst, int64_t dst_ld, const uint16_t *src, int64_t src_ld, int64_t src_z, int64_t rows,
      int64_t all_rows, int cols) {
    const int64_t units = dst_ld / 8, all = all_rows * units;        // 16-byte units, of a row and in all
    const bool narrow = all <= INT32_MAX;                            // (64-bit divisions cost as much as the copy)
#pragma unroll 2
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
        const int64_t r = narrow ? (uint32_t)i / (uint32_t)units : i / units;
        const int64_t z = narrow ? (uint32_t)r / (uint32_t)rows : r / rows;
        *(uint4 *)(dst + i * 8) = unit_of(src + z * src_z + (r - z * rows) * src_ld, (int)(i - r * units), cols);
    }
}

// ---------------------------------------------------------------------------
// Gradient clipping: one pass sums the squares, one scales.  Both are bound by
// HBM.  The tensors are cut into chunks, named by a table in device memory (read
// from kernel parameters, the table's cache misses cost more than the chunks of a
// small set of gradients); a block's chunks lie a grid apart,
// so that the whole GPU walks the tensors in order, and the second pass walks
// them backwards: it begins with what the first left in L2.

constexpr int CL_THREADS = 256;
static_assert(CLIP_UNIT == CL_THREADS * 16, "a 16-byte access a thread");

template <int DT>
struct Vec {
    static constexpr int N = DT == HWR_F32 ? 4 : 8;      // values of 16 bytes
    __device__ static void unpack(const uint4 &u, float (&f)[N]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == HWR_F32) {
                f[i] = __uint_as_float(w[i]);
            } else if (DT == HWR_BF16) {
                f[(2 * i) % N] = __uint_as_float(w[i] << 16);
                f[(2 * i + 1) % N] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                const float2 v = __half22float2(*(const __half2 *)&w[i]);
                f[(2 * i) % N] = v.x;
                f[(2 * i + 1) % N] = v.y;
            }
        }
    }
    __device__ static uint4 pack(const float (&f)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == HWR_F32) {
                w[i] = __float_as_uint(f[i]);
            } else if (DT == HWR_BF16) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(f[(2 * i) % N], f[(2 * i + 1) % N]);
                w[i] = *(const uint32_t *)&v;
            } else {
                const __half2 v = __floats2half2_rn(f[(2 * i) % N], f[(2 * i + 1) % N]);
                w[i] = *(const uint32_t *)&v;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static float load(const void *p, int i) {
        if (DT == HWR_F32) return ((const float *)p)[i];
        if (DT == HWR_BF16) return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
        return __half2float(((const __half *)p)[i]);
    }
    __device__ static void store(void *p, int i, float v) {
        if (DT == HWR_F32) ((float *)p)[i] = v;
        else if (DT == HWR_BF16) ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(v);
        else ((__half *)p)[i] = __float2half_rn(v);
    }
    static constexpr int FULL = CLIP_UNIT / (DT == HWR_F32 ? 4 : 2);      // of a unit
};

// The squares of a thread's share of a chunk once more, in 64 bits: where
// their fp32 sum left the range that fp32 holds well.
template <int DT, int CL_PER>
__device__ __noinline__ double wide_squares(const void *in, int n, bool vec) {
    double s = 0;
    auto add = [&](float f) { s += (double)f * f; };
    constexpr int N = Vec<DT>::N;
    if (vec)
        for (int i = 0; i < CL_PER; ++i)
            for (int j = 0; j < N; ++j) add(Vec<DT>::load(in, (i * CL_THREADS + threadIdx.x) * N + j));
    else
        for (int i = threadIdx.x; i < n; i += CL_THREADS) add(Vec<DT>::load(in, i));
    return s;
}

// A running sum as two fp32 values, the second what the first's roundings lost
// (exactly, so the pair holds some 48 bits however many chunks a thread walks; the
// GPU's few 64-bit units would take longer than the reads).
struct Pair {
    float hi, lo;
    __device__ __forceinline__ void add(float v) {
        const float t = hi + v, b = t - hi;
        lo += (hi - (t - b)) + (v - b);
        hi = t;
    }
};

template <int DT, int CL_PER>
__device__ __forceinline__ void sum_chunk(const ClipChunk &c, Pair &acc, double &wide) {
    constexpr int N = Vec<DT>::N;
    const bool vec = c.n == CL_PER * Vec<DT>::FULL && ((uintptr_t)c.in & 15) == 0;
    float s = 0.f;
    if (vec) {
        const uint4 *v = (const uint4 *)c.in + threadIdx.x;
        uint4 u[CL_PER];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) u[i] = v[i * CL_THREADS];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) {
            float f[N];
            Vec<DT>::unpack(u[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) s = fmaf(f[j], f[j], s);
        }
        // all zeros: nothing was lost
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) any |= u[i].x | u[i].y | u[i].z | u[i].w;
        if (any == 0) return;
    } else {
        bool any = false;
        for (int i = threadIdx.x; i < c.n; i += CL_THREADS) {
            const float f = Vec<DT>::load(c.in, i);
            any |= f != 0.f;
            s = fmaf(f, f, s);
        }
        if (!any) return;
    }
    if (s >= 1e-30f && s <= 1e30f) acc.add(s);
    else wide += wide_squares<DT, CL_PER>(c.in, c.n, vec);      // NaN and infinities too
}

template <int DT, int CL_PER>
__device__ __forceinline__ void scale_chunk(const ClipChunk &c, float k) {
    constexpr int N = Vec<DT>::N;
    if (c.n == CL_PER * Vec<DT>::FULL && (((uintptr_t)c.in | (uintptr_t)c.out) & 15) == 0) {
        // (read for the last time, written for others: neither is to push out of L2
        // what the first pass left there)
        const uint4 *v = (const uint4 *)c.in + threadIdx.x;
        uint4 *o = (uint4 *)c.out + threadIdx.x;
        uint4 u[CL_PER];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) u[i] = __ldcs(v + i * CL_THREADS);
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) {
            float f[N];
            Vec<DT>::unpack(u[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] *= k;
            __stcs(o + i * CL_THREADS, Vec<DT>::pack(f));
        }
        return;
    }
    for (int i = threadIdx.x; i < c.n; i += CL_THREADS) Vec<DT>::store(c.out, i, Vec<DT>::load(c.in, i) * k);
}

// Sums over the warp, in lane 0.  (Tested by its bits: comparing doubles in every
// thread would take the few 64-bit units a microsecond.)
__device__ __forceinline__ void warp_sum(Pair &v, double &wide) {
    for (int d = 16; d; d /= 2) {
        const float hi = __shfl_down_sync(0xffffffffu, v.hi, d), lo = __shfl_down_sync(0xffffffffu, v.lo, d);
        v.add(hi);
        v.lo += lo;
    }
    if (__any_sync(0xffffffffu, __double_as_longlong(wide) != 0))
        for (int d = 16; d; d /= 2) wide += __shfl_down_sync(0xffffffffu, wide, d);
}

// The table's entries of up to CLIP_TABLE tensors (kernel parameters), from
// chunk `at` on: for lists that are used once.
__global__ void __launch_bounds__(CL_THREADS)
k_clip_table(const __grid_constant__ ClipTable t, ClipChunk *table) {
    const int i = blockIdx.x * CL_THREADS + threadIdx.x;
    if (i >= t.chunk0[t.n]) return;
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (t.chunk0[m] <= i) lo = m;
        else hi = m - 1;
    }
    table[t.at + i] = clip_chunk(t.in[lo], t.out[lo], t.count[lo], t.dtype[lo], t.per, i - t.chunk0[lo]);
}

// The last block to finish adds the blocks' sums, in their order, and leaves
// the norm and the factor.
template <int PER>
__global__ void __launch_bounds__(CL_THREADS)
k_square_sums(const ClipChunk *table, int chunks, ClipSums sums, float max_norm, float *norm) {
    __shared__ double w[CL_THREADS / 32];
    __shared__ Pair narrow[CL_THREADS / 32];
    __shared__ bool last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Pair acc = {0.f, 0.f};
    double wide = 0;
    pdl_begin();
    int i = blockIdx.x;
    ClipChunk c;
    if (i < chunks) c = table[i];
    for (; i < chunks; i += gridDim.x) {
        const ClipChunk now = c;
        if (i + gridDim.x < chunks) c = table[i + gridDim.x];
        if (now.dtype == HWR_F32) sum_chunk<HWR_F32, PER>(now, acc, wide);
        else if (now.dtype == HWR_BF16) sum_chunk<HWR_BF16, PER>(now, acc, wide);
        else sum_chunk<HWR_F16, PER>(now, acc, wide);
    }
    warp_sum(acc, wide);
    if (lane == 0) {
        narrow[warp] = acc;
        w[warp] = wide;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Pair n = {0.f, 0.f};
        double b = 0;
        for (int k = 0; k < CL_THREADS / 32; ++k) {
            n.add(narrow[k].hi);
            n.lo += narrow[k].lo;
            if (__double_as_longlong(w[k]) != 0) b += w[k];
        }
        b += (double)n.hi + n.lo;
        sums.part[blockIdx.x] = b;
        __threadfence();
        last = atomicAdd(sums.count, 1u) == gridDim.x - 1;
        if (last) *sums.count = 0;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    double v = 0;
    for (int k = threadIdx.x; k < gridDim.x; k += CL_THREADS) v += __ldcg(&sums.part[k]);
    for (int d = 16; d; d /= 2) v += __shfl_down_sync(0xffffffffu, v, d);
    if (lane == 0) w[warp] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        double b = 0;
        for (int k = 0; k < CL_THREADS / 32; ++k) b += w[k];
        const float total = (float)sqrt(b);
        const float k = max_norm / (total + 1e-6f);
        *norm = total;
        *sums.factor = k > 1.f || isinf(max_norm) ? 1.f : k;       // NaN stays
    }
}

template <int PER>
__global__ void __launch_bounds__(CL_THREADS)
k_clip(const ClipChunk *table, int chunks, const float *factor) {
    pdl_begin();
    int i = chunks - 1 - (int)blockIdx.x;
    ClipChunk c;
    if (i >= 0) c = table[i];
    const float k = *factor;
    for (; i >= 0; i -= gridDim.x) {
        const ClipChunk now = c;
        if (i >= (int)gridDim.x) c = table[i - gridDim.x];
        if (k == 1.f && now.in == now.out) continue;
        if (now.dtype == HWR_F32) scale_chunk<HWR_F32, PER>(now, k);
        else if (now.dtype == HWR_BF16) scale_chunk<HWR_BF16, PER>(now, k);
        else scale_chunk<HWR_F16, PER>(now, k);
    }
}

}  // namespace

cudaError_t ops_prepare(int *cluster) {
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    const auto wide = cudaFuncAttributeNonPortableClusterSizeAllowed;
    cudaError_t e = cudaFuncSetAttribute(k_dispatch_place, attr, (int)place_smem(OPS_MAX_GROUPS));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_dispatch_place, wide, 1);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_dispatch_count<DP_CLUSTER>, wide, 1);
    if (e != cudaSuccess) return e;
    // (the larger of the two kernels)
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = DP_CLUSTER;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(DP_CLUSTER);
    cfg.blockDim = dim3(DP_THREADS);
    cfg.dynamicSmemBytes = place_smem(OPS_MAX_GROUPS);
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int fit = 0;
    e = cudaOccupancyMaxActiveClusters(&fit, k_dispatch_place, &cfg);
    if (e != cudaSuccess) cudaGetLastError();        // (a size that the device does not have)
    *cluster = e == cudaSuccess && fit > 0 ? DP_CLUSTER : DP_CLUSTER_LEAST;
    return cudaSuccess;
}

// Blocks and rows per block of a dispatch: whole rounds, two blocks an SM at most.
static int dispatch_blocks(int rows, int nsm, int64_t *per_block) {
    const int64_t rounds = ((int64_t)rows + DP_ROWS - 1) / DP_ROWS;
    const int64_t each = (rounds + 2 * nsm - 1) / (2 * nsm);
    *per_block = (each < 1 ? 1 : each) * DP_ROWS;
    const int64_t b = (rows + *per_block - 1) / *per_block;
    return b < 1 ? 1 : (int)b;
}

size_t dispatch_scratch_ints(int rows, int groups, int nsm, int cluster) {
    int64_t per;
    const int b = dispatch_blocks(rows, nsm, &per);
    const int counted = (b + cluster - 1) / cluster * cluster;
    return b > cluster ? (size_t)(counted + counted / cluster) * (groups + 1) : 0;
}

// A launch that may begin while the kernel before it ends (it waits by itself).
static cudaLaunchConfig_t relaxed(int grid, int block, size_t smem, cudaStream_t s, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

cudaError_t launch_dispatch(int rows, int groups, const int32_t *choice, int32_t *offsets, int32_t *order,
                            int32_t *scratch, int nsm, int cluster, cudaStream_t s) {
    cudaLaunchAttribute at[2];
    if (rows <= DP_FEW) {
        const cudaLaunchConfig_t cfg = relaxed(1, DP_FEW, 0, s, at);
        return cudaLaunchKernelEx(&cfg, k_dispatch_few, rows, groups, choice, offsets, order);
    }
    int64_t per;
    const int b = dispatch_blocks(rows, nsm, &per);
    const int32_t *hist = b > cluster ? scratch : nullptr;
    const int counted = (b + cluster - 1) / cluster * cluster;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = hist ? cluster : b;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    if (hist) {
        cudaLaunchConfig_t cfg = relaxed(counted, DP_THREADS, (groups + 1) * 4, s, at);
        cfg.numAttrs = 2;
        const cudaError_t e = cluster == DP_CLUSTER
            ? cudaLaunchKernelEx(&cfg, k_dispatch_count<DP_CLUSTER>, rows, groups, per, choice, scratch)
            : cudaLaunchKernelEx(&cfg, k_dispatch_count<DP_CLUSTER_LEAST>, rows, groups, per, choice, scratch);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = relaxed(b, DP_THREADS, place_smem(groups), s, at);
    if (!hist && b > 1) cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_dispatch_place, rows, groups, per, choice, hist, counted, cluster, offsets, order);
}

cudaError_t launch_sort_rows(const GroupPlan &plan, const SortRows &m, int places, int32_t *padded_offsets,
                             int32_t *padded_order, int nsm, cudaStream_t s) {
    const int64_t want = ((int64_t)places + SR_THREADS / 32 - 1) / (SR_THREADS / 32), most = (int64_t)nsm * 8;
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = relaxed((int)(want < most ? want : most), SR_THREADS, (plan.groups + 1) * 8, s, at);
    // slices of at least four steps of a warp
    int64_t widest = 1;
    for (int k = 0; k < m.n; ++k) widest = widest < m.dst_ld[k] / (8 * 32 * 4) ? m.dst_ld[k] / (8 * 32 * 4) : widest;
    const int64_t slices = want < 1 ? 1 : most / want;
    cfg.gridDim.y = (unsigned)(slices < 1 ? 1 : slices < widest ? slices : widest);
    return cudaLaunchKernelEx(&cfg, k_sort_rows, plan, m, places, padded_offsets, padded_order);
}

cudaError_t launch_split_low(const GroupPlan &plan, int rank, int64_t ld, const SplitLow *s, int n, int nsm,
                             cudaStream_t st) {
    Split split;
    for (int i = 0; i < 2; ++i) split.of[i] = s[i < n ? i : 0];
    const int64_t want = ((int64_t)plan.places + SP_THREADS / 32 - 1) / (SP_THREADS / 32), most = (int64_t)nsm * 8;
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = relaxed((int)(want < most ? want : most), SP_THREADS, (plan.groups + 1) * 4, st, at);
    cfg.gridDim.y = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, k_split_low, plan, split, rank, ld);
}

cudaError_t launch_ext_terms(uint16_t *dst, int64_t dst_ld, const uint16_t *src, int groups, int rows, int rank, bool mn,
                             int nsm, cudaStream_t s) {
    const int64_t units = (int64_t)groups * (mn ? ext_terms_ranks(rank, mn) / 2 : rows) * (mn ? dst_ld / 8 : dst_ld / 16);
    const int64_t want = (units + SP_THREADS - 1) / SP_THREADS, most = (int64_t)nsm * 8;
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = relaxed((int)(want < most ? want : most), SP_THREADS, 0, s, at);
    return mn ? cudaLaunchKernelEx(&cfg, k_ext_terms<true>, dst, dst_ld, src, groups, rows, rank)
              : cudaLaunchKernelEx(&cfg, k_ext_terms<false>, dst, dst_ld, src, groups, rows, rank);
}

cudaError_t launch_low_few(const LowFew &p, bool f16, cudaStream_t s) {
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = relaxed(p.plan.rows, LF_THREADS, 0, s, at);
    cfg.gridDim.y = (unsigned)((p.rank + LF_RANKS - 1) / LF_RANKS);
    return f16 ? cudaLaunchKernelEx(&cfg, k_low_few<true>, p) : cudaLaunchKernelEx(&cfg, k_low_few<false>, p);
}

cudaError_t launch_pad(void *dst, int64_t dst_ld, const void *src, int64_t src_ld, int64_t src_z, int64_t nz,
                       int64_t rows, int cols, int nsm, cudaStream_t s) {
    const int64_t units = nz * rows * (dst_ld / 8);
    if (units <= 0) return cudaSuccess;
    const int64_t want = (units + 255) / 256;
    const int grid = (int)(want < (int64_t)nsm * 8 ? want : (int64_t)nsm * 8);
    k_pad<<<grid, 256, 0, s>>>((uint16_t *)dst, dst_ld, (const uint16_t *)src, src_ld, src_z, rows, nz * rows, cols);
    return cudaGetLastError();
}

int clip_blocks(int64_t chunks, int nsm) {
    const int64_t most = (int64_t)nsm * 8;
    return (int)(chunks < 1 ? 1 : chunks < most ? chunks : most);
}

cudaError_t launch_clip_table(const ClipTable &t, ClipChunk *table, cudaStream_t s) {
    const int chunks = t.chunk0[t.n];
    if (chunks) k_clip_table<<<(chunks + CL_THREADS - 1) / CL_THREADS, CL_THREADS, 0, s>>>(t, table);
    return cudaGetLastError();
}

cudaError_t launch_clip(const ClipChunk *table, int chunks, int per, int nsm, const ClipSums &sums, float max_norm,
                        float *norm, cudaStream_t s) {
    const int blocks = clip_blocks(chunks, nsm);
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = relaxed(blocks, CL_THREADS, 0, s, at);
    const float *factor = sums.factor;
    cudaError_t e = per == 1 ? cudaLaunchKernelEx(&cfg, k_square_sums<1>, table, chunks, sums, max_norm, norm)
                             : cudaLaunchKernelEx(&cfg, k_square_sums<CLIP_PER>, table, chunks, sums, max_norm, norm);
    if (e != cudaSuccess || chunks == 0) return e;
    return per == 1 ? cudaLaunchKernelEx(&cfg, k_clip<1>, table, chunks, factor)
                    : cudaLaunchKernelEx(&cfg, k_clip<CLIP_PER>, table, chunks, factor);
}

}  // namespace hwr
