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
// that share a key find each other by a match over the warp, so a row's place
// is its key's first place (over the blocks, rounds and warps before it) plus
// the peers in lower lanes: no atomics decide an order.

constexpr int DP_THREADS = 1024, DP_WARPS = DP_THREADS / 32;
constexpr int DP_PER = 8;
constexpr int DP_ROWS = DP_THREADS * DP_PER;

__device__ __forceinline__ int key_of(const int32_t *choice, int64_t row, int64_t end, int G) {
    if (row >= end) return G + 1;            // no row
    const int c = choice[row];
    return (uint32_t)c < (uint32_t)G ? c : G;
}

// Rows of each key in each block: hist [blocks][G + 1].
__global__ void __launch_bounds__(DP_THREADS)
k_dispatch_count(int rows, int G, int64_t per_block, const int32_t *choice, int32_t *hist) {
    extern __shared__ int32_t sh[];
    for (int i = threadIdx.x; i <= G; i += DP_THREADS) sh[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * per_block;
    const int64_t end = begin + per_block < rows ? begin + per_block : rows;
    const int lane = threadIdx.x & 31;
    for (int64_t r0 = begin; r0 < end; r0 += DP_ROWS) {
        int key[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) key[i] = key_of(choice, r0 + i * DP_THREADS + threadIdx.x, end, G);
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) {
            const uint32_t peers = __match_any_sync(0xffffffffu, key[i]);
            if (key[i] <= G && lane == __ffs(peers) - 1) atomicAdd(&sh[key[i]], __popc(peers));
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i <= G; i += DP_THREADS) hist[(int64_t)blockIdx.x * (G + 1) + i] = sh[i];
}

// hist: counts per block of k_dispatch_count, or null with a single block.
__global__ void __launch_bounds__(DP_THREADS)
k_dispatch_place(int rows, int G, int64_t per_block, const int32_t *choice, const int32_t *hist,
                 int32_t *offsets, int32_t *order) {
    extern __shared__ int32_t sh[];
    const int G1 = G + 1, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t *wh = sh;                        // [DP_WARPS][G1] counts, then first places
    int32_t *base = sh + DP_WARPS * G1;      // [G1] next place of each key
    int32_t *total = base + G1;              // [G1] rows of each key in all
    int32_t *round = total + G1;             // [G1] rows of each key in this round
    __shared__ int32_t wsum[DP_WARPS];
    const int64_t begin = blockIdx.x * per_block;
    const int64_t end = begin + per_block < rows ? begin + per_block : rows;

    for (int i = tid; i < G1; i += DP_THREADS) base[i] = total[i] = 0;
    for (int64_t r0 = begin; r0 < end || r0 == begin; r0 += DP_ROWS) {
        int key[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i)
            key[i] = key_of(choice, r0 + (warp * DP_PER + i) * 32 + lane, end, G);
        for (int i = tid; i < DP_WARPS * G1; i += DP_THREADS) wh[i] = 0;
        __syncthreads();
        if (hist && r0 == begin) {
            // rows of each key in the blocks before this one, and in all
            const int subs = max(1, DP_THREADS / G1), nb = gridDim.x;
            for (int j = tid; j < G1 * subs; j += DP_THREADS) {
                const int g = j % G1, sub = j / G1;
                int before = 0, all = 0;
                for (int b = sub; b < nb; b += subs) {
                    const int c = hist[(int64_t)b * G1 + g];
                    all += c;
                    if (b < (int)blockIdx.x) before += c;
                }
                atomicAdd(&base[g], before);
                atomicAdd(&total[g], all);
            }
        }
        // counts of each warp's rows
        int rank[DP_PER];
#pragma unroll
        for (int i = 0; i < DP_PER; ++i) {
            const uint32_t peers = __match_any_sync(0xffffffffu, key[i]);
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
        __syncthreads();
        // over the warps: counts become first places within the round
        for (int g = tid; g < G1; g += DP_THREADS) {
            int sum = 0;
            for (int w = 0; w < DP_WARPS; ++w) {
                const int c = wh[w * G1 + g];
                wh[w * G1 + g] = sum;
                sum += c;
            }
            if (!hist) total[g] = sum;      // a single block has a single round
            round[g] = sum;
        }
        __syncthreads();
        if (r0 == begin) {
            // first place of each key: a running sum of the totals
            int v = tid < G ? total[tid] : 0, s = v;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int o = __shfl_up_sync(0xffffffffu, s, d);
                if (lane >= d) s += o;
            }
            if (lane == 31) wsum[warp] = s;
            __syncthreads();
            if (warp == 0) {
                int x = wsum[lane];
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int o = __shfl_up_sync(0xffffffffu, x, d);
                    if (lane >= d) x += o;
                }
                wsum[lane] = x;
            }
            __syncthreads();
            const int upto = s + (warp ? wsum[warp - 1] : 0);
            if (tid < G) base[tid] += upto - v;
            if (tid == 0) base[G] += wsum[DP_WARPS - 1];
            if (blockIdx.x == 0) {
                if (tid < G) offsets[tid + 1] = upto;
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
}

size_t place_smem(int G) { return (size_t)(DP_WARPS + 3) * (G + 1) * 4; }

// ---------------------------------------------------------------------------
// Rows by place: a warp copies a row (reads and writes of 512 bytes at a time).

constexpr int SR_THREADS = 256;

__global__ void __launch_bounds__(SR_THREADS)
k_sort_rows(const __grid_constant__ GroupPlan plan, const __grid_constant__ SortRows m, int places,
            int32_t *padded_offsets, int32_t *padded_order) {
    extern __shared__ int32_t sh[];
    const int G = plan.groups, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int32_t *offs = sh, *pad = sh + G + 1;       // first place of each group, in either plan
    int total = plan.rows;
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
        if (blockIdx.x == 0) {
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
        if (padded_offsets && lane == 0) padded_order[at] = r;
        for (int k = 0; k < m.n; ++k) {
            uint4 *dst = (uint4 *)(m.dst[k] + at * m.dst_ld[k]);
            const int units = (int)(m.dst_ld[k] / 8), cols = m.cols[k];
            const uint16_t *src = r < 0 ? nullptr : m.src[k] + r * m.src_ld[k];
            if (src && ((uintptr_t)src & 15) == 0 && cols % 8 == 0) {
#pragma unroll 4
                for (int i = lane; i < units; i += 32) dst[i] = __ldg((const uint4 *)src + i);
                continue;
            }
            for (int i = lane; i < units; i += 32) {
                uint32_t v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = src && i * 8 + j < cols ? src[i * 8 + j] : 0;
                dst[i] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Low-rank inner products of a few rows: u[place] = scale[g] A[g] x[order[place]]
// as two 16-bit terms a value, in the layout of the tensor-core kernel.  A few
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
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = p.plan.order[place];
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
    if (threadIdx.x < LF_RANKS) {
        const int r = r0 + threadIdx.x;
        float v = 0.f;
        for (int w = 0; w < LF_WARPS; ++w) v += part[w][threadIdx.x];
        v = r < p.rank && g < p.plan.groups ? v * p.scale[g] : 0.f;
        // high and low terms (an infinite high one takes a zero low one)
        uint16_t *u = p.u + (int64_t)place * p.u_ld + r / GP_RC * (2 * GP_RC) + r % GP_RC;
        if (F16) {
            const __half h = __float2half_rn(v);
            const float f = __half2float(h);
            u[0] = __half_as_ushort(h);
            u[GP_RC] = __half_as_ushort(__float2half_rn(isinf(f) ? 0.f : v - f));
        } else {
            const __nv_bfloat16 h = __float2bfloat16_rn(v);
            const float f = __bfloat162float(h);
            u[0] = __bfloat16_as_ushort(h);
            u[GP_RC] = __bfloat16_as_ushort(__float2bfloat16_rn(isinf(f) ? 0.f : v - f));
        }
    }
}

// ---------------------------------------------------------------------------
// Padding copy of 16-bit elements.

__global__ void __launch_bounds__(256)
k_pad(uint16_t *dst, int64_t dst_ld, const uint16_t *src, int64_t src_ld, int64_t src_z, int64_t rows,
      int64_t all_rows, int cols) {
    const int64_t units = dst_ld / 8;        // 16-byte units of a row
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all_rows * units; i += gridDim.x * 256ll) {
        const int64_t r = i / units;
        const int c = (int)(i - r * units) * 8;
        const uint16_t *s = src + (r / rows) * src_z + (r % rows) * src_ld + c;
        uint32_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? s[j] : 0;
        *(uint4 *)(dst + r * dst_ld + c) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16,
                                                      v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
}

// ---------------------------------------------------------------------------
// Gradient clipping: one pass sums the squares, one scales.  Both are bound by
// HBM; a block's chunks lie a grid apart, so that the whole GPU walks the
// tensors in order, and the second pass walks them backwards: it begins with
// what the first left in L2.

constexpr int CL_THREADS = 256;
constexpr int CL_BYTES = 16;                         // of one access
constexpr int CL_PER = 8;                            // accesses of a thread in a chunk

__host__ __device__ inline int dtype_size(int d) { return d == HWR_F32 ? 4 : 2; }
__host__ __device__ inline int chunk_elems(int d) { return CL_THREADS * CL_PER * CL_BYTES / dtype_size(d); }

// Eight 16-byte units (or the ragged, unaligned rest) of a chunk as floats.
template <int DT>
struct Vec {
    static constexpr int N = DT == HWR_F32 ? 4 : 8;
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
};

template <int DT>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    if (DT == HWR_F32) return ((const float *)p)[i];
    if (DT == HWR_BF16) return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
    return __half2float(((const __half *)p)[i]);
}
template <int DT>
__device__ __forceinline__ void store1(void *p, int64_t i, float v) {
    if (DT == HWR_F32) ((float *)p)[i] = v;
    else if (DT == HWR_BF16) ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(v);
    else ((__half *)p)[i] = __float2half_rn(v);
}

// Adds the squares of some values, s their fp32 sum: into `acc` where fp32
// holds it well, else (squares near fp32's limits) into `wide`, exactly
// enough.  NaN and infinite values go the ordinary way.
template <int N>
__device__ __forceinline__ void add_squares(const float (&f)[N], float &acc, double &wide) {
    float s = 0.f, m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s = fmaf(f[i], f[i], s);
        m = fmaxf(m, fabsf(f[i]));
    }
    if ((s > 1e30f && m <= 3.4028234e38f) || (s < 1e-30f && m > 0.f)) {
        for (int i = 0; i < N; ++i) wide += (double)f[i] * f[i];
        return;
    }
    acc += s;
}

template <int DT>
__device__ __forceinline__ void sum_chunk(const void *in, int64_t e0, int64_t n, float &acc, double &wide) {
    constexpr int N = Vec<DT>::N, SZ = DT == HWR_F32 ? 4 : 2;
    const int64_t left = n - e0;
    if (left >= chunk_elems(DT) && ((uintptr_t)in & 15) == 0) {
        const uint4 *v = (const uint4 *)((const char *)in + e0 * SZ) + threadIdx.x;
        uint4 u[CL_PER];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) u[i] = v[i * CL_THREADS];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) {
            float f[N];
            Vec<DT>::unpack(u[i], f);
            add_squares(f, acc, wide);
        }
        return;
    }
    const int64_t stop = left < chunk_elems(DT) ? left : chunk_elems(DT);
    for (int64_t i = threadIdx.x; i < stop; i += CL_THREADS) {
        float f[1] = {load1<DT>(in, e0 + i)};
        add_squares(f, acc, wide);
    }
}

template <int DT>
__device__ __forceinline__ void scale_chunk(const void *in, void *out, int64_t e0, int64_t n, float k) {
    constexpr int N = Vec<DT>::N, SZ = DT == HWR_F32 ? 4 : 2;
    const int64_t left = n - e0;
    if (left >= chunk_elems(DT) && (((uintptr_t)in | (uintptr_t)out) & 15) == 0) {
        const uint4 *v = (const uint4 *)((const char *)in + e0 * SZ) + threadIdx.x;
        uint4 *o = (uint4 *)((char *)out + e0 * SZ) + threadIdx.x;
        uint4 u[CL_PER];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) u[i] = v[i * CL_THREADS];
#pragma unroll
        for (int i = 0; i < CL_PER; ++i) {
            float f[N];
            Vec<DT>::unpack(u[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] *= k;
            o[i * CL_THREADS] = Vec<DT>::pack(f);
        }
        return;
    }
    const int64_t stop = left < chunk_elems(DT) ? left : chunk_elems(DT);
    for (int64_t i = threadIdx.x; i < stop; i += CL_THREADS)
        store1<DT>(out, e0 + i, load1<DT>(in, e0 + i) * k);
}

__device__ __forceinline__ int tensor_of(const ClipTable &t, int chunk) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (t.chunk0[m] <= chunk) lo = m;
        else hi = m - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double w[CL_THREADS / 32];
    for (int d = 16; d; d /= 2) v += __shfl_down_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0;
    for (int i = 0; i < CL_THREADS / 32; ++i) s += w[i];
    return s;
}

__global__ void __launch_bounds__(CL_THREADS)
k_square_sums(const __grid_constant__ ClipTable t, double *part) {
    float acc = 0.f;
    double wide = 0;
    const int chunks = t.chunk0[t.n];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int k = tensor_of(t, c);
        const int64_t n = t.count[k];
        const int64_t e0 = (int64_t)(c - t.chunk0[k]) * chunk_elems(t.dtype[k]);
        if (t.dtype[k] == HWR_F32) sum_chunk<HWR_F32>(t.in[k], e0, n, acc, wide);
        else if (t.dtype[k] == HWR_BF16) sum_chunk<HWR_BF16>(t.in[k], e0, n, acc, wide);
        else sum_chunk<HWR_F16>(t.in[k], e0, n, acc, wide);
    }
    const double s = block_sum((double)acc + wide);
    if (threadIdx.x == 0) part[t.first_block + blockIdx.x] = s;
}

__global__ void __launch_bounds__(CL_THREADS)
k_clip(const __grid_constant__ ClipTable t, const double *part, int nparts, float max_norm, float *norm) {
    double s = 0;
    for (int i = threadIdx.x; i < nparts; i += CL_THREADS) s += part[i];
    const float total = (float)sqrt(block_sum(s));
    if (blockIdx.x == 0 && t.first_block == 0 && threadIdx.x == 0) *norm = total;
    float k = max_norm / (total + 1e-6f);
    if (k > 1.f || isinf(max_norm)) k = 1.f;        // NaN stays
    const int chunks = t.chunk0[t.n];
    for (int c = chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
        const int i = tensor_of(t, c);
        if (k == 1.f && t.in[i] == t.out[i]) continue;
        const int64_t n = t.count[i];
        const int64_t e0 = (int64_t)(c - t.chunk0[i]) * chunk_elems(t.dtype[i]);
        if (t.dtype[i] == HWR_F32) scale_chunk<HWR_F32>(t.in[i], t.out[i], e0, n, k);
        else if (t.dtype[i] == HWR_BF16) scale_chunk<HWR_BF16>(t.in[i], t.out[i], e0, n, k);
        else scale_chunk<HWR_F16>(t.in[i], t.out[i], e0, n, k);
    }
}

}  // namespace

cudaError_t ops_prepare() {
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    return cudaFuncSetAttribute(k_dispatch_place, attr, (int)place_smem(OPS_MAX_GROUPS));
}

// Blocks and rows per block of a dispatch: whole rounds, a block an SM at most.
static int dispatch_blocks(int rows, int nsm, int64_t *per_block) {
    const int64_t rounds = ((int64_t)rows + DP_ROWS - 1) / DP_ROWS;
    const int64_t each = (rounds + nsm - 1) / nsm;
    *per_block = (each < 1 ? 1 : each) * DP_ROWS;
    const int64_t b = (rows + *per_block - 1) / *per_block;
    return b < 1 ? 1 : (int)b;
}

size_t dispatch_scratch_ints(int rows, int groups, int nsm) {
    int64_t per;
    const int b = dispatch_blocks(rows, nsm, &per);
    return b > 1 ? (size_t)b * (groups + 1) : 0;
}

cudaError_t launch_dispatch(int rows, int groups, const int32_t *choice, int32_t *offsets, int32_t *order,
                            int32_t *scratch, int nsm, cudaStream_t s) {
    int64_t per;
    const int b = dispatch_blocks(rows, nsm, &per);
    if (b > 1)
        k_dispatch_count<<<b, DP_THREADS, (groups + 1) * 4, s>>>(rows, groups, per, choice, scratch);
    k_dispatch_place<<<b, DP_THREADS, place_smem(groups), s>>>(rows, groups, per, choice,
                                                              b > 1 ? scratch : nullptr, offsets, order);
    return cudaGetLastError();
}

cudaError_t launch_sort_rows(const GroupPlan &plan, const SortRows &m, int places, int32_t *padded_offsets,
                             int32_t *padded_order, int nsm, cudaStream_t s) {
    const int64_t want = ((int64_t)places + SR_THREADS / 32 - 1) / (SR_THREADS / 32), most = (int64_t)nsm * 8;
    k_sort_rows<<<(int)(want < most ? want : most), SR_THREADS, (plan.groups + 1) * 8, s>>>(plan, m, places, padded_offsets,
                                                                                            padded_order);
    return cudaGetLastError();
}

cudaError_t launch_low_few(const LowFew &p, bool f16, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)p.plan.rows, (unsigned)((p.rank + 2 * GP_RC - 1) / (2 * GP_RC) * (2 * GP_RC / LF_RANKS)));
    cfg.blockDim = dim3(LF_THREADS);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
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

int64_t clip_chunks(int64_t n, int dtype) { return (n + chunk_elems(dtype) - 1) / chunk_elems(dtype); }

cudaError_t launch_square_sums(const ClipTable &t, int blocks, double *part, cudaStream_t s) {
    k_square_sums<<<blocks, CL_THREADS, 0, s>>>(t, part);
    return cudaGetLastError();
}

cudaError_t launch_clip(const ClipTable &t, int blocks, const double *part, int nparts, float max_norm,
                        float *norm, cudaStream_t s) {
    k_clip<<<blocks, CL_THREADS, 0, s>>>(t, part, nparts, max_norm, norm);
    return cudaGetLastError();
}

}  // namespace hwr
