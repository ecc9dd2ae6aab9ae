// A shared projection with low-rank terms for a few rows: decode steps, whose
// time is that of reading W.  A block takes 16 output columns and its eight warps
// an eighth of the contraction each, 32 columns of it in turn, so that the block
// reads 512 consecutive bytes of each row of W; nothing is staged, cut or joined
// through memory.  Bound by memory latency: a warp has at most four steps' loads in
// flight (48 registers), and reading W waits for the inner products though only the
// epilogue needs them (33.5 MB of W alone and with cold caches: 16.5 us, 2.0 TB/s).  The
// multiplications are warp-level 16 x 8 x 16 MMAs: a tile of 256 rows on tcgen05
// would be filled by 8 or 16 (one row, 4,096 -> 4,096, rank 16, with its dispatch:
// 28.0 us there, 21.4 us here when both were measured, 19.5 by now; the weights'
// bytes take 4.9).
//
// The contraction's order is free, so a lane takes eight consecutive columns of
// its row with one 16-byte load and uses them as the column pairs (2q, 2q + 1)
// and (2q + 8, 2q + 9) of two MMAs, in both operands alike.
#include "ops_internal.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hwr {
namespace {

constexpr int FW_THREADS = 256, FW_WARPS = FW_THREADS / 32;
constexpr int FW_ROWS = 16;        // output columns (rows of W) of a block
constexpr int FW_TOKENS = FEW_ROWS;   // rows of x

template <bool F16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight elements from column c on of a row of n, zeros beyond it and for no row.
__device__ __forceinline__ uint4 eight(const uint16_t *row, int c, int n) {
    if (!row || c >= n) return make_uint4(0, 0, 0, 0);
    if (c + 8 <= n) return __ldg((const uint4 *)(row + c));
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < n ? row[c + j] : 0;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

template <bool F16>
__device__ __forceinline__ float widen(uint16_t v) {
    if (F16) return __half2float(__ushort_as_half(v));
    return __uint_as_float((uint32_t)v << 16);
}

static_assert(FW_TOKENS == 16 && FW_ROWS * FW_TOKENS == FW_THREADS, "a value a thread; two places a warp");

template <bool F16>
__global__ void __launch_bounds__(FW_THREADS)
k_few_rows(const __grid_constant__ FewRows p) {
    __shared__ float sums[FW_WARPS][FW_ROWS][FW_TOKENS + 1];
    __shared__ int rows[FW_TOKENS], low[FW_TOKENS];     // by place: row of x and output; its adapter
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, q = lane & 3;
    const int G = p.plan.groups, n0 = blockIdx.x * FW_ROWS;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int blocks = (p.k + 31) / 32;

    const uint16_t *wa = n0 + g8 < p.n ? p.w + (int64_t)(n0 + g8) * p.w_ld : nullptr;
    const uint16_t *wb = n0 + g8 + 8 < p.n ? p.w + (int64_t)(n0 + g8 + 8) * p.w_ld : nullptr;
    const int last = p.plan.rows;
    if (tid < FW_TOKENS) {
        const int r = tid < last ? p.plan.order[tid] : -1;
        rows[tid] = (uint32_t)r < (uint32_t)last ? r : -1;
    }
    if (warp < FW_TOKENS / 2) {
        // the adapters of two places: how many groups end at or before them
        int m0 = 0, m1 = 0;
        for (int g = lane; g < G; g += 32) {
            const int end = p.plan.offsets[g + 1];
            m0 += end <= 2 * warp;
            m1 += end <= 2 * warp + 1;
        }
        m0 = __reduce_add_sync(0xffffffffu, m0);
        m1 = __reduce_add_sync(0xffffffffu, m1);
        if (lane == 0) {
            low[2 * warp] = m0 < G ? m0 : -1;
            low[2 * warp + 1] = m1 < G ? m1 : -1;
        }
    }
    __syncthreads();
    const bool two = last > 8;
    const uint16_t *xa = rows[g8] >= 0 ? p.x + rows[g8] * p.x_ld : nullptr;
    const uint16_t *xb = rows[g8 + 8] >= 0 ? p.x + rows[g8 + 8] * p.x_ld : nullptr;
    float c0[4] = {}, c1[4] = {};
#pragma unroll 4
    for (int b = warp; b < blocks; b += FW_WARPS) {
        const int c = b * 32 + q * 8;
        const uint4 a = eight(wa, c, p.k), d = eight(wb, c, p.k);
        const uint4 x = eight(xa, c, p.k);
        mma16816<F16>(c0, a.x, d.x, a.y, d.y, x.x, x.y);
        mma16816<F16>(c0, a.z, d.z, a.w, d.w, x.z, x.w);
        if (two) {
            const uint4 y = eight(xb, c, p.k);
            mma16816<F16>(c1, a.x, d.x, a.y, d.y, y.x, y.y);
            mma16816<F16>(c1, a.z, d.z, a.w, d.w, y.z, y.w);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = g8 + (i >> 1) * 8, t = 2 * q + (i & 1);
        sums[warp][r][t] = c0[i];
        sums[warp][r][t + 8] = c1[i];
    }
    __syncthreads();
    // 16 x 16 values, one a thread: output column r of the row at place t
    const int r = tid & 15, t = tid >> 4, n = n0 + r;
    if (rows[t] < 0 || n >= p.n) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < FW_WARPS; ++w) v += sums[w][r][t];
    if (low[t] >= 0) {
        const float *u = p.u + (int64_t)t * p.rank;
        const uint16_t *b = p.b + low[t] * p.b_z + (int64_t)n * p.b_ld;
        float s = 0.f;
#pragma unroll 8
        for (int j = 0; j < p.rank; ++j) s = fmaf(u[j], widen<F16>(b[j]), s);
        v += s;
    }
    uint16_t *out = p.out + rows[t] * p.ld + n;
    if (F16) *(__half *)out = __float2half_rn(v);
    else *(__nv_bfloat16 *)out = __float2bfloat16_rn(v);
}

}  // namespace

cudaError_t launch_few_rows(const FewRows &p, bool f16, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)((p.n + FW_ROWS - 1) / FW_ROWS));
    cfg.blockDim = dim3(FW_THREADS);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return f16 ? cudaLaunchKernelEx(&cfg, k_few_rows<true>, p) : cudaLaunchKernelEx(&cfg, k_few_rows<false>, p);
}

}  // namespace hwr
