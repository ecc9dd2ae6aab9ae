// The AdamW step over many tensors: one launch, a pass over parameters, gradients and
// moments, bound by HBM.  A thread takes eight consecutive elements, a block 2,048 of
// one tensor, named by a table in device memory as in gradient clipping (read a chunk
// ahead); the gradients' addresses, which change from step to step, are kernel parameters.
//
// With moments in 8 bits, 256 elements (a warp's) share a power of two: the largest
// magnitude lies in [2^7, 2^8) of e4m3's values, and those down to 2^-16 of it keep
// their three bits.  Kept are m and sqrt(v), whose ratios to their block's largest are
// alike.  A value is rounded up or down by 16 bits of a hash of seed, step, tensor and
// element, so that its expectation is the value: a step changes v by 0.1 % (beta2 0.999),
// and rounding to the nearest of values 6 to 12 % apart would leave it where it is for
// good.  A positive sqrt(v) is never rounded to 0, which would make the next update of a
// quiet element large.  Everything up to the codes is done in single fp32 operations
// that round to nearest (no fused multiply-add), so that a restatement of the formula
// gives the same codes.
#include "ops_internal.cuh"
#include "values.cuh"

namespace hwr {
namespace {

constexpr int AW_THREADS = 256, AW_BLOCKS = 3;        // blocks that an SM holds
static_assert(AW_THREADS * 8 == ADAMW_CHUNK && ADAMW_BLOCK == 32 * 8, "eight elements a thread; a warp's share a scale");

// Eight values as they lie in memory: 16 bytes (16-bit types: `a`), or 32.
struct Raw {
    uint4 a, b;
};

__device__ __forceinline__ void widen(const Raw &r, int dtype, float (&f)[8]) {
    if (dtype == HWR_F32) {
        float lo[4], hi[4];
        Vec<HWR_F32>::unpack(r.a, lo);
        Vec<HWR_F32>::unpack(r.b, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = lo[i];
            f[i + 4] = hi[i];
        }
    } else if (dtype == HWR_BF16) {
        Vec<HWR_BF16>::unpack(r.a, f);
    } else {
        Vec<HWR_F16>::unpack(r.a, f);
    }
}

// n values from element i on (full: eight, 16-byte aligned), zeros beyond.
__device__ __forceinline__ Raw take(const void *p, int dtype, int64_t i, int n, bool full) {
    Raw r = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (dtype == HWR_F32) {
        const float *q = (const float *)p + i;
        if (full) {
            r.a = __ldcs((const uint4 *)q);
            r.b = __ldcs((const uint4 *)q + 1);
        } else {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? __float_as_uint(q[j]) : 0u;
            r.a = make_uint4(v[0], v[1], v[2], v[3]);
            r.b = make_uint4(v[4], v[5], v[6], v[7]);
        }
    } else {
        const uint16_t *q = (const uint16_t *)p + i;
        if (full) {
            r.a = __ldcs((const uint4 *)q);
        } else {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? q[j] : 0u;
            r.a = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
    }
    return r;
}

__device__ __forceinline__ void put32(float *q, const float (&f)[8], int n, bool full) {
    if (full) {
        __stcs((float4 *)q, make_float4(f[0], f[1], f[2], f[3]));
        __stcs((float4 *)q + 1, make_float4(f[4], f[5], f[6], f[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) q[j] = f[j];
    }
}

template <int DT>
__device__ __forceinline__ void put16(void *p, int64_t i, const float (&f)[8], int n, bool full) {
    if (full) {
        __stcs((uint4 *)((uint16_t *)p + i), Vec<DT>::pack(f));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) Vec<DT>::store((uint16_t *)p + i, j, f[j]);
    }
}

__device__ __forceinline__ uint2 take8(const void *p, int64_t i, int n, bool full) {
    const uint8_t *q = (const uint8_t *)p + i;
    if (full) return __ldcs((const uint2 *)q);
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) (j < 4 ? lo : hi) |= (uint32_t)q[j] << 8 * (j & 3);
    return make_uint2(lo, hi);
}

__device__ __forceinline__ void put8(void *p, int64_t i, uint2 c, int n, bool full) {
    uint8_t *q = (uint8_t *)p + i;
    if (full) {
        __stcs((uint2 *)q, c);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) q[j] = (uint8_t)((j < 4 ? c.x : c.y) >> 8 * (j & 3));
}

// max(a, b), NaN where one of them is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// A 32-bit hash of whole numbers, each output bit of which depends on every input bit
// about evenly (tested on the rounding that it drives): two multiplications between shifts, the
// form and the first multiplier of C. Wellons, "Prospecting for Hash Functions" (2018).
__device__ __forceinline__ uint32_t mixed(uint32_t x) {
    x = (x ^ x >> 16) * 0x7feb352du;
    x = (x ^ x >> 15) * 0x68e31da5u;
    return x ^ x >> 16;
}

constexpr float DOWN = 0x1p-120f;         // from e4m3's exponents to fp32's last ones

// Eight e4m3 values times their block's power of two.
__device__ __forceinline__ void values8(uint2 c, float scale, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t pair = (uint16_t)((i < 2 ? c.x : c.y) >> 16 * (i & 1));
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(pair));
        const float2 x = __half22float2(*(const __half2 *)&h);
        (Two(x.x, x.y) * Two(scale, scale)).get(f[2 * i], f[2 * i + 1]);
    }
}

// The power of two of a warp's block with this largest magnitude (its bits), and its inverse.
__device__ __forceinline__ uint32_t scale_field(uint32_t most) {
    const int f = (int)(most >> 23) - 7;
    return (uint32_t)(f < 1 ? 1 : f) << 23;
}

// Bytes of eight values (root: not negative, and above 0 where the value is), rounded up or
// down by the high or the low 16 random bits of each.
template <bool ROOT>
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float *scale, const uint32_t (&random)[8], bool write) {
    float largest = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) largest = max_nan(largest, fabsf(x[j]));
    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(largest));
    const uint32_t field = scale_field(most);
    const float inverse = __uint_as_float((254u << 23) - field);
    if (write) *scale = most >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(field);
    // (both powers of two in one multiplication, where their product is a normal number: the
    // result is the same, as the first one's is exact unless the second makes 0 of it)
    const bool one = field < 134u << 23;
    const float down = one ? __uint_as_float((134u << 23) - field) : DOWN;
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        float a = x[j], b = x[j + 1];
        if (!one) (Two(a, b) * Two(inverse, inverse)).get(a, b);
        (Two(a, b) * Two(down, down)).get(a, b);
        c[j] = __float_as_uint(a);
        c[j + 1] = __float_as_uint(b);
    }
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = ROOT ? random[j] >> 12 & 0xffff0u : random[j] << 4 & 0xffff0u;
        // (the value's bits below the sign, whose place in the byte is four lower)
        c[j] = (c[j] + (bits | 8)) >> 20;
        if (ROOT) c[j] = max(c[j], min(__float_as_uint(x[j]), 1u));
        else c[j] = (c[j] & ~0x80u) | (c[j] >> 4 & 0x80u);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
    return make_uint2(w[0], w[1]);
}

// Within a unit of the last place, for values whose bits nobody keeps.
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float root(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A thread's eight elements as they lie in memory.
template <int BITS>
struct Chunk {
    const void *grad;                     // null: there is nothing to do
    int64_t at;                           // the first one's place in its tensor
    int tensor, n;
    bool full;
    Raw p, g, m, v;
    uint2 cm, cv;
    float sm, sv;
    __device__ __forceinline__ void load(const AdamWStep &s, const AdamWChunk &chunk) {
        tensor = chunk.tensor;
        const AdamWTensor &c = s.tensors[tensor];
        grad = s.grad[tensor - s.tensor0];
        at = (int64_t)chunk.chunk * ADAMW_CHUNK + threadIdx.x * 8;
        const int64_t own = c.n - at;
        n = own < 0 ? 0 : own < 8 ? (int)own : 8;
        // (the last elements, and tensors that are not aligned to 16 bytes, go one by one)
        full = n == 8 && c.aligned && ((uintptr_t)grad & 15) == 0;
        if (!grad) return;
        p = take(c.param, HWR_F32, at, n, full);
        g = take(grad, s.dtype[tensor - s.tensor0], at, n, full);
        if (BITS == 32) {
            m = take(c.m, HWR_F32, at, n, full);
            v = take(c.v, HWR_F32, at, n, full);
        } else {
            cm = take8(c.m, at, n, full);
            cv = take8(c.v, at, n, full);
            sm = n ? c.m_scale[at / ADAMW_BLOCK] : 0.f;
            sv = n ? c.v_scale[at / ADAMW_BLOCK] : 0.f;
        }
    }
    __device__ __forceinline__ void moments(float (&a)[8], float (&b)[8]) const {
        if (BITS == 32) {
            widen(m, HWR_F32, a);
            widen(v, HWR_F32, b);
        } else {
            values8(cm, sm, a);
            values8(cv, sv, b);
        }
    }
};

template <int BITS>
__global__ void __launch_bounds__(AW_THREADS, AW_BLOCKS)
k_adamw(const __grid_constant__ AdamWStep p) {
    const int tid = threadIdx.x, lane = tid & 31;
    // (the tables were there before the call)
    AdamWChunk first = {p.tensor0, 0};
    if ((int)blockIdx.x < p.chunks) first = p.table[blockIdx.x];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int32_t t = *p.step + 1;
    const float norm = p.norm ? *p.norm : 0.f, rate = p.lr ? *p.lr : p.rate;
    const bool skip = !(fabsf(norm) < INFINITY);          // nothing changes, the step's number neither
    float k = 1.f;
    if (p.norm) {
        k = __fdiv_rn(p.max_norm, norm + 1e-6f);
        k = k > 1.f || isinf(p.max_norm) ? 1.f : k;
    }
    const float c1 = -expm1f((float)t * p.log_b1), c2 = -expm1f((float)t * p.log_b2);
    const float by1 = 1.f / c1, by2 = rsqrtf(c2);
    const uint32_t key_t = mixed((uint32_t)t + p.seed * 0x9e3779b1u);
    Chunk<BITS> now;
    int i = blockIdx.x;
    if (!skip && i < p.chunks) now.load(p, first);
    // (all threads have read the step's number before thread 0 can say so below)
    __syncthreads();
    for (; !skip && i < p.chunks; i += gridDim.x) {
        // 8 bits: the next chunk's loads are under way while this one's codes are made
        Chunk<BITS> next;
        const bool more = i + gridDim.x < p.chunks;
        if (more) first = p.table[i + gridDim.x];
        if (BITS == 8 && more) next.load(p, first);
        if (now.grad) {
            const AdamWTensor &c = p.tensors[now.tensor];
            const int n = now.n;
            const bool full = now.full;
            const int64_t at = now.at, block = at / ADAMW_BLOCK;
            float w[8], g[8], m[8], v[8];
            widen(now.p, HWR_F32, w);
            widen(now.g, p.dtype[now.tensor - p.tensor0], g);
            now.moments(m, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = __fmul_rn(g[j], k), old = BITS == 32 ? v[j] : __fmul_rn(v[j], v[j]);
                m[j] = __fadd_rn(__fmul_rn(m[j], p.b1), __fmul_rn(f, p.one_b1));
                v[j] = __fadd_rn(__fmul_rn(old, p.b2), __fmul_rn(__fmul_rn(f, f), p.one_b2));
            }
            if (BITS == 32) {
                put32((float *)c.m + at, m, n, full);
                put32((float *)c.v + at, v, n, full);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = BITS == 8 ? __fsqrt_rn(v[j]) : root(v[j]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float step = m[j] * by1 * reciprocal(fmaf(v[j], by2, p.eps));
                w[j] = fmaf(-rate, fmaf(p.decay, w[j], step), w[j]);
            }
            put32(c.param + at, w, n, full);
            if (c.copy) {
                if (c.copy_dtype == HWR_BF16) put16<HWR_BF16>(c.copy, at, w, n, full);
                else put16<HWR_F16>(c.copy, at, w, n, full);
            }
            if (BITS == 8) {
                const uint32_t tensor = mixed(key_t + (uint32_t)(now.tensor + 1) * 0x85157af5u);
                // (elements from 2^32 on: others' bits, turned)
                const uint32_t key = at >> 32 ? mixed(tensor ^ (uint32_t)(at >> 32)) : tensor;
                uint32_t random[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) random[j] = mixed((uint32_t)(at + j) * 0x9e3779b1u + key);
                if (n < 8)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j >= n) m[j] = v[j] = 0.f;
                put8(c.m, at, codes8<false>(m, c.m_scale + block, random, lane == 0 && n), n, full);
                put8(c.v, at, codes8<true>(v, c.v_scale + block, random, lane == 0 && n), n, full);
            }
        }
        if (BITS == 8) now = next;
        else if (more) now.load(p, first);
    }
    // the last block of the call to have read the step's number counts it up
    if (tid == 0 && atomicAdd(p.arrivals, 1u) == p.blocks - 1) {
        *p.arrivals = 0;
        if (!skip) *p.step = t;
    }
}

}  // namespace

// Many more blocks than run at a time, so that the GPU's ends are even; with 8-bit moments
// a block's own start costs more.  113 M elements, in blocks an SM: 32 bits 507 us with 3, 464
// with 24, 447 with 192; 8 bits (bf16 gradients and copies) 361, 337 and 374.
int adamw_grid(int chunks, int bits, int nsm) {
    const int64_t most = (int64_t)nsm * (bits == 8 ? 24 : 192);
    return chunks < 1 ? 1 : chunks < most ? chunks : (int)most;
}

cudaError_t launch_adamw(const AdamWStep &p, int bits, int grid, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(AW_THREADS);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return bits == 8 ? cudaLaunchKernelEx(&cfg, k_adamw<8>, p) : cudaLaunchKernelEx(&cfg, k_adamw<32>, p);
}

}  // namespace hwr
