// Log probabilities of given tokens, entropies and best alternatives over rows of
// logits, and their gradient.
//
// A row z is read once, with a running maximum m and the sums S of exp(z - m) and D
// of exp(z - m) (z - m), both scaled by exp(m - m') where a larger maximum m' comes up:
//   logprob[v] = (z[v] - m) - log S,   entropy = log S - D / S.
// A block takes a row, or where rows are few one of its `splits` pieces, which the
// last block to finish joins in their order.  Every value is fp32; a value 10^30 below
// the maximum (a masked one's -inf among them) counts as exp = 0 times a finite
// distance, so that it adds nothing, not NaN.
//
// Alternatives: a warp keeps its best ones sorted, one a lane, as 64-bit keys (the
// value's order above, the index's complement below: equal values go by the lowest
// index).  Values come in the order of their indices from one step of a warp to the
// next, so a step in which no value is above the warp's last alternative has none to
// offer, and costs one vote.
#include "ops_internal.cuh"
#include "values.cuh"

namespace hwr {
namespace {

constexpr int TK_THREADS = 256, TK_WARPS = TK_THREADS / 32;
constexpr int TK_VECS = 4;             // 16-byte loads of a step
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FAR = -1e30f;
constexpr uint32_t ALL = 0xffffffffu;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// max(a, b), NaN where one of them is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

struct Sums {
    float m, s, d;
    __device__ __forceinline__ void raise(float to) {       // to > m
        const float by = fmaxf(m - to, FAR), f = exp2_fast(by * LOG2E);
        d = f * (d + by * s);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void join(float om, float os, float od) {
        const float to = fmaxf(m, om);
        const float a = fmaxf(m - to, FAR), b = fmaxf(om - to, FAR);
        const float fa = m == to ? 1.f : exp2_fast(a * LOG2E), fb = om == to ? 1.f : exp2_fast(b * LOG2E);
        d = (m == to ? d : fa * (d + a * s)) + (om == to ? od : fb * (od + b * os));
        s = s * fa + os * fb;
        m = to;
    }
};

// Order of a value among keys: larger ones above, -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return z != z ? 0u : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order >> 31 ? order ^ 0x80000000u : ~order);      // (0: a NaN)
}

constexpr uint32_t MASKED = 0x007fffffu;      // order_of(-inf)

// A warp's sorted list: lane i has the i-th best key (0: none yet).
struct Best {
    uint64_t key, last;       // mine; that of the last alternative
    __device__ __forceinline__ void insert(uint64_t k, int top, int lane) {
        const int at = __popc(__ballot_sync(ALL, key > k));
        const uint64_t up = __shfl_up_sync(ALL, key, 1);
        if (lane >= at) key = lane == at ? k : up;
        last = __shfl_sync(ALL, key, top - 1);
    }
    // The lanes' candidates.
    __device__ __forceinline__ void offer(uint64_t k, bool valid, int top, int lane) {
        for (;;) {
            const uint32_t who = __ballot_sync(ALL, valid && k > last);
            if (!who) return;
            const int from = __ffs(who) - 1;
            insert(__shfl_sync(ALL, k, from), top, lane);
            if (lane == from) valid = false;
        }
    }
    // Joined with another sorted list: the largest 32 of both form a bitonic
    // sequence, which five exchanges sort.
    __device__ __forceinline__ void join(uint64_t other, int lane) {
        const uint64_t turned = __shfl_sync(ALL, other, 31 - lane);
        key = key > turned ? key : turned;
#pragma unroll
        for (int d = 16; d; d /= 2) {
            const uint64_t o = __shfl_xor_sync(ALL, key, d);
            const bool lower = lane & d;
            key = (key > o) != lower ? key : o;
        }
    }
};

// The order below which none of a step's values can be among the `top` best, before the
// list is full: the top-th largest of the lanes' maxima.
__device__ __forceinline__ uint32_t floor_of(uint32_t mine, int top, int lane) {
    int rank = 0;
    for (int i = 0; i < 32; ++i) {
        const uint32_t o = __shfl_sync(ALL, mine, i);
        rank += o > mine || (o == mine && i < lane);
    }
    const uint32_t who = __ballot_sync(ALL, rank == top - 1);
    return __shfl_sync(ALL, mine, __ffs(who) - 1);
}

// Where a row's 16-byte vectors begin, and how many there are.
template <int DT>
struct Cut {
    int head, vecs;
    __device__ __forceinline__ Cut(const void *row, int n) {
        constexpr int size = DT == HWR_F32 ? 4 : 2;
        head = (int)((0 - (uintptr_t)row) & 15) / size;
        if (head > n) head = n;
        vecs = (n - head) / Vec<DT>::N;
    }
};

__device__ __forceinline__ const char *row_at(const void *p, int64_t row, int64_t ld, int dt) {
    return (const char *)p + row * ld * (dt == HWR_F32 ? 4 : 2);
}

// What the row's sums say, by lane 0 of a warp; the alternatives by all of it.
template <bool TOP>
__device__ __forceinline__ void finish(const TokenRows &p, int64_t row, const Sums &a, uint64_t key, float z, bool has,
                                       int lane) {
    const bool empty = a.m == -INFINITY;              // nothing but -inf
    const float ls = empty ? -INFINITY : logf(a.s);
    if (lane == 0) {
        p.logprob[row] = !has ? 0.f : empty ? z : (z - a.m) - ls;
        p.entropy[row] = empty ? 0.f : ls - a.d / a.s;
        p.stats[2 * row] = a.m;
        p.stats[2 * row + 1] = empty ? 0.f : ls;
    }
    if (TOP && lane < p.top) {
        const float v = value_of((uint32_t)(key >> 32));
        p.top_token[row * p.top + lane] = (int32_t)~(uint32_t)key;
        p.top_logprob[row * p.top + lane] = empty ? v : (v - a.m) - ls;
    }
}

template <int DT, bool TOP>
__global__ void __launch_bounds__(TK_THREADS)
k_token_rows(const __grid_constant__ TokenRows p) {
    constexpr int N = Vec<DT>::N;
    __shared__ Sums sums[TK_WARPS];
    __shared__ uint64_t keys[TOP ? TK_WARPS : 1][32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, top = p.top;
    const int64_t row = blockIdx.x / (uint32_t)p.splits;
    const int piece = blockIdx.x % (uint32_t)p.splits;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const void *base = row_at(p.logits, row, p.ld, DT);
    const Cut<DT> cut(base, p.vocab);
    const int per = (cut.vecs + p.splits - 1) / p.splits;
    const int v0 = min(piece * per, cut.vecs), v1 = min(v0 + per, cut.vecs);
    const uint4 *vecs = (const uint4 *)((const char *)base + (DT == HWR_F32 ? 4 : 2) * cut.head);
    const int token = p.token ? p.token[row] : -1;
    const bool has = (uint32_t)token < (uint32_t)p.vocab;
    const float z_token = has ? Vec<DT>::load(base, token) : 0.f;

    Sums a = {-INFINITY, 0.f, 0.f};
    Best best = {0, 0};
    auto add = [&](float z, float m) {
        const float d = max_nan(z - m, FAR), e = exp2_fast(d * LOG2E);
        a.s += e;
        a.d = fmaf(e, d, a.d);
    };
    // one value a lane
    auto single = [&](int i, bool valid) {
        const float z = valid ? Vec<DT>::load(base, i) : -INFINITY;
        if (z > a.m) a.raise(z);
        if (valid) add(z, a.m == -INFINITY ? 0.f : a.m);
        if (TOP) best.offer((uint64_t)order_of(z) << 32 | (uint32_t)~i, valid, top, lane);
    };
    if (warp == 0 && piece == 0 && cut.head) single(lane, lane < cut.head);
    for (int b = v0; b < v1; b += TK_THREADS * TK_VECS) {
        uint4 u[TK_VECS];
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            const int i = b + k * TK_THREADS + tid;
            if (i < v1) u[k] = __ldcs(vecs + i);
            else u[k] = Vec<DT>::lowest();
        }
        float z[TK_VECS][N], mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            Vec<DT>::unpack(u[k], z[k]);
#pragma unroll
            for (int j = 0; j < N; ++j) mx = fmaxf(mx, z[k][j]);
        }
        if (mx > a.m) a.raise(mx);
        const float m = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) add(z[k][j], m);
        if (TOP) {
            const uint32_t mine = order_of(mx);
            uint64_t least = 0;
            if (best.last == 0) {
                const uint32_t f = floor_of(mine, top, lane);
                least = f > MASKED ? (uint64_t)f << 32 : 0;      // (lanes without a number have -inf)
            }
            if (__any_sync(ALL, mine > (uint32_t)(best.last >> 32) || best.last == 0)) {
#pragma unroll 1
                for (int k = 0; k < TK_VECS; ++k) {
                    const int i = b + k * TK_THREADS + tid;
#pragma unroll 1
                    for (int j = 0; j < N; ++j) {
                        const bool valid = i < v1;
                        const int at = cut.head + i * N + j;
                        const float v = valid ? Vec<DT>::load(base, at) : 0.f;
                        const uint64_t key = (uint64_t)order_of(v) << 32 | (uint32_t)~at;
                        best.offer(key, valid && key >= least, top, lane);
                    }
                }
            }
        }
    }
    if (warp == 0 && piece == p.splits - 1) {
        const int at = cut.head + cut.vecs * N + lane;
        single(at, at < p.vocab);
    }

    for (int d = 16; d; d /= 2)
        a.join(__shfl_xor_sync(ALL, a.m, d), __shfl_xor_sync(ALL, a.s, d), __shfl_xor_sync(ALL, a.d, d));
    if (lane == 0) sums[warp] = a;
    if (TOP) keys[warp][lane] = lane < top ? best.key : 0;
    __syncthreads();
    if (warp) return;
    a = sums[0];
    for (int w = 1; w < TK_WARPS; ++w) a.join(sums[w].m, sums[w].s, sums[w].d);
    if (TOP)
        for (int w = 1; w < TK_WARPS; ++w) best.join(keys[w][lane], lane);
    if (p.splits > 1) {
        TokenPart *part = p.part + row * p.splits;
        if (lane == 0) {
            part[piece].m = a.m;
            part[piece].s = a.s;
            part[piece].d = a.d;
        }
        if (TOP) part[piece].key[lane] = best.key;
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        if (lane == 0) before = atomicAdd(p.arrivals + row, 1u);
        if (__shfl_sync(ALL, before, 0) != (uint32_t)p.splits - 1) return;
        if (lane == 0) p.arrivals[row] = 0;
        __threadfence();
        a = {-INFINITY, 0.f, 0.f};
        best.key = 0;
        for (int i = 0; i < p.splits; ++i) {
            a.join(__ldcg(&part[i].m), __ldcg(&part[i].s), __ldcg(&part[i].d));
            if (TOP) best.join(__ldcg(&part[i].key[lane]), lane);
        }
    }
    finish<TOP>(p, row, a, best.key, z_token, has, lane);
}

// dz = a (1[token] - q) - b q (log q + entropy), q = exp((z - m) - log S): bound by
// HBM, a read and a write of every value.
template <int DT>
__global__ void __launch_bounds__(TK_THREADS)
k_token_grad(const __grid_constant__ TokenGrad p) {
    constexpr int N = Vec<DT>::N;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / (uint32_t)p.splits;
    const int piece = blockIdx.x % (uint32_t)p.splits;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const void *in = row_at(p.logits, row, p.ld, DT);
    void *out = (void *)row_at(p.out, row, p.out_ld, DT);
    const int token = p.token ? p.token[row] : -1;
    float m = p.stats[2 * row];
    const float ls = p.stats[2 * row + 1], h = p.entropy[row];
    const bool empty = m == -INFINITY;
    const float a = p.da && (uint32_t)token < (uint32_t)p.vocab && !empty ? p.da[row] : 0.f;
    const float b = p.db ? p.db[row] : 0.f;
    if (empty) m = 0.f;
    auto grad = [&](float z, int at) {
        const float lq = max_nan((z - m) - ls, FAR), q = exp2_fast(lq * LOG2E);
        const float g = -q * fmaf(b, lq + h, a);
        return at == token ? g + a : g;
    };
    // (vectors where both rows begin alike, else value by value)
    const bool alike = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    const Cut<DT> cut(in, p.vocab);
    const int vecs = alike ? cut.vecs : 0, head = alike ? cut.head : 0;
    const int per = (vecs + p.splits - 1) / p.splits;
    const int v0 = min(piece * per, vecs), v1 = min(v0 + per, vecs);
    const uint4 *src = (const uint4 *)((const char *)in + (DT == HWR_F32 ? 4 : 2) * head);
    uint4 *dst = (uint4 *)((char *)out + (DT == HWR_F32 ? 4 : 2) * head);
    for (int i0 = v0 + tid; i0 < v1; i0 += TK_THREADS * TK_VECS) {
        uint4 u[TK_VECS];
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k)
            if (i0 + k * TK_THREADS < v1) u[k] = __ldcs(src + i0 + k * TK_THREADS);
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            const int i = i0 + k * TK_THREADS;
            if (i >= v1) break;
            float z[N];
            Vec<DT>::unpack(u[k], z);
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = grad(z[j], head + i * N + j);
            __stcs(dst + i, Vec<DT>::pack(z));
        }
    }
    // what the vectors leave: before them and after them
    const int left = p.vocab - vecs * N;
    for (int i = piece * TK_THREADS + tid; i < left; i += p.splits * TK_THREADS) {
        const int at = i < head ? i : i + vecs * N;
        Vec<DT>::store(out, at, grad(Vec<DT>::load(in, at), at));
    }
}

}  // namespace

// Pieces of a row: enough blocks for the GPU where rows are few, none shorter than a
// step of a block.
static int row_pieces(int rows, int vocab, int size, int blocks, int most) {
    const int64_t steps = ((int64_t)vocab * size + TK_THREADS * TK_VECS * 16 - 1) / (TK_THREADS * TK_VECS * 16);
    int64_t n = (blocks + rows - 1) / rows;
    if (n > steps) n = steps;
    return (int)(n < 1 ? 1 : n > most ? most : n);
}

int token_splits(int rows, int vocab, hwr_dtype dtype, int nsm) {
    return row_pieces(rows, vocab, dtype == HWR_F32 ? 4 : 2, 2 * nsm, TOKEN_SPLITS);
}

static cudaLaunchConfig_t early(int64_t grid, cudaStream_t s, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(TK_THREADS);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

template <int DT>
static cudaError_t rows_of(const TokenRows &p, const cudaLaunchConfig_t &cfg) {
    return p.top ? cudaLaunchKernelEx(&cfg, k_token_rows<DT, true>, p) : cudaLaunchKernelEx(&cfg, k_token_rows<DT, false>, p);
}

cudaError_t launch_token_rows(const TokenRows &p, hwr_dtype dtype, cudaStream_t s) {
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early((int64_t)p.rows * p.splits, s, at);
    return dtype == HWR_F32    ? rows_of<HWR_F32>(p, cfg)
           : dtype == HWR_BF16 ? rows_of<HWR_BF16>(p, cfg)
                               : rows_of<HWR_F16>(p, cfg);
}

cudaError_t launch_token_grad(TokenGrad p, hwr_dtype dtype, int nsm, cudaStream_t s) {
    p.splits = row_pieces(p.rows, p.vocab, dtype == HWR_F32 ? 4 : 2, 8 * nsm, 1024);
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early((int64_t)p.rows * p.splits, s, at);
    return dtype == HWR_F32    ? cudaLaunchKernelEx(&cfg, k_token_grad<HWR_F32>, p)
           : dtype == HWR_BF16 ? cudaLaunchKernelEx(&cfg, k_token_grad<HWR_BF16>, p)
                               : cudaLaunchKernelEx(&cfg, k_token_grad<HWR_F16>, p);
}

}  // namespace hwr
