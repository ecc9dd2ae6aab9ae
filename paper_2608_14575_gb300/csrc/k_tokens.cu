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
// Alternatives: 64-bit keys (the value's order above, the index's complement below: equal
// values go by the lowest index).  A block's first step has its threads' largest values,
// and from the few largest of each warp a bound that at least `top` values reach, and few
// more.  Each warp gathers the values that reach it in shared memory, and says what its few
// largest candidates are now, so that the bound rises without a barrier.  (Other warps may be
// ahead: what equals their bound is kept.)  Where candidates get too many a key's place is the
// number of larger ones, and the last of the best a bound of the warp's own: values of its
// later steps have higher indices, so those that only equal it have no place.  At the end a
// bound as in the first step, among the candidates, leaves few of them to be placed by the
// block.  (One list for the block, with barriers in each step: 512 rows of 131,072 bf16 logits
// with 20 alternatives 51.5 us for 48.5, 2,048 of 50,001 90.6 for 82.5.  With each warp's own
// bound alone 64 for 48.5.)
#include <type_traits>

#include "ops_internal.cuh"
#include "values.cuh"

namespace hwr {
namespace {

constexpr int TK_THREADS = 256, TK_WARPS = TK_THREADS / 32;
constexpr int TK_VECS = 4;             // 16-byte loads of a step
// Blocks of rows alone are smaller, so that more of them are at different stages of a row:
// 4,099 rows of 50,001 bf16 logits 77 us with 256 threads, 70 with 128 (5.9 TB/s); 2,048 in
// fp32 68 and 71, and 62 (6.6 TB/s) where a step is loaded ahead (bf16 71 so, fp16 67 for 68:
// not done).  Alternatives want few blocks, each of which finds a bound of its own: 64 rows
// of 131,072 with 20 take 18 us with 256 threads, 24 with 128.
__host__ __device__ constexpr int threads_of(bool top) { return top ? TK_THREADS : 128; }
// Blocks of rows with alternatives an SM: 3, which may use 80 registers, where all are there
// at once, else 4 (64 rows of 131,072 in bf16, 20 alternatives: 14.4 us with 3, 16.7 with 4;
// 512 rows 58 and 49).
constexpr int TK_FEW = 3, TK_LOT = 4;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FAR = -1e30f;
constexpr uint32_t ALL = 0xffffffffu;

// Within 2 units of the last place, 0 below 2^-126: an exp here is a term of a sum beside 1, or a
// probability, each of which has that much from its argument's roundings already.
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

constexpr int TK_READ = 32;                   // keys that are compared at a time
constexpr int TK_ROOM = 32 * 8 + 32;          // of a warp: a vector of each lane, beside the best
constexpr int TK_MANY = 64;                   // candidates of a warp that are sorted out
constexpr int TK_ALL = (TK_WARPS * TK_MANY > TOKEN_SPLITS * 32 ? TK_WARPS * TK_MANY : TOKEN_SPLITS * 32) + TK_READ;
constexpr uint32_t MASKED = 0x007fffffu;      // order_of(-inf)
static_assert(TK_ROOM % TK_READ == 0, "lists are filled up to whole reads");

// Keys of a warp's candidates, and of a block's.
struct alignas(16) Best {
    uint64_t key[TK_WARPS][TK_ROOM], kept[TK_WARPS][32], all[TK_ALL], sorted[32];
    uint32_t most[3][TK_WARPS];           // of the first step, now (raised), and of the candidates
    int offered[TK_WARPS];                // more than there is room for: some are missing
    int n;
};

// The least value that is above (equal: or at) the bound.
__device__ __forceinline__ float least_of(uint32_t bound, bool equal) { return value_of(bound + (equal ? 0 : 1)); }

// A thread's values at or above `least`, N from index i on, the largest of which is given,
// to its warp's candidates.  (Few threads have any, after the first steps.)
template <int N>
__device__ __forceinline__ void offer(Best &b, const float (&z)[N], float largest, uint32_t i, float least) {
    if (!(largest >= least)) return;
    const int warp = threadIdx.x >> 5;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) mine |= (uint32_t)(z[j] >= least) << j;
    int at = atomicAdd(&b.offered[warp], __popc(mine));
    // (one, nearly always)
#pragma unroll 1
    for (; mine; mine &= mine - 1, ++at) {
        const int j = __ffs(mine) - 1;
        float v = z[0];
#pragma unroll
        for (int k = 1; k < N; ++k) v = j == k ? z[k] : v;
        if (at < TK_ROOM) b.key[warp][at] = (uint64_t)order_of(v) << 32 | ~(i + j);
    }
}

// How many of n keys (filled up with zeros) are larger, as far as `top`.
__device__ __forceinline__ int place_of(uint64_t mine, const uint64_t *key, int n, int top) {
    int place = 0;
    for (int j = 0; j < n && place < top; j += TK_READ) {
        const ulonglong2 *o = (const ulonglong2 *)(key + j);
#pragma unroll
        for (int k = 0; k < TK_READ / 2; ++k) {
            const ulonglong2 v = o[k];
            place += (v.x > mine) + (v.y > mine);
        }
    }
    return place;
}

// A warp's best, left as its only candidates; the bound is the last one's value.
__device__ __noinline__ uint32_t squeeze(Best &b, int top, uint32_t bound) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t *key = b.key[warp], *kept = b.kept[warp];
    __syncwarp();
    const int n = min(b.offered[warp], TK_ROOM);
    kept[lane] = 0;
    if (n + lane < TK_ROOM) key[n + lane] = 0;
    __syncwarp();
    for (int i = lane; i < n; i += 32) {
        const uint64_t mine = key[i];
        const int place = place_of(mine, key, n, top);
        if (place < top) kept[place] = mine;
    }
    __syncwarp();
    key[lane] = kept[lane];
    if (lane == 0) b.offered[warp] = min(n, top);
    if (n >= top) bound = max(bound, (uint32_t)(kept[top - 1] >> 32));
    __syncwarp();
    return bound;
}

// The best of the block's keys, sorted (0: none).
__device__ __forceinline__ void settle(Best &b, int top) {
    __syncthreads();
    const int n = b.n;
    if (threadIdx.x < 32) b.sorted[threadIdx.x] = 0;
    if (threadIdx.x < TK_READ) b.all[n + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += TK_THREADS) {
        const uint64_t mine = b.all[i];
        const int place = place_of(mine, b.all, n, top);
        if (place < top && mine) b.sorted[place] = mine;
    }
    __syncthreads();
}

// A value that, in every warp, as many threads' keys reach as it takes for `top` in all: what
// this warp has to say.  (0: too few have one.)
__device__ __forceinline__ uint32_t most_of(uint32_t mine, int top) {
    const int lane = threadIdx.x & 31;
    uint32_t most = 0;
    for (int j = 0; j < (top + TK_WARPS - 1) / TK_WARPS; ++j) {
        most = __reduce_max_sync(ALL, mine);
        const uint32_t who = __ballot_sync(ALL, mine == most);
        if (lane == __ffs(who) - 1) mine = 0;
    }
    return most;
}
__device__ __forceinline__ uint32_t least_of_all(const uint32_t (&of)[TK_WARPS]) {
    uint32_t most = of[0];
#pragma unroll
    for (int w = 1; w < TK_WARPS; ++w) most = min(most, of[w]);
    return most;
}

// The largest of a lane's part of its warp's candidates, at most TK_MANY.
__device__ __forceinline__ uint32_t largest_of(const Best &b, int warp) {
    const int lane = threadIdx.x & 31, n = b.offered[warp];
    const uint32_t *high = (const uint32_t *)b.key[warp] + 1;
    return max(lane < n ? high[2 * lane] : 0u, lane + 32 < n ? high[2 * lane + 64] : 0u);
}

// The warps' candidates that can be among the best, sorted.
__device__ __forceinline__ void gather(Best &b, int top) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncwarp();
    if (b.offered[warp] > TK_MANY) squeeze(b, top, 0);
    const int n = b.offered[warp];
    const uint64_t one = lane < n ? b.key[warp][lane] : 0, two = lane + 32 < n ? b.key[warp][lane + 32] : 0;
    const uint32_t most = most_of((uint32_t)((one > two ? one : two) >> 32), top);
    if (lane == 0) b.most[2][warp] = most;
    __syncthreads();
    const uint32_t bound = least_of_all(b.most[2]);
    if (one && (uint32_t)(one >> 32) >= bound) b.all[atomicAdd(&b.n, 1)] = one;
    if (two && (uint32_t)(two >> 32) >= bound) b.all[atomicAdd(&b.n, 1)] = two;
    settle(b, top);
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
    // nothing but -inf (the maximum leaves NaN out, the sums do not)
    const bool empty = a.m == -INFINITY && a.s == 0.f;
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

template <int DT, bool TOP, int BLOCKS>
__global__ void __launch_bounds__(threads_of(TOP), BLOCKS)
k_token_rows(const __grid_constant__ TokenRows p) {
    constexpr int N = Vec<DT>::N, TH = threads_of(TOP);
    constexpr bool AHEAD = !TOP && DT == HWR_F32;
    __shared__ Sums sums[TH / 32];
    __shared__ bool last;
    __shared__ typename std::conditional<TOP, Best, int>::type shared_best;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, top = p.top;
    const int64_t row = blockIdx.x / (uint32_t)p.splits;
    const int piece = blockIdx.x % (uint32_t)p.splits;
    if constexpr (TOP) {
        if (tid == 0) shared_best.n = 0;
        if (lane == 0) shared_best.offered[warp] = 0;
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const void *base = row_at(p.logits, row, p.ld, DT);
    const Cut<DT> cut(base, p.vocab);
    const int per = (cut.vecs + p.splits - 1) / p.splits;
    const int v0 = min(piece * per, cut.vecs), v1 = min(v0 + per, cut.vecs);
    const uint4 *vecs = (const uint4 *)((const char *)base + (DT == HWR_F32 ? 4 : 2) * cut.head);
    const int token = p.token ? p.token[row] : -1;
    const bool has = (uint32_t)token < (uint32_t)p.vocab;
    const float z_token = has && tid == 0 ? Vec<DT>::load(base, token) : 0.f;

    uint32_t bound = MASKED;              // of my warp: values above it are candidates
    float m = -INFINITY;
    Two s(0.f, 0.f), d(0.f, 0.f);
    const auto raise = [&](float to) {
        const float by = fmaxf(m - to, FAR), f = exp2_fast(by * LOG2E);
        d = Two(f, f) * fma2(Two(by, by), s, d);
        s = s * Two(f, f);
        m = to;
    };
    const auto term = [&](float a, float b, float base) {
        (Two(a, b) + Two(-base, -base)).get(a, b);
        const Two x(max_nan(a, FAR), max_nan(b, FAR));
        (x * Two(LOG2E, LOG2E)).get(a, b);
        const Two e(exp2_fast(a), exp2_fast(b));
        d = fma2(e, x, d);
        return e;
    };
    // one value a lane of the first warp (indices of lanes without one may pass 2^31, the most
    // that a row has)
    const auto single = [&](uint32_t i, bool valid, float least) {
        float z[1] = {valid ? Vec<DT>::load(base, (int)i) : -INFINITY};
        if (z[0] > m) raise(z[0]);
        s = s + term(z[0], -INFINITY, m == -INFINITY ? 0.f : m);
        if constexpr (TOP) {
            if (valid) offer<1>(shared_best, z, z[0], i, least);
        }
    };
    __syncwarp();
    if (warp == 0 && piece == 0 && cut.head) single(lane, lane < cut.head, least_of(MASKED, false));
    // (32-bit values: a step's are on their way while the one before is taken)
    uint4 next[TK_VECS];
    const auto fetch = [&](int b) {
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            const int i = b + k * TH + tid;
            next[k] = Vec<DT>::lowest();
            if (i < v1) next[k] = __ldg(vecs + i);
        }
    };
    if (AHEAD) fetch(v0);
    for (int b = v0; b < v1; b += TH * TK_VECS) {
        uint4 u[TK_VECS];
        if (!AHEAD) fetch(b);
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) u[k] = next[k];
        if (AHEAD) fetch(b + TH * TK_VECS);
        float z[TK_VECS][N], largest[TK_VECS], mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            largest[k] = Vec<DT>::largest(u[k]);
            mx = fmaxf(mx, largest[k]);
            Vec<DT>::unpack(u[k], z[k]);
        }
        if (mx > m) raise(mx);
        const float base_m = m == -INFINITY ? 0.f : m;
        // A step's terms by halves, so that the largest, near 1, meets five others' sums, not up
        // to sixteen terms: log probabilities and entropies of 4,099 rows of 50,001 are 6.5e-8 off
        // 64 bits, one after the other 8.8e-8 (69.4 us for 69.9).  With alternatives by pairs
        // (registers: 2,048 rows 83.4 us, by halves 85.2, one after the other 82.9).
        Two sum[TK_VECS];
#pragma unroll
        for (int k = 0; k < TK_VECS; ++k) {
            Two e[N / 2];
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                e[j] = term(z[k][2 * j], z[k][2 * j + 1], base_m);
                if (TOP && j % 2) s = s + (e[j - j % 2] + e[j]);
            }
            if (!TOP) sum[k] = N == 8 ? (e[0] + e[1]) + (e[N / 2 - 2] + e[N / 2 - 1]) : e[0] + e[1];
        }
        if (!TOP) s = s + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
        if constexpr (TOP) {
            Best &best = shared_best;
            const bool first = b == v0;
            volatile uint32_t *said = best.most[1];
            if (first) {
                const uint32_t most = most_of(order_of(mx), top);
                if (lane == 0) best.most[0][warp] = said[warp] = most;
                __syncthreads();
            }
            // what `top` values reach, of any index (other warps may be ahead)
            const uint32_t floor = __reduce_min_sync(ALL, lane < TK_WARPS ? said[lane] : ~0u);
            const float any = floor > MASKED ? value_of(floor) : -INFINITY;
            // (vectors beyond the last are -inf, below any `least`)
            const uint32_t at = (uint32_t)cut.head + (uint32_t)(b + tid) * N;
            const float least = fmaxf(least_of(bound, false), any);
            if (__any_sync(ALL, mx >= least)) {
                const int before = best.offered[warp];
                __syncwarp();
                if (mx >= least)
#pragma unroll
                    for (int k = 0; k < TK_VECS; ++k) offer<N>(best, z[k], largest[k], at + k * TH * N, least);
                __syncwarp();
                const int n = best.offered[warp];
                if (n > TK_ROOM) {
                    // not all of them found room: once more, a vector at a time
                    __syncwarp();
                    if (lane == 0) best.offered[warp] = before;
                    bound = squeeze(best, top, bound);
#pragma unroll
                    for (int k = 0; k < TK_VECS; ++k) {
                        offer<N>(best, z[k], largest[k], at + k * TH * N, fmaxf(least_of(bound, false), any));
                        bound = squeeze(best, top, bound);
                    }
                } else if (n > TK_MANY) {
                    bound = squeeze(best, top, bound);
                }
                if (b + TH * TK_VECS < v1) {
                    const uint32_t most = most_of(largest_of(best, warp), top);
                    if (lane == 0 && most > said[warp]) said[warp] = most;
                }
            }
            // (not `floor`: a warp ahead may have raised it by values of higher indices than mine)
            if (first) bound = max(bound, least_of_all(best.most[0]));
        }
    }
    if (warp == 0 && piece == p.splits - 1) {
        const uint32_t at = (uint32_t)(cut.head + cut.vecs * N) + lane;
        float least = 0.f;
        if constexpr (TOP) least = least_of(bound, false);
        single(at, at < (uint32_t)p.vocab, least);
    }

    Sums a = {m, 0.f, 0.f};
    {
        float x, y;
        s.get(x, y);
        a.s = x + y;
        d.get(x, y);
        a.d = x + y;
    }
    for (int k = 16; k; k /= 2)
        a.join(__shfl_xor_sync(ALL, a.m, k), __shfl_xor_sync(ALL, a.s, k), __shfl_xor_sync(ALL, a.d, k));
    if (lane == 0) sums[warp] = a;
    if constexpr (TOP) gather(shared_best, top);
    else __syncthreads();
    a = sums[0];
    for (int w = 1; w < TH / 32; ++w) a.join(sums[w].m, sums[w].s, sums[w].d);
    if (p.splits > 1) {
        TokenPart *part = p.part + row * p.splits;
        if (warp == 0) {
            if (lane == 0) {
                part[piece].m = a.m;
                part[piece].s = a.s;
                part[piece].d = a.d;
            }
            if constexpr (TOP) part[piece].key[lane] = shared_best.sorted[lane];
            __threadfence();
            __syncwarp();
            if (lane == 0) {
                last = atomicAdd(p.arrivals + row, 1u) == (uint32_t)p.splits - 1;
                if (last) p.arrivals[row] = 0;
                __threadfence();
            }
        }
        __syncthreads();
        if (!last) return;
        a = {-INFINITY, 0.f, 0.f};
        // (all read at once, joined in their order)
        Sums mine = a;
        if (lane < p.splits) mine = {__ldcg(&part[lane].m), __ldcg(&part[lane].s), __ldcg(&part[lane].d)};
        for (int i = 0; i < p.splits; ++i)
            a.join(__shfl_sync(ALL, mine.m, i), __shfl_sync(ALL, mine.s, i), __shfl_sync(ALL, mine.d, i));
        if constexpr (TOP) {
            for (int i = tid; i < p.splits * top; i += TH) shared_best.all[i] = __ldcg(&part[i / top].key[i % top]);
            if (tid == 0) shared_best.n = p.splits * top;
            settle(shared_best, top);
        }
    }
    if (warp) return;
    uint64_t key = 0;
    if constexpr (TOP) {
        // fewer numbers than alternatives: the first masked values follow, then NaN
        uint64_t *sorted = shared_best.sorted;
        int found = __popc(__ballot_sync(ALL, lane < top && sorted[lane] != 0));
        for (int kind = 0; kind < 2; ++kind)
            for (int64_t i = 0; found < top && i < p.vocab; i += 32) {
                const float z = i + lane < p.vocab ? Vec<DT>::load(base, (int)(i + lane)) : 0.f;
                const bool is = i + lane < p.vocab && (kind ? z != z : z == -INFINITY);
                const uint32_t who = __ballot_sync(ALL, is);
                const int at = found + __popc(who & ((1u << lane) - 1));
                if (is && at < top) sorted[at] = (uint64_t)order_of(z) << 32 | (uint32_t)~(uint32_t)(i + lane);
                found += __popc(who);
            }
        __syncwarp();
        key = sorted[lane];
    }
    finish<TOP>(p, row, a, key, z_token, has, lane);
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
    const bool empty = m == -INFINITY;    // (beside NaN log S is NaN, and all of the gradient)
    const float a = p.da && (uint32_t)token < (uint32_t)p.vocab && !empty ? p.da[row] : 0.f;
    const float b = p.db ? p.db[row] : 0.f;
    if (empty) m = 0.f;
    // Where b is so large that its product with a distance (down to where q is 0, 127 at most)
    // could overflow, 2^7 q and 2^-7 of a and b: 0 times infinity would make a masked logit's
    // gradient NaN.  (b times q first costs no choice, but 133 us for the training step's 130.)
    const bool large = fabsf(b) > 0x1p120f;
    const float up = large ? 7.f : 0.f, down = large ? 0x1p-7f : 1.f, sa = a * down, sb = b * down;
    auto grad = [&](float z, int at) {
        const float lq = max_nan((z - m) - ls, -127.f), q = exp2_fast(fmaf(lq, LOG2E, up));
        const float g = -q * fmaf(sb, lq + h, sa);
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
    for (int64_t i = piece * TK_THREADS + tid; i < left; i += p.splits * TK_THREADS) {
        const int at = (int)(i < head ? i : i + vecs * N);
        Vec<DT>::store(out, at, grad(Vec<DT>::load(in, at), at));
    }
}

}  // namespace

// Pieces of a row: enough blocks for the GPU where rows are few, none shorter than a
// step of a block.
static int row_pieces(int rows, int vocab, int size, int threads, int blocks, int most) {
    const int step = threads * TK_VECS * 16;
    const int64_t steps = ((int64_t)vocab * size + step - 1) / step;
    int64_t n = blocks / rows;
    if (n > steps) n = steps;
    return (int)(n < 1 ? 1 : n > most ? most : n);
}

int token_splits(int rows, int vocab, hwr_dtype dtype, bool top, int nsm) {
    return row_pieces(rows, vocab, dtype == HWR_F32 ? 4 : 2, threads_of(top), (top ? TK_FEW : 8) * nsm, TOKEN_SPLITS);
}

static cudaLaunchConfig_t early(int64_t grid, int threads, cudaStream_t s, cudaLaunchAttribute *at) {
    cudaLaunchConfig_t cfg = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cfg;
}

template <int DT>
static cudaError_t rows_of(const TokenRows &p, int nsm, const cudaLaunchConfig_t &cfg) {
    constexpr int blocks = DT == HWR_F32 ? 8 : DT == HWR_BF16 ? 10 : 9;
    if (!p.top) return cudaLaunchKernelEx(&cfg, k_token_rows<DT, false, blocks>, p);
    return (int64_t)p.rows * p.splits <= TK_FEW * nsm ? cudaLaunchKernelEx(&cfg, k_token_rows<DT, true, TK_FEW>, p)
                                                      : cudaLaunchKernelEx(&cfg, k_token_rows<DT, true, TK_LOT>, p);
}

cudaError_t launch_token_rows(const TokenRows &p, hwr_dtype dtype, int nsm, cudaStream_t s) {
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early((int64_t)p.rows * p.splits, threads_of(p.top > 0), s, at);
    return dtype == HWR_F32    ? rows_of<HWR_F32>(p, nsm, cfg)
           : dtype == HWR_BF16 ? rows_of<HWR_BF16>(p, nsm, cfg)
                               : rows_of<HWR_F16>(p, nsm, cfg);
}

cudaError_t launch_token_grad(TokenGrad p, hwr_dtype dtype, int nsm, cudaStream_t s) {
    p.splits = row_pieces(p.rows, p.vocab, dtype == HWR_F32 ? 4 : 2, TK_THREADS, 8 * nsm, 1024);
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = early((int64_t)p.rows * p.splits, TK_THREADS, s, at);
    return dtype == HWR_F32    ? cudaLaunchKernelEx(&cfg, k_token_grad<HWR_F32>, p)
           : dtype == HWR_BF16 ? cudaLaunchKernelEx(&cfg, k_token_grad<HWR_BF16>, p)
                               : cudaLaunchKernelEx(&cfg, k_token_grad<HWR_F16>, p);
}

}  // namespace hwr
