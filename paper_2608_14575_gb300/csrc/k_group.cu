// Products with ragged groups of rows on the tensor cores, fp32 accumulation in
// TMEM.  One kernel serves
//   grouped products   out[t] = W[g(t)] x[t], or W[g(t)]^T x[t] (W MN-major);
//   shared products    out[t] = W x[t] + a low-rank term of t's group;
//   weight gradients   out[g] = sum over the group's rows of l[t] r[t]^T.
//
// A pair of CTAs (cta_group::2) computes a tile of 256 x up to 256: per 64-deep
// stage each CTA holds 128 rows of the A side and half of the B side, which
// halves the B bytes that every SM takes from L2.  W comes by TMA, and so do
// the rows of x once they lie by place; or, without a copy, each is picked by its
// index with 16-byte cp.async (65,536 x 1024 x 2048 over 64 groups: 258 us picked,
// 259 with the copy, 650 with TMA's row gather in an early form; 8,191 rows of a
// shared product of 4,096 x 4,096 with adapters of rank 64: 248 picked, 230 with the
// copy, as its rows are the A side).
//
// In a grouped product the rows of x are the B side, whose extent moves in
// steps of 16: a group's last rows cost no whole tile, and a few rows of a
// decode step cost 16.  In a shared product they are the A side, because the
// low-rank extension must keep groups apart: after the contraction, for each
// group with rows in the tile, the tile's rows of u (two 16-bit terms a value)
// times the group's [n][rank] matrix are accumulated with the MMA's row mask
// into that group's rows only; no value of one group's matrix ever meets
// another group's rows.  The terms are bf16 whatever the rows' type: they hold 16
// bits at any magnitude, where fp16's would overflow above 65,504 and lose bits
// below 2^-3; an fp16 matrix is then taken as two bf16 terms too (exactly), one
// after the other.  In the gradients of fp16 rows an inner product meets fp16 rows,
// so its terms are fp16, scaled by a power of two of each group's own.
//
// The iterations (stages of the contraction) of all tiles are dealt evenly:
// whole tiles first, one to a pair a round, then the tiles of the last rounds
// as one line of iterations cut into equal pieces.  The pieces of a tile leave
// fp32 partials; the last to arrive adds them in the order of the contraction,
// so the result does not depend on who that is.
#include "ops_internal.cuh"
#include "umma_pair.cuh"

#include <stddef.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace hwr {
namespace {

using namespace umma;

// warps 0-3 epilogue, 4-7 epilogue too (sorted rows) or picking rows, 8 TMA, 9
// MMA (even CTA), 10 dealing the pieces, 11 announcing picked rows
constexpr int THREADS = 384;
constexpr int PIECES = 4;          // pieces dealt ahead
constexpr int GATHER_WARPS = 4;
constexpr int A_BYTES = 128 * GP_BK * 2;
constexpr int MAX_STAGES = 24;
constexpr int SMEM_MAX = 227 * 1024;
constexpr int MIN_PIECE = 6 * GP_BK;   // columns of the smallest piece of a cut tile
// Joining a tile's pieces, in blocks of 64 columns of the contraction (about 0.3 us
// each): leaving, arriving and the last fences (less for the inner products), and
// what the last to arrive reads, for each piece and 64 columns of it, with eight
// warps or four.  From 110 shapes with all last tiles cut and with none.  (256 rows
// through 4,096 x 1,024: 17 us whole, 37 cut; through 8,192 columns 52 whole, 44 cut.)
constexpr float JOIN_FIXED = 20.f, JOIN_LOW = 8.f, JOIN_PIECE_8 = 1.8f, JOIN_PIECE_4 = 2.7f;
constexpr int BAND = 8;            // row tiles (32: 666 us for 8,192^3, 8: 635 us)
constexpr int WRITE_COST = 4;      // iterations that writing a gradient's tile counts for

constexpr int OUT_PITCH = 64;      // bytes of a staged output row (32 columns)
constexpr int OUT_BYTES = 32 * OUT_PITCH;   // of a warp
// Staged rows keep their four 16-byte units in an order of their own, so that
// neither writing a row a lane nor reading a row by 4 lanes meets a bank twice.
__device__ __forceinline__ int staged_at(int row, int unit) {
    return row * OUT_PITCH + ((unit ^ ((row >> 1) & 3)) << 4);
}

// What a kernel is compiled for (the epilogue's registers are those of its kind).
// The last two are launched with two products (a product's parameters at an
// address, not in the instructions, cost a single one 4 of 25 us).
enum : int { K_GROUPED = 0, K_SHARED = 1, K_PACK = 2, K_GRAD = 3, K_LOW = 4, K_PACKS = 5, KINDS = 6 };

struct Work {
    int g, xt, ot;        // group; tile of rows (gradients: of result rows); tile of columns
    int k0, k1, ki;       // iterations of this piece, and of the tile
    int c0, c1;           // first and last pair with a piece of the tile
    int first, count;     // places of the tile (gradients: of the group)
    int e0, e1;           // steps of the extension that go with the piece
};

template <int N>
struct Launch {
    GroupCall call[N];
};

// Shared memory behind the stages: this, then the group tables.
struct Tables {
    // per stage: full (even CTA: both CTAs' bytes, and their word on picked rows),
    // rows (this CTA's picked rows have landed), empty
    uint64_t full[MAX_STAGES], rowsf[MAX_STAGES], empty[MAX_STAGES], accf[2], acce[2], done;
    alignas(16) uint8_t out[8][OUT_BYTES];   // epilogue staging, a warp each
    int32_t rows[GP_TILE];               // the tile's rows of the output (epilogue)
    // pieces dealt, for the warps that work on them
    Work work[PIECES];
    uint64_t dealt[PIECES], taken[PIECES];
    uint32_t tmem;
    int abort_f;
    // epilogue: its piece and whether there is one, the accumulator is there, this
    // piece writes the tile
    Work mine;
    int go, ready, last;
    // group tables: ng groups of the tiles, and the extension's
    int ng;
    int nseg;            // groups of the extension that have rows
    int64_t *iter0;      // [ng + 1] first iteration of each group (gradients)
    int32_t *offs;       // [ng + 1] first place of each group, clamped
    int32_t *tile0;      // [ng + 1] first tile of each group (rows products)
    int32_t *eoffs;      // [groups + 1] first place of each of the extension's groups
    int32_t *seg;        // [nseg] its groups that have rows
};

static_assert(OUT_PITCH % 16 == 0 && OUT_BYTES % 16 == 0 && offsetof(Tables, out) % 16 == 0 && sizeof(Tables) % 16 == 0,
              "staged rows are read and written 16 bytes at a time");

// A group's matrix in an extension stage of one CTA: 32 ranks of blocks of 64
// columns (MN-major), or rows of 32 or, with a small rank, 16 ranks.
__host__ __device__ inline int ext_bytes(const GroupProduct &p) {      // (of one term)
    return p.dense_mn ? (p.bn / 2 + 63) / 64 * 4096 : p.bn / 2 * (p.rank <= 16 ? 32 : 64);
}

__host__ __device__ inline int ext_terms(const GroupProduct &p) { return p.f16 ? 2 : 1; }

__host__ __device__ inline int table_bytes(const GroupProduct &p) {
    const int g = p.plan.groups + 1;
    return (int)sizeof(Tables) + (p.mode == GP_WGRAD ? g * 12 : p.shared ? g * 8 + 16 : g * 8);
}

// atomicAdd that orders, across the GPU, what came before it and what comes after.
__device__ __forceinline__ uint32_t add_acq_rel(uint32_t *p, uint32_t v) {
    uint32_t old;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
}

// Bounded wait for MMAs that were issued, without flags.
__device__ __forceinline__ void drain(uint64_t *bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity))
        if (clock64() - t0 > WAIT_CYCLES) return;
}

// Time for copies in flight to land, where a barrier cannot tell.
__device__ __forceinline__ void linger() {
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000) __nanosleep(1000);     // about 10 ms
}

__host__ __device__ inline int up16(int v) { return (v + 15) & ~15; }

// A place in the ring of stages (a division a stage would cost what an MMA does).
struct Ring {
    int s = 0, stages;
    uint32_t ph = 0, n = 0;       // phase, steps in all
    __device__ explicit Ring(int stages_) : stages(stages_) {}
    __device__ void step() {
        ++n;
        if (++s == stages) {
            s = 0;
            ph ^= 1;
        }
    }
};

// a * b / c; 32-bit where that holds (a 64-bit division costs some 100 instructions)
__device__ __forceinline__ int64_t mul_div(int64_t a, int b, int c) {
    const uint64_t v = (uint64_t)a * (uint32_t)b;
    if (v >> 32) return (int64_t)(v / (uint32_t)c);
    return (uint32_t)v / (uint32_t)c;
}
__device__ __forceinline__ int64_t div_small(int64_t a, int64_t b) {
    if ((a | b) >> 32) return a / b;
    return (uint32_t)a / (uint32_t)b;
}

// The groups with rows in a tile, as places in the list of those with any.
__device__ __forceinline__ void ext_groups(const Tables &t, const Work &w, int &s0, int &s1) {
    int lo = 0, hi = t.nseg;
    while (lo < hi) {                    // the first that ends behind the tile's first place
        const int m = (lo + hi) >> 1;
        if (t.eoffs[t.seg[m] + 1] > w.first) hi = m;
        else lo = m + 1;
    }
    s0 = lo;
    hi = t.nseg;
    while (lo < hi) {                    // the first that begins behind its last
        const int m = (lo + hi) >> 1;
        if (t.eoffs[t.seg[m]] >= w.first + w.count) hi = m;
        else lo = m + 1;
    }
    s1 = lo;
}

// Steps of rank of each group of the extension.
__device__ __forceinline__ int ext_steps(const GroupProduct &p) {
    return p.rank <= GP_RC ? 1 : (p.rank + GP_RC - 1) / GP_RC;
}

template <class T>
__device__ __forceinline__ int find(const T *v, int n, T x) {   // last g with v[g] <= x
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (v[m] <= x) lo = m;
        else hi = m - 1;
    }
    return lo;
}

// Iterations that a gradient's tile counts for: its own, or what writing it takes.
__device__ __forceinline__ int grad_cost(const Tables &t, int g) {
    return max(WRITE_COST, (max(0, t.offs[g + 1] - t.offs[g]) + GP_BK - 1) / GP_BK);
}

// How the iterations of all tiles are dealt: the first dp tiles whole, one to a
// pair a round, the others as one line cut into `cutters` equal pieces.
struct Walk {
    const GroupProduct &p;
    const Tables &t;
    int me, pairs, dp, kiters, cutters, next_tile;
    int64_t base, rest;       // where the line begins (gradients), and its length
    int64_t pos, end;         // of this pair's piece of it, what is left

    __device__ Walk(const GroupProduct &p_, const Tables &t_) : p(p_), t(t_) {
        const bool grad = p.mode == GP_WGRAD, shared = p.rank > 0;
        const int per = p.mtiles * p.ntiles, tiles = grad ? t.ng * per : t.tile0[t.ng];
        me = next_tile = (blockIdx.x >> 1) - p.pair0;
        pairs = p.pairs;
        const int deep = GP_BK * p.kk;
        kiters = (p.k + deep - 1) / deep;
        dp = tiles >= 2 * pairs ? (tiles / pairs - 1) * pairs : 0;
        base = 0;
        if (grad) {
            const int g = dp / per;           // (dp < tiles: the group exists)
            base = t.iter0[g] + (int64_t)(dp - g * per) * grad_cost(t, g);
            rest = t.iter0[t.ng] - base;
        } else {
            rest = (int64_t)(tiles - dp) * kiters;
        }
        const int last = tiles - dp, rounds = (last + pairs - 1) / pairs;
        // Cut only where evening out the last rounds saves more than joining costs:
        // whole rounds of the average tile against its share of the line.
        const float work = (float)rest * p.kk + (shared && tiles ? __fdividef((float)ext_work() * last, tiles) : 0.f);
        const float fixed = p.mode == GP_ROWS && !p.shared ? JOIN_LOW : JOIN_FIXED;
        bool cut = work * rounds > fixed * last;
        cutters = 1;
        if (cut) {
            // Pieces of a tile that take the least time, its blocks / pieces + what a
            // piece costs the join * pieces; whole pieces of each tile where the pairs
            // suffice for two and more (a pair's piece of two tiles is joined twice).
            const float piece = (p.sorted ? JOIN_PIECE_8 : JOIN_PIECE_4) / 64 * join_cols(tiles);
            const float tile = __fdividef(work, last), best = max(1.f, sqrtf(__fdividef(tile, piece)));
            const int most = (int)min((int64_t)pairs, max(div_small(rest, max(1, MIN_PIECE / deep)), (int64_t)last));
            cutters = max(1, (int)min((float)most, best * last));
            cutters = cutters >= 2 * last ? cutters / last * last : max(1, most);
            const float pieces = max(2.f, __fdividef(cutters, last));
            cut = tile * rounds - __fdividef(work, cutters) > fixed + piece * (pieces + 1.f);
        }
        if (!cut) {
            dp = tiles;
            rest = 0;
            cutters = 1;
        }
        pos = end = 0;
        if (me < cutters) {
            pos = mul_div(rest, me, cutters);
            end = mul_div(rest, me + 1, cutters);
        }
    }
    // Columns of a tile's partials (of a few rows as many as take the same time).
    __device__ float join_cols(int tiles) const {
        if (p.mode == GP_GROUPED) return max(1.f, min((float)GP_TILE, __fdividef((float)t.offs[t.ng] * p.ntiles, max(1, tiles))));
        return p.mode == GP_ROWS && p.shared ? p.bn * max(1, min(t.offs[1], 128)) * (1.f / 128) : p.bn;
    }
    // The extension's steps in all of a shared product's tiles, about a block each.
    __device__ int64_t ext_work() const { return (int64_t)t.nseg * ext_steps(p) * ext_terms(p) * p.ntiles; }
    __device__ bool next(Work &w) {
        const bool grad = p.mode == GP_WGRAD;
        w.e0 = 0;
        w.e1 = INT32_MAX;
        while (true) {
            int tile = next_tile, cost = kiters;
            int64_t start = 0;       // of the tile, on the line
            const bool whole = tile < dp;
            if (whole) {
                next_tile += pairs;
            } else {
                if (pos >= end) return false;
                if (grad) {
                    const int g = find(t.iter0, t.ng, base + pos);
                    cost = grad_cost(t, g);
                    const int local = (int)div_small(base + pos - t.iter0[g], cost);
                    start = t.iter0[g] + (int64_t)local * cost - base;
                    tile = g * p.mtiles * p.ntiles + local;
                } else {
                    const int i = (int)div_small(pos, kiters);
                    start = (int64_t)i * kiters;
                    tile = dp + i;
                }
            }
            if (grad) {
                const int per = p.mtiles * p.ntiles, local = tile % per;
                w.g = tile / per;
                w.first = t.offs[w.g];
                w.count = max(0, t.offs[w.g + 1] - w.first);
                w.ki = max(1, (w.count + GP_BK - 1) / GP_BK);
                w.ot = local / p.mtiles;
                w.xt = local - w.ot * p.mtiles;
            } else {
                w.g = find(t.tile0, t.ng, tile);
                const int local = tile - t.tile0[w.g];
                const int n = t.offs[w.g + 1] - t.offs[w.g], xts = (n + GP_TILE - 1) / GP_TILE;
                // bands of BAND row tiles, column by column: the pairs at work are
                // about as many columns as rows of tiles, so that each tile of W and
                // of x that L2 serves is wanted by several at a time
                const int band = local / (BAND * p.ntiles), in = local - band * BAND * p.ntiles;
                const int h = min(BAND, xts - band * BAND);
                w.ot = in / h;
                w.xt = band * BAND + (in - w.ot * h);
                // rows on the B side: tiles of about equal extent
                const int width = p.mode == GP_GROUPED && xts <= 8 ? up16((n + xts - 1) / xts) : GP_TILE;
                w.first = t.offs[w.g] + w.xt * width;
                w.count = min(width, n - w.xt * width);
                w.ki = kiters;
            }
            if (whole) {
                w.k0 = 0;
                w.k1 = w.ki;
                w.c0 = w.c1 = me;
                return true;
            }
            const int64_t stop = start + cost < end ? start + cost : end;
            w.k0 = (int)(pos - start);
            w.k1 = min((int)(stop - start), w.ki);
            pos = stop;
            if (w.k0 >= w.k1) continue;       // (of a gradient: nothing but what writing counts for)
            // the pairs with the tile's first and last iteration
            w.c0 = (int)div_small((start + 1) * cutters - 1, rest);
            w.c1 = (int)div_small((start + w.ki) * cutters - 1, rest);
            if (p.rank && w.c0 != w.c1) {
                // a piece takes its share of the extension
                int s0, s1;
                ext_groups(t, w, s0, s1);
                const int all = (s1 - s0) * ext_steps(p);
                w.e0 = (int)mul_div(all, w.k0, w.ki);
                w.e1 = (int)mul_div(all, w.k1, w.ki);
            }
            return true;
        }
    }
};

// Warp 10's thread: deals the pair's pieces to the warps of its CTA, a few
// ahead of them.  (Every warp for itself, they took 3 to 5 us before the first
// load, in code fetched five times, and a bubble a tile.)
__device__ void deal(const GroupProduct &p, Tables &t) {
    Walk walk(p, t);
    Work w;
    for (int i = 0;; ++i) {
        const bool more = walk.next(w);
        const int s = i % PIECES;
        if (!mbar_wait(&t.taken[s], ((i / PIECES) & 1) ^ 1, &t.abort_f, p.status)) return;
        if (!more) w.g = -1;
        t.work[s] = w;
        mbar_arrive(&t.dealt[s]);
        if (!more) return;
    }
}

// The pieces as a warp takes them: all its lanes, or (ALONE) its first lane.
template <bool ALONE>
struct Pieces {
    const GroupProduct &p;
    Tables &t;
    int i = 0;
    __device__ Pieces(const GroupProduct &p_, Tables &t_) : p(p_), t(t_) {}
    __device__ bool next(Work &w) {
        const int s = i % PIECES;
        bool ok = mbar_wait(&t.dealt[s], (i / PIECES) & 1, &t.abort_f, p.status);
        if (!ALONE) ok = __all_sync(0xffffffffu, ok);
        if (!ok) return false;
        w = t.work[s];
        if (!ALONE) __syncwarp();
        if (ALONE || (threadIdx.x & 31) == 0) mbar_arrive(&t.taken[s]);
        ++i;
        return w.g >= 0;
    }
};

// The extension's stages of a piece, out of the tile's: for each group with rows
// in the tile, the rank in steps of GP_RC.  Where one step holds the whole rank,
// the tile's rows of u are the same for all groups, and a stage takes up to
// p.ext_pack groups' matrices beside them.
struct Ext {
    const GroupProduct &p;
    const Tables &t;
    int steps, i, end;            // steps of a group; this step (of all groups'), the piece's last
    int s, r;                     // its group's place in the list, its step of the rank
    __device__ Ext(const GroupProduct &p_, const Tables &t_, const Work &w) : p(p_), t(t_) {
        int s0, s1;
        ext_groups(t, w, s0, s1);
        steps = ext_steps(p);
        const int n = (s1 - s0) * steps;
        i = min(n, w.e0);
        end = min(n, w.e1);
        s = steps == 1 ? i : i / steps;
        r = i - s * steps;
        s += s0;
    }
    __device__ bool more() const { return i < end; }
    __device__ int here() const { return min(p.ext_pack, end - i); }       // groups of this stage
    __device__ int group(int q) const { return t.seg[s + q]; }
    __device__ int rank0() const { return r * GP_RC; }
    __device__ void step() {
        i += p.ext_pack;
        if (steps == 1) {
            s += p.ext_pack;
        } else if (++r == steps) {
            r = 0;
            ++s;
        }
    }
};

// 32 bits, the first n of them set (n at most 32; none below 0).
__device__ __forceinline__ uint32_t first_bits(int n) {
    uint32_t v;
    asm("shl.b32 %0, 0xffffffff, %1;" : "=r"(v) : "r"(max(n, 0)));     // (a shift by 32 or more gives 0)
    return ~v;
}

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

// A warp's 32 staged rows of 32 values to where they belong, V values an access
// (what the result's rows are aligned to): 32 / V lanes write 64 bytes of a row.
// to(j): where row j's values go (null: nowhere); left: how many of them count.
template <int V, class To>
__device__ __forceinline__ void flush(const uint8_t *stage, int left, To to) {
    constexpr int LANES = 32 / V, STEPS = 32 / V;
    const int lane = threadIdx.x & 31, e = lane % LANES * V;
#pragma unroll
    for (int i0 = 0; i0 < STEPS; i0 += 4) {
        uint16_t *dst[4];
        uint4 d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = (i0 + i) * V + lane / LANES;
            const uint8_t *src = stage + staged_at(j, e >> 3) + (e & 7) * 2;
            if (V == 8) d[i] = *(const uint4 *)src;
            if (V == 4) *(uint2 *)&d[i] = *(const uint2 *)src;
            if (V == 2) d[i].x = *(const uint32_t *)src;
            if (V == 1) d[i].x = *(const uint16_t *)src;
            dst[i] = to(j);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!dst[i]) continue;
            uint16_t *o = dst[i] + e;
            if (e + V <= left) {
                if (V == 8) *(uint4 *)o = d[i];
                if (V == 4) *(uint2 *)o = *(const uint2 *)&d[i];
                if (V == 2) *(uint32_t *)o = d[i].x;
                if (V == 1) *o = (uint16_t)d[i].x;
            } else if (V > 1) {
                const uint16_t *src =
                    (const uint16_t *)(stage + staged_at((i0 + i) * V + lane / LANES, e >> 3) + (e & 7) * 2);
                for (int k = 0; e + k < left; ++k) o[k] = src[k];
            }
        }
    }
}

// Index of the row at a place of the order, -1 where there is none.
__device__ __forceinline__ int row_at(const GroupProduct &p, int place) {
    const int r = p.plan.order[place];
    return (uint32_t)r < (uint32_t)p.plan.rows ? r : -1;
}

// ---- picked rows ------------------------------------------------------------------
//
// A stage's rows are 64 columns K-major in the 128-byte swizzle: the 16-byte
// unit c of smem row r lies at unit c ^ (r mod 8).  Eight lanes copy one row's
// 128 bytes.

__device__ void pick_rows(const GroupProduct &p, Tables &t, uint8_t *sm, int rank) {
    Work w;
    Ring at(p.stages);
    bool ok = true;
    const int tid = threadIdx.x & 127, sub = tid >> 3, c = tid & 7;
    const bool grouped = p.mode == GP_GROUPED;
    const uint32_t dst = (grouped ? p.b_off : 0) + sub * 128 + ((c ^ (sub & 7)) << 4);
    const uint32_t block = grouped ? p.b_sub : p.a_sub;
    Pieces<false> pieces(p, t);
    while (ok && pieces.next(w)) {
        // this CTA's rows of the tile: its 128 of the A side, or its half of the B side
        const int half = grouped ? up16(w.count) >> 1 : 128;
        const int mine = min(half, w.count - rank * half);
        const uint16_t *row[8];     // 16 rows apart: 2,048 bytes of smem
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = sub + i * 16, r = q < mine ? row_at(p, w.first + rank * half + q) : -1;
            row[i] = r < 0 ? nullptr : p.x + r * p.x_ld;
        }
        for (int kb = w.k0; kb < w.k1; ++kb, at.step()) {
            ok = mbar_wait(&t.empty[at.s], at.ph ^ 1, &t.abort_f, p.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const uint32_t st = smem_u32(sm + (size_t)at.s * p.stage_bytes) + dst;
            for (int j = 0; j < p.kk; ++j) {
                const int col = (kb * p.kk + j) * GP_BK + c * 8, left = p.k - col;
                const uint32_t bytes = left >= 8 ? 16 : left > 0 ? left * 2 : 0;   // beyond: zeros
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (row[i]) cp_async16(st + j * block + i * 2048, row[i] + (bytes ? col : 0), bytes);
            }
            cp_async_arrive(&t.rowsf[at.s]);
        }
        // of the extension's stages only the arrival is due
        if (p.rank && ok)
            for (Ext e(p, t, w); e.more(); e.step(), at.step()) {
                ok = mbar_wait(&t.empty[at.s], at.ph ^ 1, &t.abort_f, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                cp_async_arrive(&t.rowsf[at.s]);
            }
    }
    cp_async_wait_all();
}

// ---- the kernel -------------------------------------------------------------------

template <bool F16, int KIND>
__global__ void __launch_bounds__(THREADS, 1) __cluster_dims__(2, 1, 1)
k_group(const __grid_constant__ Launch<KIND >= K_LOW ? 2 : 1> launch) {
    constexpr int CALLS = KIND >= K_LOW ? 2 : 1;
    const GroupCall &call = launch.call[CALLS > 1 && (int)(blockIdx.x >> 1) >= launch.call[CALLS - 1].p.pair0];
    const GroupProduct &p = call.p;
    const GroupMaps &maps = call.maps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Tables &t = *(Tables *)(sm + (size_t)p.stages * p.stage_bytes);
    volatile int *abort_f = &t.abort_f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    constexpr bool grad = KIND == K_GRAD || KIND == K_LOW;
    constexpr bool grouped = KIND == K_GROUPED, shared = KIND == K_SHARED, low = KIND == K_LOW;
    constexpr bool pack = KIND == K_PACK || KIND == K_PACKS;
    constexpr int TERMS = F16 ? 2 : 1;      // of the extension's matrices
    constexpr int CS = GP_TILE;      // TMEM columns of one of the two accumulators

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&t.full[s], p.sorted ? 1 : 3);
            mbar_init(&t.rowsf[s], 32 * GATHER_WARPS);
            mbar_init(&t.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&t.accf[b], 1);
            mbar_init(&t.acce[b], p.sorted ? 16 : 8);
        }
        mbar_init(&t.done, 1);
        for (int i = 0; i < PIECES; ++i) {
            mbar_init(&t.dealt[i], 1);
            // the epilogue and TMA, the picking warps and their word, MMA
            mbar_init(&t.taken[i], (p.sorted ? 2 : 3 + GATHER_WARPS) + (rank == 0));
        }
        t.abort_f = 0;
        t.ng = shared ? 1 : p.plan.groups;
        // the tables of 8-byte values come first
        t.iter0 = (int64_t *)(&t + 1);
        t.offs = (int32_t *)(&t + 1) + (grad ? 2 * (t.ng + 1) : 0);
        t.tile0 = t.offs + t.ng + 1;
        t.eoffs = t.tile0 + t.ng + 1;
        t.seg = t.eoffs + p.plan.groups + 1;
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc_pair(&t.tmem, 2 * CS);
        tmem_relinquish_pair();
    }
    if (warp == 8 && lane == 0) {
        if (!grad) tma_prefetch_desc(&maps.w);
        if (p.sorted) tma_prefetch_desc(&maps.x);
        if (shared) tma_prefetch_desc(&maps.eb);
    }
    // everything above overlaps the kernel before; everything below may read
    // what it wrote
    grid_launch_dependents();
    grid_dependency_wait();
    __syncthreads();
    // Group tables.  Offsets are the caller's: clamped here, so that no value
    // of theirs reads or writes outside the arrays.
    {
        int32_t *dst = shared ? t.eoffs : t.offs;
        for (int i = threadIdx.x; i <= p.plan.groups; i += THREADS) {
            const int v = p.plan.offsets[i];
            dst[i] = v < 0 ? 0 : v > p.plan.places ? p.plan.places : v;
        }
        if (shared && threadIdx.x == 0) {
            const int v = p.plan.padded ? p.plan.offsets[p.plan.groups + 1] : p.plan.rows;
            t.offs[0] = 0;
            t.offs[1] = v < 0 ? 0 : v > p.plan.places ? p.plan.places : v;
        }
    }
    __syncthreads();
    if (warp == 0) {
        // first tile (or iteration) of each group: a running sum over 32 groups at a time
        int64_t run = 0;
        for (int g0 = 0; g0 < t.ng; g0 += 32) {
            const int g = g0 + lane;
            int64_t v = 0;
            if (g < t.ng) {
                const int n = max(0, t.offs[g + 1] - t.offs[g]);
                // (an empty group's zero gradient is written too: see grad_cost)
                v = grad ? (int64_t)p.mtiles * p.ntiles * max(WRITE_COST, (n + GP_BK - 1) / GP_BK)
                         : (int64_t)((n + GP_TILE - 1) / GP_TILE) * p.ntiles;
            }
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int64_t o = __shfl_up_sync(0xffffffffu, v, d);
                if (lane >= d) v += o;
            }
            if (g < t.ng) {
                if (grad) t.iter0[g + 1] = run + v;
                else t.tile0[g + 1] = (int)(run + v);
            }
            run += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) {
            if (grad) t.iter0[0] = 0;
            else t.tile0[0] = 0;
        }
    }
    if (shared && warp == 1) {
        int n = 0;
        for (int g0 = 0; g0 < p.plan.groups; g0 += 32) {
            const int g = g0 + lane;
            const bool any = g < p.plan.groups && t.eoffs[g] < t.eoffs[g + 1];
            const uint32_t v = __ballot_sync(0xffffffffu, any);
            if (any) t.seg[n + __popc(v & ((1u << lane) - 1))] = g;
            n += __popc(v);
        }
        if (lane == 0) t.nseg = n;
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();          // the other CTA's barriers and TMEM are there
    tc_fence_after();
    const uint32_t tmem = t.tmem;

    if (warp == 10) {
        if (lane == 0) deal(p, t);
        __syncwarp();
    } else if (warp == 11) {
        // Tells the even CTA that a stage's picked rows are here.  They are copied
        // by threads: the first fence makes them visible to the tensor cores' proxy, the
        // second to the even CTA's MMA thread.  (A picking thread cannot: its fence
        // would wait for all of its copies in flight, 1.75 us a stage.  The MMA
        // thread spent 0.2 us a stage on it.)
        if (lane == 0 && !p.sorted) {
            const uint32_t full0 = smem_of(&t.full[0], 0);
            Ring at(p.stages);
            bool ok = true;
            Work w;
            auto pass = [&]() {
                ok = mbar_wait(&t.rowsf[at.s], at.ph, abort_f, p.status);
                if (!ok) return false;
                fence_proxy_async_smem();
                fence_release_smem();
                mbar_arrive_cluster(full0 + at.s * 8);
                at.step();
                return true;
            };
            Pieces<true> pieces(p, t);
            while (ok && pieces.next(w)) {
                for (int kb = w.k0; kb < w.k1; ++kb)
                    if (!pass()) break;
                if (shared && ok)
                    for (Ext e(p, t, w); e.more(); e.step())
                        if (!pass()) break;
            }
        }
        __syncwarp();
    } else if (!p.sorted && warp >= 4 && warp < 8) {
        pick_rows(p, t, sm, rank);
    } else if (warp == 8) {
        // TMA: W (each CTA its 128 rows of the A side or its half of the B side),
        // sorted rows, the extension's operands, a gradient's two sides.  All bytes
        // count on the even CTA's barrier.
        if (lane == 0) {
            Ring at(p.stages);
            bool ok = true;
            Work w;
            const int half = grouped ? 128 : p.bn >> 1;           // of the dense operand
            const int blocks = (half + 63) >> 6;                  // MN-major blocks of 64
            const uint32_t dbytes = p.dense_mn ? blocks * 8192 : half * 128;
            const uint32_t ebytes = ext_bytes(p);
            const uint32_t dside = grouped ? 0 : p.b_off, xside = grouped ? p.b_off : 0;
            const uint32_t full0 = smem_of(&t.full[0], 0);
            auto claim = [&](uint32_t bytes) {
                ok = mbar_wait(&t.empty[at.s], at.ph ^ 1, abort_f, p.status);
                if (ok && rank == 0) mbar_arrive_expect_tx(&t.full[at.s], bytes);
                return ok;
            };
            Pieces<true> pieces(p, t);
            while (!p.test_stall && ok && pieces.next(w)) {
                if (grad) {
                    const int l0 = w.xt * GP_TILE + rank * 128, r0 = w.ot * p.bn + rank * half;
                    for (int kb = w.k0; kb < w.k1; ++kb, at.step()) {
                        if (!claim(2 * (2 + blocks) * 8192)) break;
                        uint8_t *st = sm + (size_t)at.s * p.stage_bytes;
                        const int row = w.first + kb * GP_BK;
                        for (int b = 0; b < 2; ++b)
                            tma_load_3d_pair(st + b * 8192, &maps.x, full0 + at.s * 8, l0 + b * 64, row, 0);
                        for (int b = 0; b < blocks; ++b)
                            tma_load_3d_pair(st + A_BYTES + b * 8192, &maps.w, full0 + at.s * 8, r0 + b * 64, row, 0);
                    }
                    continue;
                }
                const int o0 = w.ot * (grouped ? GP_TILE : p.bn) + rank * half;
                // boxes of rows: this CTA's, and both CTAs'
                const int xhalf = grouped ? up16(w.count) >> 1 : 128;
                const int x0 = w.first + rank * xhalf;
                const int c0 = min(xhalf, w.count), c1 = max(0, w.count - xhalf);
                const int boxes = ((rank ? c1 : c0) + GP_ROW_BOX - 1) / GP_ROW_BOX;
                const uint32_t xbytes = ((c0 + GP_ROW_BOX - 1) / GP_ROW_BOX + (c1 + GP_ROW_BOX - 1) / GP_ROW_BOX) *
                                        GP_ROW_BOX * 128;
                for (int kb = w.k0; kb < w.k1; ++kb, at.step()) {
                    if (!claim(2 * p.kk * dbytes + (p.sorted ? xbytes : 0))) break;
                    uint8_t *st = sm + (size_t)at.s * p.stage_bytes;
                    // (sorted rows: kk = 1)
                    if (p.sorted && boxes == 4)
                        tma_load_3d_pair(st + xside, &maps.xx, full0 + at.s * 8, kb * GP_BK, x0, 0);
                    else if (p.sorted)
                        for (int b = 0; b < boxes; ++b)
                            tma_load_3d_pair(st + xside + b * GP_ROW_BOX * 128, &maps.x, full0 + at.s * 8, kb * GP_BK,
                                             x0 + b * GP_ROW_BOX, 0);
                    auto dense = [&](uint8_t *dst, int k) {
                        if (p.dense_mn)
                            for (int b = 0; b < blocks; ++b)
                                tma_load_3d_pair(dst + b * 8192, &maps.w, full0 + at.s * 8, o0 + b * 64, k, w.g);
                        else
                            tma_load_3d_pair(dst, &maps.w, full0 + at.s * 8, k, o0, w.g);
                    };
                    dense(st + dside, kb * p.kk * GP_BK);
                    for (int j = 1; j < p.kk; ++j)
                        dense(st + dside + j * (grouped ? p.a_sub : p.b_sub), (kb * p.kk + j) * GP_BK);
                }
                if (shared && ok)
                    for (Ext e(p, t, w); e.more(); e.step(), at.step()) {
                        const int n = e.here(), r0 = e.rank0();
                        if (!claim(2 * n * TERMS * ebytes + xbytes)) break;
                        uint8_t *st = sm + (size_t)at.s * p.stage_bytes;
                        for (int b = 0; b < boxes; ++b)
                            tma_load_3d_pair(st + b * GP_ROW_BOX * 128, &maps.u, full0 + at.s * 8, r0 * 2,
                                             x0 + b * GP_ROW_BOX, 0);
                        for (int q = 0; q < n * TERMS; ++q) {
                            uint8_t *eb = st + p.b_off + q * ebytes;
                            const int g = e.group(q / TERMS), term = q % TERMS;
                            if (p.dense_mn)
                                for (int b = 0; b < blocks; ++b)
                                    tma_load_3d_pair(eb + b * 4096, &maps.eb, full0 + at.s * 8, o0 + b * 64,
                                                     r0 * TERMS + term * GP_RC, g);
                            else
                                tma_load_3d_pair(eb, &maps.eb, full0 + at.s * 8,
                                                 r0 * TERMS + term * (p.rank <= 16 ? 16 : GP_RC), o0, g);
                        }
                    }
            }
            // every stage loaded is waited for by the MMA thread, unless it gave up
            if (!ok || *abort_f) linger();
        }
        __syncwarp();
    } else if (warp == 9) {
        if (lane == 0 && rank == 0) {
            uint32_t lt = 0;
            Ring at(p.stages);
            bool ok = true;
            Work w;
            const bool a_mn = grad || (grouped && p.dense_mn);
            const bool b_mn = grad || (!grad && !grouped && p.dense_mn);
            // both CTAs' operands have landed
            auto stage_ready = [&]() {
                if (p.sorted) {
                    if (!mbar_wait(&t.full[at.s], at.ph, abort_f, p.status)) return false;
                } else {
                    if (!mbar_wait<true>(&t.full[at.s], at.ph, abort_f, p.status)) return false;
                    fence_acquire_smem();
                }
                tc_fence_after();
                return true;
            };
            // per 16-deep MMA: 16 rows of 128 bytes further (MN-major), or 32 bytes (K-major)
            const uint32_t astep = a_mn ? 2048 >> 4 : 2, bstep = b_mn ? 2048 >> 4 : 2;
            Pieces<true> pieces(p, t);
            for (; ok && pieces.next(w); ++lt) {
                const int b = lt & 1;
                const uint32_t d = tmem + b * CS;
                const int N = grouped ? up16(w.count) : p.bn;
                const uint32_t idesc = idesc_16bit(GP_TILE, N, F16, a_mn, b_mn);
                ok = mbar_wait<true>(&t.acce[b], ((lt >> 1) & 1) ^ 1, abort_f, p.status);
                if (!ok) break;
                tc_fence_after();
                for (int kb = w.k0; kb < w.k1; ++kb, at.step()) {
                    ok = stage_ready();
                    if (!ok) break;
                    const uint32_t st = smem_u32(sm + (size_t)at.s * p.stage_bytes);
                    // a gradient's last stage: whole 16s of rows, the group's padding
                    // among them (zeros), nothing of the next group
                    const int steps = grad ? min(4, max(1, (w.count - kb * GP_BK + 15) >> 4)) : 4;
                    auto block = [&](uint32_t a, uint32_t bb, bool add) {
                        const uint64_t ad = sdesc(a, 8192, 1024, 2), bd = sdesc(bb, 8192, 1024, 2);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < steps) mma_pair(d, ad + astep * k, bd + bstep * k, idesc, add || k);
                    };
                    block(st, st + p.b_off, kb > w.k0);
                    for (int j = 1; j < p.kk; ++j) block(st + j * p.a_sub, st + p.b_off + j * p.b_sub, true);
                    mma_commit_pair(&t.empty[at.s]);
                }
                if (!ok) break;
                if (shared) {
                    const uint32_t eidesc = idesc_16bit(GP_TILE, p.bn, false, false, p.dense_mn), ebytes = ext_bytes(p);
                    const uint64_t bdesc0 = p.dense_mn ? sdesc(0, 4096, 1024, 2)
                                            : p.rank <= 16 ? sdesc(0, 0, 256, 6) : sdesc(0, 0, 512, 4);
                    for (Ext e(p, t, w); e.more(); e.step(), at.step()) {
                        ok = stage_ready();
                        if (!ok) break;
                        const uint32_t st = smem_u32(sm + (size_t)at.s * p.stage_bytes);
                        const uint64_t ad = sdesc(st, 0, 1024, 2);
                        const int steps = min(GP_RC, p.rank - e.rank0()) > 16 ? 2 : 1;
                        uint64_t bd = bdesc0 + ((st + p.b_off) >> 4);
                        int g = e.group(0), a = t.eoffs[g], z = t.eoffs[g + 1];
                        for (int q = 0, n = e.here(); q < n; ++q) {
                            // rows [a, z) take part.  Without branches, and the next
                            // group's fetched ahead: one thread issues all (64
                            // adapters, 200 rows: 44 us against 55)
                            uint32_t off[8];
                            a -= w.first;
                            z = min(z - w.first, w.count);
#pragma unroll
                            for (int i = 0; i < 8; ++i) off[i] = ~first_bits(z - 32 * i) | first_bits(a - 32 * i);
                            if (q + 1 < n) {
                                g = e.group(q + 1);
                                a = t.eoffs[g];
                                z = t.eoffs[g + 1];
                            }
#pragma unroll
                            for (int term = 0; term < TERMS; ++term) {
                                for (int k = 0; k < steps; ++k) {
                                    const uint64_t bk = bd + (p.dense_mn ? (2048 >> 4) * k : 2 * k);
                                    mma_pair_rows(d, ad + 2 * k, bk, eidesc, off);
                                    mma_pair_rows(d, ad + 4 + 2 * k, bk, eidesc, off);
                                }
                                bd += ebytes >> 4;
                            }
                        }
                        mma_commit_pair(&t.empty[at.s]);
                    }
                    if (!ok) break;
                }
                mma_commit_pair(&t.accf[b]);
            }
            mma_commit_pair(&t.done);
            drain(&t.done, 0);
        }
        __syncwarp();
    } else {
        // epilogue: thread = TMEM lane = row of the A side; with eight warps, two
        // take every other 32 columns of the same rows
        const int row = threadIdx.x & 127, quad = warp & 3, half = warp >> 2;
        const int halves = p.sorted ? 2 : 1, threads = 128 * halves;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t acce0 = smem_of(&t.acce[0], 0);
        uint16_t *const out0 = (uint16_t *)p.out;
        uint8_t *const stage = t.out[warp];
        if (grouped) {
            // rows without a group: zeros
            const int total = p.plan.padded ? p.plan.offsets[p.plan.groups + 1] : p.plan.rows;
            for (int64_t pos = (int64_t)t.offs[t.ng] + blockIdx.x * (4 * halves) + warp; pos < min(total, p.plan.places);
                 pos += (int64_t)gridDim.x * (4 * halves)) {
                const int r = row_at(p, (int)pos);
                if (r < 0) continue;
                uint16_t *dst = out0 + (int64_t)r * p.ld;
                const bool wide = p.vec == 8;
                if (wide)
                    for (int j = lane * 8; j + 8 <= p.n; j += 256) *(uint4 *)(dst + j) = make_uint4(0, 0, 0, 0);
                for (int j = (wide ? p.n & ~7 : 0) + lane; j < p.n; j += 32) dst[j] = 0;
            }
        }
        uint32_t lt = 0;
        Work w;
        Pieces<false> pieces(p, t);
        for (;; ++lt) {
            // one warp waits for all, here and for the accumulator: they go on, or
            // give up, together
            if (warp == 0) {
                const bool more = pieces.next(w);
                if (lane == 0) {
                    t.go = more;
                    t.mine = w;
                }
            }
            named_bar_sync(1, threads);
            if (!*(volatile int *)&t.go) break;
            w = t.mine;
            const int b = lt & 1;
            int nrows;                 // rows of the A side that count
            int cols;                  // columns that count
            if (grad) {
                nrows = min(128, p.m - w.xt * GP_TILE - (int)rank * 128);
                cols = min(p.bn, p.n - w.ot * p.bn);
            } else if (grouped) {
                nrows = min(128, p.n - w.ot * GP_TILE - (int)rank * 128);
                cols = w.count;
                for (int i = threadIdx.x; i < w.count; i += threads) t.rows[i] = row_at(p, w.first + i);
            } else {
                nrows = min(128, w.count - (int)rank * 128);
                cols = min(p.bn, p.n - w.ot * p.bn);
                if (half == 0 && row < nrows) t.rows[row] = row_at(p, w.first + rank * 128 + row);
            }
            if (warp == 0) {
                bool ok = mbar_wait(&t.accf[b], (lt >> 1) & 1, abort_f, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (lane == 0) t.ready = ok;
            }
            named_bar_sync(1, threads);
            if (!*(volatile int *)&t.ready) break;
            tc_fence_after();
            const bool cut = w.c0 != w.c1;
            bool write = true;
            const uint32_t acc = tmem + lane_base + b * CS;
            auto release = [&]() {     // this warp has read its part of the accumulator
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acce0 + b * 8);
            };
            if (cut) {
                // leave this piece's sums (slot 1: the tile's first piece, which
                // ends its pair's line; slot 0: a later one, which begins it); the
                // last of the tile's pieces to arrive adds them all
                const int slot = 2 * blockIdx.x + (w.k0 == 0);
                float4 *dst = (float4 *)(p.part + (size_t)slot * 128 * GP_TILE) + row;
                for (int c = half * 32; c < cols; c += 32 * halves) {
                    uint32_t v[32];
                    tmem_ld32(acc + c, v);
                    tmem_wait_ld32(v);
                    if (row < nrows)
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (c + j < cols)
                                __stcg(dst + (c + j) / 4 * 128,
                                       make_float4(__uint_as_float(v[j]), __uint_as_float(v[j + 1]),
                                                   __uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])));
                }
                release();
                named_bar_sync(1, threads);
                if (threadIdx.x == 0) {
                    // (released and acquired for all behind the barriers)
                    uint32_t *count = p.count + 2 * (p.pair0 + w.c0) + rank;
                    t.last = add_acq_rel(count, 1u) == (uint32_t)(w.c1 - w.c0);
                    if (t.last) *count = 0;
                }
                named_bar_sync(1, threads);
                write = *(volatile int *)&t.last != 0;
            }
            auto out_row = [&](int r) -> uint16_t * {     // of the A side: null where there is none
                if (r >= nrows) return nullptr;
                if (grad) return out0 + w.g * p.gstride + (int64_t)(w.xt * GP_TILE + rank * 128 + r) * p.ld;
                const int at = t.rows[r];
                return at < 0 ? nullptr : out0 + (int64_t)at * p.ld;
            };
            // Chunks of 32 columns of this thread's row.  A joined tile of a few
            // rows is dealt to all threads instead, a row's chunk at a time.
            const int chunks = pack ? (p.n + 63) / 64 * 2 : low ? (cols + 63) / 64 * 2 : (cols + 31) / 32;
            const bool dealt = !grad && !grouped && cut && nrows <= 64;
            const int items = !write ? 0 : dealt ? nrows * chunks : chunks;
            // (low: both chunks of a pair in one warp)
            auto column = [&](int i) {
                return (low ? (i >> 1) * 2 * halves + half * 2 + (i & 1) : i * halves + half) * 32;
            };
            // staged rows go out 64 bytes each, by 4 lanes: this lane's 4 rows
            const bool staged = !low && !pack && p.vec == 8 && !dealt;
            const int piece = (lane & 3) * 8;
            uint16_t *base[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                base[q] = staged && !grouped ? out_row(quad * 32 + q * 8 + (lane >> 2)) : nullptr;
            // Rows that are less aligned, and those of the low-rank gradients, with
            // narrower accesses that still run along a row: against each lane writing
            // its own, 2 bytes at a time, the gradients of 4,096 rows in 16 groups of
            // 1,023 x 1,025 take 140 us (242), those of 43 adapters of rank 128 346
            // (385).  The grouped products' lanes lie along the row anyhow: 66 us so,
            // 76 through the stage
            auto send = [&](int left, auto to) {
                __syncwarp();
                if (low && p.vec == 8) flush<8>(stage, left, to);
                else if (p.vec >= 4) flush<4>(stage, left, to);
                else if (p.vec == 2) flush<2>(stage, left, to);
                else flush<1>(stage, left, to);
                __syncwarp();
            };
            auto stage_row = [&](const float (&v)[32]) {     // the lane's own row
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *(uint4 *)(stage + staged_at(lane, j)) =
                        make_uint4(pack2<F16>(v[8 * j], v[8 * j + 1]), pack2<F16>(v[8 * j + 2], v[8 * j + 3]),
                                   pack2<F16>(v[8 * j + 4], v[8 * j + 5]), pack2<F16>(v[8 * j + 6], v[8 * j + 7]));
            };
            float prev[32];
            uint32_t u[32];
            const bool tm = !cut && write;
            bool held = tm;
            if (tm && column(0) < chunks * 32) tmem_ld32(acc + column(0), u);
            for (int i = dealt ? threadIdx.x : 0; dealt ? i < items : column(i) < items * 32; i += dealt ? threads : 1) {
                const int r = dealt ? i % nrows : row, c = dealt ? i / nrows * 32 : column(i);
                const bool mine = r < nrows;
                float v[32];
                if (cut) {
                    // the pieces' sum, in the order of the contraction
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0.f;
#pragma unroll 2
                    for (int o = w.c0; o <= (mine ? w.c1 : -1); ++o) {
                        const int slot = 2 * (2 * (p.pair0 + o) + rank) + (o == w.c0);
                        const float4 *src = (const float4 *)(p.part + (size_t)slot * 128 * GP_TILE) + r;
                        float4 x[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            x[j] = c + 4 * j < cols ? __ldcg(src + (c / 4 + j) * 128) : make_float4(0, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            v[4 * j] += x[j].x;
                            v[4 * j + 1] += x[j].y;
                            v[4 * j + 2] += x[j].z;
                            v[4 * j + 3] += x[j].w;
                        }
                    }
                } else {
                    // (a gradient without rows: its stage held the next group's)
                    const bool none = grad && w.count == 0;
                    tmem_wait_ld32(u);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = none ? 0.f : __uint_as_float(u[j]);
                    if (column(i + 1) < items * 32) {
                        tmem_ld32(acc + column(i + 1), u);       // while this chunk goes out
                    } else {
                        release();
                        held = false;
                    }
                }
                if (staged) {
                    // 32 x 32 values through shared memory, rows of the output as rows.
                    // Grouped: lane = result column, TMEM column = row of x
                    if (grouped) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            *(uint16_t *)(stage + staged_at(j, lane >> 3) + (lane & 7) * 2) = (uint16_t)pack2<F16>(v[j], 0.f);
                    } else {
                        stage_row(v);
                    }
                    __syncwarp();
                    const int n = grouped ? w.ot * GP_TILE + rank * 128 + quad * 32 + piece : w.ot * p.bn + c + piece;
                    const int left = p.n - n;
                    uint16_t *dst[4];
                    uint4 d[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int j = q * 8 + (lane >> 2);
                        d[q] = *(const uint4 *)(stage + staged_at(j, lane & 3));
                        dst[q] = base[q];
                        if (grouped) {
                            const int at = c + j < cols ? t.rows[c + j] : -1;
                            dst[q] = at < 0 ? nullptr : out0 + (int64_t)at * p.ld;
                        }
                    }
                    if (left >= 8 && (grouped || c + piece < cols)) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (dst[q]) *(uint4 *)(dst[q] + n) = d[q];
                    } else if (left > 0 && (grouped || c + piece < cols)) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (dst[q])
                                for (int k = 0; k < left; ++k)
                                    dst[q][n + k] = ((const uint16_t *)(stage + staged_at(q * 8 + (lane >> 2), lane & 3)))[k];
                    }
                    __syncwarp();
                } else if (grouped) {
                    const int n = w.ot * GP_TILE + rank * 128 + row;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int at = mine && c + j < cols ? t.rows[c + j] : -1;
                        if (at >= 0) out0[(int64_t)at * p.ld + n] = (uint16_t)pack2<F16>(v[j], 0.f);
                    }
                } else if (low) {
                    // blocks of 64 columns: the products with the high terms of 32
                    // ranks, then those with the low terms (which an infinity among the
                    // rows would make a NaN of where they are 0)
                    if (!(c & 32)) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) prev[j] = v[j];
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = isfinite(prev[j]) ? prev[j] + v[j] : prev[j];
                    if (F16) {
                        const float back = peak_unscale(p.peak[w.g]);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= back;
                    }
                    uint16_t *out = out0 + w.g * p.gstride;
                    const int r0 = (w.ot * p.bn + c) >> 6 << 5, m = w.xt * GP_TILE + rank * 128 + quad * 32;
                    if (p.out_kind == GP_OUT_LOW) {
                        stage_row(v);
                        send(p.rank_out - r0, [&](int j) -> uint16_t * {
                            return m + j < p.m ? out + (int64_t)(m + j) * p.ld + r0 : nullptr;
                        });
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            *(uint16_t *)(stage + staged_at(j, lane >> 3) + (lane & 7) * 2) = (uint16_t)pack2<F16>(v[j], 0.f);
                        send(p.m - m, [&](int j) -> uint16_t * {
                            return r0 + j < p.rank_out ? out + (int64_t)(r0 + j) * p.ld + m : nullptr;
                        });
                    }
                } else if (pack) {
                    // 32 ranks of an inner product.  A place without a row (padding) has
                    // zeros, also where the adapter's values make a NaN of them
                    const float sc = p.scale[w.g];
                    const bool row_there = mine && t.rows[r] >= 0;
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = row_there && c + j < p.n ? v[j] * sc : 0.f;
                    uint16_t *dst = out0 + (int64_t)(w.first + rank * 128 + r) * p.ld + c * 2;
                    if (F16 && p.out_kind == GP_OUT_WIDE) {
                        uint32_t top = 0;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
                            top = max(top, m < 0x7f800000u ? m : 0u);
                        }
                        if (mine)
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                *(float4 *)((float *)dst + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                        // (a maximum: the order of the arrivals is free)
                        if (!dealt) top = __reduce_max_sync(0xffffffffu, top);
                        if (top && (dealt || lane == 0)) atomicMax(p.peak + w.g, top);
                    } else {
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            uint16_t h0, l0, h1, l1;
                            bf16_terms(v[j], h0, l0);
                            bf16_terms(v[j + 1], h1, l1);
                            hi[j / 2] = h0 | (uint32_t)h1 << 16;
                            lo[j / 2] = l0 | (uint32_t)l1 << 16;
                        }
                        if (mine)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                *(uint4 *)(dst + 8 * j) = make_uint4(hi[4 * j], hi[4 * j + 1], hi[4 * j + 2], hi[4 * j + 3]);
                                *(uint4 *)(dst + 32 + 8 * j) =
                                    make_uint4(lo[4 * j], lo[4 * j + 1], lo[4 * j + 2], lo[4 * j + 3]);
                            }
                    }
                } else if (!dealt) {
                    stage_row(v);
                    send(cols - c, [&](int j) -> uint16_t * {
                        uint16_t *to = out_row(quad * 32 + j);
                        return to ? to + w.ot * p.bn + c : nullptr;
                    });
                } else {
                    uint16_t *dst = out_row(r);
                    if (dst) store_row<F16>(dst + w.ot * p.bn + c, v, min(32, cols - c), p.vec == 8);
                }
            }
            if (held) release();                // (no chunk was this warp's)
            named_bar_sync(1, threads);         // what the warps share may be written again
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();          // no MMA reads this CTA's memory, no arrival is on its way
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 2 * CS);
    }
}

const void *kernel_of(int f16, int kind) {
    static const void *const all[2][KINDS] = {
        {(const void *)k_group<false, 0>, (const void *)k_group<false, 1>, (const void *)k_group<false, 2>,
         (const void *)k_group<false, 3>, (const void *)k_group<false, 4>, (const void *)k_group<false, 5>},
        {(const void *)k_group<true, 0>, (const void *)k_group<true, 1>, (const void *)k_group<true, 2>,
         (const void *)k_group<true, 3>, (const void *)k_group<true, 4>, (const void *)k_group<true, 5>}};
    return all[f16][kind];
}

int kind_of(const GroupProduct &p, int n) {
    if (p.mode == GP_GROUPED) return K_GROUPED;
    if (p.mode == GP_ROWS) return p.shared ? K_SHARED : n > 1 ? K_PACKS : K_PACK;
    return p.out_kind == GP_OUT_GROUP ? K_GRAD : K_LOW;
}

}  // namespace

cudaError_t group_prepare(int nsm, int *ctas) {
    cudaError_t e = cudaSuccess;
    for (int kind = 0; kind < KINDS && e == cudaSuccess; ++kind)
        for (int f16 = 0; f16 < 2 && e == cudaSuccess; ++f16)
            e = cudaFuncSetAttribute(kernel_of(f16, kind), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     SMEM_MAX);
    if (e != cudaSuccess) return e;
    // the pairs that run at once: the walk deals its pieces to that many
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)nsm / 2 * 2);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_MAX;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int pairs = 0;
    e = cudaOccupancyMaxActiveClusters(&pairs, kernel_of(0, K_SHARED), &cfg);
    if (e == cudaSuccess && pairs < 1) e = cudaErrorLaunchOutOfResources;
    *ctas = 2 * (pairs < nsm / 2 ? pairs : nsm / 2);
    return e;
}

size_t group_part_floats(int ctas) { return (size_t)ctas * 2 * 128 * GP_TILE; }

void group_plan(GroupProduct *p) {
    // B side: whole 1 KB; MN-major operands come in blocks of 64 columns.  Few
    // picked rows take the room of their own groups of 8 on the A side: the MMA
    // reads on into the B side for the rows that do not count
    int a = A_BYTES, b = (p->sorted ? (p->bn / 2 + GP_ROW_BOX - 1) / GP_ROW_BOX * GP_ROW_BOX : p->bn / 2) * 128;
    if (p->mode == GP_WGRAD || (p->mode == GP_ROWS && p->dense_mn)) b = (p->bn / 2 + 63) / 64 * 8192;
    if (p->mode == GP_ROWS && !p->sorted && p->plan.rows < 128) a = (p->plan.rows + GP_ROW_BOX - 1) / GP_ROW_BOX * GP_ROW_BOX * 128;
    b = (b + 1023) / 1024 * 1024;
    const int room = SMEM_MAX - 1024 - table_bytes(*p), deep = (p->k + GP_BK - 1) / GP_BK;
    // picked rows: stages of up to 256 columns, as the words and fences of a
    // stage (about 0.5 us) outlast its few bytes
    p->kk = 1;
    while (!p->sorted && p->kk < 4 && 2 * p->kk <= deep && room / ((a + b) * 2 * p->kk) >= 4) p->kk *= 2;
    p->a_sub = a;
    p->b_sub = b;
    p->b_off = a * p->kk;
    p->stage_bytes = (a + b) * p->kk;
    p->ext_pack = 1;
    if (p->rank && p->rank <= GP_RC) {
        const int fits = b * p->kk / (ext_bytes(*p) * ext_terms(*p));
        p->ext_pack = fits < 1 ? 1 : fits;
    }
    const int fit = room / p->stage_bytes;
    p->stages = fit < MAX_STAGES ? fit : MAX_STAGES;
    p->smem = 1024 + p->stages * p->stage_bytes + table_bytes(*p);
    p->ntiles = (p->n + (p->mode == GP_GROUPED ? GP_TILE : p->bn) - 1) / (p->mode == GP_GROUPED ? GP_TILE : p->bn);
    p->mtiles = (p->m + GP_TILE - 1) / GP_TILE;
}

cudaError_t launch_group(GroupCall *calls, int n, double share, int ctas, cudaStream_t s) {
    const int pairs = ctas / 2, kind = kind_of(calls[0].p, n);
    int first = pairs;
    if (n > 1) {
        first = (int)(share * pairs + 0.5);
        first = first < 1 ? 1 : first > pairs - 1 ? pairs - 1 : first;
    }
    calls[0].p.pair0 = 0;
    calls[0].p.pairs = first;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = (size_t)calls[0].p.smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    Launch<2> two;
    two.call[0] = calls[0];
    two.call[1] = calls[n - 1];
    two.call[1].p.pair0 = first;          // (one call: a pair that does not exist)
    two.call[1].p.pairs = pairs - first;
    if (n > 1 && two.call[1].p.smem > calls[0].p.smem) cfg.dynamicSmemBytes = (size_t)two.call[1].p.smem;
    void *args[1] = {&two};               // kernels of one call take the first
    return cudaLaunchKernelExC(&cfg, kernel_of(calls[0].p.f16 != 0, kind), args);
}

}  // namespace hwr
