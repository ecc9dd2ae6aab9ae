// Internal interface between the host code of the operators that follow a
// routing decision (ops_api.cu) and their kernels (k_group.cu: products on the
// tensor cores; k_few.cu: of a few rows; k_ops.cu: dispatch, row copies, low-rank
// products of a few rows, padding, gradient clipping).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hwr_internal.cuh"
#include "hwr_ops.h"

namespace hwr {

constexpr int OPS_MAX_GROUPS = HWR_OPS_MAX_GROUPS;
constexpr int OPS_MAX_RANK = HWR_OPS_MAX_RANK;

// ---- products with ragged groups of rows (k_group.cu) -----------------------

constexpr int GP_TILE = 256;       // rows of a tile's A side; B side: up to 256 in steps of 16
constexpr int GP_BK = 64;          // contraction of a pipeline stage
constexpr int GP_RC = 32;          // ranks of an extension stage (high and low terms: 64 columns)

// Which operand holds the rows of x.
enum : int {
    GP_GROUPED = 0,    // B side: out^T tile = W[g] tile (A) x rows (B): a ragged group costs
                       // whole 16s of rows
    GP_ROWS = 1,       // A side: out tile = rows x W tile
    GP_WGRAD = 2,      // contraction: both sides are columns of rows by place
};

// What a tile's values become.
enum : int {
    GP_OUT_ROWS = 0,   // out[order[p]][n], rows scattered back to their places
    GP_OUT_PACK = 1,   // scale[g] * value as two bf16 terms, a row per place
    GP_OUT_GROUP = 2,  // out[g][m][n]
    GP_OUT_LOW = 3,    // out[g][m][r]: columns j and j + 32 of each 64 added
    GP_OUT_LOW_T = 4,  // out[g][r][m]: the same, transposed
    GP_OUT_WIDE = 5,   // scale[g] * value in fp32, where GP_OUT_PACK has the terms; and
                       // each group's largest finite one
};

// A value as two bf16 terms, high + low, that give what the value gives in a sum of
// products with infinities too: the low term has the value's sign and is zero only
// where the value is (0 and inf make a NaN), so the high one is cut off, strictly below
// the value; an infinity or NaN is both terms.  16 bits of the value.
__device__ __forceinline__ void bf16_terms(float v, uint16_t &high, uint16_t &low) {
    const uint32_t u = __float_as_uint(v), m = u & 0x7fffffffu;
    const uint32_t h = (m - 1 < 0x7f7fffffu ? u - 1 : u) >> 16;          // (finite, not 0)
    const float rest = m < 0x7f800000u ? v - __uint_as_float(h << 16) : v;
    high = (uint16_t)h;
    low = __bfloat16_as_ushort(__float2bfloat16_rn(rest));
}

// The largest finite magnitude of a group's inner products (its bits) as the power of
// two that brings it into [2^14, 2^15), the end of fp16's range, and back.
__device__ __forceinline__ int peak_exponent(uint32_t peak) {
    const int e = peak >> 23 ? peak >> 23 : 1;
    return peak ? (141 - e < 126 ? 141 - e : 126) : 0;
}
__device__ __forceinline__ float peak_scale(uint32_t peak) { return __uint_as_float((127 + peak_exponent(peak)) << 23); }
__device__ __forceinline__ float peak_unscale(uint32_t peak) { return __uint_as_float((127 - peak_exponent(peak)) << 23); }

// A plan as the products read it.  The places of its order hold the groups one
// after the other, then the rows without a group; a padded plan (sort_rows)
// starts every group at a multiple of 16 places, with no row (-1) at the rest.
struct GroupPlan {
    int rows = 0;                     // rows of x and of the output
    int places = 0;                   // upper bound of the places
    int groups = 0;
    const int32_t *offsets = nullptr; // [groups + 1] (padded: and the number of places)
    const int32_t *order = nullptr;   // [places]
    int padded = 0;
};

struct GroupProduct {
    int mode = 0;
    GroupPlan plan;
    int shared = 0;                   // one W for all places; the plan's groups are the extension's
    // x (rows products) by place, through the tensor map of sorted rows, or
    // picked by index
    int sorted = 0;
    const uint16_t *x = nullptr;
    int64_t x_ld = 0;
    int k = 0, n = 0, m = 0;          // contraction (rows products), result columns, rows (gradients)
    int dense_mn = 0;                 // W is MN-major
    int bn = 0;                       // B-side extent of a tile (GP_GROUPED: at most)
    int ntiles = 0, mtiles = 0;       // column tiles; row tiles of a gradient
    int f16 = 0;
    int stages = 0, stage_bytes = 0, smem = 0;
    int kk = 1;                       // blocks of 64 columns of the contraction in a stage
    int a_sub = 0, b_sub = 0;         // bytes of a block's A and B side
    int b_off = 0;                    // of the B side in a stage
    int rank = 0;                     // of the low-rank extension of a shared product
    int ext_pack = 1;                 // groups in one of its stages
    // output
    int out_kind = 0;
    int vec = 1;                      // values of an aligned store: 8, 4, 2 or 1
    void *out = nullptr;
    int64_t ld = 0, gstride = 0;
    int rank_out = 0;                 // GP_OUT_LOW*: ranks written
    const float *scale = nullptr;
    uint32_t *peak = nullptr;         // [groups] GP_OUT_WIDE: raised; GP_OUT_LOW*: what the terms are scaled by
    // joined partial tiles and the status word
    float *part = nullptr;
    uint32_t *count = nullptr;
    int32_t *status = nullptr;
    int test_stall = 0;               // test hook: nothing is loaded (bounded waits expire)
    int pair0 = 0, pairs = 0;         // the CTA pairs at work on it
};

// x: the rows by place (or l and r of a gradient: the A and B side); w: the
// dense operand; u, eb: the extension's.
struct GroupMaps {
    CUtensorMap x, xx, w, u, eb;      // xx: x in boxes of 128 rows
};

constexpr int GP_ROW_BOX = 32;     // rows of a box of x and u

// A product as it is launched; of the kinds with small tiles (GP_OUT_PACK,
// GP_OUT_LOW*) two may share a launch, each on some of the pairs.
struct GroupCall {
    GroupMaps maps;
    GroupProduct p;
};

cudaError_t group_prepare(int nsm, int *ctas);
// Pipeline stages that fit beside the tables, and the counts of tiles.
void group_plan(GroupProduct *p);
size_t group_part_floats(int ctas);
// n calls (1 or 2, of one kind) in a launch; share: of the pairs for the first of two.
cudaError_t launch_group(GroupCall *calls, int n, double share, int ctas, cudaStream_t s);

// ---- products of a few rows (k_few.cu) ---------------------------------------

// out[t] = W x[t] + b[g(t)] u[t] for at most FEW_ROWS rows (W K-major; W and the
// rows of x 16-byte aligned).
constexpr int FEW_ROWS = 16;
struct FewRows {
    GroupPlan plan;
    int k, n;
    const uint16_t *x, *w;
    int64_t x_ld, w_ld;
    uint16_t *out;
    int64_t ld;
    int rank;
    const float *u;                   // [places][rank]
    const uint16_t *b;
    int64_t b_ld, b_z;
};
cudaError_t launch_few_rows(const FewRows &p, bool f16, cudaStream_t s);

// ---- dispatch, clipping, padding (k_ops.cu) ---------------------------------

cudaError_t ops_prepare(int *cluster);       // blocks of a dispatch's clusters
size_t dispatch_scratch_ints(int rows, int groups, int nsm, int cluster);
cudaError_t launch_dispatch(int rows, int groups, const int32_t *choice, int32_t *offsets,
                            int32_t *order, int32_t *scratch, int nsm, int cluster, cudaStream_t s);

// Rows of up to two matrices by place: dst[p] = src[order[p]], zeros where the
// order holds no row.  With padded_offsets (groups + 2 ints) the places are
// those of the padded plan, which is written there and to padded_order (places
// of its ints); without, those of the plan itself.
struct SortRows {
    int n = 0;                        // matrices
    const uint16_t *src[2];
    int64_t src_ld[2];
    int cols[2];
    uint16_t *dst[2];
    int64_t dst_ld[2];                // whole 16-byte units
    uint32_t *zero = nullptr;         // and words to be zeroed
    int nzero = 0;
};
cudaError_t launch_sort_rows(const GroupPlan &plan, const SortRows &m, int places, int32_t *padded_offsets,
                             int32_t *padded_order, int nsm, cudaStream_t s);

// Inner products in fp32 (GP_OUT_WIDE) as two fp16 terms, in place, scaled by a power of
// two of each group's own (peak_scale); where `ext` is set also as two bf16 terms there.
struct SplitLow {
    uint16_t *u, *ext;
    const uint32_t *peak;
};
cudaError_t launch_split_low(const GroupPlan &plan, int rank, int64_t ld, const SplitLow *s, int n, int nsm,
                             cudaStream_t st);

// The adapters' matrices in fp16 as two bf16 terms, exactly (8 + 3 bits), as the
// extension's stages take them: src [groups][rows][rank] (or, mn, [groups][rank][rows])
// to dst [groups][rows][ext_terms_ranks] (or [groups][ext_terms_ranks][dst_ld]), where
// a chunk of 32 ranks (16 of up to 16; mn: 32) is its high terms, then its low ones.
inline int ext_terms_ranks(int rank, bool mn) { return rank <= 16 && !mn ? 32 : (rank + GP_RC - 1) / GP_RC * 2 * GP_RC; }
cudaError_t launch_ext_terms(uint16_t *dst, int64_t dst_ld, const uint16_t *src, int groups, int rows, int rank, bool mn,
                             int nsm, cudaStream_t s);

// u[place] = scale[g] a[g] x[order[place]] as GP_OUT_PACK leaves it, for a few
// rows (a 16-byte aligned, rows of x too).
struct LowFew {
    GroupPlan plan;
    int k, rank;
    const uint16_t *x, *a;
    int64_t x_ld, a_ld, a_z;
    const float *scale;
    uint16_t *u;
    int64_t u_ld;
    float *wide;                      // or, where set, as fp32 [places][rank] here
    int by_place;                     // x lies by place already
};
cudaError_t launch_low_few(const LowFew &p, bool f16, cudaStream_t s);

// dst [z][rows][dst_ld] = src [z][rows][cols] (strides in elements, 16-bit
// elements; columns up to dst_ld are zeroed).
cudaError_t launch_pad(void *dst, int64_t dst_ld, const void *src, int64_t src_ld, int64_t src_z,
                       int64_t nz, int64_t rows, int cols, int nsm, cudaStream_t s);

// Chunks of `per` 4 KB (a 16-byte access of each of a block's threads): 4 for
// sets of gradients that fill the GPU so, 1 for small ones, whose time is that of
// the busiest SM (48 tensors of 2.8 MB in all: 12.4 us in chunks of 16 KB, 9.8 of
// 8 KB, 9.9 of 4 KB; 474 MB: 229, 232 and 241 us).
constexpr int CLIP_UNIT = 4096, CLIP_PER = 4;
constexpr int64_t CLIP_SMALL = 4 << 20;       // elements of a small set
struct alignas(16) ClipChunk {
    const void *in;
    void *out;
    int32_t n, dtype;
    int64_t unused;
};
inline __host__ __device__ int clip_elems(int dtype, int per) { return per * CLIP_UNIT / (dtype == HWR_F32 ? 4 : 2); }
inline __host__ __device__ int64_t clip_chunks(int64_t n, int dtype, int per) {
    return (n + clip_elems(dtype, per) - 1) / clip_elems(dtype, per);
}
inline __host__ __device__ ClipChunk clip_chunk(const void *in, void *out, int64_t n, int dtype, int per, int64_t i) {
    ClipChunk c;
    const int64_t left = n - i * clip_elems(dtype, per);
    c.in = (const char *)in + i * per * CLIP_UNIT;
    c.out = (char *)out + i * per * CLIP_UNIT;
    c.n = (int32_t)(left < clip_elems(dtype, per) ? left : clip_elems(dtype, per));
    c.dtype = dtype;
    c.unused = 0;
    return c;
}
constexpr int CLIP_TABLE = 256;       // tensors of one launch of the table's kernel
struct ClipTable {
    int n, at, per;                   // tensors; first chunk of them in the table; chunks' size
    const void *in[CLIP_TABLE];
    void *out[CLIP_TABLE];
    int64_t count[CLIP_TABLE];
    int32_t chunk0[CLIP_TABLE + 1];   // first chunk of each tensor
    uint8_t dtype[CLIP_TABLE];
};
int clip_blocks(int64_t chunks, int nsm);    // partial sums of a call
cudaError_t launch_clip_table(const ClipTable &t, ClipChunk *table, cudaStream_t s);
struct ClipSums {
    double *part;                     // [clip_blocks]
    uint32_t *count;                  // blocks that have finished (zeroed once, self-resetting)
    float *factor;                    // what the gradients are scaled by
};
cudaError_t launch_clip(const ClipChunk *table, int chunks, int per, int nsm, const ClipSums &sums, float max_norm,
                        float *norm, cudaStream_t s);

// ---- rows of logits (k_tokens.cu) --------------------------------------------

constexpr int TOKENS_MAX_TOP = HWR_TOKENS_MAX_TOP;
constexpr int TOKEN_SPLITS = 32;      // pieces of a row, at most
struct TokenPart {                    // of a piece: the sums, and its best keys
    float m, s, d, unused;
    uint64_t key[32];
};
struct TokenRows {
    int rows, vocab, top, splits;
    const void *logits;
    int64_t ld;
    const int32_t *token;             // may be null
    float *logprob, *entropy, *stats;
    int32_t *top_token;
    float *top_logprob;
    TokenPart *part;                  // [rows][splits] where splits > 1
    uint32_t *arrivals;               // [rows] zeroed once, self-resetting
};
int token_splits(int rows, int vocab, hwr_dtype dtype, bool top, int nsm);
cudaError_t launch_token_rows(const TokenRows &p, hwr_dtype dtype, int nsm, cudaStream_t s);
struct TokenGrad {
    int rows, vocab, splits;
    const void *logits;
    int64_t ld;
    const int32_t *token;
    const float *stats, *entropy, *da, *db;
    void *out;
    int64_t out_ld;
};
cudaError_t launch_token_grad(TokenGrad p, hwr_dtype dtype, int nsm, cudaStream_t s);

// ---- the optimizer's step (k_adamw.cu) ----------------------------------------

// A block's elements; with moments in 8 bits a warp's share one power of two.
constexpr int ADAMW_CHUNK = 2048, ADAMW_BLOCK = 256;
constexpr int ADAMW_TABLE = 256;      // tensors of one launch
struct alignas(64) AdamWTensor {
    float *param;
    void *copy, *m, *v;               // copy: may be null
    float *m_scale, *v_scale;
    int64_t n;
    int32_t copy_dtype, aligned;      // aligned: to 16 bytes, all of them
};
struct AdamWChunk {
    int32_t tensor, chunk;            // and which of its chunks
};
struct AdamWStep {
    const AdamWTensor *tensors;
    const AdamWChunk *table;
    int chunks, tensor0;              // chunks of this launch; the first of its tensors
    uint32_t blocks;                  // of all the call's launches
    uint32_t *arrivals;
    int32_t *step;
    const float *lr, *norm;           // device values, may be null
    float rate, max_norm, b1, b2, one_b1, one_b2, log_b1, log_b2, eps, decay;
    uint32_t seed;
    const void *grad[ADAMW_TABLE];    // null: the tensor is left as it is
    uint8_t dtype[ADAMW_TABLE];
};
int adamw_grid(int chunks, int bits, int nsm);
cudaError_t launch_adamw(const AdamWStep &p, int bits, int grid, cudaStream_t s);

// ---- a layer of experts for a few rows (k_experts.cu) ---------------------------

constexpr int EXPERTS_MAX_ROWS = HWR_EXPERTS_MAX_ROWS, EXPERTS_MAX_TOP = HWR_EXPERTS_MAX_TOP;
constexpr int EXPERTS_MAX_OUT = HWR_EXPERTS_MAX_OUT, EXPERTS_MAX_WIDTH = HWR_EXPERTS_MAX_WIDTH;
struct Experts {
    int rows, groups, top, n_in, hidden, n_out;
    int gated, act, over_all;
    const uint16_t *x, *w_in, *w_out;
    int64_t x_ld, w_in_ld, w_in_z, w_out_ld, w_out_z;
    const float *scores;              // null: choice and gates are given
    int64_t scores_ld;
    const int32_t *choice;
    const float *gates;
    uint16_t *y;
    int64_t y_ld;
    // workspace: h in terms [rows * top][expert_terms][h_ld], bf16 or (fp16 layers) fp32; what
    // each piece of the second product gives [rows * top][splits][n_out]
    void *h;
    int64_t h_ld;                     // whole 16-byte units
    int splits;
    float *part;
    char *tables;                     // what the routing found, for the launches after the first
    int32_t *used_splits;
    int32_t *status;
    int test_stall;                   // test hook: nothing is copied (bounded waits expire)
    // of a launch: columns of a step; where the ring of copies begins in shared memory, the
    // bytes of a step, and steps
    int cols, ring_at, step, depth;
};
__host__ __device__ constexpr int expert_terms(bool f16) { return f16 ? 2 : 3; }      // that a hidden value has
int expert_splits(int hidden);            // at most
size_t expert_tables(int rows, int top);
cudaError_t experts_prepare();
// The weights of a product as a tensor (64, rows, columns / 64, experts): boxes of 64 x 8 x
// columns / 64 of a step, and of what the last step has of them; and as one of (columns,
// rows, 1, experts): boxes of 64 x 8, where the columns are not whole 64.
struct WeightMaps {
    CUtensorMap whole, last, tail;
};
// Those of both products, where their matrices allow it, and the steps' columns.
struct ExpertMaps {
    WeightMaps in, out;
    bool in_boxes, out_boxes;
    int in_cols, out_cols;
};
void expert_plan(const Experts &p, bool f16, ExpertMaps *m);
cudaError_t launch_experts(const Experts &p, const ExpertMaps &m, bool f16, int nsm, cudaStream_t s);

}  // namespace hwr
