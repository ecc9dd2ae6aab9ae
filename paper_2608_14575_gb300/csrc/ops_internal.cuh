// Internal interface between the host code of the operators that follow a
// routing decision (ops_api.cu) and their kernels (k_group.cu: products on the
// tensor cores; k_ops.cu: dispatch, gradient clipping, padding).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "hwr_internal.cuh"
#include "hwr_ops.h"

namespace hwr {

constexpr int OPS_MAX_GROUPS = HWR_OPS_MAX_GROUPS;
constexpr int OPS_MAX_RANK = HWR_OPS_MAX_RANK;

// ---- products with ragged groups of rows (k_group.cu) -----------------------

constexpr int GP_BM = 128;         // rows of a tile (TMEM lanes)
constexpr int GP_MAX_BN = 256;     // columns of a tile
constexpr int GP_BK = 64;          // contraction of a pipeline stage
constexpr int GP_RC = 32;          // ranks of an extension stage (high and low halves: 64 columns)

// What a tile's values become.
enum : int {
    GP_OUT_ROWS = 0,   // out[order[p]][n], rows scattered back to their places
    GP_OUT_PACK = 1,   // scale[g] * value as two 16-bit terms, rows as above
    GP_OUT_GROUP = 2,  // out[g][m][n]
    GP_OUT_LOW = 3,    // out[g][m][r]: columns j and j + 32 of each 64 added
    GP_OUT_LOW_T = 4,  // out[g][r][m]: the same, transposed
};

struct GroupProduct {
    // rows and their groups
    int rows = 0, groups = 0;         // tiles lie within one of `groups` groups
    int shared = 0;                   // 1: one group of all rows (groups = 1)
    const int32_t *offsets = nullptr; // [groups or ext_groups + 1]
    const int32_t *order = nullptr;   // [rows]
    // shape: contraction length (rows products), columns of the result, and
    // for gradients (wgrad) the result's rows per group
    int wgrad = 0;
    int k = 0, n = 0, m = 0;
    int bn = 0, ntiles = 0, mtiles = 0;
    int mma_n = 0;
    int b_mn = 0;                     // B is MN-major
    int f16 = 0;
    int stages = 0, stage_bytes = 0;
    // low-rank extension of a shared product
    int rank = 0, ext_groups = 0;
    int ext_b_mn = 0;
    // output
    int out_kind = 0, vec = 0;
    void *out = nullptr;
    int64_t ld = 0, gstride = 0;
    int rank_out = 0;                 // GP_OUT_LOW*: ranks written
    const float *scale = nullptr;
    // joined partial tiles and the status word
    float *part = nullptr;
    uint32_t *count = nullptr;
    int32_t *status = nullptr;
};

struct GroupMaps {
    CUtensorMap a, b, u, eb;
};

cudaError_t group_prepare();
// Pipeline stages that fit beside the tables, for a tile of bn columns.
void group_plan(GroupProduct *p);
size_t group_part_floats(int nsm);
cudaError_t launch_group(const GroupProduct &p, const GroupMaps &maps, int nsm, cudaStream_t s);

// ---- dispatch, clipping, padding (k_ops.cu) ---------------------------------

cudaError_t ops_prepare();
size_t dispatch_scratch_ints(int rows, int groups, int nsm);
cudaError_t launch_dispatch(int rows, int groups, const int32_t *choice, int32_t *offsets,
                            int32_t *order, int32_t *scratch, int nsm, cudaStream_t s);

// dst [z][rows][dst_ld] = src [z][rows][cols] (strides in elements, 16-bit
// elements; columns up to dst_ld are zeroed).
cudaError_t launch_pad(void *dst, int64_t dst_ld, const void *src, int64_t src_ld, int64_t src_z,
                       int64_t nz, int64_t rows, int cols, int nsm, cudaStream_t s);

constexpr int CLIP_TABLE = 512;   // tensors of one launch (kernel parameters)
struct ClipTable {
    int n;
    int first_block;              // of this launch, among all partial sums
    const void *in[CLIP_TABLE];
    void *out[CLIP_TABLE];
    int64_t count[CLIP_TABLE];
    int32_t chunk0[CLIP_TABLE + 1];   // first chunk of each tensor
    uint8_t dtype[CLIP_TABLE];
};

int clip_blocks(int64_t chunks, int nsm);
int64_t clip_chunks(int64_t n, int dtype);
cudaError_t launch_square_sums(const ClipTable &t, int blocks, double *part, cudaStream_t s);
cudaError_t launch_clip(const ClipTable &t, int blocks, const double *part, int nparts, float max_norm,
                        float *norm, cudaStream_t s);

}  // namespace hwr
