// Internal declarations of the operators around the optimizer step (layer norm,
// embedding lookup, stable embedding, gradient norm and clipping), shared by
// their C-ABI layer (bq_ops_api.cpp) and their kernels (bq_norm.hip,
// bq_embedding.hip, bq_clip.hip).  Not part of the public interface.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "bq_internal.h"

namespace bq {

constexpr int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---- layer norm -----------------------------------------------------------

// Rows of `cols` values.  With ids, row i is row ids[i] of the table x, which has
// `table_rows` rows of x_stride values (an id outside of it gives a row of NaN).
struct NormArgs {
    const void *x;
    const void *weight;  // may be null: ones
    const void *bias;    // may be null: zeros
    void *y;             // rows packed
    float *mean;         // may be null, with rstd
    float *rstd;
    const void *ids;     // null for plain rows
    int64_t rows, cols, x_stride, table_rows;
    float eps;
    int32_t ids64;
};
hipError_t launch_norm_forward(int xt, int pt, int yt, const NormArgs &a, hipStream_t stream);

struct NormGradArgs {
    const void *dy;
    const void *x;
    const void *weight;  // may be null
    const float *mean;
    const float *rstd;
    void *dx;            // may be null; rows packed
    void *dweight;       // may be null
    void *dbias;         // may be null
    float *partials;     // of every workgroup [2][cols]: its rows' part of the two
    int64_t rows, cols, dy_stride, x_stride;
};
int64_t norm_workspace_bytes(int64_t rows, int64_t cols);
hipError_t launch_norm_backward(int xt, int pt, const NormGradArgs &a, hipStream_t stream);

// The sums over `groups` partial rows [2][cols] (the parameters' gradients), in
// order, to dweight and dbias (either may be null).
hipError_t launch_param_grads(int pt, const float *partials, int64_t groups, int64_t cols,
                              void *dweight, void *dbias, hipStream_t stream);

// ---- embedding ------------------------------------------------------------

struct LookupArgs {
    const void *table;
    const void *ids;
    void *out;
    int64_t count, num, dim;
    float scale;
    int32_t ids64;
};
hipError_t launch_lookup(int wt, int yt, const LookupArgs &a, hipStream_t stream);

struct LookupGradArgs {
    const void *dout;    // count x dim
    const void *ids;
    void *dtable;        // num x dim, every row written
    uint8_t *workspace;
    int64_t count, num, dim, padding;  // padding: row without a gradient, or -1
    float scale;
    int32_t ids64;
    // the stable embedding's: its table and layer norm
    const void *table;   // null for a plain lookup
    const void *weight;  // may be null
    void *dweight;       // may be null
    void *dbias;         // may be null
    float eps;
};
int64_t lookup_workspace_bytes(int64_t count, int64_t num, int64_t dim, bool stable);
hipError_t launch_lookup_backward(int wt, int yt, const LookupGradArgs &a, hipStream_t stream);
// the stable embedding holds a row on chip
constexpr int64_t kMaxStableDim = BQ_STABLE_EMBEDDING_MAX_DIM;

// ---- gradient norm and clipping --------------------------------------------

// Tensors of one launch, in kernel arguments.
constexpr int kMaxClipTensors = 180;
struct ClipArgs {
    double *partials;       // one per workgroup of every norm launch
    float *norm;            // written by the first workgroup where not null
    double max_norm;
    int32_t first_partial;  // of this launch's workgroups (norm launches)
    int32_t npartials;      // of all norm launches
    int32_t inf_norm;
    int32_t ntensors;
    int32_t total_tiles;
    void *ptr[kMaxClipTensors];
    int64_t numel[kMaxClipTensors];
    int32_t tile_begin[kMaxClipTensors];
    uint8_t dtype[kMaxClipTensors];
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel argument block must stay below 4 KiB");
constexpr int kClipTileBytes = 16384;
// Workgroups of a norm launch, at most: all run at once, five to a CU (the norm of 1.56e9
// fp16 gradients: 1.11 ms with 256, 0.71 with 512, 0.54 with 1024, 0.52 with 1280 and
// 1536).
constexpr int kClipMaxGroups = 1280;
// A clip launch's workgroups each add up the partial sums; above this many, a launch
// of its own adds them up once (behind the last of them).
constexpr int kClipMaxPartials = 2048;
hipError_t launch_grad_norm(const ClipArgs &a, int groups, hipStream_t stream);
hipError_t launch_norm_finish(const ClipArgs &a, double *total, hipStream_t stream);
hipError_t launch_clip(const ClipArgs &a, hipStream_t stream);

}  // namespace bq
