// C-ABI entry points of the operators around the optimizer step (declared in
// include/bq.h): argument checks and launches.  Every check runs before the first
// HIP call, so an error return means nothing was enqueued.
#include <cmath>
#include <cstdint>
#include <cstring>

#include "bq.h"
#include "bq_internal.h"
#include "bq_ops.h"

namespace {

bool valid_dtype(bq_dtype d) { return d == BQ_F32 || d == BQ_F16 || d == BQ_BF16; }
int64_t bytes_of(bq_dtype d) { return d == BQ_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t a)
{
    return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(a - 1)) == 0;
}
bool elements(const void *p, bq_dtype d) { return aligned(p, bytes_of(d)); }

bq_status from_hip(hipError_t e) { return e == hipSuccess ? BQ_OK : BQ_ERR_HIP; }

// Byte offsets stay far below 2^63, and the launches below 2^32 work-items.
constexpr int64_t kMaxRows = int64_t{1} << 40;
constexpr int64_t kMaxCols = int64_t{1} << 27;
constexpr int64_t kMaxDim = int64_t{1} << 24;  // at most 2^16 slabs of a launch

bq_status check_norm(bq_dtype dtype, bq_dtype param_dtype, int64_t rows, int64_t cols, float eps)
{
    if (!valid_dtype(dtype) || !valid_dtype(param_dtype) ||
        (param_dtype != BQ_F32 && param_dtype != dtype))
        return BQ_ERR_DTYPE;
    if (rows < 0 || cols < 1 || rows > kMaxRows || cols > kMaxCols ||
        rows > (int64_t{1} << 60) / cols)
        return BQ_ERR_SIZE;
    if (!(eps >= 0.0f) || std::isinf(eps))
        return BQ_ERR_ARG;
    return BQ_OK;
}

bool valid_stride(int64_t stride, int64_t rows)
{
    return stride >= 0 && stride <= (int64_t{1} << 60) / (rows < 1 ? 1 : rows);
}

// The table's and the output's types, the ids' width and the sizes of a lookup.
bq_status check_lookup(bq_dtype dtype, bq_dtype out_dtype, int64_t num, int64_t dim,
                       int32_t id_bits, int64_t count)
{
    if (!valid_dtype(dtype) || !valid_dtype(out_dtype) ||
        (dtype != BQ_F32 && out_dtype != dtype) || (id_bits != 32 && id_bits != 64))
        return BQ_ERR_DTYPE;
    if (count < 0 || num < 1 || dim < 1 || count > INT32_MAX || num >= INT32_MAX ||
        dim > kMaxDim)
        return BQ_ERR_SIZE;
    return BQ_OK;
}

}  // namespace

extern "C" {

bq_status bq_layer_norm_forward(bq_dtype dtype, bq_dtype param_dtype, const void *x, int64_t rows,
                                int64_t cols, int64_t row_stride, const void *weight,
                                const void *bias, float eps, void *y, float *mean, float *rstd,
                                hipStream_t stream)
{
    const bq_status st = check_norm(dtype, param_dtype, rows, cols, eps);
    if (st != BQ_OK)
        return st;
    if (!valid_stride(row_stride, rows))
        return BQ_ERR_SIZE;
    if (rows == 0)
        return BQ_OK;
    if (!x || !y || (mean == nullptr) != (rstd == nullptr))
        return BQ_ERR_NULL;
    if (!elements(x, dtype) || !elements(y, dtype) || !elements(weight, param_dtype) ||
        !elements(bias, param_dtype) || !aligned(mean, 4) || !aligned(rstd, 4))
        return BQ_ERR_ALIGN;
    bq::NormArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.rows = rows;
    a.cols = cols;
    a.x_stride = row_stride;
    a.table_rows = rows;
    a.eps = eps;
    return from_hip(bq::launch_norm_forward(dtype, param_dtype, dtype, a, stream));
}

int64_t bq_layer_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (check_norm(BQ_F32, BQ_F32, rows, cols, 0.0f) != BQ_OK)
        return 0;
    return bq::norm_workspace_bytes(rows, cols);
}

bq_status bq_layer_norm_backward(bq_dtype dtype, bq_dtype param_dtype, const void *dy,
                                 int64_t dy_stride, const void *x, int64_t x_stride, int64_t rows,
                                 int64_t cols, const void *weight, const float *mean,
                                 const float *rstd, void *dx, void *dweight, void *dbias,
                                 void *workspace, hipStream_t stream)
{
    const bq_status st = check_norm(dtype, param_dtype, rows, cols, 0.0f);
    if (st != BQ_OK)
        return st;
    if (!valid_stride(dy_stride, rows) || !valid_stride(x_stride, rows))
        return BQ_ERR_SIZE;
    const bool params = dweight || dbias;
    if (!params && (!dx || rows == 0))
        return BQ_OK;
    if ((params && !workspace) || (rows > 0 && (!dy || !x || !mean || !rstd)))
        return BQ_ERR_NULL;
    if (!elements(dy, dtype) || !elements(x, dtype) || !elements(dx, dtype) ||
        !elements(weight, param_dtype) || !elements(dweight, param_dtype) ||
        !elements(dbias, param_dtype) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        (params && !aligned(workspace, 16)))
        return BQ_ERR_ALIGN;
    bq::NormGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.dy = dy;
    a.x = x;
    a.weight = weight;
    a.mean = mean;
    a.rstd = rstd;
    a.dx = dx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.partials = params ? static_cast<float *>(workspace) : nullptr;
    a.rows = rows;
    a.cols = cols;
    a.dy_stride = dy_stride;
    a.x_stride = x_stride;
    return from_hip(bq::launch_norm_backward(dtype, param_dtype, a, stream));
}

bq_status bq_embedding_forward(bq_dtype dtype, bq_dtype out_dtype, const void *weight, int64_t num,
                               int64_t dim, const void *ids, int32_t id_bits, int64_t count,
                               float scale, void *out, hipStream_t stream)
{
    const bq_status st = check_lookup(dtype, out_dtype, num, dim, id_bits, count);
    if (st != BQ_OK)
        return st;
    if (!std::isfinite(scale))
        return BQ_ERR_ARG;
    if (count == 0)
        return BQ_OK;
    if (!weight || !ids || !out)
        return BQ_ERR_NULL;
    if (!elements(weight, dtype) || !elements(out, out_dtype) || !aligned(ids, id_bits / 8))
        return BQ_ERR_ALIGN;
    bq::LookupArgs a;
    std::memset(&a, 0, sizeof(a));
    a.table = weight;
    a.ids = ids;
    a.out = out;
    a.count = count;
    a.num = num;
    a.dim = dim;
    a.scale = scale;
    a.ids64 = id_bits == 64;
    return from_hip(bq::launch_lookup(dtype, out_dtype, a, stream));
}

int64_t bq_embedding_workspace_bytes(int64_t count, int64_t num, int64_t dim)
{
    if (check_lookup(BQ_F32, BQ_F32, num, dim, 64, count) != BQ_OK)
        return 0;
    return bq::lookup_workspace_bytes(count, num, dim, false);
}

bq_status bq_embedding_backward(bq_dtype dtype, bq_dtype out_dtype, const void *dout,
                                const void *ids, int32_t id_bits, int64_t count, int64_t num,
                                int64_t dim, int64_t padding, float scale, void *dweight,
                                void *workspace, hipStream_t stream)
{
    const bq_status st = check_lookup(dtype, out_dtype, num, dim, id_bits, count);
    if (st != BQ_OK)
        return st;
    if (!std::isfinite(scale) || padding < -1 || padding >= num)
        return BQ_ERR_ARG;
    if (!dweight || !workspace || (count > 0 && (!dout || !ids)))
        return BQ_ERR_NULL;
    if (!elements(dout, out_dtype) || !elements(dweight, dtype) || !aligned(ids, id_bits / 8) ||
        !aligned(workspace, 16))
        return BQ_ERR_ALIGN;
    bq::LookupGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.dout = dout;
    a.ids = ids;
    a.dtable = dweight;
    a.workspace = static_cast<uint8_t *>(workspace);
    a.count = count;
    a.num = num;
    a.dim = dim;
    a.padding = padding;
    a.scale = scale;
    a.ids64 = id_bits == 64;
    return from_hip(bq::launch_lookup_backward(dtype, out_dtype, a, stream));
}

bq_status bq_stable_embedding_forward(bq_dtype dtype, bq_dtype out_dtype, const void *weight,
                                      int64_t num, int64_t dim, const void *ids, int32_t id_bits,
                                      int64_t count, const void *norm_weight,
                                      const void *norm_bias, float eps, void *out,
                                      hipStream_t stream)
{
    bq_status st = check_lookup(dtype, out_dtype, num, dim, id_bits, count);
    if (st != BQ_OK)
        return st;
    if (dim > bq::kMaxStableDim)
        return BQ_ERR_SIZE;
    if (!(eps >= 0.0f) || std::isinf(eps))
        return BQ_ERR_ARG;
    if (count == 0)
        return BQ_OK;
    if (!weight || !ids || !out)
        return BQ_ERR_NULL;
    if (!elements(weight, dtype) || !elements(out, out_dtype) || !aligned(ids, id_bits / 8) ||
        !elements(norm_weight, dtype) || !elements(norm_bias, dtype))
        return BQ_ERR_ALIGN;
    bq::NormArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = weight;
    a.weight = norm_weight;
    a.bias = norm_bias;
    a.y = out;
    a.ids = ids;
    a.rows = count;
    a.cols = dim;
    a.x_stride = dim;
    a.table_rows = num;
    a.eps = eps;
    a.ids64 = id_bits == 64;
    return from_hip(bq::launch_norm_forward(dtype, dtype, out_dtype, a, stream));
}

int64_t bq_stable_embedding_workspace_bytes(int64_t count, int64_t num, int64_t dim)
{
    if (check_lookup(BQ_F32, BQ_F32, num, dim, 64, count) != BQ_OK || dim > bq::kMaxStableDim)
        return 0;
    return bq::lookup_workspace_bytes(count, num, dim, true);
}

bq_status bq_stable_embedding_backward(bq_dtype dtype, bq_dtype out_dtype, const void *dout,
                                       const void *ids, int32_t id_bits, int64_t count,
                                       const void *weight, int64_t num, int64_t dim,
                                       int64_t padding, const void *norm_weight, float eps,
                                       void *dweight, void *dnorm_weight, void *dnorm_bias,
                                       void *workspace, hipStream_t stream)
{
    bq_status st = check_lookup(dtype, out_dtype, num, dim, id_bits, count);
    if (st != BQ_OK)
        return st;
    if (dim > bq::kMaxStableDim)
        return BQ_ERR_SIZE;
    if (!(eps >= 0.0f) || std::isinf(eps) || padding < -1 || padding >= num)
        return BQ_ERR_ARG;
    if (!dweight || !weight || !workspace || (count > 0 && (!dout || !ids)))
        return BQ_ERR_NULL;
    if (!elements(dout, out_dtype) || !elements(weight, dtype) || !elements(dweight, dtype) ||
        !elements(norm_weight, dtype) || !elements(dnorm_weight, dtype) ||
        !elements(dnorm_bias, dtype) || !aligned(ids, id_bits / 8) || !aligned(workspace, 16))
        return BQ_ERR_ALIGN;
    bq::LookupGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.dout = dout;
    a.ids = ids;
    a.dtable = dweight;
    a.workspace = static_cast<uint8_t *>(workspace);
    a.count = count;
    a.num = num;
    a.dim = dim;
    a.padding = padding;
    a.scale = 1.0f;
    a.ids64 = id_bits == 64;
    a.table = weight;
    a.weight = norm_weight;
    a.dweight = dnorm_weight;
    a.dbias = dnorm_bias;
    a.eps = eps;
    return from_hip(bq::launch_lookup_backward(dtype, out_dtype, a, stream));
}

int64_t bq_grad_norm_workspace_bytes(int32_t ngrads)
{
    if (ngrads < 0)
        return 0;
    const int64_t launches = (int64_t{ngrads} + bq::kMaxClipTensors - 1) / bq::kMaxClipTensors;
    return (launches * bq::kClipMaxGroups + 1) * 8;
}

}  // extern "C"

namespace {

int64_t tiles_of(const bq_grad &g)
{
    const int64_t per = bq::kClipTileBytes / bytes_of(g.dtype);
    return (g.numel + per - 1) / per;
}

bq_status check_grads(const bq_grad *grads, int32_t ngrads, bq_norm kind, const void *workspace,
                      const float *norm)
{
    if (kind != BQ_NORM_L2 && kind != BQ_NORM_INF)
        return BQ_ERR_ENUM;
    if (ngrads < 0)
        return BQ_ERR_SIZE;
    if ((ngrads > 0 && !grads) || !workspace || !norm)
        return BQ_ERR_NULL;
    if (!aligned(workspace, 8) || !aligned(norm, 4))
        return BQ_ERR_ALIGN;
    int64_t tiles = 0;  // counted in 32 bits by the launches
    for (int32_t i = 0; i < ngrads; ++i) {
        const bq_grad &g = grads[i];
        if (!valid_dtype(g.dtype))
            return BQ_ERR_DTYPE;
        if (g.numel < 0 || g.numel > (int64_t{1} << 40))
            return BQ_ERR_SIZE;
        tiles += tiles_of(g);
        if (tiles > INT32_MAX / 2)
            return BQ_ERR_SIZE;
        if (g.numel == 0)
            continue;
        if (!g.data)
            return BQ_ERR_NULL;
        if (!elements(g.data, g.dtype))
            return BQ_ERR_ALIGN;
    }
    return BQ_OK;
}

// Packs non-empty gradients from `at` on into one launch's arguments; returns the
// index behind the last.
int32_t pack(const bq_grad *grads, int32_t ngrads, int32_t at, bq::ClipArgs &a)
{
    a.ntensors = 0;
    a.total_tiles = 0;
    for (; at < ngrads && a.ntensors < bq::kMaxClipTensors; ++at) {
        const bq_grad &g = grads[at];
        if (g.numel == 0)
            continue;
        a.ptr[a.ntensors] = g.data;
        a.numel[a.ntensors] = g.numel;
        a.dtype[a.ntensors] = static_cast<uint8_t>(g.dtype);
        a.tile_begin[a.ntensors] = a.total_tiles;
        a.total_tiles += static_cast<int32_t>(tiles_of(g));
        ++a.ntensors;
    }
    return at;
}

// As pack, with the last non-empty gradients before `at`; returns the first's index.
int32_t pack_below(const bq_grad *grads, int32_t at, bq::ClipArgs &a)
{
    int32_t from = at;
    for (int32_t n = 0; from > 0; --from) {
        if (grads[from - 1].numel == 0)
            continue;
        if (n++ == bq::kMaxClipTensors)
            break;
    }
    pack(grads, at, from, a);
    return from;
}

bq_status norm_and_clip(const bq_grad *grads, int32_t ngrads, bq_norm kind, bool clip,
                        double max_norm, void *workspace, float *norm, hipStream_t stream)
{
    bq::ClipArgs a;
    std::memset(&a, 0, sizeof(a));
    a.partials = static_cast<double *>(workspace);
    a.inf_norm = kind == BQ_NORM_INF;
    a.max_norm = max_norm;
    for (int32_t at = 0; at < ngrads;) {
        at = pack(grads, ngrads, at, a);
        if (a.ntensors == 0)
            break;
        a.first_partial = a.npartials;
        const int groups = a.total_tiles < bq::kClipMaxGroups ? a.total_tiles : bq::kClipMaxGroups;
        a.npartials += groups;
        const hipError_t e = bq::launch_grad_norm(a, groups, stream);
        if (e != hipSuccess)
            return from_hip(e);
    }
    a.norm = norm;
    if (!clip || a.npartials == 0 || a.npartials > bq::kClipMaxPartials) {
        double *const total = a.partials + a.npartials;
        const hipError_t e = bq::launch_norm_finish(a, total, stream);
        if (!clip || a.npartials == 0 || e != hipSuccess)
            return from_hip(e);
        a.partials = total;
        a.npartials = 1;
        a.norm = nullptr;
    }
    // the launches in the opposite order: what the norm read last comes first
    for (int32_t at = ngrads; at > 0;) {
        at = pack_below(grads, at, a);
        if (a.ntensors == 0)
            break;
        const hipError_t e = bq::launch_clip(a, stream);
        if (e != hipSuccess)
            return from_hip(e);
        a.norm = nullptr;
    }
    return BQ_OK;
}

}  // namespace

extern "C" {

bq_status bq_grad_norm(const bq_grad *grads, int32_t ngrads, bq_norm kind, void *workspace,
                       float *norm, hipStream_t stream)
{
    const bq_status st = check_grads(grads, ngrads, kind, workspace, norm);
    if (st != BQ_OK)
        return st;
    return norm_and_clip(grads, ngrads, kind, false, 0.0, workspace, norm, stream);
}

bq_status bq_clip_grad_norm(const bq_grad *grads, int32_t ngrads, bq_norm kind, double max_norm,
                            void *workspace, float *norm, hipStream_t stream)
{
    const bq_status st = check_grads(grads, ngrads, kind, workspace, norm);
    if (st != BQ_OK)
        return st;
    if (!(max_norm >= 0.0))
        return BQ_ERR_ARG;
    return norm_and_clip(grads, ngrads, kind, true, max_norm, workspace, norm, stream);
}

}  // extern "C"
