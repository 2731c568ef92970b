// Layer norm over the last axis, forward and backward, and the forward pass of the
// stable embedding (a table's row, looked up and normalized in one pass).
//
//   mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps)
//   y = xh weight + bias          with xh = (x - mean) rstd
//   g = dy weight
//   dx = rstd (g - mean(g) - xh mean(g xh))
//   dweight = sum over rows of dy xh,  dbias = sum over rows of dy
//
// Everything is formed in fp32 and rounded once where it is stored.  The statistics
// take two passes over a row held in registers: the mean first, then the sums of
// d = x - mean and of d^2; what the first mean lost in rounding is the mean of d.
#include "bq_ops_device.h"

namespace bq {
namespace {

using namespace dev;

// Elements per lane and access: 16 bytes of the wider type.
template <int A, int B>
constexpr int vec_of = (elem_bytes<A> == 4 || elem_bytes<B> == 4) ? 4 : 8;

constexpr float kNaN = __builtin_nanf("");

// ---------------------------------------------------------------------------
// Forward.  WAVES waves hold one row in registers, K vectors of V elements per
// lane; with one wave per row a workgroup takes four rows.
// ---------------------------------------------------------------------------

template <int WAVES>
constexpr int rows_per_group = WAVES == 1 ? 4 : 1;
template <int WAVES>
constexpr int group_threads = WAVES == 1 ? 256 : 64 * WAVES;

template <int XT, int PT, int YT, bool GATHER, int WAVES, int K>
__global__ __launch_bounds__(group_threads<WAVES>) void norm_forward_kernel(const NormArgs a)
{
    constexpr int V = vec_of<XT, YT>;
    __shared__ float scratch[3 * WAVES];
    const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t n = a.cols;
    // (a second row's sums go to scratch behind a barrier that follows their reading)
    for (int64_t row = (int64_t)blockIdx.x * rows_per_group<WAVES> +
                       (WAVES == 1 ? threadIdx.x >> 6 : 0);
         row < a.rows; row += (int64_t)gridDim.x * rows_per_group<WAVES>) {
        int64_t from = row;
        bool known = true;
        if constexpr (GATHER) {
            from = id_at(a.ids, row, a.ids64);
            known = from >= 0 && from < a.table_rows;
            if (!known)
                from = 0;
        }
        const void *const xp = row_of<XT>(a.x, from, a.x_stride);
        float x[K][V];
        float sum[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < K; ++k)
            load_cols<XT, V>(xp, (int64_t)(k * 64 * WAVES + lane) * V, n, x[k]);
        const float rn = 1.0f / (float)n;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int r = 0; r < V; ++r)
                sum[0] += x[k][r];
        group_sum<1, WAVES>(sum, scratch);
        const float mean0 = sum[0] * rn;
        float two[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
#pragma unroll
            for (int r = 0; r < V; ++r) {
                x[k][r] = c + r < n ? x[k][r] - mean0 : 0.0f;
                two[0] += x[k][r];
                two[1] = __builtin_fmaf(x[k][r], x[k][r], two[1]);
            }
        }
        group_sum<2, WAVES>(two, scratch + WAVES);
        const float delta = two[0] * rn;
        float var = two[1] * rn - delta * delta;
        var = var < 0.0f ? 0.0f : var;
        const float rstd = 1.0f / sqrtf(var + a.eps);
        if (a.mean && lane == 0) {
            a.mean[row] = mean0 + delta;
            a.rstd[row] = rstd;
        }
        void *const yp = row_of<YT>(a.y, row, n);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
            if (c >= n)
                break;
            float w[V], b[V];
#pragma unroll
            for (int r = 0; r < V; ++r) {
                w[r] = 1.0f;
                b[r] = 0.0f;
            }
            if (a.weight)
                load_cols<PT, V>(a.weight, c, n, w);
            if (a.bias)
                load_cols<PT, V>(a.bias, c, n, b);
            float y[V];
#pragma unroll
            for (int r = 0; r < V; ++r) {
                y[r] = __builtin_fmaf((x[k][r] - delta) * rstd, w[r], b[r]);
                if (GATHER && !known)
                    y[r] = kNaN;
            }
            store_cols<YT, V>(yp, c, n, y);
        }
    }
}

// Rows too long for the registers of a workgroup: the row is read three times.
constexpr int kLongWaves = 16;
template <int XT, int PT, int YT, bool GATHER>
__global__ __launch_bounds__(64 * kLongWaves) void norm_forward_long_kernel(const NormArgs a)
{
    constexpr int V = vec_of<XT, YT>;
    constexpr int64_t kStep = (int64_t)64 * kLongWaves * V;
    __shared__ float scratch[3 * kLongWaves];
    const int64_t n = a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        int64_t from = row;
        bool known = true;
        if constexpr (GATHER) {
            from = id_at(a.ids, row, a.ids64);
            known = from >= 0 && from < a.table_rows;
            if (!known)
                from = 0;
        }
        const void *const xp = row_of<XT>(a.x, from, a.x_stride);
        const int64_t c0 = (int64_t)threadIdx.x * V;
        const float rn = 1.0f / (float)n;
        float sum[1] = {0.0f};
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V];
            load_cols<XT, V>(xp, c, n, x);
#pragma unroll
            for (int r = 0; r < V; ++r)
                sum[0] += x[r];
        }
        group_sum<1, kLongWaves>(sum, scratch);
        const float mean0 = sum[0] * rn;
        float two[2] = {0.0f, 0.0f};
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V];
            load_cols<XT, V>(xp, c, n, x, mean0);
#pragma unroll
            for (int r = 0; r < V; ++r) {
                const float d = x[r] - mean0;
                two[0] += d;
                two[1] = __builtin_fmaf(d, d, two[1]);
            }
        }
        group_sum<2, kLongWaves>(two, scratch + kLongWaves);
        const float delta = two[0] * rn;
        float var = two[1] * rn - delta * delta;
        var = var < 0.0f ? 0.0f : var;
        const float rstd = 1.0f / sqrtf(var + a.eps);
        if (a.mean && threadIdx.x == 0) {
            a.mean[row] = mean0 + delta;
            a.rstd[row] = rstd;
        }
        void *const yp = row_of<YT>(a.y, row, n);
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V], w[V], b[V], y[V];
            load_cols<XT, V>(xp, c, n, x);
#pragma unroll
            for (int r = 0; r < V; ++r) {
                w[r] = 1.0f;
                b[r] = 0.0f;
            }
            if (a.weight)
                load_cols<PT, V>(a.weight, c, n, w);
            if (a.bias)
                load_cols<PT, V>(a.bias, c, n, b);
#pragma unroll
            for (int r = 0; r < V; ++r) {
                y[r] = __builtin_fmaf(((x[r] - mean0) - delta) * rstd, w[r], b[r]);
                if (GATHER && !known)
                    y[r] = kNaN;
            }
            store_cols<YT, V>(yp, c, n, y);
        }
    }
}

// A workgroup per row (or four), within the limit of 2^32 work-items of a launch.
unsigned forward_groups(int64_t rows, int per_group)
{
    const int64_t groups = (rows + per_group - 1) / per_group;
    return (unsigned)(groups < (1 << 20) ? groups : (1 << 20));
}

template <int XT, int PT, int YT, bool GATHER, int WAVES, int K>
void forward_k(const NormArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_forward_kernel<XT, PT, YT, GATHER, WAVES, K>),
                       dim3(forward_groups(a.rows, rows_per_group<WAVES>)),
                       dim3(group_threads<WAVES>), 0, stream, a);
}

template <int XT, int PT, int YT, bool GATHER>
hipError_t forward(const NormArgs &a, hipStream_t stream)
{
    constexpr int64_t kWave = 64 * vec_of<XT, YT>;  // a wave's elements per vector
    const int64_t k = (a.cols + kWave - 1) / kWave;
    if (k <= 1)
        forward_k<XT, PT, YT, GATHER, 1, 1>(a, stream);
    else if (k <= 2)
        forward_k<XT, PT, YT, GATHER, 1, 2>(a, stream);
    else if (k <= 4)
        forward_k<XT, PT, YT, GATHER, 1, 4>(a, stream);
    else if (k <= 8)
        forward_k<XT, PT, YT, GATHER, 1, 8>(a, stream);
    else if (k <= 16)
        forward_k<XT, PT, YT, GATHER, 4, 4>(a, stream);
    else if (k <= 32)
        forward_k<XT, PT, YT, GATHER, 4, 8>(a, stream);
    else if (k <= 64)
        forward_k<XT, PT, YT, GATHER, 16, 4>(a, stream);
    else
        hipLaunchKernelGGL((norm_forward_long_kernel<XT, PT, YT, GATHER>),
                           dim3(forward_groups(a.rows, 1)), dim3(64 * kLongWaves), 0, stream, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Backward.  Workgroups walk the rows; each keeps the sums of dy xh and dy of its
// rows per column in registers and leaves them in the workspace.
// ---------------------------------------------------------------------------

template <int XT, int PT, int WAVES, int K>
__global__ __launch_bounds__(group_threads<WAVES>) void norm_backward_kernel(const NormGradArgs a)
{
    constexpr int V = vec_of<XT, XT>;
    constexpr int kTeams = rows_per_group<WAVES>;
    __shared__ float scratch[4 * WAVES];
    const int team = WAVES == 1 ? threadIdx.x >> 6 : 0;
    const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t n = a.cols;
    const float rn = 1.0f / (float)n;
    float w[K][V], dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int r = 0; r < V; ++r) {
            w[k][r] = 1.0f;
            dw[k][r] = 0.0f;
            db[k][r] = 0.0f;
        }
        if (a.weight)
            load_cols<PT, V>(a.weight, (int64_t)(k * 64 * WAVES + lane) * V, n, w[k]);
    }
    for (int64_t row = (int64_t)blockIdx.x * kTeams + team; row < a.rows;
         row += (int64_t)gridDim.x * kTeams) {
        const void *const xp = row_of<XT>(a.x, row, a.x_stride);
        const void *const gp = row_of<XT>(a.dy, row, a.dy_stride);
        const float mean = G(a.mean)[row], rstd = G(a.rstd)[row];
        float x[K][V], dy[K][V];
        float two[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
            load_cols<XT, V>(xp, c, n, x[k], mean);
            load_cols<XT, V>(gp, c, n, dy[k]);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int r = 0; r < V; ++r) {
                x[k][r] = (x[k][r] - mean) * rstd;
                dw[k][r] = __builtin_fmaf(dy[k][r], x[k][r], dw[k][r]);
                db[k][r] += dy[k][r];
                dy[k][r] *= w[k][r];
                two[0] += dy[k][r];
                two[1] = __builtin_fmaf(dy[k][r], x[k][r], two[1]);
            }
        }
        if (a.dx) {
            if constexpr (WAVES > 1)
                __syncthreads();  // the previous row's sums have been read
            group_sum<2, WAVES>(two, scratch);
            const float c1 = two[0] * rn, c2 = two[1] * rn;
            void *const dp = row_of<XT>(a.dx, row, n);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float d[V];
#pragma unroll
                for (int r = 0; r < V; ++r)
                    d[r] = rstd * __builtin_fmaf(-x[k][r], c2, dy[k][r] - c1);
                store_cols<XT, V>(dp, (int64_t)(k * 64 * WAVES + lane) * V, n, d);
            }
        }
    }
    if (!a.partials)
        return;
    float *const out = a.partials + (int64_t)blockIdx.x * 2 * n;
    if constexpr (kTeams == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
            store_cols<kF32, V>(out, c, n, dw[k]);
            store_cols<kF32, V>(out + n, c, n, db[k]);
        }
    } else {
        // the teams' sums, in order
        __shared__ float join[kTeams][2][64 * V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < V; ++r) {
                join[team][0][r * 64 + lane] = dw[k][r];
                join[team][1][r * 64 + lane] = db[k][r];
            }
            __syncthreads();
            if (team < 2) {
                float s[V];
#pragma unroll
                for (int r = 0; r < V; ++r) {
                    s[r] = join[0][team][r * 64 + lane];
#pragma unroll
                    for (int t = 1; t < kTeams; ++t)
                        s[r] += join[t][team][r * 64 + lane];
                }
                store_cols<kF32, V>(out + team * n, (int64_t)(k * 64 + lane) * V, n, s);
            }
        }
    }
}

// Rows too long for registers: the row is read twice, and the parameters' gradients
// are summed in the workspace, by the thread that owns the column.
template <int XT, int PT>
__global__ __launch_bounds__(64 * kLongWaves) void norm_backward_long_kernel(const NormGradArgs a)
{
    constexpr int V = vec_of<XT, XT>;
    constexpr int64_t kStep = (int64_t)64 * kLongWaves * V;
    __shared__ float scratch[2 * kLongWaves];
    const int64_t n = a.cols;
    const int64_t c0 = (int64_t)threadIdx.x * V;
    const float rn = 1.0f / (float)n;
    float *const out = a.partials ? a.partials + (int64_t)blockIdx.x * 2 * n : nullptr;
    bool first = true;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
        const void *const xp = row_of<XT>(a.x, row, a.x_stride);
        const void *const gp = row_of<XT>(a.dy, row, a.dy_stride);
        const float mean = G(a.mean)[row], rstd = G(a.rstd)[row];
        float two[2] = {0.0f, 0.0f};
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V], dy[V], w[V];
            load_cols<XT, V>(xp, c, n, x, mean);
            load_cols<XT, V>(gp, c, n, dy);
#pragma unroll
            for (int r = 0; r < V; ++r)
                w[r] = 1.0f;
            if (a.weight)
                load_cols<PT, V>(a.weight, c, n, w);
            float dw[V], db[V];
#pragma unroll
            for (int r = 0; r < V; ++r)
                dw[r] = db[r] = 0.0f;
            if (out && !first) {
                load_cols<kF32, V>(out, c, n, dw);
                load_cols<kF32, V>(out + n, c, n, db);
            }
#pragma unroll
            for (int r = 0; r < V; ++r) {
                x[r] = (x[r] - mean) * rstd;
                dw[r] = __builtin_fmaf(dy[r], x[r], dw[r]);
                db[r] += dy[r];
                dy[r] *= w[r];
                two[0] += dy[r];
                two[1] = __builtin_fmaf(dy[r], x[r], two[1]);
            }
            if (out) {
                store_cols<kF32, V>(out, c, n, dw);
                store_cols<kF32, V>(out + n, c, n, db);
            }
        }
        if (!a.dx)
            continue;
        __syncthreads();  // the previous row's sums have been read
        group_sum<2, kLongWaves>(two, scratch);
        const float c1 = two[0] * rn, c2 = two[1] * rn;
        void *const dp = row_of<XT>(a.dx, row, n);
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V], dy[V], w[V];
            load_cols<XT, V>(xp, c, n, x, mean);
            load_cols<XT, V>(gp, c, n, dy);
#pragma unroll
            for (int r = 0; r < V; ++r)
                w[r] = 1.0f;
            if (a.weight)
                load_cols<PT, V>(a.weight, c, n, w);
#pragma unroll
            for (int r = 0; r < V; ++r)
                dy[r] = rstd * __builtin_fmaf(-(x[r] - mean) * rstd, c2, dy[r] * w[r] - c1);
            store_cols<XT, V>(dp, c, n, dy);
        }
    }
}

template <int XT, int PT, int WAVES, int K>
void backward_k(const NormGradArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_backward_kernel<XT, PT, WAVES, K>), dim3((unsigned)a.groups),
                       dim3(group_threads<WAVES>), 0, stream, a);
}

template <int XT, int PT>
hipError_t backward(const NormGradArgs &a, hipStream_t stream)
{
    constexpr int64_t kWave = 64 * vec_of<XT, XT>;
    const int64_t k = (a.cols + kWave - 1) / kWave;
    if (k <= 1)
        backward_k<XT, PT, 1, 1>(a, stream);
    else if (k <= 2)
        backward_k<XT, PT, 1, 2>(a, stream);
    else if (k <= 4)
        backward_k<XT, PT, 1, 4>(a, stream);
    else if (k <= 8)
        backward_k<XT, PT, 4, 2>(a, stream);
    else if (k <= 16)
        backward_k<XT, PT, 4, 4>(a, stream);
    else if (k <= 32)
        backward_k<XT, PT, 16, 2>(a, stream);
    else
        hipLaunchKernelGGL((norm_backward_long_kernel<XT, PT>), dim3((unsigned)a.groups),
                           dim3(64 * kLongWaves), 0, stream, a);
    return hipGetLastError();
}

// Sums of the partials over the groups: one workgroup per 64 columns of one of the two
// gradients; wave w takes every 16th group from w on, then the waves' sums are added
// in order.
constexpr int kSumWaves = 16;
template <int PT>
__global__ __launch_bounds__(64 * kSumWaves) void param_grads_kernel(const float *partials,
                                                                     int64_t groups, int64_t cols,
                                                                     void *dweight, void *dbias)
{
    __shared__ float part[kSumWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const int which = blockIdx.y;
    float s = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (int64_t g = wave; g < groups; g += kSumWaves)
            s += G(partials)[(2 * g + which) * cols + c];
    }
    part[wave][lane] = s;
    __syncthreads();
    void *const out = which ? dbias : dweight;
    if (wave == 0 && c < cols && out) {
        for (int w = 1; w < kSumWaves; ++w)
            s += part[w][lane];
        store1<PT>(out, c, s);
    }
}

}  // namespace

// Workgroups of the backward pass: two per CU hold the registers of the longest rows
// in flight; each leaves 8 bytes per column in the workspace.
int64_t norm_grad_groups(int64_t rows, int64_t cols)
{
    (void)cols;
    return rows < 512 ? (rows < 1 ? 1 : rows) : 512;
}

hipError_t launch_norm_forward(int xt, int pt, int yt, const NormArgs &a, hipStream_t stream)
{
    if (a.ids) {
        // x and the parameters have the table's type
        if (xt == kF32 && yt == kF32) return forward<kF32, kF32, kF32, true>(a, stream);
        if (xt == kF32 && yt == kF16) return forward<kF32, kF32, kF16, true>(a, stream);
        if (xt == kF32 && yt == kBF16) return forward<kF32, kF32, kBF16, true>(a, stream);
        if (xt == kF16) return forward<kF16, kF16, kF16, true>(a, stream);
        return forward<kBF16, kBF16, kBF16, true>(a, stream);
    }
    if (xt == kF32) return forward<kF32, kF32, kF32, false>(a, stream);
    if (xt == kF16 && pt == kF32) return forward<kF16, kF32, kF16, false>(a, stream);
    if (xt == kF16) return forward<kF16, kF16, kF16, false>(a, stream);
    if (pt == kF32) return forward<kBF16, kF32, kBF16, false>(a, stream);
    return forward<kBF16, kBF16, kBF16, false>(a, stream);
}

hipError_t launch_param_grads(int pt, const float *partials, int64_t groups, int64_t cols,
                              void *dweight, void *dbias, hipStream_t stream)
{
    const dim3 grid((unsigned)((cols + 63) / 64), 2);
    if (pt == kF32)
        hipLaunchKernelGGL(param_grads_kernel<kF32>, grid, dim3(64 * kSumWaves), 0, stream,
                           partials, groups, cols, dweight, dbias);
    else if (pt == kF16)
        hipLaunchKernelGGL(param_grads_kernel<kF16>, grid, dim3(64 * kSumWaves), 0, stream,
                           partials, groups, cols, dweight, dbias);
    else
        hipLaunchKernelGGL(param_grads_kernel<kBF16>, grid, dim3(64 * kSumWaves), 0, stream,
                           partials, groups, cols, dweight, dbias);
    return hipGetLastError();
}

hipError_t launch_norm_backward(int xt, int pt, const NormGradArgs &a, hipStream_t stream)
{
    hipError_t e;
    if (a.rows == 0) {
        e = hipSuccess;
    } else if (xt == kF32) {
        e = backward<kF32, kF32>(a, stream);
    } else if (xt == kF16) {
        e = pt == kF32 ? backward<kF16, kF32>(a, stream) : backward<kF16, kF16>(a, stream);
    } else {
        e = pt == kF32 ? backward<kBF16, kF32>(a, stream) : backward<kBF16, kBF16>(a, stream);
    }
    if (e != hipSuccess || !a.partials)
        return e;
    return launch_param_grads(pt, a.partials, a.rows == 0 ? 0 : a.groups, a.cols, a.dweight,
                              a.dbias, stream);
}

}  // namespace bq
