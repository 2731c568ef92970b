// The norm of a list of gradients as one vector, and clipping to it:
//   norm = sqrt(sum g^2), or max |g|;  c = min(1, max_norm / (norm + 1e-6));  g *= c.
//
// A norm launch adds up squares in double (no fp32 gradient overflows them, and the
// order of adding does not show in the fp32 result); each workgroup leaves one partial
// sum.  Every workgroup of the clip launch adds the partial sums up again, all in the
// same order, so no launch is needed in between; where c is 1 it ends there.
#include "bq_ops_device.h"

namespace bq {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// The tensor of tile `tile`: the last one that begins at or before it, from `from` on.
__device__ inline int tensor_of(const ClipArgs &a, int tile, int from)
{
    if (from + 1 >= a.ntensors || a.tile_begin[from + 1] > tile)
        return from;
    int lo = from + 1, hi = a.ntensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.tile_begin[mid] <= tile)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ inline double wave_add(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}
// max of non-negative values or NaN, by their bits: a NaN is above everything
__device__ inline uint32_t wave_umax(uint32_t v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}

template <int DT>
__device__ inline void tile_norm(const void *p, int64_t from, int64_t numel, bool inf_norm,
                                 double (&acc)[2], uint32_t &top)
{
    constexpr int V = DT == kF32 ? 4 : 8;
    constexpr int kVecs = kClipTileBytes / 16 / kThreads;
    float x[kVecs][V];
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        load_cols<DT, V>(p, from + (int64_t)(k * kThreads + threadIdx.x) * V, numel, x[k]);
    if (inf_norm) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
#pragma unroll
            for (int r = 0; r < V; ++r)
                top = max(top, __float_as_uint(x[k][r]) & 0x7fffffffu);
    } else {
#pragma unroll
        for (int k = 0; k < kVecs; ++k)
#pragma unroll
            for (int r = 0; r < V; ++r)
                acc[r & 1] = __builtin_fma((double)x[k][r], (double)x[k][r], acc[r & 1]);
    }
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const ClipArgs a)
{
    __shared__ double sums[kThreads / 64];
    __shared__ uint32_t tops[kThreads / 64];
    double acc[2] = {0.0, 0.0};
    uint32_t top = 0;
    int t = 0;
    for (int tile = blockIdx.x; tile < a.total_tiles; tile += gridDim.x) {
        t = tensor_of(a, tile, t);
        const void *const p = a.ptr[t];
        const int64_t at = tile - a.tile_begin[t], n = a.numel[t];
        if (a.dtype[t] == kF32)
            tile_norm<kF32>(p, at * (kClipTileBytes / 4), n, a.inf_norm, acc, top);
        else if (a.dtype[t] == kF16)
            tile_norm<kF16>(p, at * (kClipTileBytes / 2), n, a.inf_norm, acc, top);
        else
            tile_norm<kBF16>(p, at * (kClipTileBytes / 2), n, a.inf_norm, acc, top);
    }
    const double s = wave_add(acc[0] + acc[1]);
    top = wave_umax(top);
    if ((threadIdx.x & 63) == 0) {
        sums[threadIdx.x >> 6] = s;
        tops[threadIdx.x >> 6] = top;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double v = 0.0;
        if (a.inf_norm) {
            uint32_t m = 0;
            for (int w = 0; w < kThreads / 64; ++w)
                m = max(m, tops[w]);
            v = (double)__uint_as_float(m);
        } else {
            for (int w = 0; w < kThreads / 64; ++w)
                v += sums[w];
        }
        a.partials[a.first_partial + blockIdx.x] = v;
    }
}

// The partial results as one: their sum or their largest (NaN above everything), the
// same bits in every workgroup.
__device__ inline double join(const double *partials, int n, bool inf_norm)
{
    __shared__ double part[kThreads / 64];
    double v = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const double x = G(partials)[i];
        v = inf_norm ? (x > v || x != x ? x : v) : v + x;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const double x = __shfl_xor(v, o);
        v = inf_norm ? (x > v || x != x ? x : v) : v + x;
    }
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kThreads / 64; ++w)
        v = inf_norm ? (part[w] > v || part[w] != part[w] ? part[w] : v) : v + part[w];
    return v;
}

__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double *partials, int n,
                                                               int inf_norm, double *total,
                                                               float *norm)
{
    const double v = join(partials, n, inf_norm);
    if (threadIdx.x == 0) {
        if (total)
            *total = v;
        if (norm)
            *norm = (float)(inf_norm ? v : sqrt(v));
    }
}

template <int DT>
__device__ inline void tile_scale(void *p, int64_t from, int64_t numel, float c)
{
    constexpr int V = DT == kF32 ? 4 : 8;
    constexpr int kVecs = kClipTileBytes / 16 / kThreads;
    float x[kVecs][V];
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
        load_cols<DT, V>(p, from + (int64_t)(k * kThreads + threadIdx.x) * V, numel, x[k]);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
#pragma unroll
        for (int r = 0; r < V; ++r)
            x[k][r] *= c;
        store_cols<DT, V>(p, from + (int64_t)(k * kThreads + threadIdx.x) * V, numel, x[k]);
    }
}

__global__ __launch_bounds__(kThreads) void clip_kernel(const ClipArgs a)
{
    const double v = join(a.partials, a.npartials, a.inf_norm);
    const double norm = a.inf_norm ? v : sqrt(v);
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0)
        *a.norm = (float)norm;
    const double ratio = a.max_norm / (norm + 1e-6);
    const float c = (float)(ratio > 1.0 ? 1.0 : ratio);  // NaN stays
    if (c == 1.0f)
        return;
    int t = 0;
    for (int tile = blockIdx.x; tile < a.total_tiles; tile += gridDim.x) {
        t = tensor_of(a, tile, t);
        void *const p = a.ptr[t];
        const int64_t at = tile - a.tile_begin[t], n = a.numel[t];
        if (a.dtype[t] == kF32)
            tile_scale<kF32>(p, at * (kClipTileBytes / 4), n, c);
        else if (a.dtype[t] == kF16)
            tile_scale<kF16>(p, at * (kClipTileBytes / 2), n, c);
        else
            tile_scale<kBF16>(p, at * (kClipTileBytes / 2), n, c);
    }
}

}  // namespace

hipError_t launch_grad_norm(const ClipArgs &a, int groups, hipStream_t stream)
{
    hipLaunchKernelGGL(grad_norm_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_norm_finish(const ClipArgs &a, double *total, hipStream_t stream)
{
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kThreads), 0, stream, a.partials,
                       a.npartials, a.inf_norm, total, a.norm);
    return hipGetLastError();
}

hipError_t launch_clip(const ClipArgs &a, hipStream_t stream)
{
    const int groups = a.total_tiles < 2048 ? (a.total_tiles < 1 ? 1 : a.total_tiles) : 2048;
    hipLaunchKernelGGL(clip_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace bq
