// The norm of a list of gradients as one vector, and clipping to it:
//   norm = sqrt(sum g^2), or max |g|;  c = min(1, max_norm / (norm + 1e-6));  g *= c.
//
// A norm launch adds up squares in double (no fp32 gradient overflows them, and the
// order of adding does not show in the fp32 result); each workgroup leaves one partial
// sum.  Every workgroup of the clip launch adds the partial sums up again, all in the
// same order, so no launch is needed in between; where c is 1 it ends there.
//
// HBM bounds both.  1.56e9 fp16 gradients in 580 tensors, MI355X: the norm 0.52 ms (6.0
// TB/s, where reads alone reach 7), with clipping 1.68 ms (5.5 TB/s of 3 x 3.1 GB; a
// copy of that length reaches 5.1).
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

// The same where it is `from` or one before it.
__device__ inline int tensor_below(const ClipArgs &a, int tile, int from)
{
    if (a.tile_begin[from] <= tile)
        return from;
    int lo = 0, hi = from - 1;
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

constexpr int kVecs = kClipTileBytes / 16 / kThreads;  // of 16 bytes, per thread and tile

// A tile's values as they are in memory: 16 bytes at a time, zeros behind the tensor's
// end.  (A last vector's elements are loaded one by one, by one lane.)
struct Tile {
    vu4 w[kVecs];
    int dtype;
};
template <int DT>
__device__ inline vu4 load16(const void *p, int64_t e, int64_t numel)
{
    constexpr int V = 16 / elem_bytes<DT>;
    vu4 w = {0, 0, 0, 0};
    if (e + V <= numel) {
        const Raw<DT, V> x = load_raw<DT, V, true>(p, e);
        w = vu4{x.w[0], x.w[1], x.w[2], x.w[3]};
    } else if (e < numel) {
#pragma unroll
        for (int r = 0; r < V; ++r) {
            if (e + r < numel) {
                if constexpr (DT == kF32)
                    w[r] = G(static_cast<const uint32_t *>(p))[e + r];
                else
                    w[r / 2] |= (uint32_t)G(static_cast<const uint16_t *>(p))[e + r] << (16 * (r % 2));
            }
        }
    }
    return w;
}
__device__ inline void load_tile(const ClipArgs &a, int t, int tile, Tile &x)
{
    const void *const p = a.ptr[t];
    const int64_t n = a.numel[t];
    x.dtype = a.dtype[t];
    const int elems = x.dtype == kF32 ? 4 : 8;  // per vector
    const int64_t from = (int64_t)(tile - a.tile_begin[t]) * (kClipTileBytes / 16) * elems;
    if (from + kClipTileBytes / 16 * elems <= n) {
        const char *const q = static_cast<const char *>(p) + from / elems * 16;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(q) + (k * kThreads + threadIdx.x) * 16;
            x.w[k] = __builtin_nontemporal_load((gvu4_any2)at);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int64_t e = from + (int64_t)(k * kThreads + threadIdx.x) * elems;
        x.w[k] = x.dtype == kF32 ? load16<kF32>(p, e, n) : load16<kF16>(p, e, n);
    }
}

template <int DT>
__device__ inline void add_tile(const Tile &x, bool inf_norm, double (&acc)[2], uint32_t &top)
{
    constexpr int V = 16 / elem_bytes<DT>;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const Raw<DT, V> raw = {x.w[k].x, x.w[k].y, x.w[k].z, x.w[k].w};
        float f[V];
        unpack<DT, V>(raw, f);
#pragma unroll
        for (int r = 0; r < V; ++r) {
            if (inf_norm)
                top = max(top, __float_as_uint(f[r]) & 0x7fffffffu);
            else
                acc[r & 1] = __builtin_fma((double)f[r], (double)f[r], acc[r & 1]);
        }
    }
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const ClipArgs a)
{
    __shared__ double sums[kThreads / 64];
    __shared__ uint32_t tops[kThreads / 64];
    double acc[2] = {0.0, 0.0};
    uint32_t top = 0;
    // the next tile's values are on their way while this one's are added
    Tile next;
    int t = tensor_of(a, blockIdx.x, 0);
    load_tile(a, t, blockIdx.x, next);
    for (int tile = blockIdx.x; tile < a.total_tiles; tile += gridDim.x) {
        const Tile x = next;
        if (tile + (int)gridDim.x < a.total_tiles) {
            t = tensor_of(a, tile + gridDim.x, t);
            load_tile(a, t, tile + gridDim.x, next);
        }
        if (x.dtype == kF32)
            add_tile<kF32>(x, a.inf_norm, acc, top);
        else if (x.dtype == kF16)
            add_tile<kF16>(x, a.inf_norm, acc, top);
        else
            add_tile<kBF16>(x, a.inf_norm, acc, top);
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
    constexpr int kBatch = 8;  // in flight
    for (int i = threadIdx.x; i < n; i += kThreads * kBatch) {
        double x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            x[j] = 0.0;
            if (i + j * kThreads < n)
                x[j] = G(partials)[i + j * kThreads];
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            v = inf_norm ? (x[j] > v || x[j] != x[j] ? x[j] : v) : v + x[j];
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
__device__ inline void scale_tile(const ClipArgs &a, int t, int tile, const Tile &x, float c)
{
    constexpr int V = 16 / elem_bytes<DT>;
    void *const p = a.ptr[t];
    const int64_t n = a.numel[t];
    const int64_t from = (int64_t)(tile - a.tile_begin[t]) * (kClipTileBytes / 16) * V;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const Raw<DT, V> raw = {x.w[k].x, x.w[k].y, x.w[k].z, x.w[k].w};
        float f[V];
        unpack<DT, V>(raw, f);
#pragma unroll
        for (int r = 0; r < V; ++r)
            f[r] *= c;
        store_cols<DT, V>(p, from + (int64_t)(k * kThreads + threadIdx.x) * V, n, f);
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
    // from the last tile down: the norm launches read it last, and some of it may still be
    // in the memory-side cache
    int last = a.ntensors - 1;
    for (int i = blockIdx.x; i < a.total_tiles; i += gridDim.x) {
        const int tile = a.total_tiles - 1 - i;
        last = tensor_below(a, tile, last);
        Tile x;
        load_tile(a, last, tile, x);
        if (x.dtype == kF32)
            scale_tile<kF32>(a, last, tile, x, c);
        else if (x.dtype == kF16)
            scale_tile<kF16>(a, last, tile, x, c);
        else
            scale_tile<kBF16>(a, last, tile, x, c);
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
    // More workgroups than run at once clip a long list faster (4096: 1.68 ms for the
    // 580 tensors above, 1024: 1.71), but each first adds up the partial sums, which is all
    // there is to do below the limit (0.52 and 0.51 ms) and counts for a short list
    // (25.6M fp32 in 161 tensors, 6400 tiles: 25.5 and 23.0 us below, 60 and 58 above).
    const int most = a.total_tiles < 16384 ? 1024 : 4096;
    const int groups = a.total_tiles < most ? a.total_tiles : most;
    hipLaunchKernelGGL(clip_kernel, dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace bq
