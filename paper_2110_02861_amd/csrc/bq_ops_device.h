// Device helpers of the operators in bq_norm.hip, bq_embedding.hip and bq_clip.hip:
// loads and stores of fp32, fp16 and bf16 elements as fp32 values, and sums over
// a wave and a workgroup.
#pragma once

#include "bq_device.h"
#include "bq_ops.h"

namespace bq {
namespace dev {

template <int DT>
constexpr int elem_bytes = DT == kF32 ? 4 : 2;

// Vectors at any element-aligned address: rows of an odd length start there, and the
// hardware takes them (the compiler is told of the smaller alignment).
// Pointers to them are written out: a template argument would lose the alignment.
typedef uint32_t vu4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t vu4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t vu2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef __attribute__((address_space(1))) vu4_any *gvu4_any;
typedef __attribute__((address_space(1))) vu4_any2 *gvu4_any2;
typedef __attribute__((address_space(1))) vu2_any2 *gvu2_any2;

template <int DT>
__device__ inline float load1(const void *p, int64_t i)
{
    return grad_at<DT>(p, i);
}

__device__ inline uint32_t bits16(float lo, float hi, int dt)
{
    // both roundings are to nearest, ties to even
    if (dt == kF16)
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) |
               (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16;
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) |
           (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
}

template <int DT>
__device__ inline void store1(void *p, int64_t i, float v)
{
    if constexpr (DT == kF32)
        G(static_cast<float *>(p))[i] = v;
    else
        G(static_cast<uint16_t *>(p))[i] = (uint16_t)bits16(v, 0.0f, DT);
}

// V elements (4 or 8) from element i on, as fp32.
template <int DT, int V>
__device__ inline void load_vec(const void *p, int64_t i, float (&o)[V])
{
    static_assert(V == 4 || V == 8, "vector length");
    if constexpr (DT == kF32) {
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            const vu4 w = *(gvu4_any)(uintptr_t)(static_cast<const float *>(p) + i + 4 * h);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                o[4 * h + r] = __uint_as_float(w[r]);
        }
    } else if constexpr (V == 8) {
        const vu4 w = *(gvu4_any2)(uintptr_t)(static_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            o[2 * r] = g16_lo<DT>(w[r]);
            o[2 * r + 1] = g16_hi<DT>(w[r]);
        }
    } else {
        const vu2 w = *(gvu2_any2)(uintptr_t)(static_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            o[2 * r] = g16_lo<DT>(w[r]);
            o[2 * r + 1] = g16_hi<DT>(w[r]);
        }
    }
}

template <int DT, int V>
__device__ inline void store_vec(void *p, int64_t i, const float (&v)[V])
{
    if constexpr (DT == kF32) {
#pragma unroll
        for (int h = 0; h < V / 4; ++h) {
            vu4 w;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                w[r] = __float_as_uint(v[4 * h + r]);
            *(gvu4_any)(uintptr_t)(static_cast<float *>(p) + i + 4 * h) = w;
        }
    } else if constexpr (V == 8) {
        vu4 w;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            w[r] = bits16(v[2 * r], v[2 * r + 1], DT);
        *(gvu4_any2)(uintptr_t)(static_cast<uint16_t *>(p) + i) = w;
    } else {
        vu2 w;
#pragma unroll
        for (int r = 0; r < 2; ++r)
            w[r] = bits16(v[2 * r], v[2 * r + 1], DT);
        *(gvu2_any2)(uintptr_t)(static_cast<uint16_t *>(p) + i) = w;
    }
}

// Elements [c, c + V) of a row of n at p, `fill` behind its end.
template <int DT, int V>
__device__ inline void load_cols(const void *p, int64_t c, int64_t n, float (&o)[V],
                                 float fill = 0.0f)
{
    if (c + V <= n) {
        load_vec<DT, V>(p, c, o);
    } else {
#pragma unroll
        for (int r = 0; r < V; ++r)
            o[r] = c + r < n ? load1<DT>(p, c + r) : fill;
    }
}

template <int DT, int V>
__device__ inline void store_cols(void *p, int64_t c, int64_t n, const float (&v)[V])
{
    if (c + V <= n) {
        store_vec<DT, V>(p, c, v);
    } else {
#pragma unroll
        for (int r = 0; r < V; ++r)
            if (c + r < n)
                store1<DT>(p, c + r, v[r]);
    }
}

// Byte address of row `row` of rows `stride` elements apart.
template <int DT>
__device__ inline const void *row_of(const void *p, int64_t row, int64_t stride)
{
    return static_cast<const char *>(p) + row * stride * elem_bytes<DT>;
}
template <int DT>
__device__ inline void *row_of(void *p, int64_t row, int64_t stride)
{
    return static_cast<char *>(p) + row * stride * elem_bytes<DT>;
}

__device__ inline int64_t id_at(const void *ids, int64_t i, int ids64)
{
    return ids64 ? G(static_cast<const int64_t *>(ids))[i]
                 : (int64_t)G(static_cast<const int32_t *>(ids))[i];
}

template <int CTRL>
__device__ inline float dpp_fadd(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v),
                                                                  CTRL, 0xf, 0xf, true));
}
// Sum over the wave, in every lane: within rows of 16 lanes by DPP, then the four
// rows by the permlane swaps.  The order is fixed.
__device__ inline float wave_sum(float v)
{
    v = dpp_fadd<0xb1>(v);   // quad_perm [1,0,3,2]
    v = dpp_fadd<0x4e>(v);   // quad_perm [2,3,0,1]
    v = dpp_fadd<0x141>(v);  // row_half_mirror
    v = dpp_fadd<0x140>(v);  // row_mirror
    const uint32_t u = __float_as_uint(v);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const uint32_t w = __float_as_uint(v);
    const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Sums of N values over WAVES waves, in every thread; scratch holds N * WAVES
// floats.  Ends without a barrier: the next use of the same scratch needs one before.
template <int N, int WAVES>
__device__ inline void group_sum(float (&v)[N], float *scratch)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                scratch[i * WAVES + wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = scratch[i * WAVES];
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
                s += scratch[i * WAVES + w];
            v[i] = s;
        }
    }
}

}  // namespace dev
}  // namespace bq
