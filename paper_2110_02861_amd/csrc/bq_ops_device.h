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
    if (dt == kF16) {
        // the values as they are in fp32: a product would otherwise be rounded once, to
        // fp16, where the compiler finds an instruction for it, and twice elsewhere
        asm("" : "+v"(lo), "+v"(hi));
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) |
               (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16;
    }
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

// V elements (4 or 8) as they are in memory.
template <int DT, int V>
struct Raw {
    static_assert(V == 4 || V == 8, "vector length");
    static constexpr int kWords = V * elem_bytes<DT> / 4;
    uint32_t w[kWords];
};

template <int DT, int V>
__device__ inline void unpack(const Raw<DT, V> &x, float (&o)[V])
{
#pragma unroll
    for (int i = 0; i < Raw<DT, V>::kWords; ++i) {
        if constexpr (DT == kF32) {
            o[i] = __uint_as_float(x.w[i]);
        } else {
            o[2 * i] = g16_lo<DT>(x.w[i]);
            o[2 * i + 1] = g16_hi<DT>(x.w[i]);
        }
    }
}

// From element i on, NT: with the non-temporal hint.
template <int DT, int V, bool NT>
__device__ inline Raw<DT, V> load_raw(const void *p, int64_t i)
{
    Raw<DT, V> x;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p) + i * elem_bytes<DT>;
    if constexpr (Raw<DT, V>::kWords == 2) {
        const gvu2_any2 q = (gvu2_any2)at;
        const vu2 v = NT ? __builtin_nontemporal_load(q) : *q;
        x.w[0] = v.x;
        x.w[1] = v.y;
    } else {
#pragma unroll
        for (int h = 0; h < Raw<DT, V>::kWords / 4; ++h) {
            vu4 v;
            if constexpr (DT == kF32) {
                const gvu4_any q = (gvu4_any)(at + 16 * h);
                v = NT ? __builtin_nontemporal_load(q) : *q;
            } else {
                const gvu4_any2 q = (gvu4_any2)(at + 16 * h);
                v = NT ? __builtin_nontemporal_load(q) : *q;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x.w[4 * h + r] = v[r];
        }
    }
    return x;
}

// V elements from element i on, as fp32.
template <int DT, int V>
__device__ inline void load_vec(const void *p, int64_t i, float (&o)[V])
{
    unpack<DT, V>(load_raw<DT, V, false>(p, i), o);
}

// V elements from element i on, NT: with the non-temporal hint.
template <int DT, int V, bool NT = false>
__device__ inline void store_vec(void *p, int64_t i, const float (&v)[V])
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p) + i * elem_bytes<DT>;
    uint32_t w[Raw<DT, V>::kWords];
#pragma unroll
    for (int k = 0; k < Raw<DT, V>::kWords; ++k) {
        if constexpr (DT == kF32)
            w[k] = __float_as_uint(v[k]);
        else
            w[k] = bits16(v[2 * k], v[2 * k + 1], DT);
    }
    if constexpr (Raw<DT, V>::kWords == 2) {
        const vu2 x = {w[0], w[1]};
        if constexpr (NT)
            __builtin_nontemporal_store(x, (gvu2_any2)at);
        else
            *(gvu2_any2)at = x;
    } else {
#pragma unroll
        for (int h = 0; h < Raw<DT, V>::kWords / 4; ++h) {
            const vu4 x = {w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]};
            if constexpr (DT == kF32) {
                if constexpr (NT)
                    __builtin_nontemporal_store(x, (gvu4_any)(at + 16 * h));
                else
                    *(gvu4_any)(at + 16 * h) = x;
            } else {
                if constexpr (NT)
                    __builtin_nontemporal_store(x, (gvu4_any2)(at + 16 * h));
                else
                    *(gvu4_any2)(at + 16 * h) = x;
            }
        }
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

// Whether a lookup's results, of so many bytes, are stored with the non-temporal hint:
// above what the L2 caches hold together (32 MB) they would push the table out of them
// and of the memory-side cache.  Lookups of 1600 fp32 that follow each other, us, without
// / with: 4096 tokens (26 MB) 9.6 / 8.7, 8192 17.3 / 14.6, 32768 56 / 47 (with the layer
// norm 68 / 53; on three tables in turn 69 / 58).  Whoever reads them next loses 1 to 2 us
// by it, so short ones are stored as usual.  Behind what flushes the memory-side cache (a
// 1 GB fill here, the backward pass in training) the table's rows come from memory anyway
// and the hint counts for little: 32768 69 / 66 (with the layer norm 83 / 81), 65536 to
// bf16 96 / 103 (80 / 62 where they follow each other).
__device__ inline bool stream_lookup(int64_t bytes) { return bytes > (int64_t{32} << 20); }

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

// A team of lanes holds a row: 16 lanes (four teams to a wave), a wave (four to a
// workgroup), or a workgroup of as many waves as the row needs, up to 4 or up to 16 (of
// which each has half as many registers).
enum { kTeam16 = 0, kTeamWave = 1, kTeamGroup4 = 2, kTeamGroup = 3 };
template <int TEAM>
constexpr int teams_of = TEAM == kTeam16 ? 16 : TEAM == kTeamWave ? 4 : 1;
template <int TEAM>
constexpr bool is_group = TEAM == kTeamGroup4 || TEAM == kTeamGroup;
template <int TEAM>
constexpr int most_threads = TEAM == kTeamGroup ? 1024 : 256;

// Sums of N values over the team, in every lane; scratch (group teams): 16 floats per
// value.  One barrier, before the results are read: the next use of the same scratch
// needs another barrier before it.
template <int TEAM, int N>
__device__ inline void team_sum(float (&v)[N], float *scratch)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (TEAM == kTeam16) {
            v[i] = dpp_fadd<0xb1>(v[i]);
            v[i] = dpp_fadd<0x4e>(v[i]);
            v[i] = dpp_fadd<0x141>(v[i]);
            v[i] = dpp_fadd<0x140>(v[i]);
        } else {
            v[i] = wave_sum(v[i]);
        }
    }
    if constexpr (is_group<TEAM>) {
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                scratch[i * 16 + wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = scratch[i * 16];
            for (int w = 1; w < waves; ++w)
                s += scratch[i * 16 + w];
            v[i] = s;
        }
    }
}

// The columns of a row of n that a lane of its team holds: K vectors of V elements,
// `stride` columns apart, of the row's whole vectors, and with TAIL (n no multiple of V)
// one of the fewer than V elements behind those.  Every access is a vector or an
// element under one condition without an alternative: with one, lanes that are past the
// row's end would write registers that loads of the others are still to fill, and wait
// for each load in turn (32768 x 1600 in bf16: 71 us against 45).
template <int V, int K, bool TAIL>
struct Cols {
    static constexpr int kElems = K * V + (TAIL ? 1 : 0);
    uint32_t c0, stride, whole, tail;
    bool has_tail;

    __device__ Cols(int64_t n, int lane, int lanes, int64_t from = 0)
    {
        c0 = (uint32_t)(from + lane * V);
        stride = (uint32_t)(lanes * V);
        whole = (uint32_t)(n / V * V);
        tail = whole + lane;
        has_tail = TAIL && from == 0 && tail < (uint32_t)n;  // the first slab's
    }
    __device__ uint32_t col(int k) const { return c0 + k * stride; }
    __device__ bool has(int k) const { return col(k) < whole; }
    // whether element e of the lane is one of the row
    __device__ bool valid(int e) const { return e < K * V ? has(e / V) : has_tail; }
};

template <int DT, int V, int K, bool TAIL>
struct RawRow {
    Raw<DT, V> v[K];
    uint32_t t;
};

template <int DT, bool NT, int V, int K, bool TAIL>
__device__ inline void load_row(const Cols<V, K, TAIL> &c, const void *row,
                                RawRow<DT, V, K, TAIL> &x)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < Raw<DT, V>::kWords; ++i)
            x.v[k].w[i] = 0;
        if (c.has(k))
            x.v[k] = load_raw<DT, V, NT>(row, c.col(k));
    }
    if constexpr (TAIL) {
        x.t = 0;
        if (c.has_tail) {
            if constexpr (DT == kF32)
                x.t = G(static_cast<const uint32_t *>(row))[c.tail];
            else
                x.t = G(static_cast<const uint16_t *>(row))[c.tail];
        }
    }
}

template <int DT, int V, int K, bool TAIL>
__device__ inline void unpack(const RawRow<DT, V, K, TAIL> &x, float (&o)[K * V + (TAIL ? 1 : 0)])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[V];
        unpack<DT, V>(x.v[k], f);
#pragma unroll
        for (int r = 0; r < V; ++r)
            o[k * V + r] = f[r];
    }
    if constexpr (TAIL)
        o[K * V] = DT == kF32 ? __uint_as_float(x.t) : g16_lo<DT>(x.t);
}

template <int DT, int V, int K, bool TAIL>
__device__ inline void load_floats(const Cols<V, K, TAIL> &c, const void *row,
                                   float (&o)[K * V + (TAIL ? 1 : 0)])
{
    RawRow<DT, V, K, TAIL> x;
    load_row<DT, false>(c, row, x);
    unpack<DT, V, K, TAIL>(x, o);
}

template <int DT, bool NT = false, int V, int K, bool TAIL>
__device__ inline void store_row(const Cols<V, K, TAIL> &c, void *row,
                                 const float (&v)[K * V + (TAIL ? 1 : 0)])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float f[V];
#pragma unroll
        for (int r = 0; r < V; ++r)
            f[r] = v[k * V + r];
        if (c.has(k))
            store_vec<DT, V, NT>(row, c.col(k), f);
    }
    if constexpr (TAIL) {
        if (c.has_tail)
            store1<DT>(row, c.tail, v[K * V]);
    }
}

// Leaves a workgroup's sums per column of two gradients in out[2][n]: its only team's, or
// its teams' in order, a vector per lane at a time.  All threads call it.
template <int TEAM, int V, int K, bool TAIL>
__device__ inline void leave_partials(const Cols<V, K, TAIL> &c,
                                      const float (&dw)[K * V + (TAIL ? 1 : 0)],
                                      const float (&db)[K * V + (TAIL ? 1 : 0)], int64_t n,
                                      float *out)
{
    if constexpr (is_group<TEAM>) {
        store_row<kF32>(c, out, dw);
        store_row<kF32>(c, out + n, db);
    } else {
        constexpr int kTeams = teams_of<TEAM>, kLanes = 256 / kTeams;
        __shared__ float join[2][V][256];
        const auto add = [&](int which, int r, int lane) {
            float t = join[which][r][lane];
            for (int k = 1; k < kTeams; ++k)
                t += join[which][r][k * kLanes + lane];
            return t;
        };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < V; ++r) {
                join[0][r][threadIdx.x] = dw[k * V + r];
                join[1][r][threadIdx.x] = db[k * V + r];
            }
            __syncthreads();
            const uint32_t first = k * c.stride;
            const uint32_t cols = first >= c.whole ? 0 : min(c.stride, c.whole - first);
            for (uint32_t i = threadIdx.x; i < 2 * cols; i += 256) {
                const int which = i >= cols;
                const uint32_t col = i - which * cols;
                out[which * n + first + col] = add(which, col % V, col / V);
            }
        }
        if constexpr (TAIL) {
            __syncthreads();
            join[0][0][threadIdx.x] = dw[K * V];
            join[1][0][threadIdx.x] = db[K * V];
            __syncthreads();
            const uint32_t cols = (uint32_t)n - c.whole;
            if (threadIdx.x < 2 * cols) {
                const int which = threadIdx.x >= cols;
                const uint32_t col = threadIdx.x - which * cols;
                out[which * n + c.whole + col] = add(which, 0, col);
            }
        }
    }
}

}  // namespace dev
}  // namespace bq
