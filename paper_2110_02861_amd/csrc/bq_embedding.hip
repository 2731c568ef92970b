// Embedding lookup with scaling, its gradient by sorted tokens, and the gradient of
// the stable embedding (lookup, then layer norm).
//
// The gradient of a table's row is the sum of the output gradients of the tokens that
// looked it up.  The tokens are sorted by id (stable, so a row's tokens stay in their
// order and the sums have one order), then every row of the table is written once, by
// the wave that sums its tokens; a row without tokens gets zeros.  Nothing is added
// with floating-point atomics: results are the same bits every time.
//
// A row that many tokens share would be one wave's work, so the sorted list is cut into
// chunks of kChunk positions, and a chunk within one row is summed beforehand by a
// workgroup of its own; the row's wave then adds that sum in its place.
//
// The stable embedding's backward pass uses that all tokens of a row look up the same
// values x, so that xh and rstd are the row's, and the gradient is linear in dy: with S
// the sum of the row's dy and G = S weight,
//   dtable = rstd (G - mean(G) - xh mean(G xh)),
//   dweight = sum over rows of S xh,  dbias = sum over rows of S.
// Nothing of the size of the output is saved by the forward pass, and the backward
// pass normalizes each distinct row once.
#include "bq_ops_device.h"

namespace bq {
namespace {

using namespace dev;

template <int A, int B>
constexpr int vec_of = (elem_bytes<A> == 4 || elem_bytes<B> == 4) ? 4 : 8;

constexpr float kNaN = __builtin_nanf("");

// ---------------------------------------------------------------------------
// Lookup: a wave per token.
// ---------------------------------------------------------------------------

template <int WT, int YT>
__global__ __launch_bounds__(256) void lookup_kernel(const LookupArgs a)
{
    constexpr int V = vec_of<WT, YT>;
    const int lane = threadIdx.x & 63;
    for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < a.count;
         t += (int64_t)gridDim.x * 4) {
        const int64_t id = id_at(a.ids, t, a.ids64);
        const bool known = id >= 0 && id < a.num;
        const void *const from = row_of<WT>(a.table, known ? id : 0, a.dim);
        void *const to = row_of<YT>(a.out, t, a.dim);
        for (int64_t c = lane * V; c < a.dim; c += 64 * V) {
            float x[V];
            load_cols<WT, V>(from, c, a.dim, x);
#pragma unroll
            for (int r = 0; r < V; ++r)
                x[r] = known ? x[r] * a.scale : kNaN;
            store_cols<YT, V>(to, c, a.dim, x);
        }
    }
}

// ---------------------------------------------------------------------------
// Sort of (id, position) pairs by id: radix passes from the low digit up, each
// stable.  At most kSortTiles tiles of the list, one workgroup each; the counts of
// the digits in every tile give each tile its places, and a pass counts the next
// digit as it places the pairs.
// ---------------------------------------------------------------------------

constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 8;                             // per thread and subtile
constexpr int kSubtile = kSortThreads * kSortItems;       // 4096
constexpr int kSortTiles = 256;
constexpr int kMaxBins = 1024;

struct SortShape {
    int bits, passes;   // per pass; bins = 1 << bits
    int64_t tiles, tile;  // tile: elements, kSubtile times a power of two
};
SortShape sort_shape(int64_t count, int64_t num)
{
    SortShape s;
    int bits = 1;
    while ((num >> bits) != 0)  // keys 0 .. num
        ++bits;
    s.passes = bits <= 8 ? 1 : bits <= 20 ? 2 : bits <= 30 ? 3 : 4;
    s.bits = (bits + s.passes - 1) / s.passes;
    s.tile = kSubtile;
    while (s.tile * kSortTiles < count)
        s.tile *= 2;
    s.tiles = (count + s.tile - 1) / s.tile;
    return s;
}

struct SortArgs {
    const void *ids;     // the first pass reads these
    const uint2 *in;     // the others these: {key, position}
    uint2 *out;
    uint32_t *hist;      // passes x tiles x bins
    int64_t count, num, tile, tiles;
    int32_t ids64, bits, pass, passes;
};

// Id as a key: ids outside of the table get the key behind its rows.
__device__ inline uint32_t key_at(const SortArgs &a, int64_t i)
{
    const int64_t id = id_at(a.ids, i, a.ids64);
    return id >= 0 && id < a.num ? (uint32_t)id : (uint32_t)a.num;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a)
{
    __shared__ uint32_t bins[kMaxBins];
    const int n = 1 << a.bits;
    for (int i = threadIdx.x; i < n; i += kSortThreads)
        bins[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * a.tile;
    const int64_t end = begin + a.tile < a.count ? begin + a.tile : a.count;
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&bins[key_at(a, i) & (n - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        a.hist[(int64_t)blockIdx.x * n + i] = bins[i];
        for (int p = 1; p < a.passes; ++p)  // later passes count into these
            a.hist[((int64_t)p * a.tiles + blockIdx.x) * n + i] = 0;
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs a)
{
    __shared__ uint32_t place[kMaxBins];             // next place of each digit
    __shared__ uint32_t count[kSortWaves][kMaxBins];  // of the subtile, per wave
    __shared__ uint32_t sums[kSortWaves];
    const int n = 1 << a.bits;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int shift = a.bits * a.pass;
    const uint32_t mask = (uint32_t)n - 1;
    const uint32_t *const hist = a.hist + (int64_t)a.pass * a.tiles * n;

    // the digits' counts in all tiles, and in the tiles before this one
    const int per = (n + kSortThreads - 1) / kSortThreads;  // 1 or 2 digits per thread
    uint32_t total[2] = {0, 0}, before[2] = {0, 0};
    for (int j = 0; j < per; ++j) {
        const int d = threadIdx.x * per + j;
        if (d < n) {
            for (int64_t t = 0; t < a.tiles; ++t) {
                const uint32_t h = hist[t * n + d];
                total[j] += h;
                before[j] += t < (int64_t)blockIdx.x ? h : 0u;
            }
        }
    }
    const uint32_t mine = total[0] + total[1];
    const uint32_t incl = wave_scan(mine);
    if (lane == 63)
        sums[wave] = incl;
    __syncthreads();
    uint32_t run = incl - mine;
    for (int w = 0; w < wave; ++w)
        run += sums[w];
    for (int j = 0; j < per; ++j) {
        const int d = threadIdx.x * per + j;
        if (d < n)
            place[d] = run + before[j];
        run += total[j];
    }

    const int64_t begin = blockIdx.x * a.tile;
    const int64_t end = begin + a.tile < a.count ? begin + a.tile : a.count;
    const bool last = a.pass + 1 == a.passes;
    uint32_t *const next = a.hist + (int64_t)(a.pass + 1) * a.tiles * n;
    for (int64_t sub = begin; sub < end; sub += kSubtile) {
        __syncthreads();  // place is up to date, count has been read
        for (int i = threadIdx.x; i < kSortWaves * n; i += kSortThreads)
            count[i / n][i % n] = 0;
        __syncthreads();
        uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
        bool live[kSortItems];
        // a wave takes kSortItems rounds of 64 consecutive pairs
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const int64_t i = sub + wave * (64 * kSortItems) + k * 64 + lane;
            live[k] = i < end;
            key[k] = 0;
            pos[k] = 0;
            if (live[k]) {
                if (a.pass == 0) {
                    key[k] = key_at(a, i);
                    pos[k] = (uint32_t)i;
                } else {
                    const uint2 v = a.in[i];
                    key[k] = v.x;
                    pos[k] = v.y;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const uint32_t d = (key[k] >> shift) & mask;
            // the lanes with the same digit
            uint64_t same = __ballot(live[k]);
            for (int b = 0; b < a.bits; ++b) {
                const uint64_t set = __ballot((d >> b) & 1u);
                same &= (d >> b) & 1u ? set : ~set;
            }
            const int leader = same ? __ffsll((unsigned long long)same) - 1 : 0;
            uint32_t old = 0;
            if (live[k] && lane == leader)
                old = atomicAdd(&count[wave][d], (uint32_t)__popcll(same));
            old = __shfl(old, leader);
            rank[k] = old + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        // where each wave's pairs of a digit start
        for (int d = threadIdx.x; d < n; d += kSortThreads) {
            uint32_t at = place[d];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = count[w][d];
                count[w][d] = at;
                at += c;
            }
            place[d] = at;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            if (live[k]) {
                const uint32_t at = count[wave][(key[k] >> shift) & mask] + rank[k];
                a.out[at] = uint2{key[k], pos[k]};
                if (!last)
                    atomicAdd(&next[(at / a.tile) * n + ((key[k] >> (shift + a.bits)) & mask)],
                              1u);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Sums of whole chunks of one row
// ---------------------------------------------------------------------------

constexpr int kChunk = 64;

struct GradArgs {
    LookupGradArgs g;
    const uint2 *sorted;
    float *chunks;     // count / kChunk x dim
    float *partials;   // stable: groups x 2 x dim
    int64_t groups;
    int32_t rows_per_team;
};

template <int YT>
__global__ __launch_bounds__(256) void chunk_kernel(const GradArgs a)
{
    constexpr int V = elem_bytes<YT> == 4 ? 4 : 8;
    __shared__ uint32_t at[kChunk];
    const int64_t n = a.g.count / kChunk;
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const uint32_t key = a.sorted[c * kChunk].x;
        // ids outside of the table and the padding row have no gradient; the stable
        // embedding's padding row still has one in the layer norm's parameters
        if (key != a.sorted[c * kChunk + kChunk - 1].x || (int64_t)key >= a.g.num ||
            (!a.g.table && (int64_t)key == a.g.padding))
            continue;
        __syncthreads();
        if (threadIdx.x < kChunk)
            at[threadIdx.x] = a.sorted[c * kChunk + threadIdx.x].y;
        __syncthreads();
        for (int64_t col = (int64_t)threadIdx.x * V; col < a.g.dim; col += 256 * V) {
            float s[V];
#pragma unroll
            for (int r = 0; r < V; ++r)
                s[r] = 0.0f;
#pragma unroll 8
            for (int i = 0; i < kChunk; ++i) {
                float x[V];
                load_cols<YT, V>(row_of<YT>(a.g.dout, at[i], a.g.dim), col, a.g.dim, x);
#pragma unroll
                for (int r = 0; r < V; ++r)
                    s[r] += x[r];
            }
            store_cols<kF32, V>(a.chunks + c * a.g.dim, col, a.g.dim, s);
        }
    }
}

// ---------------------------------------------------------------------------
// The table's rows.  WAVES waves (a team) hold a row of K vectors of V elements per
// lane; a plain lookup's longer rows are cut into slabs (blockIdx.y).  A team takes
// rows_per_team consecutive rows, whose places in the sorted list its lanes search.
// ---------------------------------------------------------------------------

template <int WT, int YT, int WAVES, int K, bool STABLE>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void rows_kernel(const GradArgs a)
{
    constexpr int V = vec_of<WT, YT>;
    constexpr int kTeams = WAVES == 1 ? 4 : 1;
    __shared__ float scratch[5 * WAVES];
    const int team = WAVES == 1 ? threadIdx.x >> 6 : 0;
    const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t dim = a.g.dim;
    const int64_t c0 = (int64_t)blockIdx.y * (64 * WAVES * K * V);
    const float rn = 1.0f / (float)dim;
    float dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int r = 0; r < V; ++r)
            dw[k][r] = db[k][r] = 0.0f;

    const int rows = a.rows_per_team;
    const int64_t step = (int64_t)gridDim.x * kTeams * rows;
    for (int64_t row0 = ((int64_t)blockIdx.x * kTeams + team) * rows; row0 < a.g.num;
         row0 += step) {
        // lane i: the first position of a key >= row0 + i (the lanes of every wave alike)
        const uint32_t want = (uint32_t)(row0 + (threadIdx.x & 63));
        int64_t lo = 0, hi = a.g.count;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (a.sorted[mid].x < want)
                lo = mid + 1;
            else
                hi = mid;
        }
        for (int i = 0; i < rows && row0 + i < a.g.num; ++i) {
            const int64_t row = row0 + i;
            const int64_t begin = __shfl(lo, i), end = __shfl(lo, i + 1);
            float s[K][V];
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int r = 0; r < V; ++r)
                    s[k][r] = 0.0f;
            const bool padding = row == a.g.padding;
            if (STABLE || !padding) {
                for (int64_t p = begin; p < end;) {
                    float x[K][V];
                    if (p % kChunk == 0 && p + kChunk <= end) {
                        const float *const from = a.chunks + p / kChunk * dim;
#pragma unroll
                        for (int k = 0; k < K; ++k)
                            load_cols<kF32, V>(from, c0 + (int64_t)(k * 64 * WAVES + lane) * V, dim,
                                               x[k]);
                        p += kChunk;
                    } else {
                        const void *const from = row_of<YT>(a.g.dout, a.sorted[p].y, dim);
#pragma unroll
                        for (int k = 0; k < K; ++k)
                            load_cols<YT, V>(from, c0 + (int64_t)(k * 64 * WAVES + lane) * V, dim,
                                             x[k]);
                        ++p;
                    }
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int r = 0; r < V; ++r)
                            s[k][r] += x[k][r];
                }
            }
            void *const to = row_of<WT>(a.g.dtable, row, dim);
            if constexpr (!STABLE) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
#pragma unroll
                    for (int r = 0; r < V; ++r)
                        s[k][r] *= a.g.scale;
                    store_cols<WT, V>(to, c0 + (int64_t)(k * 64 * WAVES + lane) * V, dim, s[k]);
                }
            } else if (begin == end) {
#pragma unroll
                for (int k = 0; k < K; ++k)
                    store_cols<WT, V>(to, (int64_t)(k * 64 * WAVES + lane) * V, dim, s[k]);
            } else {
                // the row's statistics, as in the forward pass
                const void *const from = row_of<WT>(a.g.table, row, dim);
                float x[K][V];
                float sum[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    load_cols<WT, V>(from, (int64_t)(k * 64 * WAVES + lane) * V, dim, x[k]);
#pragma unroll
                    for (int r = 0; r < V; ++r)
                        sum[0] += x[k][r];
                }
                group_sum<1, WAVES>(sum, scratch);
                const float mean0 = sum[0] * rn;
                float two[2] = {0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
#pragma unroll
                    for (int r = 0; r < V; ++r) {
                        x[k][r] = c + r < dim ? x[k][r] - mean0 : 0.0f;
                        two[0] += x[k][r];
                        two[1] = __builtin_fmaf(x[k][r], x[k][r], two[1]);
                    }
                }
                group_sum<2, WAVES>(two, scratch + WAVES);
                const float delta = two[0] * rn;
                float var = two[1] * rn - delta * delta;
                var = var < 0.0f ? 0.0f : var;
                const float rstd = 1.0f / sqrtf(var + a.g.eps);
                float gs[2] = {0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
                    float w[V];
#pragma unroll
                    for (int r = 0; r < V; ++r)
                        w[r] = 1.0f;
                    if (a.g.weight)
                        load_cols<WT, V>(a.g.weight, c, dim, w);
#pragma unroll
                    for (int r = 0; r < V; ++r) {
                        x[k][r] = (x[k][r] - delta) * rstd;
                        dw[k][r] = __builtin_fmaf(s[k][r], x[k][r], dw[k][r]);
                        db[k][r] += s[k][r];
                        s[k][r] *= w[r];
                        gs[0] += s[k][r];
                        gs[1] = __builtin_fmaf(s[k][r], x[k][r], gs[1]);
                    }
                }
                group_sum<2, WAVES>(gs, scratch + 3 * WAVES);
                const float c1 = gs[0] * rn, c2 = gs[1] * rn;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float d[V];
#pragma unroll
                    for (int r = 0; r < V; ++r)
                        d[r] = padding ? 0.0f
                                       : rstd * __builtin_fmaf(-x[k][r], c2, s[k][r] - c1);
                    store_cols<WT, V>(to, (int64_t)(k * 64 * WAVES + lane) * V, dim, d);
                }
            }
        }
    }
    if constexpr (STABLE) {
        if (!a.partials)
            return;
        // a partial row for every team
        float *const out = a.partials + ((int64_t)blockIdx.x * kTeams + team) * 2 * dim;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t c = (int64_t)(k * 64 * WAVES + lane) * V;
            store_cols<kF32, V>(out, c, dim, dw[k]);
            store_cols<kF32, V>(out + dim, c, dim, db[k]);
        }
    }
}

// Workgroups of the stable embedding's rows: few enough that their partial sums are
// a small part of the work.
constexpr int64_t kStableGroups = 512;

struct Layout {
    int64_t pairs_a, pairs_b, hist, chunks, partials, bytes;
};
Layout layout(int64_t count, int64_t num, int64_t dim, bool stable)
{
    const SortShape s = sort_shape(count, num);
    Layout l;
    l.pairs_a = 0;
    l.pairs_b = l.pairs_a + round_up(count * 8, 256);
    l.hist = l.pairs_b + (s.passes > 1 ? round_up(count * 8, 256) : 0);
    l.chunks = l.hist + round_up((int64_t)s.passes * s.tiles * 4 << s.bits, 256);
    l.partials = l.chunks + round_up(count / kChunk * dim * 4, 256);
    l.bytes = l.partials + (stable ? kStableGroups * 4 * 2 * dim * 4 : 0);
    return l;
}

template <int WT, int YT, int WAVES, int K, bool STABLE>
void rows_k(GradArgs &a, hipStream_t stream)
{
    constexpr int V = vec_of<WT, YT>;
    constexpr int kTeams = WAVES == 1 ? 4 : 1;
    const int64_t slab = 64 * WAVES * K * V;
    const int64_t teams = (a.g.num + a.rows_per_team - 1) / a.rows_per_team;
    int64_t groups = (teams + kTeams - 1) / kTeams;
    const int64_t most = STABLE ? kStableGroups : int64_t{1} << 20;
    groups = groups < most ? groups : most;
    a.groups = groups * kTeams;
    hipLaunchKernelGGL((rows_kernel<WT, YT, WAVES, K, STABLE>),
                       dim3((unsigned)groups, STABLE ? 1u : (unsigned)((a.g.dim + slab - 1) / slab)),
                       dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, stream, a);
}

template <int WT, int YT>
hipError_t backward(const LookupGradArgs &g, hipStream_t stream)
{
    const bool stable = g.table != nullptr;
    const SortShape shape = sort_shape(g.count, g.num);
    const Layout l = layout(g.count, g.num, g.dim, stable);
    GradArgs a;
    a.g = g;
    a.sorted = nullptr;
    a.chunks = reinterpret_cast<float *>(g.workspace + l.chunks);
    a.partials = stable && (g.dweight || g.dbias)
                     ? reinterpret_cast<float *>(g.workspace + l.partials) : nullptr;
    a.groups = 0;
    // consecutive rows share a search; small tables need every wave
    a.rows_per_team = g.num >= 65536 ? 8 : g.num >= 16384 ? 4 : 1;

    if (g.count > 0) {
        uint2 *const pa = reinterpret_cast<uint2 *>(g.workspace + l.pairs_a);
        uint2 *const pb = reinterpret_cast<uint2 *>(g.workspace + l.pairs_b);
        SortArgs s;
        s.ids = g.ids;
        s.in = nullptr;
        s.out = pa;
        s.hist = reinterpret_cast<uint32_t *>(g.workspace + l.hist);
        s.count = g.count;
        s.num = g.num;
        s.tile = shape.tile;
        s.tiles = shape.tiles;
        s.ids64 = g.ids64;
        s.bits = shape.bits;
        s.passes = shape.passes;
        s.pass = 0;
        const dim3 grid((unsigned)shape.tiles), block(kSortThreads);
        hipLaunchKernelGGL(sort_count_kernel, grid, block, 0, stream, s);
        for (; s.pass < s.passes; ++s.pass) {
            s.out = s.pass % 2 ? pb : pa;
            hipLaunchKernelGGL(sort_place_kernel, grid, block, 0, stream, s);
            s.in = s.out;
        }
        a.sorted = s.in;
        const int64_t chunks = g.count / kChunk;
        if (chunks > 0)
            hipLaunchKernelGGL(chunk_kernel<YT>, dim3((unsigned)(chunks < 65536 ? chunks : 65536)),
                               dim3(256), 0, stream, a);
    }

    constexpr int kMost = 32 / vec_of<WT, YT>;  // vectors per lane
    const int64_t k = (g.dim + 64 * vec_of<WT, YT> - 1) / (64 * vec_of<WT, YT>);
    if (!stable) {
        if (k <= 1)
            rows_k<WT, YT, 1, 1, false>(a, stream);
        else if (k <= 2)
            rows_k<WT, YT, 1, 2, false>(a, stream);
        else if (k <= 4)
            rows_k<WT, YT, 1, 4, false>(a, stream);
        else
            rows_k<WT, YT, 1, kMost, false>(a, stream);
        return hipGetLastError();
    }
    if (k <= 1)
        rows_k<WT, YT, 1, 1, true>(a, stream);
    else if (k <= 2)
        rows_k<WT, YT, 1, 2, true>(a, stream);
    else if (k <= 4)
        rows_k<WT, YT, 1, 4, true>(a, stream);
    else if (k <= kMost)
        rows_k<WT, YT, 1, kMost, true>(a, stream);
    else if (k <= 2 * kMost)
        rows_k<WT, YT, 4, kMost / 2, true>(a, stream);
    else if (k <= 4 * kMost)
        rows_k<WT, YT, 4, kMost, true>(a, stream);
    else
        rows_k<WT, YT, 16, kMost / 2, true>(a, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partials)
        return e;
    return launch_param_grads(WT, a.partials, a.groups, g.dim, g.dweight, g.dbias, stream);
}

}  // namespace

int64_t lookup_workspace_bytes(int64_t count, int64_t num, int64_t dim, bool stable)
{
    return layout(count, num, dim, stable).bytes;
}

hipError_t launch_lookup(int wt, int yt, const LookupArgs &a, hipStream_t stream)
{
    const int64_t groups = (a.count + 3) / 4;
    const dim3 grid((unsigned)(groups < (1 << 20) ? groups : (1 << 20))), block(256);
    if (wt == kF32 && yt == kF32)
        hipLaunchKernelGGL((lookup_kernel<kF32, kF32>), grid, block, 0, stream, a);
    else if (wt == kF32 && yt == kF16)
        hipLaunchKernelGGL((lookup_kernel<kF32, kF16>), grid, block, 0, stream, a);
    else if (wt == kF32)
        hipLaunchKernelGGL((lookup_kernel<kF32, kBF16>), grid, block, 0, stream, a);
    else if (wt == kF16)
        hipLaunchKernelGGL((lookup_kernel<kF16, kF16>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((lookup_kernel<kBF16, kBF16>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_lookup_backward(int wt, int yt, const LookupGradArgs &a, hipStream_t stream)
{
    if (wt == kF32 && yt == kF32) return backward<kF32, kF32>(a, stream);
    if (wt == kF32 && yt == kF16) return backward<kF32, kF16>(a, stream);
    if (wt == kF32) return backward<kF32, kBF16>(a, stream);
    if (wt == kF16) return backward<kF16, kF16>(a, stream);
    return backward<kBF16, kBF16>(a, stream);
}

}  // namespace bq
