// Embedding lookup with scaling, its gradient by sorted tokens, and the gradient of
// the stable embedding (lookup, then layer norm).
//
// The gradient of a table's row is the sum of the output gradients of the tokens that
// looked it up.  The tokens are sorted by id (stable, so a row's tokens stay in their
// order and the sums have one order), then every row of the table is written once, by
// whoever sums its tokens; a row without tokens gets zeros.  Nothing is added
// with floating-point atomics: results are the same bits every time.
//
// A row that many tokens share would be one workgroup's work, so the sorted list is cut
// into chunks of kChunk positions, and a chunk within one row is summed beforehand by a
// workgroup of its own; the row's sum then takes the chunks' sums in their place.
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
// Lookup.  A wave holds R tokens' rows, K vectors per lane (16 lanes hold short ones;
// longer rows are cut into slabs, blockIdx.y).  The table's rows come from the caches
// where tokens repeat, so reading them counts as much as writing the result: 65536
// tokens, 1600 fp32 to bf16 86 us (420 MB looked up, 210 written), 32768 to fp32 51 us;
// with rows held by workgroups of 7 waves 98 and 67, 4 vectors per lane and 2 slabs 86
// and 71.
// ---------------------------------------------------------------------------

template <int WT, int YT, int TEAM, int K, int R, bool TAIL>
__global__ __launch_bounds__(256) void lookup_kernel(const LookupArgs a)
{
    constexpr int V = vec_of<WT, YT>;
    constexpr int kTeams = teams_of<TEAM>;
    using C = Cols<V, K, TAIL>;
    const int lanes = 256 / kTeams, team = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const C c(a.dim, lane, lanes, (int64_t)blockIdx.y * lanes * K * V);
    const int64_t step = (int64_t)gridDim.x * kTeams * R;
    const bool streams = stream_lookup(a.count * a.dim * elem_bytes<YT>);
    // the next tokens' rows are on their way while this round's are stored
    RawRow<WT, V, K, TAIL> next[R];
    bool next_known[R];
    const auto fetch = [&](int64_t t0) {
        int64_t id[R];
#pragma unroll
        for (int j = 0; j < R; ++j)
            id[j] = id_at(a.ids, t0 + j < a.count ? t0 + j : a.count - 1, a.ids64);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            next_known[j] = id[j] >= 0 && id[j] < a.num;
            load_row<WT, false>(c, row_of<WT>(a.table, next_known[j] ? id[j] : 0, a.dim), next[j]);
        }
    };
    int64_t t0 = ((int64_t)blockIdx.x * kTeams + team) * R;
    if (t0 < a.count)
        fetch(t0);
    for (; t0 < a.count; t0 += step) {
        RawRow<WT, V, K, TAIL> raw[R];
        bool known[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            raw[j] = next[j];
            known[j] = next_known[j];
        }
        if (t0 + step < a.count)
            fetch(t0 + step);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (t0 + j >= a.count)
                break;
            float x[C::kElems];
            unpack<WT, V, K, TAIL>(raw[j], x);
#pragma unroll
            for (int e = 0; e < C::kElems; ++e)
                x[e] = known[j] ? x[e] * a.scale : kNaN;
            if (streams)
                store_row<YT, true>(c, row_of<YT>(a.out, t0 + j, a.dim), x);
            else
                store_row<YT>(c, row_of<YT>(a.out, t0 + j, a.dim), x);
        }
    }
}

// ---------------------------------------------------------------------------
// Sort of (id, position) pairs by id: radix passes from the low digit up, each
// stable.  At most kSortTiles tiles of the list, one workgroup each; the counts of
// the digits in every tile give each tile its places.  (Counting the next pass's digits
// in global memory while pairs are placed saves a launch and loses 8 us by it: the same
// few counters take most of the additions.)
// ---------------------------------------------------------------------------

constexpr int kSortThreads = 512;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 2;                             // per thread and subtile
constexpr int kSubtile = kSortThreads * kSortItems;       // 1024
constexpr int kSortTiles = 128;
constexpr int kMaxBins = 1024;
constexpr int kSmallSort = 4096;  // tokens that one workgroup sorts by itself

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
    s.passes = count <= kSmallSort ? (bits + 7) / 8  // of at most kSmallBins digits
               : bits <= 8 ? 1 : bits <= 20 ? 2 : bits <= 30 ? 3 : 4;
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
    uint32_t *hist;      // tiles x bins, of the pass
    int64_t count, num, tile, tiles;
    int32_t ids64, bits, pass, passes;
};

// Id as a key: ids outside of the table get the key behind its rows.
__device__ inline uint32_t key_at(const SortArgs &a, int64_t i)
{
    const int64_t id = id_at(a.ids, i, a.ids64);
    return id >= 0 && id < a.num ? (uint32_t)id : (uint32_t)a.num;
}

// The pass's digit of the pairs in every tile.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortArgs a)
{
    __shared__ uint32_t bins[kMaxBins];
    const int n = 1 << a.bits, shift = a.bits * a.pass;
    for (int i = threadIdx.x; i < n; i += kSortThreads)
        bins[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * a.tile;
    const int64_t end = begin + a.tile < a.count ? begin + a.tile : a.count;
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const uint32_t key = a.pass == 0 ? key_at(a, i) : a.in[i].x;
        atomicAdd(&bins[(key >> shift) & (n - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSortThreads)
        a.hist[(int64_t)blockIdx.x * n + i] = bins[i];
}

// Rank of a pair among the wave's earlier pairs with its digit d, which `count` holds
// for the wave's earlier rounds and then for this one too.
__device__ inline uint32_t wave_rank(uint32_t d, bool live, int bits, uint32_t *count)
{
    const int lane = threadIdx.x & 63;
    uint64_t same = __ballot(live);  // the lanes with the same digit
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((d >> b) & 1u);
        same &= (d >> b) & 1u ? set : ~set;
    }
    const int leader = same ? __ffsll((unsigned long long)same) - 1 : 0;
    uint32_t old = 0;
    if (live && lane == leader)
        old = atomicAdd(&count[d], (uint32_t)__popcll(same));
    old = __shfl(old, leader);
    return old + (uint32_t)__popcll(same & ((1ull << lane) - 1));
}

// Few tokens: one workgroup, which keeps the pairs on chip from pass to pass.
constexpr int kSmallThreads = 1024;
constexpr int kSmallWaves = kSmallThreads / 64;
constexpr int kSmallItems = 4;
static_assert(kSmallSort == kSmallThreads * kSmallItems, "a pair per thread and item");
constexpr int kSmallBins = 256;
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(const SortArgs a)
{
    __shared__ uint2 pairs[kSmallSort];
    __shared__ uint32_t count[kSmallWaves][kSmallBins];
    __shared__ uint32_t sums[kSmallWaves];
    const int n = 1 << a.bits;
    const uint32_t mask = (uint32_t)n - 1;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint2 pair[kSmallItems];
    bool live[kSmallItems];
#pragma unroll
    for (int k = 0; k < kSmallItems; ++k) {
        const int i = wave * (64 * kSmallItems) + k * 64 + lane;
        live[k] = i < a.count;
        pair[k] = uint2{live[k] ? key_at(a, i) : 0u, (uint32_t)i};
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = a.bits * pass;
        for (int i = threadIdx.x; i < kSmallWaves * kSmallBins; i += kSmallThreads)
            (&count[0][0])[i] = 0;
        __syncthreads();
        uint32_t rank[kSmallItems];
#pragma unroll
        for (int k = 0; k < kSmallItems; ++k)
            rank[k] = wave_rank((pair[k].x >> shift) & mask, live[k], a.bits, count[wave]);
        __syncthreads();
        // where each wave's pairs of a digit start
        uint32_t total = 0;
        if (threadIdx.x < kSmallBins) {
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w)
                total += count[w][threadIdx.x];
        }
        const uint32_t incl = wave_scan(total);
        if (lane == 63)
            sums[wave] = incl;
        __syncthreads();
        if (threadIdx.x < kSmallBins) {
            uint32_t at = incl - total;
            for (int w = 0; w < wave; ++w)
                at += sums[w];
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w) {
                const uint32_t c = count[w][threadIdx.x];
                count[w][threadIdx.x] = at;
                at += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSmallItems; ++k) {
            const uint32_t at = count[wave][(pair[k].x >> shift) & mask] + rank[k];
            if (live[k]) {
                if (pass + 1 == a.passes)
                    a.out[at] = pair[k];
                else
                    pairs[at] = pair[k];
            }
        }
        if (pass + 1 == a.passes)
            return;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSmallItems; ++k)
            if (live[k])
                pair[k] = pairs[wave * (64 * kSmallItems) + k * 64 + lane];
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(const SortArgs a)
{
    __shared__ uint32_t place[kMaxBins];              // next place of each digit
    __shared__ uint32_t all[kMaxBins];                // of each digit, in all tiles
    __shared__ uint32_t count[kSortWaves][kMaxBins];  // of the subtile, per wave
    __shared__ uint32_t sums[kSortWaves];
    const int n = 1 << a.bits;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int shift = a.bits * a.pass;
    const uint32_t mask = (uint32_t)n - 1;
    const uint32_t *const hist = a.hist;

    // the first subtile's pairs, on their way during the count of places; a wave takes
    // kSortItems rounds of 64 consecutive pairs
    const int64_t begin = blockIdx.x * a.tile;
    const int64_t end = begin + a.tile < a.count ? begin + a.tile : a.count;
    uint32_t key[kSortItems], pos[kSortItems];
    bool live[kSortItems];
    const auto fetch = [&](int64_t sub) {
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const int64_t i = sub + wave * (64 * kSortItems) + k * 64 + lane;
            live[k] = i < end;
            key[k] = 0;
            pos[k] = (uint32_t)i;
            if (live[k]) {
                if (a.pass == 0) {
                    key[k] = key_at(a, i);
                } else {
                    const uint2 v = a.in[i];
                    key[k] = v.x;
                    pos[k] = v.y;
                }
            }
        }
    };
    fetch(begin);

    // the digits' counts in all tiles, and in the tiles before this one: where there
    // are fewer digits than threads, the threads of a digit share the tiles
    for (int d = threadIdx.x; d < n; d += kSortThreads)
        place[d] = all[d] = 0;
    __syncthreads();
    const int parts = n < kSortThreads ? kSortThreads >> a.bits : 1;
    for (int d = threadIdx.x & (n < kSortThreads ? n - 1 : kSortThreads - 1); d < n;
         d += kSortThreads) {
        uint32_t total = 0, before = 0;
#pragma unroll 8
        for (int t = (int)threadIdx.x >> (n < kSortThreads ? a.bits : 31); t < (int)a.tiles;
             t += parts) {
            const uint32_t h = hist[(int64_t)t * n + d];
            total += h;
            before += t < (int)blockIdx.x ? h : 0u;
        }
        atomicAdd(&all[d], total);
        atomicAdd(&place[d], before);
    }
    __syncthreads();
    const int per = (n + kSortThreads - 1) / kSortThreads;  // 1 or 2 digits per thread
    uint32_t mine = 0;
    for (int j = 0; j < per; ++j) {
        const int d = threadIdx.x * per + j;
        mine += d < n ? all[d] : 0u;
    }
    const uint32_t incl = wave_scan(mine);
    if (lane == 63)
        sums[wave] = incl;
    __syncthreads();
    uint32_t run = incl - mine;
    for (int w = 0; w < wave; ++w)
        run += sums[w];
    for (int j = 0; j < per; ++j) {
        const int d = threadIdx.x * per + j;
        if (d < n) {
            place[d] += run;
            run += all[d];
        }
    }

    for (int64_t sub = begin; sub < end; sub += kSubtile) {
        __syncthreads();  // place is up to date, count has been read
        for (int i = threadIdx.x; i < kSortWaves << a.bits; i += kSortThreads)
            count[i >> a.bits][i & mask] = 0;
        __syncthreads();
        uint32_t rank[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            rank[k] = wave_rank((key[k] >> shift) & mask, live[k], a.bits, count[wave]);
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
            }
        }
        if (sub + kSubtile < end)
            fetch(sub + kSubtile);
    }
}

// ---------------------------------------------------------------------------
// Sums of whole chunks of one row; and where each row of the table starts in the
// sorted list (a thread per row searches it: all of them wait at the same time).
// ---------------------------------------------------------------------------

constexpr int kChunk = 32;
constexpr int kBatch = 8;  // rows in flight per thread

// Where rows have thousands of tokens, kSpan chunks of one row are added up too: 2^18
// tokens or more (frequent words), or 32 for every row.  Elsewhere another launch (3 us)
// is not repaid.  Backward passes, plain / stable, us, without | with: 500,000 tokens,
// 50257 rows of 128 fp32 184 / 209 | 147 / 175; 60,000 tokens, 300 rows of 1600 fp32
// 131 / 152 | 126 / 132; 131,072 tokens, 50257 rows of 1024 152 / 210 | 145 / 214;
// 65,536 tokens, 50257 rows of 1600 154 / 210 | 160 / 210; 5000 tokens, 50 rows of 512
// 22 / 27 | 24 / 29.
constexpr int kSpan = 32;
bool use_spans(int64_t count, int64_t num)
{
    return count >= (int64_t{1} << 18) || (count >= (int64_t{1} << 15) && count >= 32 * num);
}

// What an earlier launch wrote, read by scalar loads where a wave's lanes agree.
typedef const __attribute__((address_space(4))) uint32_t *cptr;
__device__ inline int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}

struct GradArgs {
    LookupGradArgs g;
    const uint2 *sorted;
    uint32_t *starts;  // num + 1: first position of a key >= i
    float *chunks;     // count / kChunk x dim
    float *spans;      // count / (kChunk kSpan) x dim, or null
    float *partials;   // stable: groups x 2 x dim
    int32_t chunk_groups;
};

template <int YT>
__global__ __launch_bounds__(512) void chunk_kernel(const GradArgs a)
{
    constexpr int V = elem_bytes<YT> == 4 ? 4 : 8;
    __shared__ uint32_t at[kChunk];
    if ((int)blockIdx.x >= a.chunk_groups) {
        const int64_t row = (int64_t)(blockIdx.x - a.chunk_groups) * blockDim.x + threadIdx.x;
        if (row > a.g.num)
            return;
        uint32_t lo = 0, hi = (uint32_t)a.g.count;
        while (lo < hi) {
            const uint32_t mid = lo + ((hi - lo) >> 1);
            if ((int64_t)a.sorted[mid].x < row)
                lo = mid + 1;
            else
                hi = mid;
        }
        a.starts[row] = lo;
        return;
    }
    const int64_t n = a.g.count / kChunk;
    for (int64_t c = blockIdx.x; c < n; c += a.chunk_groups) {
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
        float *const out = a.chunks + c * a.g.dim;
        const int64_t whole = a.g.dim / V * V;
        for (int64_t col = (int64_t)threadIdx.x * V; col < whole; col += blockDim.x * V) {
            float s[V];
#pragma unroll
            for (int r = 0; r < V; ++r)
                s[r] = 0.0f;
            for (int i = 0; i < kChunk; i += kBatch) {
                Raw<YT, V> x[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    x[j] = load_raw<YT, V, false>(row_of<YT>(a.g.dout, at[i + j], a.g.dim), col);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    float f[V];
                    unpack<YT, V>(x[j], f);
#pragma unroll
                    for (int r = 0; r < V; ++r)
                        s[r] += f[r];
                }
            }
            store_vec<kF32, V>(out, col, s);
        }
        const int64_t col = whole + threadIdx.x;
        if (col < a.g.dim) {
            float s = 0.0f;
            for (int i = 0; i < kChunk; ++i)
                s += load1<YT>(row_of<YT>(a.g.dout, at[i], a.g.dim), col);
            out[col] = s;
        }
    }
}

// Sums of kSpan chunks of one row.
__global__ __launch_bounds__(256) void span_kernel(const GradArgs a)
{
    constexpr int64_t kTokens = kChunk * kSpan;
    const int64_t n = a.g.count / kTokens;
    for (int64_t c = blockIdx.x; c < n; c += gridDim.x) {
        const uint32_t key = a.sorted[c * kTokens].x;
        if (key != a.sorted[c * kTokens + kTokens - 1].x || (int64_t)key >= a.g.num ||
            (!a.g.table && (int64_t)key == a.g.padding))
            continue;
        const float *const from = a.chunks + c * kSpan * a.g.dim;
        for (int64_t col = threadIdx.x; col < a.g.dim; col += 256) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < kSpan; ++i)
                s += G(from)[i * a.g.dim + col];
            a.spans[c * a.g.dim + col] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// The table's rows.  A team of lanes holds a row, K vectors of V elements per lane; a
// plain lookup's longer rows are cut into slabs (blockIdx.y).  Teams walk the
// table with the grid, so that frequent rows, which lie together in many
// vocabularies, fall to different workgroups.
// ---------------------------------------------------------------------------

// Adds the first n of N rows of type DT, given by `row` (which is asked for all N), to a
// lane's columns, all in flight at once: most rows have fewer than N tokens (one by one,
// backward passes took: 60,000 tokens, 50257 rows of 64 fp32 61 us, now 48; 16,384 tokens,
// 50257 of 1024 bf16 61, 57; 509 tokens, 1000 of 256 fp32 17.1, 15.5).
template <int DT, int N, int V, int K, bool TAIL, typename Row>
__device__ inline void add_rows(const Cols<V, K, TAIL> &c, float (&s)[Cols<V, K, TAIL>::kElems],
                                uint32_t n, Row row)
{
    RawRow<DT, V, K, TAIL> x[N] = {};
    const void *at[N];
#pragma unroll
    for (int j = 0; j < N; ++j)
        at[j] = row(j);
#pragma unroll
    for (int j = 0; j < N; ++j)
        if ((uint32_t)j < n)
            load_row<DT, false>(c, at[j], x[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float f[Cols<V, K, TAIL>::kElems];
        unpack<DT, V, K, TAIL>(x[j], f);
#pragma unroll
        for (int e = 0; e < Cols<V, K, TAIL>::kElems; ++e)
            s[e] += f[e];
    }
}

template <int WT, int YT, int TEAM, int K, bool STABLE, bool TAIL>
__global__ __launch_bounds__(most_threads<TEAM>) void rows_kernel(const GradArgs a)
{
    constexpr int V = vec_of<WT, YT>;
    constexpr int B = kBatch / K;
    constexpr int kTeams = teams_of<TEAM>;
    using C = Cols<V, K, TAIL>;
    constexpr int E = C::kElems;
    __shared__ float scratch[STABLE && is_group<TEAM> ? 5 * 16 : 1];
    const int lanes = is_group<TEAM> ? blockDim.x : 256 / kTeams;
    const int team = is_group<TEAM> ? 0 : threadIdx.x / (256 / kTeams);
    const int lane = is_group<TEAM> ? threadIdx.x : threadIdx.x % (256 / kTeams);
    const int64_t dim = a.g.dim;
    const C c(dim, lane, lanes, (int64_t)blockIdx.y * lanes * K * V);
    const float rn = 1.0f / (float)dim;
    float dw[E], db[E];
    RawRow<WT, V, K, TAIL> weight;
#pragma unroll
    for (int e = 0; e < E; ++e)
        dw[e] = db[e] = 0.0f;
    if (STABLE && a.g.weight)
        load_row<WT, false>(c, a.g.weight, weight);

    // where a row's tokens are, asked for a round ahead
    const auto places = [&](int64_t row, uint32_t &begin, uint32_t &end) {
        begin = end = 0;
        if (row < a.g.num && (STABLE || row != a.g.padding)) {
            if constexpr (TEAM == kTeam16) {
                begin = a.starts[row];
                end = a.starts[row + 1];
            } else {
                const int64_t at = uniform(row);
                begin = ((cptr)a.starts)[at];
                end = ((cptr)a.starts)[at + 1];
            }
        }
    };
    uint32_t next_begin, next_end;
    places((int64_t)blockIdx.x * kTeams + team, next_begin, next_end);
    // (a workgroup's teams leave together, for the sums over the wave)
    for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < a.g.num;
         row0 += (int64_t)gridDim.x * kTeams) {
        const int64_t row = row0 + team;
        const bool exists = row < a.g.num;
        const bool padding = row == a.g.padding;
        const uint32_t begin = next_begin, end = next_end;
        places(row + (int64_t)gridDim.x * kTeams, next_begin, next_end);
        float s[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
            s[e] = 0.0f;
        // tokens up to the first whole chunk, the chunks, and the tokens behind them
        const uint32_t first = (begin + kChunk - 1) / kChunk, last = end / kChunk;
        const bool chunks = first < last;
        const auto token = [&](uint32_t p) {
            const uint32_t at = TEAM == kTeam16 ? a.sorted[p].y
                                                : ((cptr)a.sorted)[2 * (uint64_t)p + 1];
            return row_of<YT>(a.g.dout, at, dim);
        };
        const auto tokens = [&](uint32_t p, uint32_t to) {
            for (; p + B <= to; p += B)
                add_rows<YT, B>(c, s, B, [&](int j) { return token(p + j); });
            if (p < to)
                add_rows<YT, B>(c, s, to - p, [&](int j) { return token(min(p + j, to - 1)); });
        };
        const bool some = begin != end;
        RawRow<WT, V, K, TAIL> table;
        if constexpr (STABLE) {
            if (TEAM == kTeam16 ? __any(some) : some)
                load_row<WT, false>(c, row_of<WT>(a.g.table, exists ? row : 0, dim), table);
        }
        tokens(begin, chunks ? first * kChunk : end);
        if (chunks) {
            const auto sums = [&](const float *parts, uint32_t i, uint32_t to) {
                const auto part = [&](uint32_t k) {
                    return (const void *)(parts + (int64_t)k * dim);
                };
                for (; i + B <= to; i += B)
                    add_rows<kF32, B>(c, s, B, [&](int j) { return part(i + j); });
                if (i < to)
                    add_rows<kF32, B>(c, s, to - i, [&](int j) { return part(min(i + j, to - 1)); });
            };
            const uint32_t span = (first + kSpan - 1) / kSpan, past = last / kSpan;
            const bool spans = a.spans && span < past;
            sums(a.chunks, first, spans ? span * kSpan : last);
            if (spans) {
                sums(a.spans, span, past);
                sums(a.chunks, past * kSpan, last);
            }
            tokens(last * kChunk, end);
        }
        void *const to = row_of<WT>(a.g.dtable, exists ? row : 0, dim);
        if constexpr (!STABLE) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                s[e] *= a.g.scale;
            if (exists)
                store_row<WT>(c, to, s);
        } else {
            if (TEAM == kTeam16 ? !__any(some) : !some) {
                if (exists)
                    store_row<WT>(c, to, s);
                continue;
            }
            // the row's statistics, as in the forward pass
            float x[E];
            float sum[1] = {0.0f};
            unpack<WT, V, K, TAIL>(table, x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                sum[0] += x[e];
            team_sum<TEAM, 1>(sum, scratch);
            const float mean0 = sum[0] * rn;
            float two[2] = {0.0f, 0.0f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = c.valid(e) ? x[e] - mean0 : 0.0f;
                two[0] += x[e];
                two[1] = __builtin_fmaf(x[e], x[e], two[1]);
            }
            team_sum<TEAM, 2>(two, scratch + 16);
            const float delta = two[0] * rn;
            float var = two[1] * rn - delta * delta;
            var = var < 0.0f ? 0.0f : var;
            const float rstd = 1.0f / sqrtf(var + a.g.eps);
            float gs[2] = {0.0f, 0.0f};
            float w[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
                w[e] = 1.0f;
            if (a.g.weight)
                unpack<WT, V, K, TAIL>(weight, w);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = (x[e] - delta) * rstd;
                if (some)
                    dw[e] = __builtin_fmaf(s[e], x[e], dw[e]);
                db[e] += s[e];
                s[e] *= w[e];
                gs[0] += s[e];
                gs[1] = __builtin_fmaf(s[e], x[e], gs[1]);
            }
            team_sum<TEAM, 2>(gs, scratch + 48);
            const float c1 = gs[0] * rn, c2 = gs[1] * rn;
#pragma unroll
            for (int e = 0; e < E; ++e)
                s[e] = padding || !some ? 0.0f : rstd * __builtin_fmaf(-x[e], c2, s[e] - c1);
            if (exists)
                store_row<WT>(c, to, s);
        }
    }
    if constexpr (STABLE) {
        if (a.partials)
            leave_partials<TEAM>(c, dw, db, dim, a.partials + (int64_t)blockIdx.x * 2 * dim);
    }
}

// Workgroups of a plain lookup's rows, at most.  Walking the table evens out rows of
// many tokens; the whole backward pass, 50257 rows of 1600 fp32, 65536 tokens: 178 us at
// 1024, 158 at 2048, 151 at 4096 and at 8192, 176 with one for every row.
constexpr int64_t kRowGroups = 8192;
// Of the stable embedding's, of which each also leaves a partial row: the same 258 us at
// 512, 224 at 768, 212 at 1024, 224 at 1280; shorter rows take twice as many.  The rows and
// the partial rows' sums, 32768 tokens, 50257 rows of fp32, 1024 | 2048: 256 columns 30.2 |
// 30.9 us, 512 64 | 53, 768 78 | 66, 1024 92.5 | 91.9; 60,000 tokens on 4000 rows of 768, of
// which a workgroup has two or four, 44.6 | 46.8.
constexpr int64_t stable_groups(int64_t dim) { return dim <= 1024 ? 2048 : 1024; }

struct Layout {
    int64_t pairs_a, pairs_b, hist, starts, chunks, spans, partials, bytes;
};
Layout layout(int64_t count, int64_t num, int64_t dim, bool stable)
{
    const SortShape s = sort_shape(count, num);
    Layout l;
    l.pairs_a = 0;
    l.pairs_b = l.pairs_a + round_up(count * 8, 256);
    l.hist = l.pairs_b + (s.passes > 1 ? round_up(count * 8, 256) : 0);
    l.starts = l.hist + round_up(s.tiles * 4 << s.bits, 256);
    l.chunks = l.starts + round_up((num + 1) * 4, 256);
    l.spans = l.chunks + round_up(count / kChunk * dim * 4, 256);
    l.partials = l.spans + (use_spans(count, num)
                                ? round_up(count / (kChunk * kSpan) * dim * 4, 256) : 0);
    // of every workgroup, each with at least one row of the table
    const int64_t groups = num < stable_groups(dim) ? num : stable_groups(dim);
    l.bytes = l.partials + (stable ? groups * 2 * dim * 4 : 0);
    return l;
}

// Slabs of `slab` columns (a multiple of a vector) of the row's whole vectors; at least
// one, for the elements behind them.
template <int V>
unsigned slabs_of(int64_t dim, int64_t slab)
{
    const int64_t n = (dim / V * V + slab - 1) / slab;
    return (unsigned)(n < 1 ? 1 : n);
}

template <int WT, int YT, int TEAM, int K, bool STABLE>
int64_t rows_k(const GradArgs &a, int threads, hipStream_t stream)
{
    constexpr int V = vec_of<WT, YT>;
    constexpr int kTeams = teams_of<TEAM>;
    const int64_t most = STABLE ? stable_groups(a.g.dim) : kRowGroups;
    int64_t groups = (a.g.num + kTeams - 1) / kTeams;
    groups = groups < most ? groups : most;
    const dim3 grid((unsigned)groups, slabs_of<V>(a.g.dim, (int64_t)threads / kTeams * K * V));
    const dim3 block((unsigned)threads);
    if (a.g.dim % V == 0)
        hipLaunchKernelGGL((rows_kernel<WT, YT, TEAM, K, STABLE, false>), grid, block, 0, stream,
                           a);
    else
        hipLaunchKernelGGL((rows_kernel<WT, YT, TEAM, K, STABLE, true>), grid, block, 0, stream, a);
    return groups;
}

// Threads of a group team for rows of `vectors` vectors, K to a lane.
int threads_of(int64_t vectors, int k = 1)
{
    return (int)((vectors + 64 * k - 1) / (64 * k) * 64);
}

// The team that holds a row, and the launch; returns the workgroups.  The stable
// embedding's rows want few waves at a barrier, the plain sums many loads in flight for
// the same tokens: backward passes of 65536 tokens, 50257 rows of 1600 fp32 (400 vectors),
// in us:  one vector per lane, 7 waves: plain 151, stable 257;  4 waves, 2: 166, 212;
// 2 waves, 4: 192, 230;  a wave, 8: 235, 266.
template <int WT, int YT, bool STABLE>
int64_t rows(const GradArgs &a, hipStream_t stream)
{
    constexpr int V = vec_of<WT, YT>;
    const int64_t vectors = a.g.dim / V;
    if (vectors <= 16)
        return rows_k<WT, YT, kTeam16, 1, STABLE>(a, 256, stream);
    if (vectors <= 64)
        return rows_k<WT, YT, kTeamWave, 1, STABLE>(a, 256, stream);
    if constexpr (STABLE) {
        if (vectors <= 256)
            return rows_k<WT, YT, kTeamGroup4, 1, true>(a, threads_of(vectors), stream);
        if (vectors <= 512)
            return rows_k<WT, YT, kTeamGroup4, 2, true>(a, threads_of(vectors, 2), stream);
        if (vectors <= 1024)
            return rows_k<WT, YT, kTeamGroup4, 4, true>(a, threads_of(vectors, 4), stream);
        if constexpr (V == 4) {
            if (vectors > 2048)
                return rows_k<WT, YT, kTeamGroup, 4, true>(a, 1024, stream);
        }
        return rows_k<WT, YT, kTeamGroup, 2, true>(a, threads_of(vectors, 2), stream);
    } else {
        if (vectors <= 1024)
            return rows_k<WT, YT, kTeamGroup, 1, false>(a, threads_of(vectors), stream);
        return rows_k<WT, YT, kTeamGroup, 2, false>(a, 1024, stream);
    }
}

template <int WT, int YT, int TEAM, int K, int R>
void lookup_k(const LookupArgs &a, hipStream_t stream)
{
    constexpr int V = vec_of<WT, YT>;
    const int64_t per = teams_of<TEAM> * R;
    const int64_t groups = (a.count + per - 1) / per;
    const dim3 grid((unsigned)(groups < (1 << 16) ? groups : (1 << 16)),
                    slabs_of<V>(a.dim, (int64_t)256 / teams_of<TEAM> * K * V)), block(256);
    if (a.dim % V == 0)
        hipLaunchKernelGGL((lookup_kernel<WT, YT, TEAM, K, R, false>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((lookup_kernel<WT, YT, TEAM, K, R, true>), grid, block, 0, stream, a);
}

template <int WT, int YT>
hipError_t lookup(const LookupArgs &a, hipStream_t stream)
{
    const int64_t vectors = a.dim / vec_of<WT, YT>;
    if (vectors <= 16)
        lookup_k<WT, YT, kTeam16, 1, 4>(a, stream);
    else if (vectors <= 64)
        lookup_k<WT, YT, kTeamWave, 1, 4>(a, stream);
    else if (vectors <= 128)
        lookup_k<WT, YT, kTeamWave, 2, 2>(a, stream);
    else if (vectors <= 256)
        lookup_k<WT, YT, kTeamWave, 4, 1>(a, stream);
    else
        lookup_k<WT, YT, kTeamWave, 8, 1>(a, stream);
    return hipGetLastError();
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
    a.starts = reinterpret_cast<uint32_t *>(g.workspace + l.starts);
    a.chunks = reinterpret_cast<float *>(g.workspace + l.chunks);
    a.spans = use_spans(g.count, g.num) ? reinterpret_cast<float *>(g.workspace + l.spans) : nullptr;
    a.partials = stable && (g.dweight || g.dbias)
                     ? reinterpret_cast<float *>(g.workspace + l.partials) : nullptr;

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
        if (g.count <= kSmallSort) {
            hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(kSmallThreads), 0, stream, s);
            s.in = s.out;
        } else {
            for (; s.pass < s.passes; ++s.pass) {
                s.out = s.pass % 2 ? pb : pa;
                hipLaunchKernelGGL(sort_count_kernel, grid, block, 0, stream, s);
                hipLaunchKernelGGL(sort_place_kernel, grid, block, 0, stream, s);
                s.in = s.out;
            }
        }
        a.sorted = s.in;
    }
    const int64_t chunks = g.count / kChunk;
    a.chunk_groups = (int32_t)(chunks < 65536 ? chunks : 65536);
    // a thread for every vector of a row, where there are so many
    const int64_t vectors = g.dim / (elem_bytes<YT> == 4 ? 4 : 8);
    const int threads = vectors < 64 ? 64 : vectors < 512 ? threads_of(vectors) : 512;
    hipLaunchKernelGGL(chunk_kernel<YT>,
                       dim3((unsigned)(a.chunk_groups + (g.num + threads) / threads)),
                       dim3((unsigned)threads), 0, stream, a);
    if (a.spans) {
        const int64_t spans = g.count / (kChunk * kSpan);
        hipLaunchKernelGGL(span_kernel, dim3((unsigned)(spans < 65536 ? spans : 65536)), dim3(256),
                           0, stream, a);
    }

    if (!stable) {
        rows<WT, YT, false>(a, stream);
        return hipGetLastError();
    }
    const int64_t groups = rows<WT, YT, true>(a, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partials)
        return e;
    return launch_param_grads(WT, a.partials, groups, g.dim, g.dweight, g.dbias, stream);
}

}  // namespace

int64_t lookup_workspace_bytes(int64_t count, int64_t num, int64_t dim, bool stable)
{
    return layout(count, num, dim, stable).bytes;
}

hipError_t launch_lookup(int wt, int yt, const LookupArgs &a, hipStream_t stream)
{
    if (wt == kF32 && yt == kF32) return lookup<kF32, kF32>(a, stream);
    if (wt == kF32 && yt == kF16) return lookup<kF32, kF16>(a, stream);
    if (wt == kF32) return lookup<kF32, kBF16>(a, stream);
    if (wt == kF16) return lookup<kF16, kF16>(a, stream);
    return lookup<kBF16, kBF16>(a, stream);
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
