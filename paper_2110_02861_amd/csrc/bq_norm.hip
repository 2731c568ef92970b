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
// Forward.  A team takes R consecutive rows at a time, K vectors of V elements per lane
// and row; it keeps its columns of the parameters in registers and walks the rows with
// the grid, the next rows' loads in flight.  HBM bounds it: 2 bytes per element each way
// in 16 bits.
//
// The team for a row, measured (us, buffers larger than the memory-side cache; a wave
// with K vectors per lane, 4 waves, or one vector per lane in as many waves as needed):
//   32768 x 1600 bf16 (200 vectors)  wave, 4: 46   4 waves, 1: 57   2: 49
//   32768 x 1024 bf16 (128)          wave, 2: 27   4 waves, 1: 31   2: 28
//   16384 x 4096 bf16 (512)          wave, 8: 61   4 waves, 2: 57   4: 54   8 waves, 1: 63
//    4096 x 8192 bf16 (1024)         4 waves, 4: 29   8: 37         16 waves, 1: 43
// A row's own wave needs no barrier; above 4 vectors per lane its registers cost more.
// Looked-up rows of up to 512 vectors are a wave's with 8 all the same.  32768 tokens,
// results streamed past the caches, calls that follow each other / behind a 1 GB fill
// that flushes the memory-side cache:
//   1600 fp32 (400 vectors)            wave, 8: 53 / 81   4 waves, 4: 50 / 72
//   1300 fp32                                   45 / 69               43 / 62
//   2000 fp32 to bf16                           49 / 77               47 / 69
// On three tables in turn both take 58 with 1600 fp32.
// ---------------------------------------------------------------------------

template <int XT, int PT, int YT, bool GATHER, int TEAM, int K, int R, bool TAIL>
__global__ __launch_bounds__(most_threads<TEAM>) void norm_forward_kernel(const NormArgs a)
{
    constexpr int V = vec_of<XT, YT>;
    constexpr int kTeams = teams_of<TEAM>;
    using C = Cols<V, K, TAIL>;
    constexpr int E = C::kElems;
    __shared__ float scratch[is_group<TEAM> ? 3 * R * 16 : 1];
    const int lanes = is_group<TEAM> ? blockDim.x : 256 / kTeams;
    const int team = is_group<TEAM> ? 0 : threadIdx.x / (256 / kTeams);
    const int lane = is_group<TEAM> ? threadIdx.x : threadIdx.x % (256 / kTeams);
    const int64_t n = a.cols;
    const C c(n, lane, lanes);
    const float rn = 1.0f / (float)n;
    const bool streams = GATHER && stream_lookup(a.rows * n * elem_bytes<YT>);
    RawRow<PT, V, K, TAIL> pw, pb;
    if (a.weight)
        load_row<PT, false>(c, a.weight, pw);
    if (a.bias)
        load_row<PT, false>(c, a.bias, pb);
    // the next round's rows are on their way while this one's are worked on
    RawRow<XT, V, K, TAIL> next[R];
    bool next_known[R];
    const auto fetch = [&](int64_t group) {
        const int64_t row0 = (group * kTeams + team) * R;
        int64_t from[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            from[j] = row0 + j < a.rows ? row0 + j : a.rows - 1;
            if constexpr (GATHER)
                from[j] = id_at(a.ids, from[j], a.ids64);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            next_known[j] = true;
            if constexpr (GATHER) {
                next_known[j] = from[j] >= 0 && from[j] < a.table_rows;
                from[j] = next_known[j] ? from[j] : 0;
            }
            load_row<XT, !GATHER>(c, row_of<XT>(a.x, from[j], a.x_stride), next[j]);
        }
    };
    // (all of a workgroup's rounds are its teams' rounds, for the sums over a wave; a
    // round's sums go to scratch behind a barrier that follows their last reading)
    const int64_t groups = (a.rows + kTeams * R - 1) / (kTeams * R);
    fetch(blockIdx.x);
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t row0 = (group * kTeams + team) * R;
        RawRow<XT, V, K, TAIL> raw[R];
        bool known[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            raw[j] = next[j];
            known[j] = next_known[j];
        }
        float x[R][E];
        float sum[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            sum[j] = 0.0f;
            unpack<XT, V, K, TAIL>(raw[j], x[j]);
#pragma unroll
            for (int e = 0; e < E; ++e)
                sum[j] += x[j][e];
        }
        if (group + gridDim.x < groups)
            fetch(group + gridDim.x);
        team_sum<TEAM, R>(sum, scratch);
        float two[2 * R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float mean0 = sum[j] * rn;
            two[2 * j] = two[2 * j + 1] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[j][e] = c.valid(e) ? x[j][e] - mean0 : 0.0f;
                two[2 * j] += x[j][e];
                two[2 * j + 1] = __builtin_fmaf(x[j][e], x[j][e], two[2 * j + 1]);
            }
        }
        team_sum<TEAM, 2 * R>(two, scratch + R * 16);
        float w[E], b[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            w[e] = 1.0f;
            b[e] = 0.0f;
        }
        if (a.weight)
            unpack<PT, V, K, TAIL>(pw, w);
        if (a.bias)
            unpack<PT, V, K, TAIL>(pb, b);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = row0 + j;
            if (row >= a.rows)
                break;
            const float delta = two[2 * j] * rn;
            float var = two[2 * j + 1] * rn - delta * delta;
            var = var < 0.0f ? 0.0f : var;
            const float rstd = 1.0f / sqrtf(var + a.eps);
            if (a.mean && lane == 0) {
                a.mean[row] = sum[j] * rn + delta;
                a.rstd[row] = rstd;
            }
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                y[e] = __builtin_fmaf((x[j][e] - delta) * rstd, w[e], b[e]);
                if (GATHER && !known[j])
                    y[e] = kNaN;
            }
            // (a long lookup's results would push the table out of the caches; a plain layer
            // norm's stay there for whoever reads them next)
            if (GATHER && streams)
                store_row<YT, true>(c, row_of<YT>(a.y, row, n), y);
            else
                store_row<YT>(c, row_of<YT>(a.y, row, n), y);
        }
    }
}

// Rows too long for the registers of a workgroup (above 16384 elements): the row is read
// three times.
constexpr int kLongWaves = 16;
template <int XT, int PT, int YT>
__global__ __launch_bounds__(64 * kLongWaves) void norm_forward_long_kernel(const NormArgs a)
{
    constexpr int V = vec_of<XT, YT>;
    constexpr int64_t kStep = (int64_t)64 * kLongWaves * V;
    __shared__ float scratch[3 * 16];
    const int64_t n = a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void *const xp = row_of<XT>(a.x, row, a.x_stride);
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
        team_sum<kTeamGroup, 1>(sum, scratch);
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
        team_sum<kTeamGroup, 2>(two, scratch + 16);
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
            for (int r = 0; r < V; ++r)
                y[r] = __builtin_fmaf(((x[r] - mean0) - delta) * rstd, w[r], b[r]);
            store_cols<YT, V>(yp, c, n, y);
        }
    }
}

template <int XT, int PT, int YT, bool GATHER, int TEAM, int K, int R>
void forward_k(const NormArgs &a, int threads, hipStream_t stream)
{
    constexpr int V = vec_of<XT, YT>;
    const int64_t rows = teams_of<TEAM> * R;
    const int64_t groups = (a.rows + rows - 1) / rows;
    // as many as run at once: where a lane holds 32 values, three workgroups of 256 threads
    // to a CU (8192 x 1600 fp16 13.5 us with 768, 14.9 with 1024, 16.2 with 2048;
    // 40000 x 256 fp32 18.3, 17.1, 18.9)
    const int64_t most = (K * V >= 32 ? 768 : 1024) * 256 / threads;
    const dim3 grid((unsigned)(groups < most ? groups : most)), block((unsigned)threads);
    if (a.cols % V == 0)
        hipLaunchKernelGGL((norm_forward_kernel<XT, PT, YT, GATHER, TEAM, K, R, false>), grid,
                           block, 0, stream, a);
    else
        hipLaunchKernelGGL((norm_forward_kernel<XT, PT, YT, GATHER, TEAM, K, R, true>), grid,
                           block, 0, stream, a);
}

// Threads of a group team for rows of `vectors` vectors, K to a lane (at least a wave: a
// row's last elements, fewer than a vector, take a lane each).
int threads_of(int64_t vectors, int k = 1)
{
    return (int)((vectors + 64 * k - 1) / (64 * k) * 64);
}

// More than 2048 vectors.
template <int XT, int PT, int YT, bool GATHER>
void forward_longest(const NormArgs &a, int64_t vectors, hipStream_t stream)
{
    if constexpr (vec_of<XT, YT> == 4) {
        if (GATHER || vectors <= 4096) {  // (a looked-up row has at most 16384 elements)
            forward_k<XT, PT, YT, GATHER, kTeamGroup, 4, 1>(a, threads_of(vectors, 4), stream);
            return;
        }
    }
    if constexpr (!GATHER)
        hipLaunchKernelGGL((norm_forward_long_kernel<XT, PT, YT>),
                           dim3((unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20))),
                           dim3(64 * kLongWaves), 0, stream, a);
}

template <int XT, int PT, int YT, bool GATHER>
hipError_t forward(const NormArgs &a, hipStream_t stream)
{
    constexpr int V = vec_of<XT, YT>;
    const int64_t vectors = a.cols / V;
    if (vectors <= 16)
        forward_k<XT, PT, YT, GATHER, kTeam16, 1, 4>(a, 256, stream);
    else if (vectors <= 64)
        forward_k<XT, PT, YT, GATHER, kTeamWave, 1, 4>(a, 256, stream);
    else if (vectors <= 128)
        forward_k<XT, PT, YT, GATHER, kTeamWave, 2, 2>(a, 256, stream);
    else if (vectors <= 256)
        forward_k<XT, PT, YT, GATHER, kTeamWave, 4, 1>(a, 256, stream);
    else if (vectors <= 512)
        forward_k<XT, PT, YT, GATHER, GATHER ? kTeamWave : kTeamGroup4, GATHER ? 8 : 2, 1>(
            a, GATHER ? 256 : threads_of(vectors, 2), stream);
    else if (vectors <= 1024)
        forward_k<XT, PT, YT, GATHER, kTeamGroup4, 4, 1>(a, threads_of(vectors, 4), stream);
    else if (vectors <= 2048)
        forward_k<XT, PT, YT, GATHER, kTeamGroup4, 8, 1>(a, threads_of(vectors, 8), stream);
    else
        forward_longest<XT, PT, YT, GATHER>(a, vectors, stream);
    return hipGetLastError();
}

// Most workgroups of a backward pass, of 256 threads each (fewer of larger ones).  Two per
// CU hold enough rows in flight, and each leaves a partial row to be summed: 32768 x 1600
// bf16 71 us at 512 and 76 at 1024, 16384 x 1024 fp32 43 and 46.
constexpr int64_t kNormGradGroups = 512;

// ---------------------------------------------------------------------------
// Backward.  As the forward pass; each workgroup also keeps the sums of dy xh and dy of
// its rows per column in registers and leaves them in the workspace.  HBM bounds it: 3
// elements per element of the row.  The teams, measured (us, with the parameters' sums):
//   32768 x 1600 bf16  wave, 4: 71   one vector per lane in 4 waves: 76
//   32768 x 1024 bf16  wave, 2: 44                                   53
//    8192 x 4096 bf16  4 waves, 2: 49   4: 57   in 8 waves: 52
//    4096 x 8192 bf16  4 waves, 4: 50           in 16 waves: 60
// and above 1024 vectors, where a lane of 4 waves would hold 8:
//    4096 x  8448 bf16  up to 16 waves, 2: 57   4 waves, 8: 91    up to 8 waves, 4: 244
//    4096 x 12288 bf16                     88               106                     291
//    2048 x 16384 bf16                     74               78                      178
//    4096 x  4608 fp32                     54               48                      47
//    4096 x  6144 fp32                     76               58                      64
//    2048 x  8192 fp32                     63               46                      47
// (16-bit rows need registers for 8 elements of a vector and spill; fp32 rows would gain by
// fewer waves, and share the rule.)
// ---------------------------------------------------------------------------

template <int XT, int PT, int TEAM, int K, int R, bool TAIL>
__global__ __launch_bounds__(most_threads<TEAM>) void norm_backward_kernel(const NormGradArgs a)
{
    constexpr int V = vec_of<XT, XT>;
    constexpr int kTeams = teams_of<TEAM>;
    using C = Cols<V, K, TAIL>;
    constexpr int E = C::kElems;
    __shared__ float scratch[is_group<TEAM> ? 2 * 2 * R * 16 : 1];
    const int lanes = is_group<TEAM> ? blockDim.x : 256 / kTeams;
    const int team = is_group<TEAM> ? 0 : threadIdx.x / (256 / kTeams);
    const int lane = is_group<TEAM> ? threadIdx.x : threadIdx.x % (256 / kTeams);
    const int64_t n = a.cols;
    const C c(n, lane, lanes);
    const float rn = 1.0f / (float)n;
    float w[E], dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        w[e] = 1.0f;
        dw[e] = db[e] = 0.0f;
    }
    if (a.weight)
        load_floats<PT, V, K, TAIL>(c, a.weight, w);
    int side = 0;  // two rounds' sums take turns in scratch
    for (int64_t group = blockIdx.x; group * (kTeams * R) < a.rows; group += gridDim.x) {
        const int64_t row0 = (group * kTeams + team) * R;
        RawRow<XT, V, K, TAIL> rx[R], rg[R];
        float mean[R], rstd[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t row = row0 + j < a.rows ? row0 + j : a.rows - 1;
            load_row<XT, true>(c, row_of<XT>(a.x, row, a.x_stride), rx[j]);
            load_row<XT, true>(c, row_of<XT>(a.dy, row, a.dy_stride), rg[j]);
            mean[j] = G(a.mean)[row];
            rstd[j] = G(a.rstd)[row];
        }
        // behind the row's end x and dy are 0 (x from no mean: a large one times rstd may be
        // infinite), and so is everything that is summed
        float x[R][E], dy[R][E];
        float two[2 * R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const bool live = row0 + j < a.rows;
            two[2 * j] = two[2 * j + 1] = 0.0f;
            unpack<XT, V, K, TAIL>(rx[j], x[j]);
            unpack<XT, V, K, TAIL>(rg[j], dy[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[j][e] = (x[j][e] - (c.valid(e) ? mean[j] : 0.0f)) * rstd[j];
                if (live) {
                    dw[e] = __builtin_fmaf(dy[j][e], x[j][e], dw[e]);
                    db[e] += dy[j][e];
                }
                dy[j][e] *= w[e];
                two[2 * j] += dy[j][e];
                two[2 * j + 1] = __builtin_fmaf(dy[j][e], x[j][e], two[2 * j + 1]);
            }
        }
        if (!a.dx)
            continue;
        team_sum<TEAM, 2 * R>(two, scratch + side);
        if constexpr (is_group<TEAM>)
            side = 2 * R * 16 - side;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (row0 + j >= a.rows)
                break;
            const float c1 = two[2 * j] * rn, c2 = two[2 * j + 1] * rn;
            float d[E];
#pragma unroll
            for (int e = 0; e < E; ++e)
                d[e] = rstd[j] * __builtin_fmaf(-x[j][e], c2, dy[j][e] - c1);
            store_row<XT>(c, row_of<XT>(a.dx, row0 + j, n), d);
        }
    }
    if (a.partials)
        leave_partials<TEAM>(c, dw, db, n, a.partials + (int64_t)blockIdx.x * 2 * n);
}

// Rows too long for registers: dx in two readings of the row.
template <int XT, int PT>
__global__ __launch_bounds__(64 * kLongWaves) void norm_backward_long_kernel(const NormGradArgs a)
{
    constexpr int V = vec_of<XT, XT>;
    constexpr int64_t kStep = (int64_t)64 * kLongWaves * V;
    __shared__ float scratch[2 * 16];
    const int64_t n = a.cols;
    const int64_t c0 = (int64_t)threadIdx.x * V;
    const float rn = 1.0f / (float)n;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void *const xp = row_of<XT>(a.x, row, a.x_stride);
        const void *const gp = row_of<XT>(a.dy, row, a.dy_stride);
        const float mean = G(a.mean)[row], rstd = G(a.rstd)[row];
        const auto load = [&](int64_t c, float (&x)[V], float (&g)[V]) {
            float w[V];
            load_cols<XT, V>(xp, c, n, x, mean);
            load_cols<XT, V>(gp, c, n, g);
#pragma unroll
            for (int r = 0; r < V; ++r)
                w[r] = 1.0f;
            if (a.weight)
                load_cols<PT, V>(a.weight, c, n, w);
#pragma unroll
            for (int r = 0; r < V; ++r) {
                x[r] = (x[r] - mean) * rstd;
                g[r] *= w[r];
            }
        };
        float two[2] = {0.0f, 0.0f};
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V], g[V];
            load(c, x, g);
#pragma unroll
            for (int r = 0; r < V; ++r) {
                two[0] += g[r];
                two[1] = __builtin_fmaf(g[r], x[r], two[1]);
            }
        }
        __syncthreads();  // the previous row's sums have been read
        team_sum<kTeamGroup, 2>(two, scratch);
        const float c1 = two[0] * rn, c2 = two[1] * rn;
        void *const dp = row_of<XT>(a.dx, row, n);
        for (int64_t c = c0; c < n; c += kStep) {
            float x[V], g[V];
            load(c, x, g);
#pragma unroll
            for (int r = 0; r < V; ++r)
                g[r] = rstd * __builtin_fmaf(-x[r], c2, g[r] - c1);
            store_cols<XT, V>(dp, c, n, g);
        }
    }
}

// Their parameters' gradients, by columns: a thread holds V columns and takes a share of
// the rows (blockIdx.y), four in flight.  (Sums kept in memory by the kernel above moved
// 16 bytes per element, this reads 4 again in 16 bits: 2000 x 20000 bf16 195 -> 120 us.)
template <int XT>
__global__ __launch_bounds__(256) void norm_params_kernel(const NormGradArgs a)
{
    constexpr int V = vec_of<XT, XT>;
    constexpr int R = 4;
    const int64_t n = a.cols;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
    if (c >= n)
        return;
    float dw[V], db[V];
#pragma unroll
    for (int r = 0; r < V; ++r)
        dw[r] = db[r] = 0.0f;
    const bool whole = c + V <= n;
    for (int64_t row = blockIdx.y; row < a.rows; row += (int64_t)gridDim.y * R) {
        float x[R][V], dy[R][V], mean[R], rstd[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t at = row + (int64_t)j * gridDim.y;
#pragma unroll
            for (int r = 0; r < V; ++r)
                x[j][r] = dy[j][r] = 0.0f;
            mean[j] = rstd[j] = 0.0f;
            if (at < a.rows) {
                const void *const xp = row_of<XT>(a.x, at, a.x_stride);
                const void *const gp = row_of<XT>(a.dy, at, a.dy_stride);
                if (whole) {
                    load_vec<XT, V>(xp, c, x[j]);
                    load_vec<XT, V>(gp, c, dy[j]);
                } else {
                    load_cols<XT, V>(xp, c, n, x[j]);
                    load_cols<XT, V>(gp, c, n, dy[j]);
                }
                mean[j] = G(a.mean)[at];
                rstd[j] = G(a.rstd)[at];
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (row + (int64_t)j * gridDim.y >= a.rows)
                break;
#pragma unroll
            for (int r = 0; r < V; ++r) {
                dw[r] = __builtin_fmaf(dy[j][r], (x[j][r] - mean[j]) * rstd[j], dw[r]);
                db[r] += dy[j][r];
            }
        }
    }
    float *const out = a.partials + (int64_t)blockIdx.y * 2 * n;
    store_cols<kF32, V>(out, c, n, dw);
    store_cols<kF32, V>(out + n, c, n, db);
}

template <int XT, int PT, int TEAM, int K, int R>
int64_t backward_k(const NormGradArgs &a, int threads, hipStream_t stream)
{
    const int64_t rows = teams_of<TEAM> * R;
    int64_t groups = (a.rows + rows - 1) / rows;
    const int64_t most = kNormGradGroups * 256 / (threads < 256 ? 256 : threads);
    groups = groups < most ? groups : most;
    const dim3 grid((unsigned)groups), block((unsigned)threads);
    if (a.cols % vec_of<XT, XT> == 0)
        hipLaunchKernelGGL((norm_backward_kernel<XT, PT, TEAM, K, R, false>), grid, block, 0,
                           stream, a);
    else
        hipLaunchKernelGGL((norm_backward_kernel<XT, PT, TEAM, K, R, true>), grid, block, 0,
                           stream, a);
    return groups;
}

// Shares of the rows in a launch of norm_params_kernel with `blocks` workgroups to each:
// eight workgroups to a CU.
int64_t shares_of(int64_t rows, int64_t blocks)
{
    const int64_t shares = (2048 + blocks - 1) / blocks;
    const int64_t most = rows < kNormGradGroups ? rows : kNormGradGroups;
    return shares < most ? shares : most;
}

template <int XT, int PT>
int64_t backward(const NormGradArgs &a, hipStream_t stream)
{
    constexpr int V = vec_of<XT, XT>;
    const int64_t vectors = a.cols / V;
    if (vectors <= 16)
        return backward_k<XT, PT, kTeam16, 1, 2>(a, 256, stream);
    if (vectors <= 64)
        return backward_k<XT, PT, kTeamWave, 1, 2>(a, 256, stream);
    if (vectors <= 128)
        return backward_k<XT, PT, kTeamWave, 2, 2>(a, 256, stream);
    if (vectors <= 256)
        return backward_k<XT, PT, kTeamWave, 4, 1>(a, 256, stream);
    if (vectors <= 512)
        return backward_k<XT, PT, kTeamGroup4, 2, 1>(a, threads_of(vectors, 2), stream);
    if (vectors <= 1024)
        return backward_k<XT, PT, kTeamGroup4, 4, 1>(a, threads_of(vectors, 4), stream);
    if (vectors <= 2048)
        return backward_k<XT, PT, kTeamGroup, 2, 1>(a, threads_of(vectors, 2), stream);
    if constexpr (V == 4) {
        if (vectors <= 4096)
            return backward_k<XT, PT, kTeamGroup, 4, 1>(a, threads_of(vectors, 4), stream);
    }
    if (a.dx)
        hipLaunchKernelGGL((norm_backward_long_kernel<XT, PT>),
                           dim3((unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20))),
                           dim3(64 * kLongWaves), 0, stream, a);
    if (!a.partials)
        return 0;
    const int64_t blocks = (a.cols + 256 * V - 1) / (256 * V);
    const int64_t shares = shares_of(a.rows, blocks);
    hipLaunchKernelGGL(norm_params_kernel<XT>, dim3((unsigned)blocks, (unsigned)shares), dim3(256),
                       0, stream, a);
    return shares;
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
        constexpr int kBatch = 16;  // in flight
        for (int64_t g0 = wave; g0 < groups; g0 += kSumWaves * kBatch) {
            float v[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int64_t g = g0 + j * kSumWaves;
                v[j] = 0.0f;
                if (g < groups)
                    v[j] = G(partials)[(2 * g + which) * cols + c];
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                s += v[j];
        }
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

int64_t norm_workspace_bytes(int64_t rows, int64_t cols)
{
    int64_t groups = rows < 1 ? 1 : rows < kNormGradGroups ? rows : kNormGradGroups;
    // rows that are too long for registers in every type: the fewest workgroups to a share
    // are 16-bit rows', 8 elements to a thread
    if (cols / 8 > 2048 && rows > 0)
        groups = shares_of(rows, (cols + 2047) / 2048);
    return groups * 2 * cols * 4;
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
    int64_t groups = 0;
    if (a.rows > 0) {
        if (xt == kF32)
            groups = backward<kF32, kF32>(a, stream);
        else if (xt == kF16)
            groups = pt == kF32 ? backward<kF16, kF32>(a, stream) : backward<kF16, kF16>(a, stream);
        else
            groups = pt == kF32 ? backward<kBF16, kF32>(a, stream)
                                : backward<kBF16, kBF16>(a, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    if (!a.partials)
        return hipSuccess;
    return launch_param_grads(pt, a.partials, groups, a.cols, a.dweight, a.dbias, stream);
}

}  // namespace bq
