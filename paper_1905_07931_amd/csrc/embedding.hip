// Embedding: rows of a table as columns of the activations, and the table's gradient.
//   forward   X[d][b] = scale E[t_b][d]            (0 where t_b is no row of the table)
//   backward  dE[v][d] = add[v][d] + scale sum_{b: t_b = v} dX[d][b]
//   masked    gv[p] = scale sum_{b: t_b = row p} dX[col p][b]   on the pattern of a CSR table
// Tables are [V][D] with the features contiguous, activations [D][B] with the tokens contiguous, so every
// call transposes; each does it by tiles through LDS, with whole cache lines on both sides.
//
// The gradient's sums go by sorted tokens: the plan ranks the tokens by (token, position), the columns of dX
// are stored as rows in that order, and a row of the table adds up the run of rows that is its own.  No
// atomics: sums have one order.
#include <algorithm>
#include <climits>

#include "common.hpp"
#include "launch.hpp"
#include "typed.hpp"

namespace l1csr {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;              // tokens and features of a transposed tile
constexpr int kPitch = kTile + 1;      // of its rows in LDS: every access below touches each bank once
constexpr int kMaxGrid = 1 << 20;      // workgroups of a launch; they step over what is left

__device__ __forceinline__ bool in_table(int token, int V) { return (unsigned)token < (unsigned)V; }

// The tile of workgroup (or step) i: tiles side by side along the tokens first.  Rows of X are often a power of two long, and
// 64 rows of such a matrix lie in the same few memory channels: neighbours along the features would all wait for those
// (4096 x 8192 fp32, columns to rows: 88 us with the features first, 43 so).
struct tile_at {
    int d0, b0;
    __device__ __forceinline__ tile_at(int64_t i, int b_tiles) {
        const int64_t q = i / b_tiles;
        d0 = (int)q * kTile;
        b0 = (int)(i - q * b_tiles) * kTile;
    }
};

// Results of this size are stored past the caches: they would only displace each other
constexpr int64_t kPastBytes = 32 << 20;

// A workgroup a tile.  131072 x 4096 bf16, 8192 tokens to fp32: 41 us from cold memory (165 MB, 4.0 TB/s; storing X alone
// takes 20).  Larger tiles (59) and several tiles of the same tokens, their loads ahead (45 to 58), leave fewer
// waves to wait for the rows.
template <typename TE, typename TX, bool PAST>
__global__ __launch_bounds__(kThreads) void gather_kernel(int V, int D, int B, const TE *__restrict__ E, int64_t lde,
                                                          const int *__restrict__ tokens, float scale,
                                                          TX *__restrict__ X, int64_t ldx, int b_tiles, int64_t tiles) {
    __shared__ float tile[kTile * kPitch];
    constexpr int N = kPer16<TE>, lanes = kTile / N;
    const int d = (threadIdx.x & (lanes - 1)) * N;
    for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
        const tile_at at(i, b_tiles);
        const int d0 = at.d0, b0 = at.b0;
#pragma unroll
        for (int b = threadIdx.x / lanes; b < kTile; b += kThreads / lanes) {
            const int t = b0 + b < B ? tokens[b0 + b] : -1;
            TE e[N] = {};
            if (in_table(t, V) && d0 + d < D) load_some<TE, N>(E + (int64_t)t * lde + d0 + d, D - d0 - d, e);
#pragma unroll
            for (int n = 0; n < N; ++n) tile[(d + n) * kPitch + b] = widen(e[n]);
        }
        __syncthreads();
        constexpr int M = 4, across = kTile / M;
        const int b = (threadIdx.x & (across - 1)) * M;
#pragma unroll
        for (int k = threadIdx.x / across; k < kTile; k += kThreads / across) {
            if (d0 + k >= D || b0 + b >= B) continue;
            const float *row = tile + k * kPitch + b;
            TX x[M];
#pragma unroll
            for (int m = 0; m < M; ++m) x[m] = (TX)(scale * row[m]);
            TX *p = X + (int64_t)(d0 + k) * ldx + b0 + b;
            if (PAST && b0 + b + M <= B) store_past<TX, M>(p, x);
            else store_some<TX, M>(p, B - b0 - b, x);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// a table kept in CSR
// ---------------------------------------------------------------------------

constexpr int kCsrThreads = 1024;
constexpr int kCsrTokens = 32;     // of a tile: 128 bytes of a row of X
constexpr int kCsrFeatures = 256;  // of a tile
constexpr int kCsrPitch = kCsrTokens + 1;

// first position of [lo, hi) whose column is c or more, by a whole wave: 64 probes a step
__device__ __forceinline__ int wave_lower_bound(const int *__restrict__ col, int lo, int hi, int c, int lane) {
    while (hi - lo > 0) {
        const int step = (hi - lo + kWave - 1) / kWave;
        const int64_t at = (int64_t)lo + (int64_t)lane * step;
        const uint64_t below = wave_ballot(at < hi && col[at < hi ? at : lo] < c);
        const int n = (int)__popcll(below);  // probes 0 .. n - 1 lie below (the columns ascend)
        if (n == 0) return lo;
        const int64_t next = (int64_t)lo + (int64_t)n * step;
        lo = lo + (n - 1) * step + 1;
        hi = (int)min((int64_t)hi, next);
    }
    return lo;
}

// A wave a token: its row's entries of the tile's features, found by search, are put between zeros.
__global__ __launch_bounds__(kCsrThreads) void gather_csr_kernel(int V, int D, int B, int nnz,
                                                                 const int *__restrict__ ptr,
                                                                 const int *__restrict__ col,
                                                                 const float *__restrict__ val,
                                                                 const int *__restrict__ tokens, float scale,
                                                                 float *__restrict__ X, int64_t ldx, int b_tiles,
                                                                 int64_t tiles) {
    __shared__ float tile[kCsrFeatures * kCsrPitch];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
        const int d0 = (int)(i / b_tiles) * kCsrFeatures, b0 = (int)(i % b_tiles) * kCsrTokens;
        for (int j = threadIdx.x; j < kCsrFeatures * kCsrPitch; j += kCsrThreads) tile[j] = 0.f;
        __syncthreads();
        for (int b = wave; b < kCsrTokens && b0 + b < B; b += kCsrThreads / kWave) {
            const int t = tokens[b0 + b];
            if (!in_table(t, V)) continue;
            const int lo = max(ptr[t], 0), hi = min(ptr[t + 1], nnz);
            for (int p = wave_lower_bound(col, lo, hi, d0, lane) + lane; p < hi; p += kWave) {
                const int d = col[p] - d0;
                if ((unsigned)d >= (unsigned)kCsrFeatures) break;
                tile[d * kCsrPitch + b] = scale * val[p];
            }
        }
        __syncthreads();
        constexpr int N = 4, lanes = kCsrTokens / N;
        const int b = (threadIdx.x & (lanes - 1)) * N;
        for (int d = threadIdx.x / lanes; d < kCsrFeatures && d0 + d < D; d += kCsrThreads / lanes) {
            if (b0 + b >= B) break;
            const float *row = tile + d * kCsrPitch + b;
            const float x[N] = {row[0], row[1], row[2], row[3]};
            store_some<float, N>(X + (int64_t)(d0 + d) * ldx + b0 + b, B - b0 - b, x);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// the order of the tokens
// ---------------------------------------------------------------------------

constexpr int kRun = 1024;         // tokens that are ranked by counting
constexpr int kWays = 8;           // runs that are merged at a time
constexpr int kRankThreads = 1024;

// what the tokens are sorted by: those of no row come last
__device__ __forceinline__ int key_of(int token, int V) { return (int)min((unsigned)token, (unsigned)V); }

// Up to kCounted tokens are ranked in one launch: a workgroup has all keys in LDS and kOwn tokens, each by 64 threads, of which
// every one counts the smaller keys (and the equal ones ahead) of its share, four a step: 1656 tokens take 3.6 us, 4096 4.2
// and 8192 8.8, by runs and their merge 12.5, 14.0 and 14.7.  It grows with the square: larger batches go by runs.  (The
// limit is that of the array of keys, 32 KB; where both take the same time lies higher and has not been measured.)
constexpr int kCounted = 8192, kOwn = 16;
__global__ __launch_bounds__(kRankThreads) void count_kernel(int V, int B, const int *__restrict__ tokens,
                                                             int *__restrict__ rank, int *__restrict__ sorted) {
    constexpr int N = 4, shares = kRankThreads / kOwn;
    __shared__ __align__(16) int keys[kCounted];
    __shared__ int part[kRankThreads / kWave][kOwn];
    const int steps = (B + shares * N - 1) / (shares * N);  // the keys past the end are larger than any
    for (int i = threadIdx.x * N; i < steps * shares * N; i += kRankThreads * N) {
        int x[N];
        load_some<int, N>(tokens + i, B - i, x);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = i + k < B ? key_of(x[k], V) : INT_MAX;
        store_values<int, N>(keys + i, x);
    }
    __syncthreads();
    const int own = threadIdx.x & (kOwn - 1), share = threadIdx.x / kOwn, b = blockIdx.x * kOwn + own;
    const int key = b < B ? keys[b] : 0;
    int less = 0;
#pragma unroll 4
    for (int i = 0; i < steps; ++i) {
        const int at = (i * shares + share) * N;
        int x[N];
        load_values<int, N>(keys + at, x);
        const int limit = key + (at + N <= b ? 1 : 0);  // equal tokens ahead count
#pragma unroll
        for (int k = 0; k < N; ++k) less += x[k] < limit ? 1 : 0;
    }
    static_assert(kWave % kOwn == 0 && kOwn % N == 0, "a wave has whole shares, a workgroup's tokens whole steps");
    if (share == 0)  // those of the token's own step
        for (int j = b & ~(N - 1); j < min(b, B); ++j) less += keys[j] == key ? 1 : 0;
#pragma unroll
    for (int d = kOwn; d < kWave; d <<= 1) less += __shfl_xor(less, d, kWave);
    if (lane_id() < kOwn) part[threadIdx.x / kWave][own] = less;
    __syncthreads();
    if (threadIdx.x < kOwn && b < B) {
        int r = 0;
#pragma unroll
        for (int w = 0; w < kRankThreads / kWave; ++w) r += part[w][own];
        rank[b] = r;
        sorted[r] = key;
    }
}

// Ranks within runs of kRun tokens by counting the smaller ones (and the equal ones ahead): a lane a token, each wave of a
// workgroup goes through 64 tokens of the run.
__global__ __launch_bounds__(kRankThreads) void rank_kernel(int V, int B, const int *__restrict__ tokens,
                                                            int *__restrict__ rank, int *__restrict__ sorted) {
    constexpr int waves = kRankThreads / kWave;
    static_assert(waves * kWave == kRun, "a wave for every 64 tokens of a run");
    __shared__ int part[waves][kWave];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    const int own = blockIdx.x * kWave, base = own / kRun * kRun, at = base + wave * kWave, n = min(kWave, B - at);
    const int b = own + lane;
    const int key = b < B ? key_of(tokens[b], V) : V, others = lane < n ? key_of(tokens[at + lane], V) : 0;
    int less = 0;
    if (at == own) {
        for (int j = 0; j < n; ++j) {
            const int other = lane_bcast(others, j);
            less += other < key || (other == key && j < lane) ? 1 : 0;
        }
    } else {
        const int limit = key + (at < own ? 1 : 0);  // equal tokens ahead count
        for (int j = 0; j < n; ++j) less += lane_bcast(others, j) < limit ? 1 : 0;
    }
    part[wave][lane] = less;
    __syncthreads();
    if (wave == 0 && b < B) {
        int r = 0;
#pragma unroll
        for (int w = 0; w < waves; ++w) r += part[w][lane];
        rank[b] = r;
        sorted[base + r] = key;
    }
}

// first position of the ascending s[0 .. n) whose value is k or more
__device__ __forceinline__ int lower_bound(const int *__restrict__ s, int n, int k) {
    int lo = 0;
    while (n > 0) {
        const int half = n >> 1;
        const bool below = s[lo + half] < k;
        lo = below ? lo + half + 1 : lo;
        n = below ? n - half - 1 : half;
    }
    return lo;
}

// Eight sorted runs of `run` tokens become one: a token's rank grows by what goes before it in each of the others, whose
// searches go side by side.  The first round searches in LDS (FIRST: run = kRun), where a step's 64 x 7 scattered words
// do not queue at the cache (8192 tokens 9.2 us; searched in memory 16.6).
template <bool FIRST>
__global__ __launch_bounds__(kThreads) void merge_kernel(int V, int B, int64_t run, const int *__restrict__ tokens,
                                                         int *__restrict__ rank, const int *__restrict__ sorted,
                                                         int *__restrict__ merged) {
    __shared__ __align__(16) int runs[FIRST ? kRun * kWays + 1 : 4];  // (an empty range's step looks at the place behind it)
    const int64_t b0 = (int64_t)blockIdx.x * kThreads, b = b0 + threadIdx.x;
    if constexpr (FIRST) run = kRun;
    const int64_t first = b0 / (run * kWays) * (run * kWays);  // (a run is a multiple of kThreads tokens)
    const int token = b < B ? tokens[b] : 0, own = b < B ? rank[b] : 0;
    if constexpr (FIRST) {
        const int n = (int)min((int64_t)kRun * kWays, B - first);
        constexpr int N = 4, loads = kRun * kWays / (N * kThreads);
        int x[loads][N];
#pragma unroll
        for (int i = 0; i < loads; ++i) {
            const int at = (i * kThreads + (int)threadIdx.x) * N;
            load_some<int, N>(sorted + first + at, n - at, x[i]);
        }
#pragma unroll
        for (int i = 0; i < loads; ++i) store_values<int, N>(runs + (i * kThreads + (int)threadIdx.x) * N, x[i]);
        __syncthreads();
    }
    if (b >= B) return;
    const int key = key_of(token, V), q = (int)((b - first) / run);
    int lo[kWays], n[kWays];
#pragma unroll
    for (int w = 0; w < kWays; ++w) {
        lo[w] = 0;
        n[w] = w == q ? 0 : (int)min(run, max((int64_t)0, B - first - w * run));
    }
    for (int64_t left = run; left > 0; left >>= 1) {  // (a search of n values takes no more steps than n has bits)
#pragma unroll
        for (int w = 0; w < kWays; ++w) {
            const int half = n[w] >> 1;
            // equal tokens of an earlier run go before
            const int other = FIRST ? runs[w * kRun + lo[w] + half] : n[w] > 0 ? sorted[first + w * run + lo[w] + half] : 0;
            const bool below = n[w] > 0 && other < key + (w < q ? 1 : 0);
            lo[w] = below ? lo[w] + half + 1 : lo[w];
            n[w] = below ? n[w] - half - 1 : half;
        }
    }
    int r = own;
#pragma unroll
    for (int w = 0; w < kWays; ++w) r += lo[w];
    rank[b] = r;
    merged[first + r] = key;
}

// The plan's parts: rank[B] of every token, sorted[B] the tokens in order (V: of no row).  (Merged
// runs alternate between two arrays.)
struct plan_parts {
    int *rank, *sorted, *other;
};
plan_parts carve_plan(int B, void *plan) {
    int *p = static_cast<int *>(plan);
    plan_parts r{p, p + B, p + 2 * (size_t)B};
    if (B > kCounted)
        for (int64_t run = kRun; run < B; run *= kWays) std::swap(r.sorted, r.other);
    return r;
}

// ---------------------------------------------------------------------------
// the gradient
// ---------------------------------------------------------------------------

constexpr int kGroup = 32;  // rows that are added up ahead where all are of one token, and such groups

// What the sums read: the columns of dX as rows in the tokens' order, and sums of groups of them
template <typename T>
struct run_rows {
    const T *rows;          // [B][ld]
    const float *groups;    // [B / 32][ld], a group's where its rows are of one token; null: not summed
    const float *blocks;    // [B / 1024][ld], of 32 groups; null: not summed
    int64_t ld;
};

// adds U rows of ld values at p, their loads ahead
template <int U, typename T, int N>
__device__ __forceinline__ void add_ahead(const T *p, int64_t ld, float (&sum)[N]) {
    T x[U][N];
#pragma unroll
    for (int i = 0; i < U; ++i) load_values<T, N>(p + i * ld, x[i]);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] += widen(x[i][k]);
}

// adds n rows, eight at a time; what is left by four, two and one where a thread has one value (the pattern of 98 rows, 1656
// tokens: 13.0 -> 9.8 us), one by one where it has four (there it gains nothing, and costs large tables 3 to 5 %)
template <typename T, int N>
__device__ __forceinline__ void add_rows(const T *p, int64_t ld, int n, float (&sum)[N]) {
    for (; n >= 8; n -= 8, p += 8 * ld) add_ahead<8>(p, ld, sum);
    if constexpr (N == 1) {
        if (n & 4) {
            add_ahead<4>(p, ld, sum);
            p += 4 * ld;
        }
        if (n & 2) {
            add_ahead<2>(p, ld, sum);
            p += 2 * ld;
        }
        if (n & 1) add_ahead<1>(p, ld, sum);
    } else {
        for (; n > 0; --n, p += ld) add_ahead<1>(p, ld, sum);
    }
}

// sum over rows lo .. hi - 1 of the values at d .. d + N - 1, in one order: the rows ahead of the first whole group,
// groups (blocks of them where they are whole and summed), the rows behind
template <typename T, int N>
__device__ __forceinline__ void sum_run(const run_rows<T> &r, int lo, int hi, int64_t d, float (&sum)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) sum[n] = 0.f;
    const T *rows = r.rows + d;
    int g = (lo + kGroup - 1) / kGroup;
    const int end = hi / kGroup;
    if (g >= end || !r.groups) {
        add_rows<T, N>(rows + lo * r.ld, r.ld, hi - lo, sum);
        return;
    }
    add_rows<T, N>(rows + lo * r.ld, r.ld, g * kGroup - lo, sum);
    const float *groups = r.groups + d;
    const int b = r.blocks ? (g + kGroup - 1) / kGroup : 0, b_end = r.blocks ? end / kGroup : 0;
    if (b < b_end) {
        add_rows<float, N>(groups + g * r.ld, r.ld, b * kGroup - g, sum);
        add_rows<float, N>(r.blocks + d + b * r.ld, r.ld, b_end - b, sum);
        g = b_end * kGroup;
    }
    add_rows<float, N>(groups + g * r.ld, r.ld, end - g, sum);
    add_rows<T, N>(rows + end * kGroup * r.ld, r.ld, hi - end * kGroup, sum);
}

// bounds[v] = the first place of row v of the table in the order (row v's run is bounds[v] .. bounds[v + 1] - 1), by
// workgroup `block` of `grid`.  Where the table is not much larger than the batch every place fills in the rows since the
// one before it (a wave 64 places, each gap by all lanes), else every row is searched for.
constexpr int kRowsAPlace = 32;
__device__ __forceinline__ void fill_bounds(int V, int B, const int *__restrict__ sorted, int *__restrict__ bounds, int block,
                                            int grid) {
    const int64_t stride = (int64_t)grid * kThreads;
    if (V > (int64_t)kRowsAPlace * (B + 1)) {
        for (int64_t v = (int64_t)block * kThreads + threadIdx.x; v <= V; v += stride) bounds[v] = lower_bound(sorted, B, (int)v);
        return;
    }
    const int lane = lane_id();
    for (int64_t i0 = (int64_t)block * kThreads + (threadIdx.x & ~63); i0 <= B; i0 += stride) {
        const int64_t i = i0 + lane;
        // (key_of: a plan of a larger table holds more)
        const int from = i == 0 ? 0 : i <= B ? key_of(sorted[i - 1], V) + 1 : V + 1, to = i < B ? key_of(sorted[i], V) : V;
        for (uint64_t some = wave_ballot(i <= B && from <= to); some != 0; some &= some - 1) {
            const int j = __builtin_ctzll(some);
            const int last = lane_bcast(to, j);
            for (int v = lane_bcast(from, j) + lane; v <= last; v += kWave) bounds[v] = (int)(i0 + j);
        }
    }
}

// rows[rank of b][d] = dX[d][b]; the last workgroups fill the bounds
template <typename T>
__global__ __launch_bounds__(kThreads) void sort_columns_kernel(int V, int D, int B, const T *__restrict__ dX, int64_t ldx,
                                                                const int *__restrict__ rank,
                                                                const int *__restrict__ sorted, T *__restrict__ rows,
                                                                int64_t ld, int b_tiles, int64_t tiles, int tile_grid,
                                                                int *__restrict__ bounds) {
    __shared__ float tile[kTile * kPitch];  // [token][feature]
    if ((int)blockIdx.x >= tile_grid) {
        fill_bounds(V, B, sorted, bounds, blockIdx.x - tile_grid, gridDim.x - tile_grid);
        return;
    }
    constexpr int N = kPer16<T>, lanes = kTile / N;
    const int c = (threadIdx.x & (lanes - 1)) * N;
    constexpr int step = kThreads / lanes;
    for (int64_t i = blockIdx.x; i < tiles; i += tile_grid) {
        const tile_at at(i, b_tiles);
        const int d0 = at.d0, b0 = at.b0;
        int to[kTile / step];  // the rows that this thread stores, -1: of no token that counts
#pragma unroll
        for (int j = 0; j < kTile / step; ++j) {
            const int b = b0 + threadIdx.x / lanes + j * step;
            to[j] = b < B ? rank[b] : -1;
        }
#pragma unroll
        for (int j = 0; j < kTile / step; ++j)
            if ((unsigned)to[j] >= (unsigned)B || sorted[to[j]] >= V) to[j] = -1;
#pragma unroll
        for (int d = threadIdx.x / lanes; d < kTile; d += kThreads / lanes) {
            T x[N] = {};
            if (d0 + d < D && b0 + c < B) load_some<T, N>(dX + (int64_t)(d0 + d) * ldx + b0 + c, B - b0 - c, x);
#pragma unroll
            for (int n = 0; n < N; ++n) tile[(c + n) * kPitch + d] = widen(x[n]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kTile / step; ++j) {
            const int b = threadIdx.x / lanes + j * step;
            T x[N];
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] = (T)tile[b * kPitch + c + n];
            if (to[j] >= 0 && d0 + c < ld) store_values<T, N>(rows + to[j] * ld + d0 + c, x);  // ld: D up to a multiple of 8
        }
        __syncthreads();
    }
}

// Sums of the groups of 32 rows (rows of `from`, `width` tokens each) that are all of one token
template <typename T>
__global__ __launch_bounds__(kThreads) void group_kernel(int V, int B, int width, const T *__restrict__ from,
                                                         const int *__restrict__ sorted, float *__restrict__ to,
                                                         int64_t ld, int groups) {
    constexpr int N = 4;
    for (int g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t first = (int64_t)g * kGroup * width, last = first + (int64_t)kGroup * width - 1;
        if (last >= B || sorted[first] >= V || sorted[first] != sorted[last]) continue;
        for (int64_t d = threadIdx.x * N; d < ld; d += kThreads * N) {
            float sum[N] = {};
            const T *p = from + (int64_t)g * kGroup * ld + d;
#pragma unroll 8
            for (int i = 0; i < kGroup; ++i) {
                T x[N];
                load_values<T, N>(p + i * ld, x);
#pragma unroll
                for (int n = 0; n < N; ++n) sum[n] += widen(x[n]);
            }
            store_values<float, N>(to + g * ld + d, sum);
        }
    }
}

constexpr int64_t kFullCard = 1024;  // workgroups
constexpr int kRowBlock = 4;  // rows of a thread, whose loads are under way together; a grid apart: frequent tokens are neighbours

// dE, every row of it (ALL), or dE += where only the rows that have tokens change: then a workgroup's rows are
// places in the order, of which the first of each run has work.  blockIdx.y: a range of features.
template <typename T, typename TE, bool ALL, bool PAST>
__global__ __launch_bounds__(kThreads) void table_rows_kernel(int V, int D, int B, run_rows<T> r,
                                                              const int *__restrict__ sorted,
                                                              const int *__restrict__ bounds, float scale, const TE *add,
                                                              int64_t ldadd, TE *dE, int64_t ldde, int tx_shift) {
    constexpr int N = 4;
    const int TX = 1 << tx_shift, TY = kThreads >> tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> tx_shift;
    const int64_t total = ALL ? V : B, d = ((int64_t)blockIdx.y * TX + tx) * N;
    if (d >= D) return;
    const int64_t apart = (int64_t)gridDim.x * TY;
    for (int64_t v0 = (int64_t)blockIdx.x * TY + ty; v0 < total; v0 += apart * kRowBlock) {
        // the runs of the rows and what is added to them, all loads ahead of the first sum
        int64_t row[kRowBlock];
        int lo[kRowBlock], hi[kRowBlock];  // lo < 0: no work
        TE e[kRowBlock][N];
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i) {
            const int64_t v = min(v0 + i * apart, total - 1);
            row[i] = ALL ? v : sorted[v];
        }
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i) {
            const bool on = v0 + i * apart < total && row[i] < V;
            lo[i] = on ? bounds[row[i]] : -1;
            hi[i] = on ? bounds[row[i] + 1] : -1;
            if (!ALL && lo[i] != v0 + i * apart) lo[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i) {
            if (add && lo[i] >= 0) {
                load_some<TE, N>(add + row[i] * ldadd + d, D - d, e[i]);
            } else {
#pragma unroll
                for (int n = 0; n < N; ++n) e[i][n] = (TE)0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i) {
            if (lo[i] < 0) continue;
            float s[N] = {};
            if (lo[i] < hi[i]) sum_run<T, N>(r, lo[i], hi[i], d, s);
#pragma unroll
            for (int n = 0; n < N; ++n) e[i][n] = (TE)(widen(e[i][n]) + scale * s[n]);
            TE *p = dE + row[i] * ldde + d;
            if (PAST && D - d >= N) store_past<TE, N>(p, e[i]);
            else store_some<TE, N>(p, D - d, e[i]);
        }
    }
}

// gv on the pattern: 2^tx_shift threads a row of the table
__global__ __launch_bounds__(kThreads) void table_pattern_kernel(int V, int D, int nnz, run_rows<float> r,
                                                                 const int *__restrict__ bounds, float scale,
                                                                 const int *__restrict__ ptr, const int *__restrict__ col,
                                                                 float *__restrict__ gv, int tx_shift) {
    const int TX = 1 << tx_shift, TY = kThreads >> tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> tx_shift;
    const int64_t apart = (int64_t)gridDim.x * TY;
    for (int64_t v0 = (int64_t)blockIdx.x * TY + ty; v0 < V; v0 += apart * kRowBlock) {
        int p0[kRowBlock], p1[kRowBlock], lo[kRowBlock], hi[kRowBlock];
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i) {
            const int64_t v = min(v0 + i * apart, (int64_t)V - 1);
            p0[i] = max(ptr[v], 0);
            p1[i] = v0 + i * apart < V ? min(ptr[v + 1], nnz) : 0;
            lo[i] = bounds[v];
            hi[i] = bounds[v + 1];
        }
#pragma unroll
        for (int i = 0; i < kRowBlock; ++i)
            for (int q = p0[i] + tx; q < p1[i]; q += TX) {
                float s[1] = {};
                if (lo[i] < hi[i]) {
                    const int c = col[q];
                    if ((unsigned)c < (unsigned)D) sum_run<float, 1>(r, lo[i], hi[i], c, s);
                }
                gv[q] = scale * s[0];
            }
    }
}

int64_t padded(int D) { return ((int64_t)D + 7) & ~7ll; }

int pow2_shift(int64_t n, int most) {
    int s = 0;
    while (s < most && ((int64_t)1 << s) < n) ++s;
    return s;
}

int grid_of(int64_t work) { return (int)std::min<int64_t>(std::max<int64_t>(work, 1), kMaxGrid); }

// Workgroups for `rows` rows, `ty` of them side by side in one: kRowBlock rows to a thread, fewer while the card is not full, for
// the rows of a thread follow one another where their runs are long (1611 tokens over 103 rows of 20 fp16: 10.4 us, with
// kRowBlock rows a thread 16; 1656 tokens over 98 rows of a pattern with 71 columns: 13.6 and 23)
int row_grid(int64_t rows, int ty, int64_t chunks) {
    const int64_t full = ceil_div(rows, (int64_t)ty * kRowBlock);
    return grid_of(std::max(full, std::min(ceil_div(rows, ty), kFullCard / chunks)));
}

struct bwd_parts {
    int *bounds;
    float *groups, *blocks;
    char *rows;
    size_t bytes;
};
bwd_parts carve_bwd(int V, int D, int B, void *ws) {
    char *p = static_cast<char *>(ws);
    const size_t row = sizeof(float) * (size_t)padded(D);
    bwd_parts w;
    w.bounds = reinterpret_cast<int *>(p);
    size_t at = (sizeof(int) * ((size_t)V + 1) + 63) & ~(size_t)63;
    w.groups = reinterpret_cast<float *>(p + at);
    at += row * (B / kGroup);
    w.blocks = reinterpret_cast<float *>(p + at);
    at += row * (B / (kGroup * kGroup));
    w.rows = p + at;
    w.bytes = at + row * B;
    return w;
}

// tokens from which on groups are summed ahead (fewer: 32 times 8 rows at most, less than the launch costs for
// most batches), and from which on groups of groups are
constexpr int kGroupsFrom = 256, kBlocksFrom = 1 << 14;

// the columns of dX as rows in the tokens' order, and the sums of their groups
template <typename T>
hipError_t sort_columns(const embedding_args &a, const plan_parts &plan, const bwd_parts &w, run_rows<T> *r,
                        hipStream_t s) {
    const int64_t ld = padded(a.D);
    T *rows = reinterpret_cast<T *>(w.rows);
    const int b_tiles = (int)ceil_div(a.B, kTile);
    const int64_t tiles = b_tiles * ceil_div(a.D, kTile);
    const int tile_grid = a.B > 0 ? grid_of(tiles) : 0, bound_grid = grid_of(ceil_div(std::max(a.V, a.B) + 1ll, kThreads));
    sort_columns_kernel<T><<<tile_grid + bound_grid, kThreads, 0, s>>>(
        a.V, a.D, a.B, static_cast<const T *>(a.X), a.ldx, plan.rank, plan.sorted, rows, ld, b_tiles, tiles, tile_grid, w.bounds);
    const int groups = a.B >= kGroupsFrom ? a.B / kGroup : 0, blocks = a.B >= kBlocksFrom ? a.B / (kGroup * kGroup) : 0;
    *r = {rows, groups > 0 ? w.groups : nullptr, blocks > 0 ? w.blocks : nullptr, ld};
    if (groups > 0)
        group_kernel<T><<<grid_of(groups), kThreads, 0, s>>>(a.V, a.B, 1, rows, plan.sorted, w.groups, ld, groups);
    if (blocks > 0)
        group_kernel<float><<<grid_of(blocks), kThreads, 0, s>>>(a.V, a.B, kGroup, w.groups, plan.sorted, w.blocks, ld,
                                                                 blocks);
    return hipGetLastError();
}

}  // namespace

bool embedding_fits(int64_t V, int64_t D, int64_t B) {
    // (a launch has fewer than 2^32 threads, and fewer than 2^16 ranges of features)
    return V <= 1 << 30 && D <= 1 << 25 && B <= 1 << 24;
}

size_t embedding_plan_bytes(int B) { return sizeof(int) * 3 * (size_t)std::max(B, 0); }

size_t embedding_bwd_workspace_bytes(int V, int D, int B) {
    return V <= 0 || D <= 0 ? 0 : carve_bwd(V, D, std::max(B, 0), nullptr).bytes;
}

hipError_t launch_embedding_fwd(const embedding_args &a, hipStream_t s) {
    if (a.D == 0 || a.B == 0) return hipSuccess;
    const int b_tiles = (int)ceil_div(a.B, kTile);
    return with_types(a.dtype, a.x_dtype, [&](auto e, auto x) {
        using TE = decltype(e);
        using TX = decltype(x);
        const int64_t tiles = b_tiles * ceil_div(a.D, kTile);
        const bool past = (int64_t)a.D * a.B * (int64_t)sizeof(TX) > kPastBytes;
        (past ? gather_kernel<TE, TX, true> : gather_kernel<TE, TX, false>)<<<grid_of(tiles), kThreads, 0, s>>>(
            a.V, a.D, a.B, static_cast<const TE *>(a.E), a.lde, a.tokens, a.scale, static_cast<TX *>(a.X_out), a.ldx, b_tiles,
            tiles);
        return hipGetLastError();
    });
}

hipError_t launch_embedding_csr_fwd(const embedding_args &a, int nnz, const int *ptr, const int *col, const float *val,
                                    hipStream_t s) {
    if (a.D == 0 || a.B == 0) return hipSuccess;
    const int b_tiles = (int)ceil_div(a.B, kCsrTokens);
    const int64_t tiles = b_tiles * ceil_div(a.D, kCsrFeatures);
    gather_csr_kernel<<<grid_of(tiles), kCsrThreads, 0, s>>>(a.V, a.D, a.B, nnz, ptr, col, val, a.tokens, a.scale,
                                                             static_cast<float *>(a.X_out), a.ldx, b_tiles, tiles);
    return hipGetLastError();
}

hipError_t launch_embedding_plan(int V, int B, const int *tokens, void *plan, hipStream_t s) {
    if (B == 0) return hipSuccess;
    int *rank = static_cast<int *>(plan), *from = rank + B, *to = from + B;
    if (B <= kCounted) {
        count_kernel<<<(int)ceil_div(B, kOwn), kRankThreads, 0, s>>>(V, B, tokens, rank, from);
        return hipGetLastError();
    }
    rank_kernel<<<(int)ceil_div(B, kWave), kRankThreads, 0, s>>>(V, B, tokens, rank, from);
    for (int64_t run = kRun; run < B; run *= kWays) {
        (run == kRun ? merge_kernel<true> : merge_kernel<false>)<<<(int)ceil_div(B, kThreads), kThreads, 0, s>>>(
            V, B, run, tokens, rank, from, to);
        std::swap(from, to);
    }
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(const embedding_args &a, const void *plan_mem, void *ws, hipStream_t s) {
    if (a.D == 0 || a.V == 0) return hipSuccess;
    const bool in_place = a.add != nullptr && a.add == a.dE;
    if (in_place && a.B == 0) return hipSuccess;
    const plan_parts plan = carve_plan(a.B, const_cast<void *>(plan_mem));
    const bwd_parts w = carve_bwd(a.V, a.D, a.B, ws);
    return with_types(a.dtype, a.e_dtype, [&](auto x, auto e) {
        using T = decltype(x);
        using TE = decltype(e);
        run_rows<T> r;
        const hipError_t err = sort_columns<T>(a, plan, w, &r, s);
        if (err != hipSuccess) return err;
        const int shift = pow2_shift(ceil_div(a.D, 4), 8);
        const int64_t chunks = ceil_div(a.D, (int64_t)4 << shift);
        const TE *add = static_cast<const TE *>(a.add);
        TE *dE = static_cast<TE *>(a.dE);
        const int64_t rows = in_place ? a.B : a.V, most = std::max<int64_t>(1, kMaxGrid / chunks);
        const dim3 grid((unsigned)std::min<int64_t>(row_grid(rows, kThreads >> shift, chunks), most), (unsigned)chunks);
        const bool past = (int64_t)a.V * a.D * (int64_t)sizeof(TE) > kPastBytes;
        const auto kernel = in_place ? table_rows_kernel<T, TE, false, false>
                                     : past ? table_rows_kernel<T, TE, true, true> : table_rows_kernel<T, TE, true, false>;
        kernel<<<grid, kThreads, 0, s>>>(a.V, a.D, a.B, r, plan.sorted, w.bounds, a.scale, add, a.ldadd, dE, a.ldde, shift);
        return hipGetLastError();
    });
}

hipError_t launch_embedding_masked_bwd(const embedding_args &a, int nnz, const int *ptr, const int *col, float *gv,
                                       const void *plan_mem, void *ws, hipStream_t s) {
    if (a.V == 0 || a.D == 0 || nnz == 0) return hipSuccess;
    const plan_parts plan = carve_plan(a.B, const_cast<void *>(plan_mem));
    const bwd_parts w = carve_bwd(a.V, a.D, a.B, ws);
    run_rows<float> r;
    const hipError_t err = sort_columns<float>(a, plan, w, &r, s);
    if (err != hipSuccess) return err;
    const int shift = std::max(3, pow2_shift(nnz / a.V, 8));
    table_pattern_kernel<<<row_grid(a.V, kThreads >> shift, 1), kThreads, 0, s>>>(a.V, a.D, nnz, r, w.bounds, a.scale, ptr, col,
                                                                                  gv, shift);
    return hipGetLastError();
}

}  // namespace l1csr
