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

// A tile's features d0 .. d0 + 63 of the tokens b0 .. b0 + 63, from LDS [feature][token] to X[d][b]
template <typename T, typename F>
__device__ __forceinline__ void store_columns(const float (&tile)[kTile * kPitch], int D, int B, int d0, int b0, T *X,
                                              int64_t ldx, F value) {
    constexpr int V = 4, lanes = kTile / V;
    const int b = (threadIdx.x & (lanes - 1)) * V;
#pragma unroll
    for (int d = threadIdx.x / lanes; d < kTile; d += kThreads / lanes) {
        if (d0 + d >= D || b0 + b >= B) continue;
        const float *row = tile + d * kPitch + b;
        T x[V];
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = (T)value(row[v]);
        store_some<T, V>(X + (int64_t)(d0 + d) * ldx + b0 + b, B - b0 - b, x);
    }
}

template <typename TE, typename TX>
__global__ __launch_bounds__(kThreads) void gather_kernel(int V, int D, int B, const TE *__restrict__ E, int64_t lde,
                                                          const int *__restrict__ tokens, float scale,
                                                          TX *__restrict__ X, int64_t ldx, int d_tiles, int64_t tiles) {
    __shared__ float tile[kTile * kPitch];
    constexpr int N = kPer16<TE>, lanes = kTile / N;
    const int d = (threadIdx.x & (lanes - 1)) * N;
    for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
        const int d0 = (int)(i % d_tiles) * kTile, b0 = (int)(i / d_tiles) * kTile;
#pragma unroll
        for (int b = threadIdx.x / lanes; b < kTile; b += kThreads / lanes) {
            const int t = b0 + b < B ? tokens[b0 + b] : -1;
            TE e[N] = {};
            if (in_table(t, V) && d0 + d < D) load_some<TE, N>(E + (int64_t)t * lde + d0 + d, D - d0 - d, e);
#pragma unroll
            for (int n = 0; n < N; ++n) tile[(d + n) * kPitch + b] = widen(e[n]);
        }
        __syncthreads();
        store_columns(tile, D, B, d0, b0, X, ldx, [&](float x) { return scale * x; });
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// a table kept in CSR
// ---------------------------------------------------------------------------

constexpr int kCsrThreads = 1024;
constexpr int kCsrTokens = 32;     // of a tile: 128 bytes of a row of X
constexpr int kCsrFeatures = 512;  // of a tile
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
                                                                 float *__restrict__ X, int64_t ldx, int d_tiles,
                                                                 int64_t tiles) {
    __shared__ float tile[kCsrFeatures * kCsrPitch];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
        const int d0 = (int)(i % d_tiles) * kCsrFeatures, b0 = (int)(i / d_tiles) * kCsrTokens;
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

constexpr int kRun = 8192;         // tokens that are ranked by counting
constexpr int kRankThreads = 1024;

// what the tokens are sorted by: those of no row come last
__device__ __forceinline__ int key_of(int token, int V) { return in_table(token, V) ? token : V; }

// Ranks within runs of kRun tokens by counting the smaller ones (and the equal ones ahead): a lane a token, the waves
// of a workgroup share the run, whose tokens are read as scalars.
__global__ __launch_bounds__(kRankThreads) void rank_kernel(int V, int B, const int *__restrict__ tokens,
                                                            int *__restrict__ rank, int *__restrict__ sorted) {
    constexpr int waves = kRankThreads / kWave;
    __shared__ int part[waves][kWave];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    const int own = blockIdx.x * kWave, base = own / kRun * kRun, n = min(kRun, B - base);
    const int b = own + lane, key = key_of(b < B ? tokens[b] : -1, V);
    int less = 0;
    for (int j0 = wave * kWave; j0 < n; j0 += waves * kWave) {  // 64 tokens at a time
        const int at = base + j0, m = min(kWave, n - j0);
        if (at == own) {
            for (int j = 0; j < m; ++j) {
                const int other = key_of(tokens[at + j], V);
                less += other < key || (other == key && j < lane) ? 1 : 0;
            }
        } else {
            const int limit = key + (at < own ? 1 : 0);  // equal tokens ahead count
            if (m == kWave) {
#pragma unroll 16
                for (int j = 0; j < kWave; ++j) less += key_of(tokens[at + j], V) < limit ? 1 : 0;
            } else {
                for (int j = 0; j < m; ++j) less += key_of(tokens[at + j], V) < limit ? 1 : 0;
            }
        }
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

// Two sorted runs of `run` tokens become one: a token's rank grows by what goes before it in the other run.
__global__ __launch_bounds__(kThreads) void merge_kernel(int V, int B, int64_t run, const int *__restrict__ tokens,
                                                         int *__restrict__ rank, const int *__restrict__ sorted,
                                                         int *__restrict__ merged) {
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (b >= B) return;
    const int key = key_of(tokens[b], V);
    const int64_t q = b / run, other = (q ^ 1) * run;
    const int n = (int)min((int64_t)run, max((int64_t)0, B - other));
    // equal tokens of an earlier run go before
    const int r = rank[b] + lower_bound(sorted + other, n, key + (q & 1 ? 1 : 0));
    rank[b] = r;
    merged[(q & ~1ll) * run + r] = key;
}

// The plan's parts: rank[B] of every token, sorted[B] the tokens in order (V: of no row).  (Merged
// runs alternate between two arrays.)
struct plan_parts {
    int *rank, *sorted, *other;
};
plan_parts carve_plan(int B, void *plan) {
    int *p = static_cast<int *>(plan);
    plan_parts r{p, p + B, p + 2 * (size_t)B};
    for (int64_t run = kRun; run < B; run *= 2) std::swap(r.sorted, r.other);
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
    const float *groups;    // [B / 32][ld], a group's where its rows are of one token
    const float *blocks;    // [B / 1024][ld], of 32 groups
    int64_t ld;
};

// sum over rows lo .. hi - 1 of the values at d .. d + N - 1, in one order
template <typename T, int N>
__device__ __forceinline__ void sum_run(const run_rows<T> &r, int lo, int hi, int64_t d, float (&sum)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) sum[n] = 0.f;
    int i = lo;
    while (i < hi) {
        if (i % kGroup == 0 && hi - i >= kGroup) {
            float x[N];
            if (i % (kGroup * kGroup) == 0 && hi - i >= kGroup * kGroup) {
                load_values<float, N>(r.blocks + (int64_t)(i / (kGroup * kGroup)) * r.ld + d, x);
                i += kGroup * kGroup;
            } else {
                load_values<float, N>(r.groups + (int64_t)(i / kGroup) * r.ld + d, x);
                i += kGroup;
            }
#pragma unroll
            for (int n = 0; n < N; ++n) sum[n] += x[n];
        } else {
            T x[N];
            load_values<T, N>(r.rows + (int64_t)i * r.ld + d, x);
            ++i;
#pragma unroll
            for (int n = 0; n < N; ++n) sum[n] += widen(x[n]);
        }
    }
}

// rows[rank of b][d] = dX[d][b]
template <typename T>
__global__ __launch_bounds__(kThreads) void sort_columns_kernel(int V, int D, int B, const T *__restrict__ dX, int64_t ldx,
                                                                const int *__restrict__ rank,
                                                                const int *__restrict__ sorted, T *__restrict__ rows,
                                                                int64_t ld, int d_tiles, int64_t tiles) {
    __shared__ float tile[kTile * kPitch];  // [token][feature]
    constexpr int N = kPer16<T>, lanes = kTile / N;
    const int c = (threadIdx.x & (lanes - 1)) * N;
    for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
        const int d0 = (int)(i % d_tiles) * kTile, b0 = (int)(i / d_tiles) * kTile;
#pragma unroll
        for (int d = threadIdx.x / lanes; d < kTile; d += kThreads / lanes) {
            T x[N] = {};
            if (d0 + d < D && b0 + c < B) load_some<T, N>(dX + (int64_t)(d0 + d) * ldx + b0 + c, B - b0 - c, x);
#pragma unroll
            for (int n = 0; n < N; ++n) tile[(c + n) * kPitch + d] = widen(x[n]);
        }
        __syncthreads();
#pragma unroll
        for (int b = threadIdx.x / lanes; b < kTile; b += kThreads / lanes) {
            if (b0 + b >= B) continue;
            const int r = rank[b0 + b];
            if ((unsigned)r >= (unsigned)B || sorted[r] >= V) continue;
            T x[N];
#pragma unroll
            for (int n = 0; n < N; ++n) x[n] = (T)tile[b * kPitch + c + n];
            if (d0 + c < ld) store_values<T, N>(rows + (int64_t)r * ld + d0 + c, x);  // ld: D up to a multiple of 8
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

constexpr int kRowBlock = 8;  // least rows of a workgroup, whose runs are searched side by side

// dE, every row of it (all), or dE += where only the rows that have tokens change: then a workgroup's rows are
// places in the order, of which the first of each run has work.
template <typename T, typename TE, bool ALL>
__global__ __launch_bounds__(kThreads) void table_rows_kernel(int V, int D, int B, run_rows<T> r,
                                                              const int *__restrict__ sorted, float scale,
                                                              const TE *add, int64_t ldadd, TE *dE, int64_t ldde,
                                                              int tx_shift) {
    constexpr int N = 4;
    __shared__ int bound[kThreads + 1];
    const int TX = 1 << tx_shift, TY = kThreads >> tx_shift, per = max(TY, kRowBlock);
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> tx_shift;
    const int64_t total = ALL ? V : B;
    for (int64_t v0 = (int64_t)blockIdx.x * per; v0 < total; v0 += (int64_t)gridDim.x * per) {
        __syncthreads();
        for (int i = threadIdx.x; i < per + ALL; i += kThreads) {
            const int64_t v = v0 + i;
            if constexpr (ALL) {
                bound[i] = lower_bound(sorted, B, (int)min(v, (int64_t)V));
            } else {
                // the end of the run that begins here; 0 where none does
                int end = 0;
                if (v < B && sorted[v] < V && (v == 0 || sorted[v - 1] != sorted[v]))
                    end = (int)v + lower_bound(sorted + v, B - (int)v, sorted[v] + 1);
                bound[i] = end;
            }
        }
        __syncthreads();
        for (int y = ty; y < per && v0 + y < total; y += TY) {
            int lo, hi;
            int64_t v = v0 + y;
            if constexpr (ALL) {
                lo = bound[y];
                hi = bound[y + 1];
            } else {
                lo = (int)v;
                hi = bound[y];
                if (hi <= lo) continue;
                v = sorted[lo];
            }
            for (int64_t d = tx * N; d < D; d += TX * N) {
                float s[N];
                sum_run<T, N>(r, lo, hi, d, s);
                TE e[N] = {};
                if (add) load_some<TE, N>(add + v * ldadd + d, D - d, e);
#pragma unroll
                for (int n = 0; n < N; ++n) e[n] = (TE)(widen(e[n]) + scale * s[n]);
                store_some<TE, N>(dE + v * ldde + d, D - d, e);
            }
        }
    }
}

// gv on the pattern: a wave a row of the table
__global__ __launch_bounds__(kThreads) void table_pattern_kernel(int V, int D, int B, int nnz, run_rows<float> r,
                                                                 const int *__restrict__ sorted, float scale,
                                                                 const int *__restrict__ ptr, const int *__restrict__ col,
                                                                 float *__restrict__ gv) {
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    for (int64_t v = (int64_t)blockIdx.x * (kThreads / kWave) + wave; v < V; v += (int64_t)gridDim.x * (kThreads / kWave)) {
        const int p0 = max(ptr[v], 0), p1 = min(ptr[v + 1], nnz);
        if (p0 >= p1) continue;
        const int lo = lower_bound(sorted, B, (int)v), hi = lo + lower_bound(sorted + lo, B - lo, (int)v + 1);
        for (int p = p0 + lane; p < p1; p += kWave) {
            float s[1] = {};
            if (lo < hi && (unsigned)col[p] < (unsigned)D) sum_run<float, 1>(r, lo, hi, col[p], s);
            gv[p] = scale * s[0];
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

struct bwd_parts {
    char *rows;
    float *groups, *blocks;
};
bwd_parts carve_bwd(int D, int B, void *ws) {
    char *p = static_cast<char *>(ws);
    const int64_t ld = padded(D);
    bwd_parts w;
    w.groups = reinterpret_cast<float *>(p);
    w.blocks = w.groups + B / kGroup * ld;
    w.rows = reinterpret_cast<char *>(w.blocks + B / (kGroup * kGroup) * ld);
    return w;
}

// the columns of dX as rows in the tokens' order, and the sums of their groups
template <typename T>
hipError_t sort_columns(const embedding_args &a, const plan_parts &plan, const bwd_parts &w, run_rows<T> *r,
                        hipStream_t s) {
    const int64_t ld = padded(a.D);
    T *rows = reinterpret_cast<T *>(w.rows);
    *r = {rows, w.groups, w.blocks, ld};
    const int d_tiles = (int)ceil_div(a.D, kTile);
    const int64_t tiles = d_tiles * ceil_div(a.B, kTile);
    sort_columns_kernel<T><<<grid_of(tiles), kThreads, 0, s>>>(a.V, a.D, a.B, static_cast<const T *>(a.X), a.ldx, plan.rank,
                                                               plan.sorted, rows, ld, d_tiles, tiles);
    const int groups = a.B / kGroup, blocks = a.B / (kGroup * kGroup);
    if (groups > 0)
        group_kernel<T><<<grid_of(groups), kThreads, 0, s>>>(a.V, a.B, 1, rows, plan.sorted, w.groups, ld, groups);
    if (blocks > 0)
        group_kernel<float><<<grid_of(blocks), kThreads, 0, s>>>(a.V, a.B, kGroup, w.groups, plan.sorted, w.blocks, ld,
                                                                 blocks);
    return hipGetLastError();
}

}  // namespace

bool embedding_fits(int64_t V, int64_t D, int64_t B) {
    constexpr int64_t most = 1 << 30;
    return V <= most && D <= most && B <= 1 << 24;  // (a launch has fewer than 2^32 threads)
}

size_t embedding_plan_bytes(int B) { return sizeof(int) * 3 * (size_t)std::max(B, 0); }

size_t embedding_bwd_workspace_bytes(int D, int B) {
    if (D <= 0 || B <= 0) return 0;
    return (size_t)padded(D) * sizeof(float) * ((size_t)B + B / kGroup + B / (kGroup * kGroup));
}

hipError_t launch_embedding_fwd(const embedding_args &a, hipStream_t s) {
    if (a.D == 0 || a.B == 0) return hipSuccess;
    const int d_tiles = (int)ceil_div(a.D, kTile);
    const int64_t tiles = d_tiles * ceil_div(a.B, kTile);
    return with_types(a.dtype, a.x_dtype, [&](auto e, auto x) {
        using TE = decltype(e);
        using TX = decltype(x);
        gather_kernel<TE, TX><<<grid_of(tiles), kThreads, 0, s>>>(a.V, a.D, a.B, static_cast<const TE *>(a.E), a.lde,
                                                                  a.tokens, a.scale, static_cast<TX *>(a.X_out), a.ldx,
                                                                  d_tiles, tiles);
        return hipGetLastError();
    });
}

hipError_t launch_embedding_csr_fwd(const embedding_args &a, int nnz, const int *ptr, const int *col, const float *val,
                                    hipStream_t s) {
    if (a.D == 0 || a.B == 0) return hipSuccess;
    const int d_tiles = (int)ceil_div(a.D, kCsrFeatures);
    const int64_t tiles = d_tiles * ceil_div(a.B, kCsrTokens);
    gather_csr_kernel<<<grid_of(tiles), kCsrThreads, 0, s>>>(a.V, a.D, a.B, nnz, ptr, col, val, a.tokens, a.scale,
                                                             static_cast<float *>(a.X_out), a.ldx, d_tiles, tiles);
    return hipGetLastError();
}

hipError_t launch_embedding_plan(int V, int B, const int *tokens, void *plan, hipStream_t s) {
    if (B == 0) return hipSuccess;
    int *rank = static_cast<int *>(plan), *from = rank + B, *to = from + B;
    rank_kernel<<<(int)ceil_div(B, kWave), kRankThreads, 0, s>>>(V, B, tokens, rank, from);
    for (int64_t run = kRun; run < B; run *= 2) {
        merge_kernel<<<(int)ceil_div(B, kThreads), kThreads, 0, s>>>(V, B, run, tokens, rank, from, to);
        std::swap(from, to);
    }
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(const embedding_args &a, const void *plan_mem, void *ws, hipStream_t s) {
    if (a.D == 0 || a.V == 0) return hipSuccess;
    const plan_parts plan = carve_plan(a.B, const_cast<void *>(plan_mem));
    const bwd_parts w = carve_bwd(a.D, a.B, ws);
    return with_types(a.dtype, a.e_dtype, [&](auto x, auto e) {
        using T = decltype(x);
        using TE = decltype(e);
        run_rows<T> r{};
        if (a.B > 0) {
            const hipError_t err = sort_columns<T>(a, plan, w, &r, s);
            if (err != hipSuccess) return err;
        }
        const int shift = pow2_shift(ceil_div(a.D, 4), 8), per = std::max(kThreads >> shift, kRowBlock);
        const TE *add = static_cast<const TE *>(a.add);
        TE *dE = static_cast<TE *>(a.dE);
        if (a.add != nullptr && a.add == a.dE) {
            if (a.B > 0)
                table_rows_kernel<T, TE, false><<<grid_of(ceil_div(a.B, per)), kThreads, 0, s>>>(
                    a.V, a.D, a.B, r, plan.sorted, a.scale, add, a.ldadd, dE, a.ldde, shift);
        } else {
            table_rows_kernel<T, TE, true><<<grid_of(ceil_div(a.V, per)), kThreads, 0, s>>>(
                a.V, a.D, a.B, r, plan.sorted, a.scale, add, a.ldadd, dE, a.ldde, shift);
        }
        return hipGetLastError();
    });
}

hipError_t launch_embedding_masked_bwd(const embedding_args &a, int nnz, const int *ptr, const int *col, float *gv,
                                       const void *plan_mem, void *ws, hipStream_t s) {
    if (a.V == 0 || nnz == 0) return hipSuccess;
    const plan_parts plan = carve_plan(a.B, const_cast<void *>(plan_mem));
    const bwd_parts w = carve_bwd(a.D, a.B, ws);
    run_rows<float> r{};
    if (a.B > 0) {
        const hipError_t err = sort_columns<float>(a, plan, w, &r, s);
        if (err != hipSuccess) return err;
    }
    table_pattern_kernel<<<grid_of(ceil_div(a.V, kThreads / kWave)), kThreads, 0, s>>>(a.V, a.D, a.B, nnz, r, plan.sorted,
                                                                                       a.scale, ptr, col, gv);
    return hipGetLastError();
}

}  // namespace l1csr
