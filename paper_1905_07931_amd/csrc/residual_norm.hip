// Norms before and after a block, with its gate and its residual, for activations [K][B] (features by tokens, tokens
// contiguous); per token (column):
//   q  = 1 / sqrt(mean_k y^2 + eps),  n = y q w_post     (without post gain: n = y)
//   r' = r + alpha a(gate) n
//   s  = 1 / sqrt(mean_k r'^2 + eps), h = r' s w_pre
// and the gradients, from dr' (of r' as it is used further on) and dh:
//   u = dh w_pre,  c = mean(u r'),  t = dr' + s u - s^3 c r',  dr = t
//   k = alpha a w_post,  e = mean(k y t),  dy = q k t - q^3 e y     (without post gain: dy = alpha a t)
//   dgate = alpha t n' a'(gate),  n' = y q w_post;  dw_pre = sum_b dh r' s;  dw_post = sum_b alpha a t y q
//
// Both means of a call come from one pass.  Forward: with x = alpha a w_post y, r' = r + q x and
// sum r'^2 = sum r^2 + 2 q sum r x + q^2 sum x^2.  Backward: sum k y t = sum k y dr' + s sum k y u - s^3 c sum k y r'.
// The sums are in double (the forward one cancels where a block takes back what the residual holds), in a fixed order.
// Three launches: the sums of ranges of rows, their join to a column's factors, the results.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"
#include "typed.hpp"

namespace l1csr {

namespace {

constexpr int kThreads = 256;
constexpr int kSums = 6;       // most sums of a column
constexpr int kFactors = 4;    // most factors of a column
constexpr int kMaxSplits = 64; // most ranges of rows that a column's sums are taken over

// How a workgroup lies over [K][B]: 2^tx_shift threads of V columns each side by side, the others over the rows;
// blockIdx.y a range of rows.
struct norm_grid {
    int tx_shift, splits, rows;
};

template <int V>
struct columns {
    int col0, n;  // the first column of this thread, how many of its V exist
    __device__ columns(int tx, int tx_shift, int B) {
        const int64_t c = (((int64_t)blockIdx.x << tx_shift) + tx) * V;
        col0 = (int)min(c, (int64_t)B);
        n = min(V, B - col0);
    }
};

template <typename T, int V>
__device__ __forceinline__ void load_columns(const T *p, int n, float (&x)[V]) {
    T t[V];
    load_some<T, V>(p, n, t);
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = widen(t[v]);
}

template <typename T, int V>
__device__ __forceinline__ void store_columns(T *p, int n, const float (&x)[V]) {
    T t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t[v] = (T)x[v];
    store_some<T, V>(p, n, t);
}

// The gate of a row's columns: a(g), and its derivative
template <typename T, int V, int GATE, bool SIGMOID>
struct gate_values {
    float a[V], da[V];
    __device__ __forceinline__ void set(int v, float g) {
        if constexpr (SIGMOID) {
            a[v] = 1.f / (1.f + expf(-g));
            da[v] = a[v] * (1.f / (1.f + expf(g)));
        } else {
            a[v] = g;
            da[v] = 1.f;
        }
    }
    __device__ __forceinline__ gate_values(const norm_args &A, int k, int col0, int n) {
        if constexpr (GATE == kGateFull) {
            float g[V];
            load_columns<T, V>(static_cast<const T *>(A.gate) + (int64_t)k * A.ldg + col0, n, g);
#pragma unroll
            for (int v = 0; v < V; ++v) set(v, g[v]);
        } else if constexpr (GATE == kGateRow) {
            set(0, static_cast<const float *>(A.gate)[k]);
#pragma unroll
            for (int v = 1; v < V; ++v) {
                a[v] = a[0];
                da[v] = da[0];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                a[v] = 1.f;
                da[v] = 0.f;
            }
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ void load_row(const void *p, int64_t ld, int k, int col0, int n, float (&x)[V]) {
    load_columns<T, V>(static_cast<const T *>(p) + (int64_t)k * ld + col0, n, x);
}

// Joins the sums of a workgroup's threads over the rows and stores them: part[q][split][B]
template <int V, int NS>
__device__ __forceinline__ void store_sums(const double (&sum)[NS][V], const norm_grid &g, const columns<V> &c, int B,
                                           double *lds, double *part) {
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
#pragma unroll
    for (int q = 0; q < NS; ++q) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) lds[v * kThreads + threadIdx.x] = sum[q][v];
        __syncthreads();
        if (ty == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                double t = 0;
                for (int y = 0; y < TY; ++y) t += lds[v * kThreads + (y << g.tx_shift) + tx];
                if (v < c.n) part[((int64_t)q * g.splits + blockIdx.y) * B + c.col0 + v] = t;
            }
        }
    }
}

constexpr int kJoinColumns = 32;  // of a workgroup of the join; the other threads share the ranges of rows

// Joins the sums over the ranges of rows; true in the threads that hold a column's
template <int NS>
__device__ __forceinline__ bool join_sums(const double *__restrict__ part, int splits, int B, int col, double *lds,
                                          double (&sum)[NS]) {
    constexpr int ways = kThreads / kJoinColumns;
    const int way = threadIdx.x / kJoinColumns;
#pragma unroll
    for (int q = 0; q < NS; ++q) {
        double t = 0;
        if (col < B)
            for (int i = way; i < splits; i += ways) t += part[((int64_t)q * splits + i) * B + col];
        lds[q * kThreads + threadIdx.x] = t;
    }
    __syncthreads();
    if (way != 0 || col >= B) return false;
#pragma unroll
    for (int q = 0; q < NS; ++q) {
        sum[q] = 0;
        for (int i = 0; i < ways; ++i) sum[q] += lds[q * kThreads + i * kJoinColumns + threadIdx.x];
    }
    return true;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// what a call has: y (with gate), a norm of y, a norm of r'
enum { kHasY = 1, kHasPost = 2, kHasPre = 4 };

template <typename T, int V, int GATE, bool SIGMOID, int HAS>
__global__ __launch_bounds__(kThreads) void forward_sums_kernel(norm_args A, norm_grid g, double *__restrict__ part) {
    constexpr int NS = 4;  // y^2; r^2, r x, x^2 (without post: r'^2 alone)
    __shared__ double lds[kThreads * V];
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> c(tx, g.tx_shift, A.B);
    double sum[NS][V] = {};
    const int k1 = min(A.K, (int)(blockIdx.y + 1) * g.rows);
    if (c.n > 0)
        for (int k = blockIdx.y * g.rows + ty; k < k1; k += TY) {
            float r[V], y[V];
            if constexpr (HAS & kHasPre) load_row<T, V>(A.r, A.ldr, k, c.col0, c.n, r);
            if constexpr (HAS & kHasY) load_row<T, V>(A.y, A.ldy, k, c.col0, c.n, y);
            const gate_values<T, V, GATE, SIGMOID> gate(A, k, c.col0, c.n);
            const float w = HAS & kHasPost ? A.post_gain[k] : 1.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (HAS & kHasPost) sum[0][v] += (double)y[v] * y[v];
                if constexpr (HAS & kHasPre) {
                    if constexpr (HAS & kHasPost) {
                        const double x = (double)(A.alpha * gate.a[v] * w) * y[v];
                        sum[1][v] += (double)r[v] * r[v];
                        sum[2][v] += r[v] * x;
                        sum[3][v] += x * x;
                    } else {
                        double x = r[v];
                        if constexpr (HAS & kHasY) x += (double)(A.alpha * gate.a[v]) * y[v];
                        sum[1][v] += x * x;
                    }
                }
            }
        }
    store_sums<V, NS>(sum, g, c, A.B, lds, part);
}

// a column's factors: q, s
__global__ __launch_bounds__(kThreads) void forward_join_kernel(int K, int B, float eps, int splits, bool post, bool pre,
                                                                const double *__restrict__ part, float *__restrict__ fac) {
    __shared__ double lds[4 * kThreads];
    const int col = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    double sum[4];
    if (!join_sums<4>(part, splits, B, col, lds, sum)) return;
    const double q = post ? 1 / sqrt(sum[0] / K + eps) : 1.0;
    fac[col] = (float)q;
    if (!pre) return;
    const double square = sum[1] + q * (2 * sum[2] + q * sum[3]);
    fac[B + col] = (float)(1 / sqrt((square < 0 ? 0 : square) / K + eps));  // (a NaN stays one)
}

template <typename T, int V, int GATE, bool SIGMOID, int HAS>
__global__ __launch_bounds__(kThreads) void forward_kernel(norm_args A, norm_grid g, const float *__restrict__ fac) {
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> c(tx, g.tx_shift, A.B);
    if (c.n <= 0) return;
    float q[V], s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = c.col0 + min(v, c.n - 1);
        q[v] = HAS & kHasPost ? fac[col] : 1.f;
        s[v] = HAS & kHasPre ? fac[A.B + col] : 0.f;
    }
    const int k1 = min(A.K, (int)(blockIdx.y + 1) * g.rows);
    for (int k = blockIdx.y * g.rows + ty; k < k1; k += TY) {
        float r[V], y[V];
        load_row<T, V>(A.r, A.ldr, k, c.col0, c.n, r);
        if constexpr (HAS & kHasY) {
            load_row<T, V>(A.y, A.ldy, k, c.col0, c.n, y);
            const gate_values<T, V, GATE, SIGMOID> gate(A, k, c.col0, c.n);
            const float w = HAS & kHasPost ? A.post_gain[k] : 1.f;
#pragma unroll
            for (int v = 0; v < V; ++v) r[v] += A.alpha * gate.a[v] * w * (y[v] * q[v]);
            store_columns<T, V>(static_cast<T *>(A.r_out) + (int64_t)k * A.ldro + c.col0, c.n, r);
        }
        if constexpr (HAS & kHasPre) {
            const float w = A.pre_gain[k];
#pragma unroll
            for (int v = 0; v < V; ++v) r[v] = r[v] * s[v] * w;
            store_columns<T, V>(static_cast<T *>(A.h) + (int64_t)k * A.ldh + c.col0, c.n, r);
        }
    }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------

template <typename T, int V, int GATE, bool SIGMOID, int HAS>
__global__ __launch_bounds__(kThreads) void backward_sums_kernel(norm_args A, norm_grid g, double *__restrict__ part) {
    constexpr int NS = kSums;  // r'^2, u r'; y^2, k y dr', k y u, k y r'
    __shared__ double lds[kThreads * V];
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> c(tx, g.tx_shift, A.B);
    double sum[NS][V] = {};
    const int k1 = min(A.K, (int)(blockIdx.y + 1) * g.rows);
    if (c.n > 0)
        for (int k = blockIdx.y * g.rows + ty; k < k1; k += TY) {
            float r[V], u[V] = {}, y[V], dr[V] = {};
            if constexpr (HAS & kHasPre) {
                load_row<T, V>(A.r_out, A.ldro, k, c.col0, c.n, r);
                load_row<T, V>(A.dh, A.lddh, k, c.col0, c.n, u);
                const float w = A.pre_gain[k];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    u[v] *= w;
                    sum[0][v] += (double)r[v] * r[v];
                    sum[1][v] += (double)u[v] * r[v];
                }
            }
            if constexpr (HAS & kHasPost) {
                load_row<T, V>(A.y, A.ldy, k, c.col0, c.n, y);
                if (A.dr_out) load_row<T, V>(A.dr_out, A.lddro, k, c.col0, c.n, dr);
                const gate_values<T, V, GATE, SIGMOID> gate(A, k, c.col0, c.n);
                const float w = A.post_gain[k];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const double ky = (double)(A.alpha * gate.a[v] * w) * y[v];
                    sum[2][v] += (double)y[v] * y[v];
                    sum[3][v] += ky * dr[v];
                    if constexpr (HAS & kHasPre) {
                        sum[4][v] += ky * u[v];
                        sum[5][v] += ky * r[v];
                    }
                }
            }
        }
    store_sums<V, NS>(sum, g, c, A.B, lds, part);
}

// a column's factors: s, f = s^2 c, q, g = q^2 e
__global__ __launch_bounds__(kThreads) void backward_join_kernel(int K, int B, float eps, int splits, bool post, bool pre,
                                                                 const double *__restrict__ part, float *__restrict__ fac) {
    __shared__ double lds[kSums * kThreads];
    const int col = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    double sum[kSums];
    if (!join_sums<kSums>(part, splits, B, col, lds, sum)) return;
    double s = 0, f = 0;
    if (pre) {
        s = 1 / sqrt(sum[0] / K + eps);
        f = s * s * sum[1] / K;
        fac[col] = (float)s;
        fac[B + col] = (float)f;
    }
    if (post) {
        const double q = 1 / sqrt(sum[2] / K + eps), m = sum[3] + s * (sum[4] - f * sum[5]);
        fac[2 * (int64_t)B + col] = (float)q;
        fac[3 * (int64_t)B + col] = (float)(q * q * m / K);
    }
}

// Sums over a workgroup's columns of a row go to rows[i][column block][K], i = dw_pre, dw_post, dgate
template <typename T, int V, int GATE, bool SIGMOID, int HAS>
__global__ __launch_bounds__(kThreads) void backward_kernel(norm_args A, norm_grid g, const float *__restrict__ fac,
                                                            float *__restrict__ rows) {
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> c(tx, g.tx_shift, A.B);
    float s[V] = {}, f[V] = {}, q[V], e[V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = min(c.col0 + v, A.B - 1);
        s[v] = HAS & kHasPre ? fac[col] : 0.f;
        f[v] = HAS & kHasPre ? fac[A.B + col] : 0.f;
        q[v] = HAS & kHasPost ? fac[2 * (int64_t)A.B + col] : 1.f;
        e[v] = HAS & kHasPost ? fac[3 * (int64_t)A.B + col] : 0.f;
    }
    const int k1 = min(A.K, (int)(blockIdx.y + 1) * g.rows);
    for (int k = blockIdx.y * g.rows + ty; k < k1; k += TY) {
        float t[V] = {}, sums[3] = {};
        if (c.n > 0) {
            if (A.dr_out) load_row<T, V>(A.dr_out, A.lddro, k, c.col0, c.n, t);
            if constexpr (HAS & kHasPre) {
                float r[V], dh[V];
                load_row<T, V>(A.r_out, A.ldro, k, c.col0, c.n, r);
                load_row<T, V>(A.dh, A.lddh, k, c.col0, c.n, dh);
                const float w = A.pre_gain[k];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float rs = r[v] * s[v];
                    sums[0] += v < c.n ? dh[v] * rs : 0.f;
                    t[v] += s[v] * (dh[v] * w) - f[v] * rs;
                }
            }
            if (A.dr) store_columns<T, V>(static_cast<T *>(A.dr) + (int64_t)k * A.lddr + c.col0, c.n, t);
            if constexpr (HAS & kHasY) {
                float y[V], dy[V], dg[V];
                load_row<T, V>(A.y, A.ldy, k, c.col0, c.n, y);
                const gate_values<T, V, GATE, SIGMOID> gate(A, k, c.col0, c.n);
                const float w = HAS & kHasPost ? A.post_gain[k] : 1.f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float at = A.alpha * t[v], yq = y[v] * q[v];
                    dy[v] = gate.a[v] * at * w * q[v] - e[v] * yq;
                    dg[v] = at * yq * w * gate.da[v];
                    sums[1] += v < c.n ? gate.a[v] * at * yq : 0.f;
                    sums[2] += v < c.n ? dg[v] : 0.f;
                }
                store_columns<T, V>(static_cast<T *>(A.dy) + (int64_t)k * A.lddy + c.col0, c.n, dy);
                if constexpr (GATE == kGateFull)
                    store_columns<T, V>(static_cast<T *>(A.dgate) + (int64_t)k * A.lddg + c.col0, c.n, dg);
            }
        }
        const int lanes = min(TX, kWave);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (i == 0 ? !(HAS & kHasPre) : i == 1 ? !(HAS & kHasPost) : GATE != kGateRow) continue;
            for (int d = lanes / 2; d >= 1; d >>= 1) sums[i] += __shfl_xor(sums[i], d, kWave);
            if (tx == 0) rows[((int64_t)i * gridDim.x + blockIdx.x) * A.K + k] = sums[i];
        }
    }
}

// a row's sum over the column blocks
__global__ __launch_bounds__(kThreads) void row_sums_kernel(int K, int blocks, const float *__restrict__ rows,
                                                            float *pre, float *post, float *gate) {
    const int k = blockIdx.x * kThreads + threadIdx.x;
    if (k >= K) return;
    float *out[3] = {pre, post, gate};
    for (int i = 0; i < 3; ++i) {
        if (out[i] == nullptr) continue;
        double t = 0;
        for (int b = 0; b < blocks; ++b) t += rows[((int64_t)i * blocks + b) * K + k];
        out[i][k] = (float)t;
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

int vector_of(int B, int dtype) {
    const int v = dtype == kTypeF32 ? 4 : 8;
    return B >= v ? v : 1;
}

norm_grid grid_for(int K, int B, int dtype, int *col_blocks) {
    norm_grid g;
    const int64_t lanes = ceil_div(B, vector_of(B, dtype));
    g.tx_shift = 0;
    while (g.tx_shift < 6 && (1 << g.tx_shift) < lanes) ++g.tx_shift;
    *col_blocks = (int)ceil_div(lanes, 1 << g.tx_shift);
    const int TY = kThreads >> g.tx_shift;
    // about 2048 workgroups, of 8 rows a thread at least
    const int64_t most = std::min<int64_t>(kMaxSplits, ceil_div(K, 8 * TY));
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(most, 2048 / *col_blocks));
    g.rows = (int)(ceil_div(ceil_div(K, splits), TY) * TY);
    g.splits = (int)ceil_div(K, g.rows);
    return g;
}

template <typename F>
hipError_t with_gate(int gate, bool sigmoid, F f) {
    using std::integral_constant;
    using std::false_type;
    using std::true_type;
    if (gate == kGateRow) return sigmoid ? f(integral_constant<int, kGateRow>{}, true_type{}) : f(integral_constant<int, kGateRow>{}, false_type{});
    if (gate == kGateFull) return sigmoid ? f(integral_constant<int, kGateFull>{}, true_type{}) : f(integral_constant<int, kGateFull>{}, false_type{});
    return f(integral_constant<int, kGateNone>{}, false_type{});
}

// f(T, V, GATE, SIGMOID, HAS) as compile-time values
template <typename F>
hipError_t with_variant(const norm_args &a, F f) {
    using std::integral_constant;
    auto typed = [&](auto t) {
        using T = decltype(t);
        auto wide = [&](auto v) {
            if (a.y == nullptr) return f(t, v, integral_constant<int, kGateNone>{}, std::false_type{}, integral_constant<int, kHasPre>{});
            return with_gate(a.gate_kind, a.sigmoid, [&](auto gate, auto sig) {
                if (a.post_gain && a.pre_gain) return f(t, v, gate, sig, integral_constant<int, kHasY | kHasPost | kHasPre>{});
                if (a.post_gain) return f(t, v, gate, sig, integral_constant<int, kHasY | kHasPost>{});
                if (a.pre_gain) return f(t, v, gate, sig, integral_constant<int, kHasY | kHasPre>{});
                return f(t, v, gate, sig, integral_constant<int, kHasY>{});
            });
        };
        return vector_of(a.B, a.dtype) == 1 ? wide(integral_constant<int, 1>{}) : wide(integral_constant<int, kPer16<T>>{});
    };
    if (a.dtype == kTypeF32) return typed(float{});
    if (a.dtype == kTypeBF16) return typed(__bf16{});
    return typed(_Float16{});
}

}  // namespace

size_t residual_norm_workspace_bytes(int K, int B) {
    if (K <= 0 || B <= 0) return 0;
    size_t most = 0;
    for (int dtype : {kTypeF32, kTypeBF16}) {
        int col_blocks;
        const norm_grid g = grid_for(K, B, dtype, &col_blocks);
        most = std::max(most, sizeof(double) * kSums * (size_t)g.splits * B +
                                  sizeof(float) * (kFactors * (size_t)B + 3 * (size_t)col_blocks * K));
    }
    return most;
}

hipError_t launch_residual_norm_fwd(const norm_args &a, void *ws, hipStream_t s) {
    if (a.K == 0 || a.B == 0) return hipSuccess;
    int col_blocks;
    const norm_grid g = grid_for(a.K, a.B, a.dtype, &col_blocks);
    const dim3 grid(col_blocks, g.splits);
    double *part = static_cast<double *>(ws);
    float *fac = reinterpret_cast<float *>(part + kSums * (size_t)g.splits * a.B);
    return with_variant(a, [&](auto t, auto v, auto gate, auto sig, auto has) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, G = decltype(gate)::value, H = decltype(has)::value;
        constexpr bool S = decltype(sig)::value;
        if constexpr ((H & (kHasPost | kHasPre)) != 0) {
            forward_sums_kernel<T, V, G, S, H><<<grid, kThreads, 0, s>>>(a, g, part);
            forward_join_kernel<<<(int)ceil_div(a.B, kJoinColumns), kThreads, 0, s>>>(
                a.K, a.B, a.eps, g.splits, (H & kHasPost) != 0, (H & kHasPre) != 0, part, fac);
        }
        forward_kernel<T, V, G, S, H><<<grid, kThreads, 0, s>>>(a, g, fac);
        return hipGetLastError();
    });
}

hipError_t launch_residual_norm_bwd(const norm_args &a, void *ws, hipStream_t s) {
    if (a.K == 0) return hipSuccess;
    if (a.B == 0) {
        row_sums_kernel<<<(int)ceil_div(a.K, kThreads), kThreads, 0, s>>>(a.K, 0, nullptr, a.dpre_gain, a.dpost_gain,
                                                                         a.gate_kind == kGateRow ? static_cast<float *>(a.dgate) : nullptr);
        return hipGetLastError();
    }
    int col_blocks;
    const norm_grid g = grid_for(a.K, a.B, a.dtype, &col_blocks);
    const dim3 grid(col_blocks, g.splits);
    double *part = static_cast<double *>(ws);
    float *fac = reinterpret_cast<float *>(part + kSums * (size_t)g.splits * a.B), *rows = fac + kFactors * (size_t)a.B;
    return with_variant(a, [&](auto t, auto v, auto gate, auto sig, auto has) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, G = decltype(gate)::value, H = decltype(has)::value;
        constexpr bool S = decltype(sig)::value;
        if constexpr ((H & (kHasPost | kHasPre)) != 0) {
            backward_sums_kernel<T, V, G, S, H><<<grid, kThreads, 0, s>>>(a, g, part);
            backward_join_kernel<<<(int)ceil_div(a.B, kJoinColumns), kThreads, 0, s>>>(
                a.K, a.B, a.eps, g.splits, (H & kHasPost) != 0, (H & kHasPre) != 0, part, fac);
        }
        backward_kernel<T, V, G, S, H><<<grid, kThreads, 0, s>>>(a, g, fac, rows);
        float *dgate = G == kGateRow ? static_cast<float *>(a.dgate) : nullptr;
        if (a.dpre_gain || a.dpost_gain || dgate)
            row_sums_kernel<<<(int)ceil_div(a.K, kThreads), kThreads, 0, s>>>(a.K, col_blocks, rows, a.dpre_gain, a.dpost_gain, dgate);
        return hipGetLastError();
    });
}

}  // namespace l1csr
