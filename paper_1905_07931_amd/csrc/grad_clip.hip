// The norm of many gradients together, and their clipping to it:
//   norm = sqrt(sum over all tensors of g^2) * inv_scale
//   g   <- g f inv_scale,  f = min(1, max_norm / (norm + eps))
// inv_scale takes out a factor that the gradients hold (the losses' grad_scale).
// Squares are added in double (no value of the three types overflows there), in a fixed order.
//
// The tensors' addresses and sizes go to the kernels as arguments, kTable of them a launch: nothing is copied
// to the device, and a captured call holds its own.  A tensor is cut into chunks of 32 KB (8 KB where all of them are
// few), dealt to the workgroups one after another: a thread's 8 loads of a chunk are under way together.  Reading 436 MB
// so takes 7.1 TB/s past the caches and 6.3 through them, 5.2 where a workgroup's loads lie a whole grid apart.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"
#include "typed.hpp"

namespace l1csr {

namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 2048;  // most workgroups (and partial sums) of a launch
constexpr int kTable = 48;     // tensors of a launch (of the 4 KB of arguments)

struct table_entry {
    const void *g;
    void *out;
    int64_t cols, ld, ldo;
    int64_t first;   // chunk
    int rows, block; // rows; rows of a chunk, or 0: a row has several chunks
    int chunk;       // values of a chunk
    int type, out_type;
};
struct table {
    int n;
    int64_t chunks;
    table_entry t[kTable];
};

// The rows and columns of chunk `i` of a tensor
struct chunk_range {
    int64_t r0, r1, c0, c1;
    __device__ __forceinline__ chunk_range(const table_entry &e, int64_t i) {
        if (e.block > 0) {
            r0 = i * e.block;
            r1 = min(r0 + e.block, (int64_t)e.rows);
            c0 = 0;
            c1 = e.cols;
        } else {
            r0 = 0;
            if (e.rows > 1) {
                const int64_t pieces = (e.cols + e.chunk - 1) / e.chunk;
                r0 = i / pieces;
                i -= r0 * pieces;
            }
            r1 = r0 + 1;
            c0 = i * e.chunk;
            c1 = min(c0 + e.chunk, e.cols);
        }
    }
};

__device__ __forceinline__ int tensor_of(const table &t, int64_t chunk) {
    int lo = 0, n = t.n;  // the last whose first chunk is no later
    while (n > 1) {
        const int half = n >> 1;
        if (t.t[lo + half].first <= chunk) lo += half, n -= half; else n = half;
    }
    return lo;
}

constexpr int kAhead = 8;  // loads of 16 bytes that a thread has under way

// f(row, column, values, how many) for the vectors of a chunk that are this thread's (fewer than a vector at a row's end)
template <typename T, int V, typename F>
__device__ __forceinline__ void for_vectors(const table_entry &e, const chunk_range &r, F f) {
    const int TX = e.block > 1 ? kWave : kThreads, tx = threadIdx.x & (TX - 1), ty = threadIdx.x / TX;
    for (int64_t row = r.r0 + ty; row < r.r1; row += kThreads / TX) {
        const T *p = static_cast<const T *>(e.g) + row * e.ld;
        int64_t c = r.c0 + tx * V;
        const int step = TX * V;
        for (; r.c1 - c >= (kAhead - 1) * step + V; c += kAhead * step) {
            T x[kAhead][V];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) load_past<T, V>(p + c + u * step, x[u]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) f(row, c + u * step, x[u], V);
        }
        for (; c < r.c1; c += 2 * step) {
            T x[2][V];
            const int64_t left = r.c1 - c;
            load_some<T, V>(p + c, left, x[0]);
            load_some<T, V>(p + c + step, left - step, x[1]);
            f(row, c, x[0], (int)min((int64_t)V, left));
            if (left > step) f(row, c + step, x[1], (int)min((int64_t)V, left - step));
        }
    }
}

template <typename T>
__device__ __forceinline__ double squares(const table_entry &e, const chunk_range &r) {
    double sum = 0;
    for_vectors<T, kPer16<T>>(e, r, [&](int64_t, int64_t, const T(&x)[kPer16<T>], int) {  // (what is past the end is 0)
#pragma unroll
        for (int v = 0; v < kPer16<T>; ++v) sum += (double)widen(x[v]) * widen(x[v]);
    });
    return sum;
}

__device__ __forceinline__ double block_sum(double x, double *lds, int waves) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0;
    for (int i = 0; i < waves; ++i) t += lds[i];
    return t;
}

__global__ __launch_bounds__(kThreads) void squares_kernel(table t, double *__restrict__ part) {
    __shared__ double lds[kThreads / kWave];
    double sum = 0;
    for (int64_t i = blockIdx.x; i < t.chunks; i += gridDim.x) {
        const table_entry &e = t.t[tensor_of(t, i)];
        const chunk_range r(e, i - e.first);
        if (e.type == kTypeF32) sum += squares<float>(e, r);
        else if (e.type == kTypeBF16) sum += squares<__bf16>(e, r);
        else sum += squares<_Float16>(e, r);
    }
    sum = block_sum(sum, lds, kThreads / kWave);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The factor of the gradients from the partial sums, by a whole workgroup (every thread has it); stats by one of them
__device__ __forceinline__ double factor_of(int n, const double *__restrict__ part, const clip_args &a, double *lds,
                                            bool store) {
    double sum = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) sum += part[i];
    sum = block_sum(sum, lds, kThreads / kWave);
    const double norm = sqrt(sum) * a.inv_scale;
    double f = a.inv_scale;
    if (a.clip) {
        const double x = a.max_norm / (norm + a.eps);
        if (!(x >= 1)) f *= x;  // a NaN stays one
        if (a.zero_nonfinite && !(norm < INFINITY)) f = 0;
    }
    if (store && threadIdx.x == 0) {
        a.stats[0] = (float)norm;
        a.stats[1] = (float)f;
    }
    return f;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(int n, const double *__restrict__ part, clip_args a) {
    __shared__ double lds[kThreads / kWave];
    factor_of(n, part, a, lds, true);
}

// one partial sum from many
__global__ __launch_bounds__(kThreads) void join_kernel(int n, const double *__restrict__ part, double *__restrict__ one) {
    __shared__ double lds[kThreads / kWave];
    double sum = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) sum += part[i];
    sum = block_sum(sum, lds, kThreads / kWave);
    if (threadIdx.x == 0) *one = sum;
}

template <typename T, typename TO>
__device__ __forceinline__ void scaled(const table_entry &e, const chunk_range &r, double f, bool zero) {
    constexpr int V = kPer16<TO>;  // whole lines are written
    for_vectors<T, V>(e, r, [&](int64_t row, int64_t col, const T(&x)[V], int n) {
        TO y[V];
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] = zero ? (TO)0.f : (TO)(float)(widen(x[v]) * f);
        TO *p = static_cast<TO *>(e.out) + row * e.ldo + col;
        if (n == V) {
            store_past<TO, V>(p, y);
        } else {
            store_some<TO, V>(p, n, y);
        }
    });
}

// From the last chunk to the first: what was read last by the norm is read first.
__global__ __launch_bounds__(kThreads) void scale_kernel(table t, int n, const double *__restrict__ part, clip_args a,
                                                         bool store) {
    __shared__ double lds[kThreads / kWave];
    const double f = factor_of(n, part, a, lds, store && blockIdx.x == 0);
    const bool zero = a.zero_nonfinite && f == 0;
    for (int64_t j = blockIdx.x; j < t.chunks; j += gridDim.x) {
        const int64_t i = t.chunks - 1 - j;
        const table_entry &e = t.t[tensor_of(t, i)];
        if (f == 1 && e.out == e.g) continue;
        const chunk_range r(e, i - e.first);
        const bool same = e.out_type == e.type;
        if (e.type == kTypeF32) scaled<float, float>(e, r, f, zero);
        else if (e.type == kTypeBF16) same ? scaled<__bf16, __bf16>(e, r, f, zero) : scaled<__bf16, float>(e, r, f, zero);
        else same ? scaled<_Float16, _Float16>(e, r, f, zero) : scaled<_Float16, float>(e, r, f, zero);
    }
}

// Entry of a tensor; its number of chunks
int64_t enter(const grad_tensor &g, int chunk_bytes, table_entry *e) {
    const bool whole = g.rows == 1 || (g.ld == g.cols && (g.out == nullptr || g.ldo == g.cols));
    const int64_t rows = whole ? 1 : g.rows, cols = whole ? g.rows * g.cols : g.cols;
    const int chunk = chunk_bytes / (g.dtype == kTypeF32 ? 4 : 2);
    *e = {g.g, g.out, cols, g.ld, g.ldo, 0, (int)rows, 0, chunk, g.dtype, g.out_dtype};
    if (rows == 0 || cols == 0) return 0;
    if (rows == 1 || cols > chunk / 2) return rows * ceil_div(cols, chunk);
    e->block = (int)(chunk / cols);
    return ceil_div(rows, e->block);
}

}  // namespace

// (the partial sums of a launch for every kTable tensors, and one that joins them)
size_t grad_norm_workspace_bytes(int n) {
    if (n < 0) return 0;
    return sizeof(double) * (1 + (size_t)kBlocks * std::max<int64_t>(1, ceil_div(n, kTable)));
}

hipError_t launch_clip_grad_norm(int n, const grad_tensor *g, const clip_args &a, void *ws, hipStream_t s) {
    double *one = static_cast<double *>(ws), *part = one + 1;
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) bytes += g[i].rows * g[i].cols * (g[i].dtype == kTypeF32 ? 4 : 2);
    const int chunk = bytes >= (int64_t)kBlocks << 15 ? 1 << 15 : 1 << 13;
    table t;
    auto fill = [&](int first) {
        t.n = 0;
        t.chunks = 0;
        for (int i = first; i < std::min(n, first + kTable); ++i) {
            const int64_t chunks = enter(g[i], chunk, &t.t[t.n]);
            if (chunks == 0) continue;
            t.t[t.n++].first = t.chunks;
            t.chunks += chunks;
        }
        return (int)std::min<int64_t>(t.chunks, kBlocks);
    };
    int parts = 0, filled = -1;
    for (int first = 0; first < n; first += kTable) {
        const int blocks = fill(filled = first);
        if (blocks > 0) squares_kernel<<<blocks, kThreads, 0, s>>>(t, part + parts);
        parts += blocks;
    }
    if (parts == 0 || !a.clip) {
        norm_kernel<<<1, kThreads, 0, s>>>(parts, part, a);
        return hipGetLastError();
    }
    if (n > kTable) {
        join_kernel<<<1, kThreads, 0, s>>>(parts, part, one);
        part = one;
        parts = 1;
    }
    bool store = true;
    for (int last = (n - 1) / kTable * kTable; last >= 0; last -= kTable) {
        const int blocks = last == filled ? (int)std::min<int64_t>(t.chunks, kBlocks) : fill(filled = last);
        if (blocks == 0) continue;
        scale_kernel<<<blocks, kThreads, 0, s>>>(t, parts, part, a, store);
        store = false;
    }
    return hipGetLastError();
}

}  // namespace l1csr
