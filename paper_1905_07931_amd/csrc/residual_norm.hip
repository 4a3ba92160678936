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
// Two ways, by whether a strip of columns stays on the chip:
// - strips: a workgroup of 1024 threads holds a few columns, all their rows, in registers; every mean is taken in its turn
//   and everything is read once (the backward gate twice).
// - two passes, for longer columns: both means of a call come from one pass over ranges of rows.  Forward: with
//   x = alpha a w_post y, r' = r + q x and sum r'^2 = sum r^2 + 2 q sum r x + q^2 sum x^2.  Backward:
//   sum k y t = sum k y dr' + s sum k y u - s^3 c sum k y r'.
// Sums over a column are in double (the forward expansion cancels where a block takes back what the residual holds; squares
// of bf16 values leave fp32), in a fixed order.  Sums over tokens are fp32 over the columns of a wave, 512 at most, and double over
// those.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"
#include "typed.hpp"

namespace l1csr {

namespace {

constexpr int kSums = 6;        // most sums of a column
constexpr int kFactors = 4;     // most factors of a column

// The logistic function and its complement.  For fp32 from exp(-|g|) (the rounding of the exponent's product put back) and
// a reciprocal refined once: each within about 4 steps of 2^-24.  For 16-bit gates as the instructions give it, within
// (6 + |g|) steps of 2^-24, a quarter of the instructions.
__device__ __forceinline__ void logistic(float g, float, float &a, float &b) {
    constexpr float log2e = 1.44269504088896340736f, log2e_rest = 1.92596299112661746887e-8f, ln2 = 0.69314718055994530942f;
    const float x = -fabsf(g), y = x * log2e;
    const float rest = fmaf(x, log2e_rest, fmaf(x, log2e, -y)) * ln2;
    float e = __builtin_amdgcn_exp2f(y);
    if (y > -INFINITY) e = fmaf(e, rest, e);  // (the product leaves fp32 ahead of g: its rest is infinite then)
    const float d = 1.f + e, r0 = __builtin_amdgcn_rcpf(d), r = fmaf(fmaf(-d, r0, 1.f), r0, r0), small = e * r;
    a = g >= 0.f ? r : small;  // (a NaN is in both)
    b = g >= 0.f ? small : r;
}
template <typename T>
__device__ __forceinline__ void logistic(float g, T, float &a, float &b) {
    const float y = g * 1.44269504088896340736f;
    a = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-y));
    b = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y));
}

// The gate of a row's columns from its values (a row of them, or one for all): a(g), and a'(g)
template <typename T, int V>
struct gate_values {
    float a[V], da[V];
    __device__ __forceinline__ gate_values(const norm_args &A, int k, const T (&raw)[V]) {
        if (A.gate_kind == kGateFull) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                a[v] = widen(raw[v]);
                da[v] = 1.f;
            }
            if (A.sigmoid) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float b;
                    logistic(a[v], T{}, a[v], b);
                    da[v] = a[v] * b;
                }
            }
        } else {
            float one = 1.f, d = 0.f;
            if (A.gate_kind == kGateRow) {
                one = static_cast<const float *>(A.gate)[k];
                d = 1.f;
                if (A.sigmoid) {
                    float b;
                    logistic(one, 0.f, one, b);
                    d = one * b;
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                a[v] = one;
                da[v] = d;
            }
        }
    }
};

// rounded to nearest even, two 16-bit values an instruction
template <typename T, int V>
__device__ __forceinline__ void narrow(const float (&x)[V], T (&t)[V]) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int v = 0; v < V; v += 2) {
            const t2 y = __builtin_convertvector((f2{x[v], x[v + 1]}), t2);
            __builtin_memcpy(&t[v], &y, 4);
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] = (T)x[v];
    }
}

// ---------------------------------------------------------------------------
// strips
// ---------------------------------------------------------------------------

constexpr int kStripThreads = 1024;
constexpr int kStripWaves = kStripThreads / kWave;
constexpr int kMaxStripColumns = 64;

// 2^tx_shift threads of V columns each side by side, the others over the rows: thread row ty has the rows ty, ty + TY, ...
// The strips of a cache line go to workgroups of one XCD that start together (32-byte pieces of rows: 4.4 to 6.0 TB/s so,
// 1.6 to 1.9 where neighbours lie on other XCDs).
struct strip_grid {
    int tx_shift, strips, line;  // line: strips of 128 bytes
    int blocks() const { return (int)(ceil_div(strips, 8 * line) * 8 * line); }
};

struct strip_place {
    int strip, tx, ty, TY;
    __device__ __forceinline__ explicit strip_place(const strip_grid &g) {
        const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
        strip = (j / g.line * 8 + x) * g.line + j % g.line;
        tx = threadIdx.x & ((1 << g.tx_shift) - 1);
        ty = threadIdx.x >> g.tx_shift;
        TY = kStripThreads >> g.tx_shift;
    }
};

struct strip_shared {
    double part[kStripWaves][kMaxStripColumns];
    float factor[2][kMaxStripColumns];
};

// Adds up a wave's values over its rows: while a lane holds several columns each step halves them (V = 8: 9 exchanges
// for 40); col: the column that is left.
template <int D, int HELD, int V>
__device__ __forceinline__ void fold(double (&x)[V], int lane, int TX, int &col) {
    if constexpr (HELD > 1) {
        constexpr int half = HELD / 2;
        const bool upper = (lane & D) != 0;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const double keep = upper ? x[i + half] : x[i], send = upper ? x[i] : x[i + half];
            x[i] = keep + __shfl_xor(send, D, kWave);
        }
        col += upper ? half : 0;
        fold<D / 2, half, V>(x, lane, TX, col);
    } else if constexpr (D >= 1) {
        if (D >= TX) x[0] += __shfl_xor(x[0], D, kWave);
        fold<D / 2, 1, V>(x, lane, TX, col);
    }
}

// Sums over the rows of NS values of each of a thread's V columns; f(column of the strip, its sums) in one thread a column.
template <int V, int NS, typename F>
__device__ __forceinline__ void strip_sums(double (&sum)[NS][V], int tx_shift, strip_shared (&sh)[NS], F f) {
    const int lane = lane_id(), wave = threadIdx.x >> 6, TX = 1 << tx_shift;
#pragma unroll
    for (int q = 0; q < NS; ++q) {
        int col = 0;
        fold<kWave / 2, V, V>(sum[q], lane, TX, col);
        // one lane of each column: those whose bits above tx that chose no column are 0
        constexpr int chosen = (kWave - 1) & ~(kWave / V - 1);
        if ((lane & ~chosen & ~(TX - 1)) == 0) sh[q].part[wave][(lane & (TX - 1)) * V + col] = sum[q][0];
    }
    __syncthreads();
    if ((int)threadIdx.x < TX * V) {
        double t[NS];
#pragma unroll
        for (int q = 0; q < NS; ++q) {
            t[q] = 0;
#pragma unroll
            for (int w = 0; w < kStripWaves; ++w) t[q] += sh[q].part[w][threadIdx.x];
        }
        f((int)threadIdx.x, t);
    }
    __syncthreads();
}

// A thread's columns of a matrix, row after row of its own: byte offsets of 32 bits, the last row again past the end.  Loads are
// whole vectors: where the columns end inside one it lies further back, over the neighbour's columns, whose values
// are not used.
template <typename T, int V>
struct strip_rows {
    unsigned first, step, last;
    __device__ __forceinline__ strip_rows(const norm_args &A, int64_t ld, int at_col, int ty, int TY)
        : first((unsigned)((ty * ld + at_col) * sizeof(T))), step((unsigned)(TY * ld * sizeof(T))),
          last((unsigned)(((A.K - 1) * ld + at_col) * sizeof(T))) {}
    __device__ __forceinline__ void load(const void *p, int j, T (&x)[V]) const {
        load_values<T, V>(reinterpret_cast<const T *>(static_cast<const char *>(p) + min(first + j * step, last)), x);
    }
    // own: the first of the values that is a column of this thread
    __device__ __forceinline__ void store(void *p, int j, const float (&x)[V], int own) const {
        T t[V];
        narrow<T, V>(x, t);
        T *q = reinterpret_cast<T *>(static_cast<char *>(p) + (first + j * step));
        if (own == 0) {
            store_values<T, V>(q, t);
        } else {
#pragma unroll
            for (int v = 1; v < V; ++v)
                if (v >= own) q[v] = t[v];
        }
    }
};

// a value of a vector over the rows, by an offset of 32 bits
__device__ __forceinline__ float row_value(const float *p, int k) {
    return *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p) + 4u * (unsigned)k);
}

// The same row of a thread, as the compiler cannot know: offsets of one phase are not kept for the next
__device__ __forceinline__ int anew(int ty) {
    asm volatile("" : "+v"(ty));
    return ty;
}

// Forward: y stays in registers and becomes r'.  J rows of V columns a thread (J <= 8); r and the gate
// come ahead, the first of them before the first mean is known.
template <typename T, int V, int J>
__global__ __launch_bounds__(kStripThreads) void forward_strip_kernel(norm_args A, strip_grid g) {
    __shared__ strip_shared sh[1];
    constexpr int P = J * V > 64 ? 1 : 2;  // rows of r and the gate that are under way
    const strip_place at(g);
    if (at.strip >= g.strips) return;
    const int64_t c = (((int64_t)at.strip << g.tx_shift) + at.tx) * V;
    const int col = (int)min(c, (int64_t)A.B - V), own = (int)min(c - col, (int64_t)V);
    const bool has_y = A.y != nullptr, post = A.post_gain != nullptr, pre = A.pre_gain != nullptr, full = A.gate_kind == kGateFull;
    const int rows = at.ty < A.K ? (A.K - 1 - at.ty) / at.TY + 1 : 0;  // of this thread
    T raw[J][V];  // y, or r without it
    {
        const strip_rows<T, V> m(A, has_y ? A.ldy : A.ldr, col, at.ty, at.TY);
#pragma unroll
        for (int j = 0; j < J; ++j) m.load(has_y ? A.y : A.r, j, raw[j]);
    }
    const int ty2 = anew(at.ty);
    const strip_rows<T, V> mr(A, A.ldr, col, ty2, at.TY), mg(A, full ? A.ldg : 0, full ? col : 0, ty2, at.TY),
        mo(A, A.ldro, col, ty2, at.TY);
    T r[P][V], gate[P][V];
    auto ahead = [&](int j) {
        if (j >= J) return;
        mr.load(A.r, j, r[j % P]);
        if (full) mg.load(A.gate, j, gate[j % P]);
    };
    float x[J][V], q[V];
    const float *factor = sh[0].factor[0] + at.tx * V;
    auto mean_square = [&](auto value) {
        double sum[1][V] = {};  // (squares of bf16 values and of r' leave fp32)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j >= rows) continue;
#pragma unroll
            for (int v = 0; v < V; ++v) sum[0][v] += (double)value(j, v) * value(j, v);
        }
        strip_sums<V, 1>(sum, g.tx_shift, sh, [&](int i, const double(&t)[1]) {
            sh[0].factor[0][i] = (float)(1 / sqrt(t[0] / A.K + A.eps));
        });
    };
    if (has_y) {
#pragma unroll
        for (int j = 0; j < P; ++j) ahead(j);
        if (post) mean_square([&](int j, int v) { return widen(raw[j][v]); });
#pragma unroll
        for (int v = 0; v < V; ++v) q[v] = post ? factor[v] : 1.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = min(ty2 + j * at.TY, A.K - 1);
            const gate_values<T, V> a(A, k, gate[j % P]);
            const float w = A.alpha * (post ? row_value(A.post_gain, k) : 1.f);
#pragma unroll
            for (int v = 0; v < V; ++v) x[j][v] = widen(r[j % P][v]) + a.a[v] * w * (widen(raw[j][v]) * q[v]);
            ahead(j + P);
            if (j < rows) mo.store(A.r_out, j, x[j], own);
        }
    } else {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) x[j][v] = widen(raw[j][v]);
    }
    if (!pre) return;
    mean_square([&](int j, int v) { return x[j][v]; });
    float s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = factor[v];
    const int ty3 = anew(at.ty);
    const strip_rows<T, V> mh(A, A.ldh, col, ty3, at.TY);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (j >= rows) continue;
        const float w = row_value(A.pre_gain, ty3 + j * at.TY);
#pragma unroll
        for (int v = 0; v < V; ++v) x[j][v] = x[j][v] * s[v] * w;
        mh.store(A.h, j, x[j], own);
    }
}

// A row's sum over the threads side by side, stored by the first: rows[i][block][K]
__device__ __forceinline__ void store_row_sum(const norm_args &A, float *rows, int i, int blocks, int block, int k, int tx,
                                              int TX, float x) {
    for (int d = TX / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d, kWave);
    if (tx == 0 && k < A.K) rows[((int64_t)i * blocks + block) * A.K + k] = x;
}

// Backward: r' and dh stay in registers and become t and y (J <= 4, or 8 of one column)
template <typename T, int V, int J>
__global__ __launch_bounds__(kStripThreads) void backward_strip_kernel(norm_args A, strip_grid g, float *__restrict__ rows) {
    __shared__ strip_shared sh[2];
    const strip_place at(g);
    if (at.strip >= g.strips) return;
    const int TX = 1 << g.tx_shift;
    const int64_t c = (((int64_t)at.strip << g.tx_shift) + at.tx) * V;
    const int col = (int)min(c, (int64_t)A.B - V), own = (int)min(c - col, (int64_t)V);
    const bool has_y = A.y != nullptr, post = A.post_gain != nullptr, pre = A.pre_gain != nullptr;
    const bool full = A.gate_kind == kGateFull, row = A.gate_kind == kGateRow;
    const int held = at.ty < A.K ? (A.K - 1 - at.ty) / at.TY + 1 : 0;  // rows of this thread
    float t[J][V], y[J][V];
    float s[V] = {}, f[V] = {};
    double sum[2][V] = {};
    if (pre) {
        const strip_rows<T, V> mr(A, A.ldro, col, at.ty, at.TY), mh(A, A.lddh, col, at.ty, at.TY);
        T raw[J][V], raw2[J][V];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            mr.load(A.r_out, j, raw[j]);
            mh.load(A.dh, j, raw2[j]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const float w = row_value(A.pre_gain, min(at.ty + j * at.TY, A.K - 1));
#pragma unroll
            for (int v = 0; v < V; ++v) {
                t[j][v] = j < held ? widen(raw[j][v]) : 0.f;
                y[j][v] = j < held ? widen(raw2[j][v]) : 0.f;
                sum[0][v] += (double)t[j][v] * t[j][v];
                sum[1][v] += (double)(y[j][v] * w) * t[j][v];
            }
        }
        strip_sums<V, 2>(sum, g.tx_shift, sh, [&](int i, const double(&x)[2]) {
            const double s2 = 1 / (x[0] / A.K + A.eps);
            sh[0].factor[0][i] = (float)sqrt(s2);
            sh[0].factor[1][i] = (float)(s2 * x[1] / A.K);
        });
#pragma unroll
        for (int v = 0; v < V; ++v) {
            s[v] = sh[0].factor[0][at.tx * V + v];
            f[v] = sh[0].factor[1][at.tx * V + v];
            sum[0][v] = sum[1][v] = 0;
        }
    }
    // t; y is read behind it
    const void *dr_out = A.dr_out ? A.dr_out : A.r_out, *yp = has_y ? A.y : dr_out;
    const int ty2 = anew(at.ty);
    const strip_rows<T, V> md(A, A.dr_out ? A.lddro : A.ldro, col, ty2, at.TY),
        my(A, has_y ? A.ldy : A.dr_out ? A.lddro : A.ldro, col, ty2, at.TY),
        mg(A, full ? A.ldg : 0, full ? col : 0, ty2, at.TY), mo(A, A.lddr, col, ty2, at.TY);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        T dr[V], yr[V], gate[V];
        md.load(dr_out, j, dr);
        if (has_y) my.load(yp, j, yr);
        if (full && post) mg.load(A.gate, j, gate);
        const int k = min(ty2 + j * at.TY, A.K - 1);
        float z[V];
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = A.dr_out && j < held ? widen(dr[v]) : 0.f;
        if (pre) {
            const float w = row_value(A.pre_gain, k);
            float sums = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float rs = t[j][v] * s[v], dh = y[j][v];
                sums += v >= own ? dh * rs : 0.f;
                z[v] += s[v] * (dh * w) - f[v] * rs;
            }
            store_row_sum(A, rows, 0, g.strips, at.strip, ty2 + j * at.TY, at.tx, TX, sums);
            if (j < held) mo.store(A.dr, j, z, own);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) t[j][v] = z[v];
        if (!has_y) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) y[j][v] = j < held ? widen(yr[v]) : 0.f;
        if (!post) continue;
        const gate_values<T, V> a(A, k, gate);
        const float w = A.alpha * row_value(A.post_gain, k);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            sum[0][v] += (double)y[j][v] * y[j][v];
            sum[1][v] += j < held ? (double)(a.a[v] * w * t[j][v]) * y[j][v] : 0;
        }
    }
    if (!has_y) return;
    float q[V], e[V];
    if (post)
        strip_sums<V, 2>(sum, g.tx_shift, sh, [&](int i, const double(&x)[2]) {
            const double q2 = 1 / (x[0] / A.K + A.eps);
            sh[0].factor[0][i] = (float)sqrt(q2);
            sh[0].factor[1][i] = (float)(q2 * x[1] / A.K);
        });
#pragma unroll
    for (int v = 0; v < V; ++v) {
        q[v] = post ? sh[0].factor[0][at.tx * V + v] : 1.f;
        e[v] = post ? sh[0].factor[1][at.tx * V + v] : 0.f;
    }
    const int ty3 = anew(at.ty);
    const strip_rows<T, V> mdy(A, A.lddy, col, ty3, at.TY), mdg(A, A.lddg, col, ty3, at.TY),
        mg3(A, full ? A.ldg : 0, full ? col : 0, ty3, at.TY);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        T gate[V];
        if (full) mg3.load(A.gate, j, gate);
        const int k = min(ty3 + j * at.TY, A.K - 1);
        const gate_values<T, V> a(A, k, gate);
        const float w = post ? row_value(A.post_gain, k) : 1.f;
        float dy[V], dg[V], sums[2] = {};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float at_ = A.alpha * t[j][v], yq = y[j][v] * q[v];
            dy[v] = a.a[v] * at_ * w * q[v] - (post ? e[v] * yq : 0.f);  // (y may be infinite where it has no norm)
            dg[v] = at_ * yq * w * a.da[v];
            sums[0] += v >= own ? a.a[v] * at_ * yq : 0.f;
            sums[1] += v >= own ? dg[v] : 0.f;
        }
        if (post) store_row_sum(A, rows, 1, g.strips, at.strip, ty3 + j * at.TY, at.tx, TX, sums[0]);
        if (row) store_row_sum(A, rows, 2, g.strips, at.strip, ty3 + j * at.TY, at.tx, TX, sums[1]);
        if (j >= held) continue;
        mdy.store(A.dy, j, dy, own);
        if (full) mdg.store(A.dgate, j, dg, own);
    }
}

// ---------------------------------------------------------------------------
// two passes
// ---------------------------------------------------------------------------

constexpr int kPassThreads = 512;
constexpr int kPassVector = 4;  // columns of a thread of the sums (those of 8 take 96 registers); of the results: 16 bytes

// How a workgroup lies over [K][B]: 2^tx_shift threads of V columns each side by side, the others over the rows;
// blockIdx.y a range of rows.
struct norm_grid {
    int tx_shift, col_blocks, splits, rows;
};

// A thread's columns.  Loads are whole vectors as in the strips: own is the first of the values that is a column of
// this thread.  They go past the caches, which hold nothing that is read again: the backward sums of 9216 x 2048 fp32 (378
// MB) take 67 us so and 96 through them.
template <typename T, int V>
struct columns {
    int col, own;
    __device__ columns(int tx, int tx_shift, int B) {
        const int64_t c = (((int64_t)blockIdx.x << tx_shift) + tx) * V;
        col = (int)min(c, (int64_t)B - V);
        own = (int)min(c - col, (int64_t)V);
    }
    __device__ __forceinline__ void load(const void *p, int64_t ld, int k, T (&x)[V]) const {
        const T *q = static_cast<const T *>(p) + (int64_t)k * ld + col;
        if constexpr (V > 1) load_past<T, V>(q, x);
        else load_values<T, V>(q, x);
    }
    __device__ __forceinline__ void store(void *p, int64_t ld, int k, const float (&x)[V]) const {
        T t[V];
        narrow<T, V>(x, t);
        T *q = static_cast<T *>(p) + (int64_t)k * ld + col;
        if (own == 0) {
            store_values<T, V>(q, t);
        } else {
#pragma unroll
            for (int v = 1; v < V; ++v)
                if (v >= own) q[v] = t[v];
        }
    }
};

// Rows of every matrix that a thread has under way.  Forward, 4096 x 8192 bf16: two everywhere 117 us, four in the
// sums 112, in the 16-bit results too 109, six 120, eight 115; fp32 220, 217 and 226.  Backward, 9216 x 2048: two everywhere
// 179 (fp32) and 115 (bf16), one in the sums 177 and 112, in the 16-bit results too 109, in the fp32 ones 183; four 178 and 127.
constexpr int kSumRows = 4;
template <typename T>
constexpr int kResultRows = sizeof(T) == 2 ? 4 : 2;
template <typename T>
constexpr int kBackwardResultRows = sizeof(T) == 2 ? 1 : 2;

// f(rows, k): the rows k, k + TY, ... of a range, U of them at a time while there are as many
template <int U, typename F>
__device__ __forceinline__ void for_rows(int k, int k1, int TY, F f) {
    for (; k + (U - 1) * TY < k1; k += U * TY) f(std::integral_constant<int, U>{}, k);
    for (; k < k1; k += TY) f(std::integral_constant<int, 1>{}, k);
}

// Joins the sums of a workgroup's threads over the rows and stores them: part[q][split][B].  Two sums at a time lie in LDS,
// and the threads share the columns of them.
template <int V>
constexpr int kSumsValues = 2 * V * kPassThreads;
template <typename T, int V, int NS>
__device__ __forceinline__ void store_sums(const double (&sum)[NS][V], const norm_grid &g, const columns<T, V> &c, int B,
                                           double *lds, double *part) {
    static_assert(NS % 2 == 0, "two sums at a time");
    const int TX = 1 << g.tx_shift, TY = kPassThreads >> g.tx_shift, width = TX * V;
    const int ty = threadIdx.x >> g.tx_shift;
    const int64_t first = ((int64_t)blockIdx.x << g.tx_shift) * V;
    // (the place of a column: its thread's within those of the same v)
    auto place = [&](int column) { return column % V * TX + column / V; };
#pragma unroll
    for (int q = 0; q < NS; q += 2) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v >= c.own) {
                const int at = place((int)(c.col + v - first));
                lds[ty * width + at] = sum[q][v];
                lds[(TY + ty) * width + at] = sum[q + 1][v];
            }
        __syncthreads();
        // 2 * width sums of TY values, each by `ways` threads (9216 x 1 fp32: 6.8 us, by one thread each 17.2)
        const int sums = 2 * width, ways = min(16, kPassThreads / sums), i = (threadIdx.x & (sums - 1)) / width;
        const int at = threadIdx.x & (width - 1);
        double t = 0;
        if ((int)threadIdx.x < sums * ways)
            for (int y = threadIdx.x / sums; y < TY; y += ways) t += lds[(i * TY + y) * width + at];
        if (ways > 1) {
            __syncthreads();
            lds[threadIdx.x] = t;
            __syncthreads();
            if ((int)threadIdx.x < sums)
                for (int w = 1; w < ways; ++w) t += lds[w * sums + threadIdx.x];
        }
        const int64_t col = first + (at & (TX - 1)) * V + (at >> g.tx_shift);
        if ((int)threadIdx.x < sums && col < B) part[((int64_t)(q + i) * g.splits + blockIdx.y) * B + col] = t;
    }
}

// 256 columns in 288 ranges: 5.6 us (four sums) and 7.7 (six); 14.4 and 20.7 with 256 threads on 32 columns
constexpr int kJoinThreads = 1024;
constexpr int kJoinColumns = 16;  // of a workgroup of the join; the other threads share the ranges of rows

// Joins the sums over the ranges of rows; true in the threads that hold a column's
template <int NS>
__device__ __forceinline__ bool join_sums(const double *__restrict__ part, int splits, int B, int col, double *lds,
                                          double (&sum)[NS]) {
    constexpr int ways = kJoinThreads / kJoinColumns;
    static_assert(NS <= ways, "a thread's share of the second step is one sum");
    const int way = threadIdx.x / kJoinColumns, column = threadIdx.x % kJoinColumns;
#pragma unroll
    for (int q = 0; q < NS; ++q) {
        double t = 0;
        if (col < B)
#pragma unroll 4
            for (int i = way; i < splits; i += ways) t += part[((int64_t)q * splits + i) * B + col];
        lds[q * kJoinThreads + threadIdx.x] = t;
    }
    __syncthreads();
    if (way < NS) {  // a sum each
        double t = 0, *p = lds + way * kJoinThreads + column;
#pragma unroll 8
        for (int i = 0; i < ways; ++i) t += p[i * kJoinColumns];
        p[0] = t;
    }
    __syncthreads();
    if (way != 0 || col >= B) return false;
#pragma unroll
    for (int q = 0; q < NS; ++q) sum[q] = lds[q * kJoinThreads + column];
    return true;
}

// What a call has: y, a norm of y, a norm of r'
enum { kHasY = 1, kHasPost = 2, kHasPre = 4 };

template <typename T, int V, int HAS>
__global__ __launch_bounds__(kPassThreads) void forward_sums_kernel(norm_args A, norm_grid g, double *__restrict__ part) {
    constexpr int NS = 4;  // y^2; r^2, r x, x^2 (without post: r'^2 alone)
    constexpr bool has_y = (HAS & kHasY) != 0, post = (HAS & kHasPost) != 0, pre = (HAS & kHasPre) != 0;
    __shared__ double lds[kSumsValues<V>];
    const int TX = 1 << g.tx_shift, TY = kPassThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<T, V> c(tx, g.tx_shift, A.B);
    const int k0 = blockIdx.y * g.rows + ty, k1 = (int)min((int64_t)A.K, (int64_t)(blockIdx.y + 1) * g.rows);
    const bool full = A.gate_kind == kGateFull;
    double sum[NS][V] = {};
    for_rows<kSumRows>(k0, k1, TY, [&](auto rows, int k) {
        constexpr int U = decltype(rows)::value;
        T r[U][V], y[U][V], gate[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (pre) c.load(A.r, A.ldr, k + u * TY, r[u]);
            if (has_y) c.load(A.y, A.ldy, k + u * TY, y[u]);
        }
        if (full && pre) {
#pragma unroll
            for (int u = 0; u < U; ++u) c.load(A.gate, A.ldg, k + u * TY, gate[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (post) {
#pragma unroll
                for (int v = 0; v < V; ++v) sum[0][v] += (double)widen(y[u][v]) * widen(y[u][v]);
            }
            if constexpr (pre && !has_y) {
#pragma unroll
                for (int v = 0; v < V; ++v) sum[1][v] += (double)widen(r[u][v]) * widen(r[u][v]);
            }
            if constexpr (pre && has_y) {
                const gate_values<T, V> a(A, k + u * TY, gate[u]);
                const float w = A.alpha * (post ? A.post_gain[k + u * TY] : 1.f);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const double x = (double)(a.a[v] * w) * widen(y[u][v]), rr = widen(r[u][v]);
                    if constexpr (post) {
                        sum[1][v] += rr * rr;
                        sum[2][v] += rr * x;
                        sum[3][v] += x * x;
                    } else {
                        sum[1][v] += (rr + x) * (rr + x);
                    }
                }
            }
        }
    });
    if constexpr (post && pre) {
        // Squares of finite values are finite: a column with an infinite r or x comes here.  r' is infinite there, or NaN, and so
        // is its square, whatever r x gave (0 times infinity, or one infinity less another).  Looked at once behind the sums: in
        // the loop it takes 12 to 15 % of the call in 16 bits (4096 x 8192 104 -> 119 us).
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (sum[1][v] + sum[3][v] < INFINITY) continue;
            bool nan = false;
            for (int k = k0; k < k1; k += TY) {
                T r[V], y[V], gate[V];
                c.load(A.r, A.ldr, k, r);
                c.load(A.y, A.ldy, k, y);
                if (full) c.load(A.gate, A.ldg, k, gate);
                const gate_values<T, V> a(A, k, gate);
                const float w = A.alpha * A.post_gain[k];
                const double z = widen(r[v]) + (double)(a.a[v] * w) * widen(y[v]);
                nan = nan || z != z;
            }
            sum[2][v] = nan ? NAN : INFINITY;
        }
    }
    store_sums<T, V, NS>(sum, g, c, A.B, lds, part);
}

// a column's factors: q, s
__global__ __launch_bounds__(kJoinThreads) void forward_join_kernel(int K, int B, float eps, int splits, bool post, bool pre,
                                                                const double *__restrict__ part, float *__restrict__ fac) {
    __shared__ double lds[4 * kJoinThreads];
    const int col = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    double sum[4];
    if (!join_sums<4>(part, splits, B, col, lds, sum)) return;
    const double q = post ? 1 / sqrt(sum[0] / K + eps) : 1.0;
    fac[col] = (float)q;
    if (!pre) return;
    const double square = sum[1] + q * (2 * sum[2] + q * sum[3]);
    fac[B + col] = (float)(1 / sqrt((square < 0 ? 0 : square) / K + eps));  // (a NaN stays one)
}

template <typename T, int V>
__global__ __launch_bounds__(kPassThreads) void forward_kernel(norm_args A, norm_grid g, const float *__restrict__ fac) {
    const int TX = 1 << g.tx_shift, TY = kPassThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<T, V> c(tx, g.tx_shift, A.B);
    const int k0 = blockIdx.y * g.rows + ty, k1 = (int)min((int64_t)A.K, (int64_t)(blockIdx.y + 1) * g.rows);
    if (c.own >= V) return;
    const bool has_y = A.y != nullptr, post = A.post_gain != nullptr, pre = A.pre_gain != nullptr, full = A.gate_kind == kGateFull;
    float q[V], s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        q[v] = post ? fac[c.col + v] : 1.f;
        s[v] = pre ? fac[A.B + c.col + v] : 0.f;
    }
    for_rows<kResultRows<T>>(k0, k1, TY, [&](auto rows, int k) {
        constexpr int U = decltype(rows)::value;
        T r[U][V], y[U][V], gate[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            c.load(A.r, A.ldr, k + u * TY, r[u]);
            if (has_y) c.load(A.y, A.ldy, k + u * TY, y[u]);
        }
        if (full) {
#pragma unroll
            for (int u = 0; u < U; ++u) c.load(A.gate, A.ldg, k + u * TY, gate[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[V];
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = widen(r[u][v]);
            if (has_y) {
                const gate_values<T, V> a(A, k + u * TY, gate[u]);
                const float w = A.alpha * (post ? A.post_gain[k + u * TY] : 1.f);
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] += a.a[v] * w * (widen(y[u][v]) * q[v]);
                c.store(A.r_out, A.ldro, k + u * TY, x);
            }
            if (pre) {
                const float w = A.pre_gain[k + u * TY];
#pragma unroll
                for (int v = 0; v < V; ++v) x[v] = x[v] * s[v] * w;
                c.store(A.h, A.ldh, k + u * TY, x);
            }
        }
    });
}

template <typename T, int V, int HAS>
__global__ __launch_bounds__(kPassThreads) void backward_sums_kernel(norm_args A, norm_grid g, double *__restrict__ part) {
    constexpr int NS = kSums;  // r'^2, u r'; y^2, k y dr', k y u, k y r'
    constexpr bool post = (HAS & kHasPost) != 0, pre = (HAS & kHasPre) != 0;
    __shared__ double lds[kSumsValues<V>];
    const int TX = 1 << g.tx_shift, TY = kPassThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<T, V> c(tx, g.tx_shift, A.B);
    const int k0 = blockIdx.y * g.rows + ty, k1 = (int)min((int64_t)A.K, (int64_t)(blockIdx.y + 1) * g.rows);
    const bool full = A.gate_kind == kGateFull, more = A.dr_out != nullptr;
    // (without dr_out r' is read in its place and not used: zeros put there instead would wait for every load ahead)
    const void *dr_out = more ? A.dr_out : A.r_out;
    const int64_t lddro = more ? A.lddro : A.ldro;
    double sum[NS][V] = {};
    for_rows<1>(k0, k1, TY, [&](auto rows, int k) {
        constexpr int U = decltype(rows)::value;
        T r[U][V], dh[U][V], y[U][V], dr[U][V], gate[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (pre) c.load(A.r_out, A.ldro, k + u * TY, r[u]);
            if (pre) c.load(A.dh, A.lddh, k + u * TY, dh[u]);
            if (post) c.load(A.y, A.ldy, k + u * TY, y[u]);
            if (post) c.load(dr_out, lddro, k + u * TY, dr[u]);
        }
        if (post && full) {
#pragma unroll
            for (int u = 0; u < U; ++u) c.load(A.gate, A.ldg, k + u * TY, gate[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float d[V];
            if constexpr (pre) {
                const float w = A.pre_gain[k + u * TY];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    d[v] = widen(dh[u][v]) * w;
                    sum[0][v] += (double)widen(r[u][v]) * widen(r[u][v]);
                    sum[1][v] += (double)d[v] * widen(r[u][v]);
                }
            }
            if constexpr (post) {
                const gate_values<T, V> a(A, k + u * TY, gate[u]);
                const float w = A.alpha * A.post_gain[k + u * TY];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const double yy = widen(y[u][v]), ky = (double)(a.a[v] * w) * yy;
                    sum[2][v] += yy * yy;
                    sum[3][v] += more ? ky * widen(dr[u][v]) : 0;
                    if constexpr (pre) {
                        sum[4][v] += ky * d[v];
                        sum[5][v] += ky * widen(r[u][v]);
                    }
                }
            }
        }
    });
    store_sums<T, V, NS>(sum, g, c, A.B, lds, part);
}

// a column's factors: s, f = s^2 c, q, g = q^2 e
__global__ __launch_bounds__(kJoinThreads) void backward_join_kernel(int K, int B, float eps, int splits, bool post, bool pre,
                                                                 const double *__restrict__ part, float *__restrict__ fac) {
    __shared__ double lds[kSums * kJoinThreads];
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
template <typename T, int V>
__global__ __launch_bounds__(kPassThreads) void backward_kernel(norm_args A, norm_grid g, const float *__restrict__ fac,
                                                                float *__restrict__ rows_out) {
    const int TX = 1 << g.tx_shift, TY = kPassThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<T, V> c(tx, g.tx_shift, A.B);
    const int k0 = blockIdx.y * g.rows + ty, k1 = (int)min((int64_t)A.K, (int64_t)(blockIdx.y + 1) * g.rows);
    const bool has_y = A.y != nullptr, post = A.post_gain != nullptr, pre = A.pre_gain != nullptr, more = A.dr_out != nullptr;
    const bool full = A.gate_kind == kGateFull, row = A.gate_kind == kGateRow;
    const void *dr_out = more ? A.dr_out : A.r_out;  // (as in the sums)
    const int64_t lddro = more ? A.lddro : A.ldro;
    float s[V], f[V], q[V], e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = c.col + v;
        s[v] = pre ? fac[col] : 0.f;
        f[v] = pre ? fac[A.B + col] : 0.f;
        q[v] = post ? fac[2 * (int64_t)A.B + col] : 1.f;
        e[v] = post ? fac[3 * (int64_t)A.B + col] : 0.f;
    }
    for_rows<kBackwardResultRows<T>>(k0, k1, TY, [&](auto rows, int k2) {
        constexpr int U = decltype(rows)::value;
        T r[U][V], dh[U][V], y[U][V], dr[U][V], gate[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) c.load(dr_out, lddro, k2 + u * TY, dr[u]);
        if (pre) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                c.load(A.r_out, A.ldro, k2 + u * TY, r[u]);
                c.load(A.dh, A.lddh, k2 + u * TY, dh[u]);
            }
        }
        if (has_y) {
#pragma unroll
            for (int u = 0; u < U; ++u) c.load(A.y, A.ldy, k2 + u * TY, y[u]);
        }
        if (full) {
#pragma unroll
            for (int u = 0; u < U; ++u) c.load(A.gate, A.ldg, k2 + u * TY, gate[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k2 + u * TY;
            float t[V];
#pragma unroll
            for (int v = 0; v < V; ++v) t[v] = more ? widen(dr[u][v]) : 0.f;
            if (pre) {
                const float w = A.pre_gain[k];
                float sums = 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float rs = widen(r[u][v]) * s[v], d = widen(dh[u][v]);
                    sums += v >= c.own ? d * rs : 0.f;
                    t[v] += s[v] * (d * w) - f[v] * rs;
                }
                c.store(A.dr, A.lddr, k, t);
                store_row_sum(A, rows_out, 0, g.col_blocks, blockIdx.x, k, tx, TX, sums);
            }
            if (!has_y) continue;
            const gate_values<T, V> a(A, k, gate[u]);
            const float w = post ? A.post_gain[k] : 1.f;
            float dy[V], dg[V], sums[2] = {};
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float at = A.alpha * t[v], yq = widen(y[u][v]) * q[v];
                dy[v] = a.a[v] * at * w * q[v] - (post ? e[v] * yq : 0.f);  // (y may be infinite where it has no norm)
                dg[v] = at * yq * w * a.da[v];
                sums[0] += v >= c.own ? a.a[v] * at * yq : 0.f;
                sums[1] += v >= c.own ? dg[v] : 0.f;
            }
            c.store(A.dy, A.lddy, k, dy);
            if (full) c.store(A.dgate, A.lddg, k, dg);
            if (post) store_row_sum(A, rows_out, 1, g.col_blocks, blockIdx.x, k, tx, TX, sums[0]);
            if (row) store_row_sum(A, rows_out, 2, g.col_blocks, blockIdx.x, k, tx, TX, sums[1]);
        }
    });
}

// a row's sum over the blocks of columns: 32 rows and 32 threads to each of a workgroup, blockIdx.y one of the three sums
constexpr int kRowSumThreads = 1024;
__global__ __launch_bounds__(kRowSumThreads) void row_sums_kernel(int K, int blocks, const float *__restrict__ rows,
                                                                  float *pre, float *post, float *gate) {
    constexpr int width = 32, ways = kRowSumThreads / width;
    __shared__ double lds[kRowSumThreads];
    float *out = blockIdx.y == 0 ? pre : blockIdx.y == 1 ? post : gate;
    if (out == nullptr) return;
    const int64_t k = (int64_t)blockIdx.x * width + threadIdx.x % width;
    const int way = threadIdx.x / width;
    double t = 0;
    if (k < K) {
        const float *p = rows + (int64_t)blockIdx.y * blocks * K + k;
#pragma unroll 8
        for (int b = way; b < blocks; b += ways) t += p[(int64_t)b * K];
    }
    lds[threadIdx.x] = t;
    __syncthreads();
    if (way != 0 || k >= K) return;
    t = 0;
    for (int i = 0; i < ways; ++i) t += lds[i * width + threadIdx.x];
    out[k] = (float)t;
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

int pass_vector(int B) { return B < kPassVector ? 1 : kPassVector; }

int vector_of(int B, int dtype) {
    const int v = dtype == kTypeF32 ? 4 : 8;
    return B >= v ? v : 1;
}

// (the forward results take twice the workgroups: 4096 x 8192 bf16, two rows under way, 78 -> 68 us; the backward ones 108 -> 113)
norm_grid grid_for(int K, int B, int V, int workgroups = 512) {
    norm_grid g;
    const int64_t lanes = ceil_div(B, V);
    g.tx_shift = 0;
    while (g.tx_shift < 6 && (1 << g.tx_shift) < lanes) ++g.tx_shift;
    g.col_blocks = (int)ceil_div(lanes, 1 << g.tx_shift);
    const int TY = kPassThreads >> g.tx_shift;
    // two workgroups a CU (twice as many leave the join twice the sums and gain nothing), of 4 rows a thread at least
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(ceil_div(K, 4 * TY), workgroups / g.col_blocks));
    g.rows = (int)(ceil_div(ceil_div(K, splits), TY) * TY);
    g.splits = (int)ceil_div(K, g.rows);
    return g;
}

constexpr int kStripFill = 256;      // strips that fill the card

// The widest strips that leave kStripFill of them (a thread's V columns at least) and whose rows are `held` values of a
// thread at most; returns its rows, 0: there are none
int rows_held(int K, int B, int V, int dtype, int held, strip_grid *g) {
    const int64_t lanes = ceil_div(B, V);
    int shift = 3;
    auto rows = [&] { return ceil_div(K, kStripThreads >> shift); };
    if (V == 1) {
        shift = 0;
        while ((1 << shift) < lanes) ++shift;  // (fewer than 8 columns)
    } else {
        while (shift > 0 && (ceil_div(lanes, 1 << shift) < kStripFill || rows() * V > held)) --shift;
    }
    if (rows() * V > held) return 0;
    *g = {shift, (int)ceil_div(lanes, 1 << shift), std::max(1, 128 / (V * (dtype == kTypeF32 ? 4 : 2) << shift))};
    return (int)rows();
}

// f(T, V, J) as compile-time values, J at least the rows (MOST of them, of a vector's kernels); V is 1 or WIDE (0: 16 bytes)
template <int MOST, int WIDE, typename F>
hipError_t with_rows(int V, int dtype, int rows, F f) {
    using std::integral_constant;
    auto by_rows = [&](auto t, auto v) {
        if (rows <= 2) return f(t, v, integral_constant<int, 2>{});
        if (rows <= 4) return f(t, v, integral_constant<int, 4>{});
        if constexpr (MOST >= 8 || decltype(v)::value == 1) {
            if (rows <= 8) return f(t, v, integral_constant<int, 8>{});
        }
        return hipErrorInvalidValue;
    };
    auto by_type = [&](auto t) {
        constexpr int wide = WIDE > 0 ? WIDE : kPer16<decltype(t)>;
        return V == 1 ? by_rows(t, integral_constant<int, 1>{}) : by_rows(t, integral_constant<int, wide>{});
    };
    if (dtype == kTypeF32) return by_type(float{});
    if (dtype == kTypeBF16) return by_type(__bf16{});
    return by_type(_Float16{});
}

// f(T, V): V is 1, or WIDE (0: 16 bytes)
template <int WIDE, typename F>
hipError_t with_vectors(int V, int dtype, F f) {
    using std::integral_constant;
    auto by_type = [&](auto t) {
        constexpr int wide = WIDE > 0 ? WIDE : kPer16<decltype(t)>;
        return V == 1 ? f(t, integral_constant<int, 1>{}) : f(t, integral_constant<int, wide>{});
    };
    if (dtype == kTypeF32) return by_type(float{});
    if (dtype == kTypeBF16) return by_type(__bf16{});
    return by_type(_Float16{});
}

// (offsets within a matrix are 32 bits)
bool short_enough(const norm_args &a) {
    const int64_t ld = std::max({a.ldr, a.ldy, a.ldg, a.ldro, a.ldh, a.lddro, a.lddh, a.lddr, a.lddy, a.lddg, (int64_t)a.B});
    return a.K * ld < (int64_t)1 << 30;
}

// Strips of up to 2048 rows leave room for several workgroups a CU (us, strips and two passes, gate and both norms:
// fp32 1024 x 8192 45 and 64, 2048 x 8192 105 and 112, 2000 x 64 13 and 17, bf16 2048 x 8192 50 and 66).  Up to 4096 rows one
// workgroup fills a CU and nothing hides its reductions: that still pays where the launches and the join are most of the
// time (fp32 2800 x 64 17 and 17, 2800 x 1024 31 and 35; bf16, inputs in the caches, 4000 x 256 18.7 and 20.5, 4000 x 1024 24
// and 28, but 24.5 and 22, 41 and 29 from cold memory), but not for large matrices (fp32 4096 x 8192 259 and 217, bf16 124 and
// 113), nor for the longest fp32 columns, which are held four a thread at least (4000 x 64 23.6 and 17.4, 4000 x 512 33 and 27;
// rows of under 64 bytes are soon read: 4000 x 8 11 and 17).  Longer columns would spill.  Everything is read once and
// still takes 1.4 to 1.9 times its bytes (5.1 TB/s, cold): a workgroup's loads wait while it takes its means.
constexpr int kStripRows = 2048, kMostStripRows = 4096, kMostFp32Rows = 2816;
constexpr int64_t kStripBytes = 32 << 20;  // of a matrix of more than kStripRows rows
constexpr int kShortRow = 64;              // bytes
int forward_rows(int K, int B, int dtype, strip_grid *g) {
    const int V = vector_of(B, dtype), size = dtype == kTypeF32 ? 4 : 2;
    if (V > 1 && (K > kMostStripRows || (K > kStripRows && (int64_t)K * B * size > kStripBytes))) return 0;
    if (V > 1 && dtype == kTypeF32 && K > kMostFp32Rows && B * (int64_t)size >= kShortRow) return 0;
    return rows_held(K, B, V, dtype, V == 1 ? 8 : 8 * V, g);
}

// Backward strips hold two matrices and leave three sums a row each (37 % of a matrix in pieces of 32 bytes).  us, strips
// and two passes (from cold memory the strips take 73 and 46 in bf16, 98 and 55 in fp32, 1.8 to 3 times their bytes): bf16
// 1024 x 8192 49 and 70, 300 x 16384 40 and 59; fp32 94 and 100, 48 and 69; but fp32 2048 x 8192 252
// and 163, 100 x 100000 (3125 strips, whose sums few rows join) 160 and 122.  Of more than 2048 rows only those of
// under 64 bytes: fp32 4000 x 8 21 and 24, 2000 x 64 24.2 and 24.5, 2800 x 64 37 and 25, 4000 x 64 50 and 25, 4000 x 512 62
// and 40, bf16 2000 x 64 22 and 27, 4000 x 64 40 and 28, 4000 x 512 48 and 43, 2800 x 256 36 and 37.
constexpr int kBackwardRows = 1024, kMostBackwardStrips = 1024;
constexpr int64_t kSmallBytes = 8 << 20, kBackwardBytes = 128 << 20;  // of a matrix: any rows that fit, kBackwardRows of them
int backward_rows(int K, int B, int dtype, strip_grid *g) {
    const int64_t row = B * (dtype == kTypeF32 ? 4ll : 2ll), bytes = K * row;
    if (bytes > kSmallBytes && (K > kBackwardRows || bytes > kBackwardBytes)) return 0;
    if (K > kStripRows && row >= kShortRow) return 0;
    const int rows = rows_held(K, B, pass_vector(B), dtype, B < kPassVector ? 8 : 4 * kPassVector, g);
    return rows > 0 && g->strips <= kMostBackwardStrips ? rows : 0;
}

}  // namespace

size_t residual_norm_workspace_bytes(int K, int B) {
    if (K <= 0 || B <= 0) return 0;
    size_t most = 0, blocks = 0;
    for (int dtype : {kTypeF32, kTypeBF16}) blocks = std::max(blocks, (size_t)grid_for(K, B, vector_of(B, dtype)).col_blocks);
    most = sizeof(double) * kSums * (size_t)grid_for(K, B, pass_vector(B)).splits * B + sizeof(float) * (kFactors * (size_t)B + 3 * blocks * K);
    for (int dtype : {kTypeF32, kTypeBF16}) {
        strip_grid sg;
        if (backward_rows(K, B, dtype, &sg) > 0) most = std::max(most, sizeof(float) * 3 * (size_t)sg.strips * K);
    }
    return most;
}

hipError_t launch_residual_norm_fwd(const norm_args &a, void *ws, hipStream_t s) {
    if (a.K == 0 || a.B == 0) return hipSuccess;
    strip_grid sg;
    const int rows = short_enough(a) ? forward_rows(a.K, a.B, a.dtype, &sg) : 0;
    if (rows > 0)
        return with_rows<8, 0>(vector_of(a.B, a.dtype), a.dtype, rows, [&](auto t, auto v, auto j) {
            forward_strip_kernel<decltype(t), decltype(v)::value, decltype(j)::value><<<sg.blocks(), kStripThreads, 0, s>>>(a, sg);
            return hipGetLastError();
        });
    const norm_grid sums = grid_for(a.K, a.B, pass_vector(a.B)), g = grid_for(a.K, a.B, vector_of(a.B, a.dtype), 1024);
    const bool post = a.post_gain != nullptr, pre = a.pre_gain != nullptr;
    double *part = static_cast<double *>(ws);
    float *fac = reinterpret_cast<float *>(part + kSums * (size_t)sums.splits * a.B);
    if (post || pre) {
        const hipError_t err = with_vectors<kPassVector>(pass_vector(a.B), a.dtype, [&](auto t, auto v) {
            using T = decltype(t);
            constexpr int N = decltype(v)::value;
            (a.y == nullptr  ? forward_sums_kernel<T, N, kHasPre>
             : !post         ? forward_sums_kernel<T, N, kHasY | kHasPre>
             : !pre          ? forward_sums_kernel<T, N, kHasY | kHasPost>
                             : forward_sums_kernel<T, N, kHasY | kHasPost | kHasPre>)
                <<<dim3(sums.col_blocks, sums.splits), kPassThreads, 0, s>>>(a, sums, part);
            forward_join_kernel<<<(int)ceil_div(a.B, kJoinColumns), kJoinThreads, 0, s>>>(a.K, a.B, a.eps, sums.splits, post, pre, part,
                                                                                    fac);
            return hipGetLastError();
        });
        if (err != hipSuccess) return err;
    }
    return with_vectors<0>(vector_of(a.B, a.dtype), a.dtype, [&](auto t, auto v) {
        forward_kernel<decltype(t), decltype(v)::value><<<dim3(g.col_blocks, g.splits), kPassThreads, 0, s>>>(a, g, fac);
        return hipGetLastError();
    });
}

hipError_t launch_residual_norm_bwd(const norm_args &a, void *ws, hipStream_t s) {
    if (a.K == 0) return hipSuccess;
    const bool post = a.post_gain != nullptr, pre = a.pre_gain != nullptr;
    float *dgate = a.gate_kind == kGateRow ? static_cast<float *>(a.dgate) : nullptr;
    auto join_rows = [&](int blocks, const float *rows) {
        if (a.dpre_gain || a.dpost_gain || dgate)
            row_sums_kernel<<<dim3((unsigned)ceil_div(a.K, 32), 3), kRowSumThreads, 0, s>>>(a.K, blocks, rows, a.dpre_gain, a.dpost_gain,
                                                                                    dgate);
        return hipGetLastError();
    };
    if (a.B == 0) return join_rows(0, nullptr);
    strip_grid sg;
    const int held = short_enough(a) ? backward_rows(a.K, a.B, a.dtype, &sg) : 0;
    if (held > 0) {
        float *rows = static_cast<float *>(ws);
        const hipError_t err = with_rows<4, kPassVector>(pass_vector(a.B), a.dtype, held, [&](auto t, auto v, auto j) {
            backward_strip_kernel<decltype(t), decltype(v)::value, decltype(j)::value>
                <<<sg.blocks(), kStripThreads, 0, s>>>(a, sg, rows);
            return hipGetLastError();
        });
        return err != hipSuccess ? err : join_rows(sg.strips, rows);
    }
    const norm_grid sums = grid_for(a.K, a.B, pass_vector(a.B)), g = grid_for(a.K, a.B, vector_of(a.B, a.dtype));
    double *part = static_cast<double *>(ws);
    float *fac = reinterpret_cast<float *>(part + kSums * (size_t)sums.splits * a.B), *rows = fac + kFactors * (size_t)a.B;
    hipError_t err = hipSuccess;
    if (post || pre)
        err = with_vectors<kPassVector>(pass_vector(a.B), a.dtype, [&](auto t, auto v) {
            using T = decltype(t);
            constexpr int N = decltype(v)::value;
            (!post  ? backward_sums_kernel<T, N, kHasPre>
             : !pre ? backward_sums_kernel<T, N, kHasPost>
                    : backward_sums_kernel<T, N, kHasPost | kHasPre>)
                <<<dim3(sums.col_blocks, sums.splits), kPassThreads, 0, s>>>(a, sums, part);
            backward_join_kernel<<<(int)ceil_div(a.B, kJoinColumns), kJoinThreads, 0, s>>>(a.K, a.B, a.eps, sums.splits, post, pre,
                                                                                     part, fac);
            return hipGetLastError();
        });
    if (err == hipSuccess)
        err = with_vectors<0>(vector_of(a.B, a.dtype), a.dtype, [&](auto t, auto v) {
            backward_kernel<decltype(t), decltype(v)::value>
                <<<dim3(g.col_blocks, g.splits), kPassThreads, 0, s>>>(a, g, fac, rows);
            return hipGetLastError();
        });
    return err != hipSuccess ? err : join_rows(g.col_blocks, rows);
}

}  // namespace l1csr
