// Losses on the log-probabilities of taken tokens and their gradients with
// respect to the logits z[C][B] (class-major, tokens contiguous):
//   lp_b = z[a_b][b] - log sum_c exp z[c][b]
//   policy      r = exp(lp - old), pg = -min(r A, clip(r, 1 - cl, 1 + ch) A),
//               kl = exp(ref - lp) - (ref - lp) - 1,
//               loss = sum_b w (pg + beta kl) / sum_b w
//   preference  S_s = sum_{b in s} w lp, reward_s = beta (S_s - R_s),
//               D = reward_chosen - reward_rejected,
//               loss = mean_p( -(1 - ls) log sig(D) - ls log sig(-D) )
// Both gradients are dz[c][b] = coef_b (1[c = a_b] - softmax(z_.b)_c) with one
// coefficient a token, coef_b = d loss / d lp_b, times a factor of the caller's
// that comes before dz's rounding (fp16 holds nothing under 2^-24).
//
// Three passes: partial (maximum, sum of exponentials) of every column over
// ranges of classes; a token pass that joins them and takes the loss and the
// coefficient; the gradient pass.  (The preference loss has a pass over the
// pairs before the last.)  Sums over tokens are taken in double in a fixed order.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace l1csr {

namespace {

constexpr int kThreads = 256;
constexpr int kTokenBlocks = 1024;  // most workgroups (and partial sums) of the token pass
constexpr int kJoin = 8;            // partial sums that a lane of it has in flight
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }

// exp(x) for x <= 0 (or NaN); results under 2^-126 are zero.  (The difference z - m is taken first: z log2 e
// overflows for masks of the type's lowest value.)
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// V values at any alignment of T: the hardware takes unaligned 16-byte accesses
template <typename T, int V>
__device__ __forceinline__ void load_vec(const T *p, T (&x)[V]) {
    __builtin_memcpy(x, p, sizeof(T) * V);
}

typedef unsigned word4 __attribute__((ext_vector_type(4), aligned(2)));

// Past the caches, where dz would only displace what is read (the whole call: 32768 x 8192 bf16 370 ->
// 315 us, 32768 x 4099 230 -> 181)
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const T (&x)[V]) {
    if constexpr (sizeof(T) * V == 16) {
        word4 w;
        __builtin_memcpy(&w, x, 16);
        __builtin_nontemporal_store(w, reinterpret_cast<word4 *>(p));
    } else {
        __builtin_nontemporal_store(x[0], p);
        static_assert(V == 1, "16 bytes or one value");
    }
}

// a word's two 16-bit values, and back (to nearest even)
__device__ __forceinline__ void unpack(unsigned w, __bf16, float &a, float &b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack(unsigned w, _Float16, float &a, float &b) {
    _Float16 x[2];
    __builtin_memcpy(x, &w, 4);
    a = (float)x[0];
    b = (float)x[1];
}
template <typename T>
__device__ __forceinline__ unsigned pack(float a, float b) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef T t2 __attribute__((ext_vector_type(2)));
    const t2 y = __builtin_convertvector((f2{a, b}), t2);
    unsigned w;
    __builtin_memcpy(&w, &y, 4);
    return w;
}

// How a workgroup lies over [C][B]: 2^tx_shift threads of V columns each side by
// side, the others over the classes; blockIdx.y a range of classes.
struct grid_shape {
    int tx_shift, col_blocks, splits, rows;
};

template <int V>
struct columns {
    int col0;   // the first column of this thread
    int at;     // where its loads begin: col0, or B - V where the columns end inside the vector
    bool any;   // it has a column
    __device__ columns(int tx, int tx_shift, int B) {
        col0 = (((int)blockIdx.x << tx_shift) + tx) * V;
        any = col0 < B;
        at = V == 1 ? col0 : min(col0, B - V);
    }
    // element v of the loads is a column of this thread (not its neighbour's)
    __device__ bool mine(int v) const { return at + v >= col0; }
};

__device__ __forceinline__ bool live(const int *labels, const float *w, int b, int C) {
    const int a = labels[b];
    return a >= 0 && a < C && (w == nullptr || w[b] != 0.f);
}

// Partial (maximum, sum of exponentials) of the columns over a range of classes.  Memory-bound: 112 us for 537 MB at
// 32768 x 8192 bf16 (4.8 TB/s); the vector units, at 10 instructions and an exponential (a quarter of their
// rate) a logit, are half busy, which is why the rescaling comes once in eight rows.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void column_sums_kernel(int C, int B, const T *__restrict__ z, int64_t ld,
                                                               const int *__restrict__ labels,
                                                               const float *__restrict__ w, grid_shape g,
                                                               float2 *__restrict__ part) {
    constexpr int U = 8;
    __shared__ float sm[kThreads * V], ss[kThreads * V];
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> k(tx, g.tx_shift, B);
    bool work = false;  // a column that counts: the others' logits are not read
    if (k.any)
#pragma unroll
        for (int v = 0; v < V; ++v) work |= k.mine(v) && live(labels, w, k.at + v, C);
    float m[V], s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        m[v] = -INFINITY;
        s[v] = 0.f;
    }
    const int c0 = blockIdx.y * g.rows, c1 = min(C, c0 + g.rows);
    // n rows (of U) of the columns' values, the others as excluded classes
    auto add = [&](const T(&x)[U][V], int n) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float y[U], top = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                y[u] = u < n ? to_f32(x[u][v]) : -INFINITY;
                top = fmaxf(top, y[u]);
            }
            top = fmaxf(top, m[v]);
            const float base = top == -INFINITY ? 0.f : top;  // only excluded classes so far
            float sum = s[v] * exp_neg(m[v] - base);
#pragma unroll
            for (int u = 0; u < U; ++u) sum += exp_neg(y[u] - base);
            m[v] = top;
            s[v] = sum;
        }
    };
    if (work) {
        int c = c0 + ty;
        const T *p = z + (int64_t)c * ld + k.at;
        const int64_t step = (int64_t)TY * ld;
        for (; c + (U - 1) * TY < c1; c += U * TY, p += U * step) {
            T x[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_vec<T, V>(p + u * step, x[u]);
            add(x, U);
        }
        if (c < c1) {
            const int n = (c1 - c + TY - 1) / TY;
            T x[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_vec<T, V>(p + min(u, n - 1) * step, x[u]);
            add(x, n);
        }
    }
    const int first = ((int)blockIdx.x << g.tx_shift) * V;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = k.at + v - first;
        if (k.any && k.mine(v)) {
            sm[ty * TX * V + col] = m[v];
            ss[ty * TX * V + col] = s[v];
        }
    }
    __syncthreads();
    const int n = min(TX * V, B - first);
    for (int col = threadIdx.x; col < n; col += kThreads) {
        float top = -INFINITY, sum = 0.f;
        for (int t = 0; t < TY; ++t) top = fmaxf(top, sm[t * TX * V + col]);
        const float base = top == -INFINITY ? 0.f : top;
        for (int t = 0; t < TY; ++t) sum += ss[t * TX * V + col] * exp_neg(sm[t * TX * V + col] - base);
        part[(int64_t)(first + col) * g.splits + blockIdx.y] = make_float2(top, sum);
    }
}

// What the token pass leaves for the others
struct token_out {
    float *m, *inv;   // the column's maximum and 1 / (sum of exponentials)
    float *coef;      // d loss / d lp (policy: times the sum of weights)
    float *lp;        // log-probability; 0 where the token does not count
    double *sums;     // [4][kTokenBlocks] weights, and weighted loss, kl, clipped
};

struct policy_args {
    const float *old_lp, *adv, *ref_lp;
    float low, high, kl_coef;  // 1 - clip_low, 1 + clip_high
};

enum { kLogp = 0, kPolicy = 1, kPreference = 2 };

struct policy_sums {
    double weight = 0, pg = 0, kl = 0, off = 0;  // the last three weighted
};

// w d loss / d lp of a token (times the sum of weights), its loss added to the sums
__device__ __forceinline__ float policy_token(const policy_args &P, const float *w, int b, float lp, policy_sums &s) {
    const float wt = w ? w[b] : 1.f, A = P.adv[b], r = expf(lp - P.old_lp[b]);
    const bool off = (A > 0.f && r > P.high) || (A < 0.f && r < P.low);
    const float used = off ? (A > 0.f ? P.high : P.low) : r;
    float kl = 0.f, dlp = off ? 0.f : -A * r;
    if (P.ref_lp) {
        const float q = P.ref_lp[b] - lp, e = expm1f(q);
        kl = e - q;
        dlp -= P.kl_coef * e;
    }
    s.weight += wt;
    s.pg += (double)wt * (-A * used);
    s.kl += (double)wt * kl;
    s.off += off ? wt : 0.f;
    return wt * dlp;
}

// A token's coefficient times the factor of all of them (grad_scale over the sum of weights), in double where that
// is no normal float: weights of any size enter by their shares, and a token that does not count keeps 0.
struct coef_scale {
    double wide;
    float narrow;
    bool normal;
    __device__ __forceinline__ explicit coef_scale(double x)
        : wide(x), narrow((float)x), normal(fabsf(narrow) >= 0x1p-126f && fabsf(narrow) < INFINITY) {}
    __device__ __forceinline__ float operator()(float coef) const {
        if (coef == 0.f) return 0.f;
        return normal ? coef * narrow : (float)(coef * wide);
    }
};

// A pair's loss, its rewards given, and d loss / d (sum of the preferred sequence), which is minus the other's
struct pair_terms {
    double loss, slope;
    __device__ __forceinline__ pair_terms(double chosen, double rejected, float smoothing, float beta, int pairs) {
        const double D = chosen - rejected, e = exp(-fabs(D)), up = D >= 0 ? 1 / (1 + e) : e / (1 + e);  // sig(D)
        const double down = D >= 0 ? e / (1 + e) : 1 / (1 + e);
        // -log sig(D) = log(1 + e) + max(-D, 0)
        loss = log1p(e) + (1 - (double)smoothing) * fmax(-D, 0.0) + smoothing * fmax(D, 0.0);
        slope = (smoothing * up - (1 - (double)smoothing) * down) * beta / pairs;
    }
};

// tokens lo .. mid - 1 and mid .. hi - 1 of a pair, within [0, B] whatever the offsets are
__device__ __forceinline__ void pair_range(const int *seq, int p, int B, int &lo, int &mid, int &hi) {
    lo = min(max(seq[2 * p], 0), B);
    mid = min(max(seq[2 * p + 1], lo), B);
    hi = min(max(seq[2 * p + 2], mid), B);
}

__device__ __forceinline__ double block_sum(double x, double *lds) {
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0;
    for (int i = 0; i < kThreads / kWave; ++i) t += lds[i];
    return t;
}

// 2^lane_shift lanes a token join its partial sums
template <typename T, int KIND>
__global__ __launch_bounds__(kThreads) void token_kernel(int C, int B, const T *__restrict__ z, int64_t ld,
                                                         const int *__restrict__ labels, const float *__restrict__ w,
                                                         int splits, int lane_shift, const float2 *__restrict__ part,
                                                         policy_args P, token_out o) {
    __shared__ double lds[kThreads / kWave];
    const int L = 1 << lane_shift, per = kThreads >> lane_shift;
    const int lane = threadIdx.x & (L - 1);
    policy_sums sums;
    for (int64_t b0 = (int64_t)blockIdx.x * per; b0 < B; b0 += (int64_t)gridDim.x * per) {
        const int64_t b = b0 + (threadIdx.x >> lane_shift);
        const bool on = b < B && live(labels, w, (int)b, C);
        float top = -INFINITY, s = 0.f;
        if (on)
            for (int i0 = lane; i0 < splits; i0 += L * kJoin) {
                float2 p[kJoin];
#pragma unroll
                for (int u = 0; u < kJoin; ++u) p[u] = part[b * splits + min(i0 + u * L, splits - 1)];
                float t = top;
#pragma unroll
                for (int u = 0; u < kJoin; ++u) t = fmaxf(t, p[u].x);  // (past the end the last again)
                const float base = t == -INFINITY ? 0.f : t;
                s *= exp_neg(top - base);
#pragma unroll
                for (int u = 0; u < kJoin; ++u) s += i0 + u * L < splits ? p[u].y * exp_neg(p[u].x - base) : 0.f;
                top = t;
            }
        const float mine = top;
        for (int d = L / 2; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, kWave));
        s *= exp_neg(mine - (top == -INFINITY ? 0.f : top));
        for (int d = L / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, kWave);
        if (lane != 0 || b >= B) continue;
        const float lp = on ? (to_f32(z[(int64_t)labels[b] * ld + b]) - top) - logf(s) : 0.f;
        if (o.lp) o.lp[b] = lp;
        if constexpr (KIND == kLogp) continue;
        o.m[b] = top;
        o.inv[b] = on ? 1.f / s : 0.f;
        o.coef[b] = KIND == kPolicy && on ? policy_token(P, w, (int)b, lp, sums) : 0.f;
    }
    if constexpr (KIND == kPolicy) {
        const double t[4] = {block_sum(sums.weight, lds), block_sum(sums.pg, lds), block_sum(sums.kl, lds), block_sum(sums.off, lds)};
        if (threadIdx.x < 4) o.sums[threadIdx.x * kTokenBlocks + blockIdx.x] = t[threadIdx.x];
    }
}

// A workgroup a pair: the sums over its two sequences, the loss, the tokens' coefficients.
__global__ __launch_bounds__(kThreads) void pair_kernel(int C, int B, int pairs, const int *__restrict__ labels,
                                                        const float *__restrict__ w, const int *__restrict__ seq,
                                                        const float *__restrict__ ref, float beta, float smoothing,
                                                        const float *__restrict__ lp, float *__restrict__ coef,
                                                        float *__restrict__ rewards, double *__restrict__ loss) {
    __shared__ double lds[kThreads / kWave];
    const int p = blockIdx.x;
    int lo, mid, hi;
    pair_range(seq, p, B, lo, mid, hi);
    double s0 = 0, s1 = 0;
    for (int b = lo + (int)threadIdx.x; b < hi; b += kThreads) {
        if (!live(labels, w, b, C)) continue;
        const double x = (double)lp[b] * (w ? w[b] : 1.f);
        if (b < mid) s0 += x; else s1 += x;
    }
    s0 = beta * (block_sum(s0, lds) - (ref ? ref[2 * p] : 0.f));
    s1 = beta * (block_sum(s1, lds) - (ref ? ref[2 * p + 1] : 0.f));
    const pair_terms t(s0, s1, smoothing, beta, pairs);
    if (threadIdx.x == 0) {
        if (rewards) {
            rewards[2 * p] = (float)s0;
            rewards[2 * p + 1] = (float)s1;
        }
        loss[p] = t.loss;
    }
    for (int b = lo + (int)threadIdx.x; b < hi; b += kThreads)
        if (live(labels, w, b, C)) coef[b] = (float)((b < mid ? t.slope : -t.slope) * (w ? w[b] : 1.f));
}

// The loss from the partial sums, by one workgroup: out[0..3] = loss, policy part, kl, clipped share,
// or out[0] = the mean over the pairs.  Returns what the policy's coefficients are scaled with.
template <int KIND>
__device__ double finish(int n, const double *__restrict__ sums, float kl_coef, double *lds, bool write, float *out) {
    auto sum = [&](const double *x) {
        double t = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) t += x[i];
        return block_sum(t, lds);
    };
    if constexpr (KIND == kPolicy) {
        const double sw = sum(sums), inv = sw != 0 ? 1 / sw : 0.0;
        if (!write) return inv;
        double t[3];
        for (int q = 0; q < 3; ++q) t[q] = sum(sums + (q + 1) * kTokenBlocks) * inv;
        if (threadIdx.x == 0) {
            out[0] = (float)(t[0] + kl_coef * t[1]);
            out[1] = (float)t[0];
            out[2] = (float)t[1];
            out[3] = (float)t[2];
        }
        return inv;
    } else {
        if (!write) return 1;
        const double x = sum(sums);
        if (threadIdx.x == 0) out[0] = n > 0 ? (float)(x / n) : 0.f;
        return 1;
    }
}

template <int KIND>
__global__ __launch_bounds__(kThreads) void finish_kernel(int n, const double *__restrict__ sums, float kl_coef,
                                                          float *__restrict__ out) {
    __shared__ double lds[kThreads / kWave];
    finish<KIND>(n, sums, kl_coef, lds, true, out);
}

// dz, over the layout of column_sums_kernel; z and dz may be the same matrix (every
// element is read by the thread that writes it; a thread's loads of its
// neighbour's columns are not used).  A token's own class comes last, from lp.
// Memory-bound: 205 us for 1074 MB at 32768 x 8192 bf16 (5.2 TB/s, a large copy 4.9).
template <typename T, int V, int KIND>
__global__ __launch_bounds__(kThreads) void gradient_kernel(int C, int B, const T *z, int64_t ld,
                                                            const int *__restrict__ labels, grid_shape g, token_out t,
                                                            T *dz, int64_t ldd, int n_sums, float kl_coef,
                                                            float grad_scale, float *__restrict__ out) {
    constexpr int U = 4;
    __shared__ double lds[kThreads / kWave];
    const coef_scale scale(grad_scale *
                           finish<KIND>(n_sums, t.sums, kl_coef, lds, blockIdx.x == 0 && blockIdx.y == 0, out));
    const int TX = 1 << g.tx_shift, TY = kThreads >> g.tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> g.tx_shift;
    const columns<V> k(tx, g.tx_shift, B);
    if (!k.any) return;
    float m[V], f[V];  // dz = f exp(z - m)
    constexpr int words = sizeof(T) * V / 4;
    unsigned keep[words > 0 ? words : 1];  // the bits of the columns that count: the others' may hold anything
    T ones[V];
    bool work = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float coef = scale(t.coef[k.at + v]);
        const bool on = coef != 0.f;
        m[v] = on ? t.m[k.at + v] : 0.f;
        f[v] = on ? -coef * t.inv[k.at + v] : 0.f;
        work |= k.mine(v) && on;
        __builtin_memset(&ones[v], on ? 0xff : 0, sizeof(T));
    }
    __builtin_memcpy(keep, ones, sizeof(T) * V);
    const int c0 = blockIdx.y * g.rows, c1 = min(C, c0 + g.rows);
    const bool whole = k.at == k.col0;
    const int64_t step = (int64_t)TY * ld, stepd = (int64_t)TY * ldd;
    // from the range's end, whose logits the sums read last (the whole call: 326 -> 316 us)
    for (int c = c0 + ty + max(0, c1 - c0 - ty - 1) / (U * TY) * (U * TY); c >= c0; c -= U * TY) {
        if (c >= c1) continue;
        const T *p = z + (int64_t)c * ld + k.at;
        T *d = dz + (int64_t)c * ldd + k.at;
        T x[U][V];
        const int n = min(U, (c1 - c + TY - 1) / TY);
        if (work) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_vec<T, V>(p + min(u, n - 1) * step, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= n) continue;
            T y[V] = {};
            if (work) {
                auto value = [&](float x, int v) { return f[v] * exp_neg(x - m[v]); };
                if constexpr (words > 0) {
                    unsigned b[words];
                    __builtin_memcpy(b, x[u], sizeof(b));
#pragma unroll
                    for (int i = 0; i < words; ++i) {
                        b[i] &= keep[i];
                        if constexpr (sizeof(T) == 4) {
                            b[i] = __float_as_uint(value(__uint_as_float(b[i]), i));
                        } else {
                            float lo, hi;
                            unpack(b[i], T{}, lo, hi);
                            b[i] = pack<T>(value(lo, 2 * i), value(hi, 2 * i + 1));
                        }
                    }
                    __builtin_memcpy(y, b, sizeof(b));
                } else {
                    y[0] = f[0] == 0.f ? (T)0.f : (T)value(to_f32(x[u][0]), 0);
                }
            }
            if (whole) {
                store_vec<T, V>(d + u * stepd, y);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (k.mine(v)) d[u * stepd + v] = y[v];
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int b = k.at + v, a = labels[b];
        if (!k.mine(v) || a < c0 || a >= c1 || (a - c0) % TY != ty) continue;
        const float coef = scale(t.coef[b]);
        if (coef != 0.f) dz[(int64_t)a * ldd + b] = (T)(-coef * expm1f(t.lp[b]));
    }
}

// A small problem in one workgroup: its launches are all that such a call costs (us, three or four of them and one:
// policy loss 10 x 128 19.4 and 13.1, 32768 x 1 20.8 and 16.7, 32 x 1000 19.6 and 15.4). 2^tx_shift threads over
// the columns, the others over the classes, the tokens' values in LDS.
constexpr int kSmallThreads = 1024;
constexpr int kSmallTokens = 1024;       // most columns
constexpr int kSmallElements = 1 << 15;  // most logits

template <typename T, int KIND>
__global__ __launch_bounds__(kSmallThreads) void small_loss_kernel(token_loss_args a, policy_args P, int tx_shift) {
    constexpr int waves = kSmallThreads / kWave;
    __shared__ float part_m[kSmallThreads], part_s[kSmallThreads];  // (2^tx_shift columns of as many waves as have them)
    __shared__ float tm[kSmallTokens], tinv[kSmallTokens], tcoef[kSmallTokens], tlp[kSmallTokens];
    __shared__ double lds[waves];
    const int C = a.C, B = a.B, TX = 1 << tx_shift, TY = kSmallThreads >> tx_shift;
    const int tx = threadIdx.x & (TX - 1), ty = threadIdx.x >> tx_shift;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const T *z = static_cast<const T *>(a.logits) + tx;  // B <= TX
    const bool on = tx < B && live(a.labels, a.weights, tx, C);
    auto sum = [&](double x) {
#pragma unroll
        for (int d = kWave / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d, kWave);
        __syncthreads();
        if (lane == 0) lds[wave] = x;
        __syncthreads();
        double t = 0;
        for (int i = 0; i < waves; ++i) t += lds[i];
        return t;
    };
    float m = -INFINITY, s = 0.f;
    if (on)
        for (int c = ty; c < C; c += 4 * TY) {
            float y[4], top = m;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = c + u * TY;
                const float v = to_f32(z[(int64_t)min(r, C - 1) * a.ld]);
                y[u] = r < C ? v : -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) top = fmaxf(top, y[u]);
            const float base = top == -INFINITY ? 0.f : top;
            s *= exp_neg(m - base);
#pragma unroll
            for (int u = 0; u < 4; ++u) s += exp_neg(y[u] - base);
            m = top;
        }
    auto join = [&](float m2, float s2) {
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
        s = s * exp_neg(m - base) + s2 * exp_neg(m2 - base);
        m = top;
    };
    for (int d = TX; d < kWave; d <<= 1) {
        const float m2 = __shfl_xor(m, d, kWave), s2 = __shfl_xor(s, d, kWave);
        join(m2, s2);
    }
    part_m[threadIdx.x] = m;
    part_s[threadIdx.x] = s;
    __syncthreads();
    policy_sums ps;
    if (ty == 0) {
        // (a wave's rows are joined already where it has several)
        for (int t = TX > kWave ? TX : kWave; t < kSmallThreads; t += TX > kWave ? TX : kWave)
            join(part_m[t + tx], part_s[t + tx]);
        const float lp = on ? (to_f32(z[(int64_t)a.labels[tx] * a.ld]) - m) - logf(s) : 0.f;
        if (tx < B) {
            if (a.logp) a.logp[tx] = lp;
            if constexpr (KIND != kLogp) {
                tm[tx] = m;
                tinv[tx] = on ? 1.f / s : 0.f;
                tlp[tx] = lp;
                tcoef[tx] = KIND == kPolicy && on ? policy_token(P, a.weights, tx, lp, ps) : 0.f;
            }
        }
    }
    if constexpr (KIND == kLogp) return;
    double factor = a.grad_scale;
    if constexpr (KIND == kPolicy) {
        const double sw = sum(ps.weight), inv = sw != 0 ? 1 / sw : 0.0;
        const double pg = sum(ps.pg) * inv, kl = sum(ps.kl) * inv, off = sum(ps.off) * inv;
        if (threadIdx.x == 0) {
            a.out[0] = (float)(pg + P.kl_coef * kl);
            a.out[1] = (float)pg;
            a.out[2] = (float)kl;
            a.out[3] = (float)off;
        }
        factor *= inv;
    } else {
        __syncthreads();
        double loss = 0;
        for (int p = wave; p < a.pairs; p += waves) {
            int lo, mid, hi;
            pair_range(a.seq_ptr, p, B, lo, mid, hi);
            double s0 = 0, s1 = 0;
            for (int b = lo + lane; b < hi; b += kWave) {
                const double x = (double)tlp[b] * (a.weights ? a.weights[b] : 1.f);
                if (!live(a.labels, a.weights, b, C)) continue;
                if (b < mid) s0 += x; else s1 += x;
            }
#pragma unroll
            for (int d = kWave / 2; d >= 1; d >>= 1) {
                s0 += __shfl_xor(s0, d, kWave);
                s1 += __shfl_xor(s1, d, kWave);
            }
            s0 = a.beta * (s0 - (a.ref_logp ? a.ref_logp[2 * p] : 0.f));
            s1 = a.beta * (s1 - (a.ref_logp ? a.ref_logp[2 * p + 1] : 0.f));
            const pair_terms t(s0, s1, a.smoothing, a.beta, a.pairs);
            if (lane == 0) {
                if (a.rewards) {
                    a.rewards[2 * p] = (float)s0;
                    a.rewards[2 * p + 1] = (float)s1;
                }
                loss += t.loss;
            }
            for (int b = lo + lane; b < hi; b += kWave)
                if (live(a.labels, a.weights, b, C))
                    tcoef[b] = (float)((b < mid ? t.slope : -t.slope) * (a.weights ? a.weights[b] : 1.f));
        }
        loss = sum(loss);
        if (threadIdx.x == 0) a.out[0] = a.pairs > 0 ? (float)(loss / a.pairs) : 0.f;
    }
    if (a.dlogits == nullptr || tx >= B) return;
    __syncthreads();
    const float coef = coef_scale(factor)(tcoef[tx]), f = coef != 0.f ? -coef * tinv[tx] : 0.f;
    const float own = coef != 0.f ? -coef * expm1f(tlp[tx]) : 0.f;
    const int label = a.labels[tx];
    T *dz = static_cast<T *>(a.dlogits) + tx;
    m = tm[tx];
    for (int c = ty; c < C; c += 4 * TY) {
        float y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = to_f32(z[(int64_t)min(c + u * TY, C - 1) * a.ld]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = c + u * TY;
            if (r >= C) continue;
            dz[(int64_t)r * a.ldd] = (T)(r == label ? own : (coef != 0.f ? f * exp_neg(y[u] - m) : 0.f));
        }
    }
}

template <typename T>
constexpr int kVec = 16 / sizeof(T);

// (more leave a last partial round: with 2048 the whole policy loss at 32768 x 8192 bf16 took 405 us for 370, with
// 768 369, 32768 x 4099 259, 232 and 253)
constexpr int kWorkgroups = 1024;

// ranges of a round of loads at least
grid_shape shape_of(int C, int B, int V) {
    grid_shape g;
    const int64_t threads = ceil_div(B, V);
    g.tx_shift = 0;
    while ((1 << g.tx_shift) < threads && g.tx_shift < 6) ++g.tx_shift;
    g.col_blocks = (int)ceil_div(threads, 1 << g.tx_shift);
    const int TY = kThreads >> g.tx_shift;
    int64_t s = ceil_div(kWorkgroups, g.col_blocks);
    const int64_t most = ceil_div(C, 8 * TY);
    s = s < most ? s : most;
    g.rows = (int)ceil_div(C, s);
    g.splits = (int)ceil_div(C, g.rows);
    return g;
}

struct carved {
    float2 *part;
    token_out t;
    double *pair_loss;
    size_t bytes;
};

carved carve(int C, int B, int pairs, void *ws) {
    carved r;
    char *p = static_cast<char *>(ws);
    auto take = [&](size_t n) {
        char *q = p;
        p += (n + 255) / 256 * 256;
        return q;
    };
    // room for every vector width
    int64_t most = 0;
    for (int v : {1, 4, 8})
        if (B >= v) most = std::max<int64_t>(most, (int64_t)B * shape_of(C, B, v).splits);
    r.part = reinterpret_cast<float2 *>(take(sizeof(float2) * (size_t)most));
    r.t.m = reinterpret_cast<float *>(take(sizeof(float) * B));
    r.t.inv = reinterpret_cast<float *>(take(sizeof(float) * B));
    r.t.coef = reinterpret_cast<float *>(take(sizeof(float) * B));
    r.t.lp = reinterpret_cast<float *>(take(sizeof(float) * B));
    r.t.sums = reinterpret_cast<double *>(take(sizeof(double) * 4 * kTokenBlocks));
    r.pair_loss = reinterpret_cast<double *>(take(sizeof(double) * pairs));
    r.bytes = (size_t)(p - static_cast<char *>(ws));
    return r;
}

template <typename T, int V, int KIND>
hipError_t run(const token_loss_args &a, const policy_args &P, void *ws, hipStream_t s) {
    if (a.B <= kSmallTokens && (int64_t)a.C * a.B <= kSmallElements) {
        int shift = 0;
        while ((1 << shift) < a.B) ++shift;
        small_loss_kernel<T, KIND><<<1, kSmallThreads, 0, s>>>(a, P, shift);
        return hipGetLastError();
    }
    const grid_shape g = shape_of(a.C, a.B, V);
    carved w = carve(a.C, a.B, a.pairs, ws);
    token_out t = w.t;
    if (a.logp) t.lp = a.logp;
    const T *z = static_cast<const T *>(a.logits);
    const dim3 grid((unsigned)g.col_blocks, (unsigned)g.splits);
    column_sums_kernel<T, V><<<grid, kThreads, 0, s>>>(a.C, a.B, z, a.ld, a.labels, a.weights, g, w.part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int shift = 0;
    while ((1 << shift) < g.splits && shift < 4) ++shift;
    int n = std::min((int)ceil_div(a.B, kThreads >> shift), kTokenBlocks);
    token_kernel<T, KIND><<<n, kThreads, 0, s>>>(a.C, a.B, z, a.ld, a.labels, a.weights, g.splits, shift, w.part, P, t);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if constexpr (KIND == kLogp) {
        return hipSuccess;
    } else {
        if (KIND == kPreference) {
            n = a.pairs;
            if (n > 0) {
                pair_kernel<<<n, kThreads, 0, s>>>(a.C, a.B, n, a.labels, a.weights, a.seq_ptr, a.ref_logp, a.beta,
                                                   a.smoothing, t.lp, t.coef, a.rewards, w.pair_loss);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            t.sums = w.pair_loss;
        }
        if (a.dlogits == nullptr)
            finish_kernel<KIND><<<1, kThreads, 0, s>>>(n, t.sums, P.kl_coef, a.out);
        else
            gradient_kernel<T, V, KIND><<<grid, kThreads, 0, s>>>(a.C, a.B, z, a.ld, a.labels, g, t,
                                                                  static_cast<T *>(a.dlogits), a.ldd, n, P.kl_coef,
                                                                  a.grad_scale, a.out);
        return hipGetLastError();
    }
}

template <typename T, int KIND>
hipError_t run_vec(const token_loss_args &a, const policy_args &P, void *ws, hipStream_t s) {
    return a.B >= kVec<T> ? run<T, kVec<T>, KIND>(a, P, ws, s) : run<T, 1, KIND>(a, P, ws, s);
}

template <int KIND>
hipError_t run_type(const token_loss_args &a, const policy_args &P, void *ws, hipStream_t s) {
    if (a.dtype == kTypeF32) return run_vec<float, KIND>(a, P, ws, s);
    if (a.dtype == kTypeBF16) return run_vec<__bf16, KIND>(a, P, ws, s);
    return run_vec<_Float16, KIND>(a, P, ws, s);
}

}  // namespace

// 32-bit class and column numbers with room for a round of a workgroup's loads; the threads of a grid
bool token_loss_fits(int C, int B, int pairs) { return C <= (1 << 30) && B <= (1 << 30) && pairs < (1 << 24); }

size_t token_loss_workspace_bytes(int C, int B, int pairs) {
    return C > 0 && B >= 0 && pairs >= 0 && (B > 0 || pairs > 0) && token_loss_fits(C, B, pairs) ? carve(C, B, pairs, nullptr).bytes : 0;
}

hipError_t launch_token_logp(const token_loss_args &a, void *ws, hipStream_t s) {
    return a.B == 0 ? hipSuccess : run_type<kLogp>(a, policy_args{}, ws, s);
}

hipError_t launch_policy_loss(const token_loss_args &a, void *ws, hipStream_t s) {
    if (a.B == 0) return launch_fill_f32(a.out, 4, 0.f, s);
    return run_type<kPolicy>(a, policy_args{a.old_logp, a.adv, a.ref_logp, 1.f - a.clip_low, 1.f + a.clip_high, a.kl_coef},
                             ws, s);
}

hipError_t launch_preference_loss(const token_loss_args &a, void *ws, hipStream_t s) {
    if (a.B == 0) {  // empty sequences: the loss of the reference alone
        const carved w = carve(a.C, 0, a.pairs, ws);
        if (a.pairs > 0)
            pair_kernel<<<a.pairs, kThreads, 0, s>>>(a.C, 0, a.pairs, a.labels, a.weights, a.seq_ptr, a.ref_logp,
                                                     a.beta, a.smoothing, nullptr, nullptr, a.rewards, w.pair_loss);
        finish_kernel<kPreference><<<1, kThreads, 0, s>>>(a.pairs, w.pair_loss, 0.f, a.out);
        return hipGetLastError();
    }
    return run_type<kPreference>(a, policy_args{}, ws, s);
}

}  // namespace l1csr
