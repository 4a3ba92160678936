// Orthogonalised momentum (the Muon update; K. Jordan et al., 2024):
//   M' = mu M + G,  U = G + mu M' (Nesterov) or M' (without momentum: U = G)
//   X  = U / (|U|_F + eps), transposed where it has more rows than columns
//   `steps` times:  A = X X^T,  X <- a X + (b A + c A^2) X
//   O  = scale X
// The quintic f(x) = a x + b x^3 + c x^5 moves every singular value in (0, 1]
// towards [0.7, 1.2] and leaves the singular vectors alone.
//
// Form.  X is m x n, m <= n.  With P(A) = a I + b A + c A^2 a step is X <- P X,
// and the next Gram matrix is P A P: g steps need X only for A and for the last
// product, Q X with Q = P_g ... P_1:  3 m^2 n + (4 g - 3) m^3 multiplications
// (A, and every product of the polynomials of one symmetric matrix, is
// symmetric: half a product) against g (3 m^2 n + m^3).  A small eigenvalue of A
// grows 11.9-fold a step and the error that A was made with grows along, so A is made again from X
// after three steps at most; in one group of five a matrix of rank 8 of 500 x
// 800 came out twice as far from the 64-bit result, a square random one of 1024 thirty times.
//
// Arithmetic.  Operands are fp16 parts of 2^e x: two (hi, lo: 22 bits) with the
// three products hi hi, lo hi, hi lo, summed in fp32, the small ones apart (the
// fp32 result: 4e-7 to 1e-6 off the 64-bit one over the five steps where fp32
// matrix products give 2e-6), or one part with one product (2^-12 an operand,
// 1e-3 off).  |X| <= 1.3, |A| <= 1.7, |P| <= 3.5 and |Q| <= 41, so the scales
// 2^14 and 2^10 keep every part in range and the second part's last bit at 2^-38
// or 2^-34.  U is brought into range by a power of two; the rest of 1 / (|U|_F +
// eps) is multiplied in behind the first products.  One part keeps X itself in
// two: a X is added from both, or the rounding of X, which spreads into
// directions that U lacks, would grow 3.4-fold a step (1.4e-2 off at rank 64 of
// 300 x 784 against 8e-4).
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "common.hpp"
#include "launch.hpp"
#include "lds_dma.hpp"

namespace l1csr {

namespace {

typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int kGroup = 32, kStep = 16, kBlock = 1024;
constexpr int kScaleX = 14, kScaleP = 10;  // exponents of the parts: X, A and P A; P and Q
constexpr int kNormBlocks = 1024;          // most partial sums of |U|^2
constexpr int kMaxGroup = 3;               // steps between two products with X

// A packed operand: [32-row group][16-index step][part][lane][8] fp16.  Lane l of
// a block holds row l % 32 and reduction indices 8 (l / 32) .. + 7: the fragment of one
// v_mfma_f32_32x32x16_f16, so copies into LDS and fragment reads are linear in
// the lane.  An even number of steps; rows and indices past the matrix are zeros.
struct packed_half {
    char *data;
    int groups, steps;
    int parts;  // stored (a product with one part reads the first)
};

int even_steps(int k) { return 2 * (int)ceil_div(k, 32); }
size_t packed_half_bytes(int rows, int k, int parts) {
    return (size_t)ceil_div(rows, kGroup) * even_steps(k) * parts * kBlock;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(__bf16 x) { return (float)x; }

template <int waves>
__device__ __forceinline__ double block_sum(double x, double *lds) {
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = lds[0];
#pragma unroll
    for (int w = 1; w < waves; ++w) t += lds[w];
    return t;
}

// ---------------------------------------------------------------------------
// momentum, norm, packing
// ---------------------------------------------------------------------------

struct update_src {
    const void *G;     // [N][ldg]
    int64_t ldg;
    const float *M;    // [N][ldm], null: U = G
    int64_t ldm;
    float *M_out;      // [N][ldo], null: not stored
    int64_t ldo;
    float mu;
    int nesterov;
    int N, K;
};

__device__ __forceinline__ float update_at(const update_src &u, float g, float m_new) {
    return u.M == nullptr ? g : (u.nesterov ? fmaf(u.mu, m_new, g) : m_new);
}

// M' and the partial sums of U^2, four columns a thread.  Memory-bound: 79 us for 453 MB at 4096 x 9216 (5.7 TB/s)
template <typename T>
__global__ __launch_bounds__(256) void momentum_kernel(update_src u, double *__restrict__ part) {
    __shared__ double lds[4];
    const T *G = static_cast<const T *>(u.G);
    const unsigned per_row = (unsigned)(u.K + 3) / 4;
    const uint64_t chunks = (uint64_t)per_row * (unsigned)u.N;
    double sum = 0;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < chunks; i += gridDim.x * 256ull) {
        const unsigned row = (unsigned)i / per_row, k = ((unsigned)i - row * per_row) * 4;  // chunks < 2^31
        const T *g = G + (int64_t)row * u.ldg + k;
        const float *m = u.M ? u.M + (int64_t)row * u.ldm + k : nullptr;
        float *o = u.M_out ? u.M_out + (int64_t)row * u.ldo + k : nullptr;
        const int n = min(4, u.K - (int)k);
        T gv[4];
        float mv[4] = {0.f, 0.f, 0.f, 0.f};
        if (n == 4) {
            __builtin_memcpy(gv, g, sizeof(gv));
            if (m) __builtin_memcpy(mv, m, sizeof(mv));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gv[e] = e < n ? g[e] : (T)0.f;
                if (m && e < n) mv[e] = m[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            mv[e] = fmaf(u.mu, mv[e], to_f32(gv[e]));
            const double x = (double)update_at(u, to_f32(gv[e]), mv[e]);
            if (e < n) sum = fma(x, x, sum);
        }
        if (o == nullptr) continue;
        if (n == 4)
            __builtin_memcpy(o, mv, sizeof(mv));
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) o[e] = mv[e];
    }
    sum = block_sum<4>(sum, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// hi (and lo) of 8 values
template <int N>
struct parts_of {
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    vec hi, lo;
    __device__ __forceinline__ explicit parts_of(const float (&x)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            hi[e] = (_Float16)x[e];
            lo[e] = (_Float16)(x[e] - (float)hi[e]);
        }
    }
};

// 2^-e |U|_F in [1/2, 1) and s = 1 / (2^-e (|U|_F + eps)), at most 2.  U = 0: s = 0, not 1 / eps, whose square, taken
// in float, would be infinite below eps = 5.4e-20 and NaN times the zero Gram matrix.
struct norm_scale {
    int e = 0;
    float s;
    __device__ __forceinline__ norm_scale(double norm, float eps) {
        if (norm < INFINITY) {
            (void)frexp(norm, &e);
            s = norm > 0 ? (float)(1 / ldexp(norm + (double)eps, -e)) : 0.f;
        } else {
            s = NAN;  // an infinity or a NaN in U, or a norm past double: nothing to give
        }
    }
};

// e of U's norm from its partial sums; scal[0] = s, scal[1] = s^2
template <int waves>
__device__ __forceinline__ int scale_of(const double *part, int n_part, float eps, float *scal, bool write,
                                        double *lds) {
    double sum = 0;
    for (int i = threadIdx.x; i < n_part; i += waves * kWave) sum += part[i];
    const norm_scale ns(sqrt(block_sum<waves>(sum, lds)), eps);
    if (write && threadIdx.x == 0) {
        scal[0] = ns.s;
        scal[1] = ns.s * ns.s;
    }
    return ns.e;
}

// V elements of U (0 past its ends): every load in flight before the first is used
template <typename T, int V, typename At>
__device__ __forceinline__ void load_update(const update_src &u, At at, float (&x)[V]) {
    const T *G = static_cast<const T *>(u.G);
    T g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        int r, c;
        at(v, r, c);
        g[v] = G[(int64_t)min(r, u.N - 1) * u.ldg + min(c, u.K - 1)];
    }
    float m[V] = {};
    if (u.M) {
        const float *M = u.M_out ? u.M_out : u.M;
        const int64_t ld = u.M_out ? u.ldo : u.ldm;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            int r, c;
            at(v, r, c);
            m[v] = M[(int64_t)min(r, u.N - 1) * ld + min(c, u.K - 1)];
        }
        if (u.M_out == nullptr)
#pragma unroll
            for (int v = 0; v < V; ++v) m[v] = fmaf(u.mu, m[v], to_f32(g[v]));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        int r, c;
        at(v, r, c);
        x[v] = r < u.N && c < u.K ? update_at(u, to_f32(g[v]), m[v]) : 0.f;
    }
}

// 2^14 2^-e U packed by rows (X) and by columns (X^T).  A workgroup takes 64 x 64 of X.  Memory-bound: 118 us
// for 604 MB at 4096 x 9216 (5.1 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void pack_update_kernel(update_src u, int tall, const double *__restrict__ part,
                                                          int n_part, float eps, packed_half X, packed_half Xt,
                                                          float *__restrict__ scal) {
    constexpr int LD = 65;
    __shared__ float tile[64 * LD];
    __shared__ double lds[4];
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;  // of X
    const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;    // of U
    const int col = threadIdx.x & 63, q = threadIdx.x >> 6;
    float x[16];
    load_update<T>(u, [&](int v, int &r, int &c) { r = r0 + q + 4 * v; c = c0 + col; }, x);
    const int e = scale_of<4>(part, n_part, eps, scal, blockIdx.x == 0 && blockIdx.y == 0, lds);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = q + 4 * v;
        tile[tall ? col * LD + r : r * LD + col] = ldexpf(x[v], kScaleX - e);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
#pragma unroll
    for (int b = 0; b < 16; b += 4) {  // blocks of X, then of X^T
        const bool t = b >= 8;
        const packed_half &o = t ? Xt : X;
        const int gg = b >> 2 & 1, ss = q;
        const int g = (t ? j0 : i0) / kGroup + gg, st = (t ? i0 : j0) / kStep + ss;
        if (g >= o.groups || st >= o.steps) continue;
        float y[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int row = gg * 32 + l, k = ss * 16 + h * 8 + v;
            y[v] = t ? tile[k * LD + row] : tile[row * LD + k];
        }
        const parts_of<8> p(y);
        char *d = o.data + ((int64_t)g * o.steps + st) * (o.parts * kBlock) + lane * 16;
        *reinterpret_cast<halfx8 *>(d) = p.hi;
        if (o.parts == 2) *reinterpret_cast<halfx8 *>(d + kBlock) = p.lo;
    }
}

// ---------------------------------------------------------------------------
// m <= 128: a step in one launch
// ---------------------------------------------------------------------------
//
// Such matrices are bound by the launches' own time.  A workgroup holds all of A (the
// sums over the column ranges of X, added up by every workgroup) and a slice of
// 64 columns of X: it takes Y = A X, X' = a X + b Y + c A Y and, with X' still in LDS,
// the slice's part of X' X'^T.  One product more than with the polynomial of A made
// ahead, on a slice that one workgroup multiplies in a microsecond.  Many ranges are
// summed by a launch of their own first.

constexpr int kSmall = 128;       // most rows of X
constexpr int kSlice = 64;        // columns of X a workgroup takes at a time
constexpr int kSliceSteps = kSlice / kStep;
constexpr int kMostRanges = 192;  // partial sums of A
constexpr int kSumRanges = 8;     // more are summed ahead

// partial sums of A: [range][32 x 32 tile, ti <= tj by columns][register][lane]
__host__ __device__ constexpr int tiles_of(int g) { return g * (g + 1) / 2; }
__device__ __forceinline__ void tile_of(int t, int &ti, int &tj) {
    tj = t >= 6 ? 3 : (t >= 3 ? 2 : (t >= 1 ? 1 : 0));
    ti = t - tj * (tj + 1) / 2;
}

// byte of element (row, k) of a two-part operand, first part
__device__ __forceinline__ int element_at(int row, int k, int steps) {
    return ((row >> 5) * steps + (k >> 4)) * (2 * kBlock) + ((row & 31) + 32 * ((k >> 3) & 1)) * 16 + (k & 7) * 2;
}

__device__ __forceinline__ void product_step(const char *pa, const char *pb, floatx16 &acc, floatx16 &low) {
    const halfx8 ah = *reinterpret_cast<const halfx8 *>(pa), al = *reinterpret_cast<const halfx8 *>(pa + kBlock);
    const halfx8 bh = *reinterpret_cast<const halfx8 *>(pb), bl = *reinterpret_cast<const halfx8 *>(pb + kBlock);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc, 0, 0, 0);
    low = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, low, 0, 0, 0);
    low = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, low, 0, 0, 0);
}

// The products of this wave's tiles of X X^T over a slice, packed by rows in LDS
template <int g, int waves, int per>
__device__ __forceinline__ void gram_slice(const char *X, int wave, int lane, floatx16 (&acc)[per], floatx16 (&low)[per]) {
#pragma unroll
    for (int x = 0; x < per; ++x) {
        const int t = wave + waves * x;
        if (t >= tiles_of(g)) continue;
        int ti, tj;
        tile_of(t, ti, tj);
#pragma unroll
        for (int st = 0; st < kSliceSteps; ++st)
            product_step(X + (ti * kSliceSteps + st) * (2 * kBlock) + lane * 16,
                         X + (tj * kSliceSteps + st) * (2 * kBlock) + lane * 16, acc[x], low[x]);
    }
}

template <int g, int waves, int per>
__device__ __forceinline__ void store_gram(float *partial, int wave, int lane, const floatx16 (&acc)[per],
                                           const floatx16 (&low)[per]) {
#pragma unroll
    for (int x = 0; x < per; ++x) {
        const int t = wave + waves * x;
        if (t >= tiles_of(g)) continue;
        float *d = partial + ((int64_t)blockIdx.x * tiles_of(g) + t) * (16 * kWave) + lane;
#pragma unroll
        for (int r = 0; r < 16; ++r) d[r * kWave] = acc[x][r] + low[x][r];
    }
}

// 2^14 2^-e U by slices: X^T packed, and the first A's partial sums
template <int g>
constexpr int kPackWaves = g > 2 ? 8 : 4;

template <typename T, int g>
__global__ __launch_bounds__(kPackWaves<g> *kWave) void small_pack_kernel(update_src u, int tall,
                                                         const double *__restrict__ part, int n_part, float eps, packed_half Xt, int m, int n,
                                                         float *__restrict__ scal, float *__restrict__ partial) {
    constexpr int LD = kSlice + 1, rows = 32 * g, waves = kPackWaves<g>, each = rows / waves;
    __shared__ float tile[rows * LD];
    __shared__ __attribute__((aligned(16))) char X[g * kSliceSteps * 2 * kBlock];
    __shared__ double lds[waves];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int l = lane & 31, h = lane >> 5;
    constexpr int per = (tiles_of(g) + waves - 1) / waves;
    floatx16 acc[per] = {}, low[per] = {};
    int e = 0;
    for (int j0 = blockIdx.x * kSlice; j0 < n; j0 += gridDim.x * kSlice) {
        // along U's rows; element v of a thread is (i, j) of X
        float x[each];
        auto at = [&](int v, int &i, int &j) {
            const int f = threadIdx.x + waves * kWave * v;
            i = tall ? f % rows : f / kSlice;
            j = tall ? f / rows : f % kSlice;
        };
        load_update<T>(u, [&](int v, int &r, int &c) {
            int i, j;
            at(v, i, j);
            r = tall ? j0 + j : i;
            c = tall ? i : j0 + j;
        }, x);
        if (j0 == (int)blockIdx.x * kSlice) e = scale_of<waves>(part, n_part, eps, scal, blockIdx.x == 0, lds);
        __syncthreads();  // the last slice is read
#pragma unroll
        for (int v = 0; v < each; ++v) {
            int i, j;
            at(v, i, j);
            tile[i * LD + j] = ldexpf(x[v], kScaleX - e);
        }
        __syncthreads();
        for (int b = wave; b < 8 * g; b += waves) {  // blocks of X^T, then of X
            const bool t = b < 4 * g;
            const int c = t ? b : b - 4 * g;
            const int gr = t ? c & 1 : c / kSliceSteps, st = t ? c >> 1 : c % kSliceSteps;
            float y[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                const int k = st * kStep + 8 * h + v, r = gr * 32 + l;
                y[v] = t ? tile[k * LD + r] : tile[r * LD + k];
            }
            const parts_of<8> p(y);
            char *d = X + (gr * kSliceSteps + st) * (2 * kBlock) + lane * 16;
            if (t) {
                const int row = j0 / kGroup + gr;
                if (row >= Xt.groups) continue;
                d = Xt.data + ((int64_t)row * Xt.steps + st) * (2 * kBlock) + lane * 16;
            }
            *reinterpret_cast<halfx8 *>(d) = p.hi;
            *reinterpret_cast<halfx8 *>(d + kBlock) = p.lo;
        }
        __syncthreads();
        gram_slice<g, waves, per>(X, wave, lane, acc, low);
    }
    store_gram<g, waves, per>(partial, wave, lane, acc, low);
}

// s[q] = the sum over the ranges of the four floats at p + q * apart, a range every
// `stride` floats, U ranges in flight (past the last the last again, not added)
template <int n, int U>
__device__ __forceinline__ void sum_ranges(const float *p, int apart, int ranges, int64_t stride, float4 (&s)[n]) {
#pragma unroll
    for (int q = 0; q < n; ++q) s[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = 0; r < ranges; r += U) {
        float4 v[U][n];
#pragma unroll
        for (int w = 0; w < U; ++w)
#pragma unroll
            for (int q = 0; q < n; ++q)
                v[w][q] = *reinterpret_cast<const float4 *>(p + min(r + w, ranges - 1) * stride + q * apart);
#pragma unroll
        for (int w = 0; w < U; ++w)
#pragma unroll
            for (int q = 0; q < n; ++q) {
                const bool on = r + w < ranges;
                s[q].x += on ? v[w][q].x : 0.f;
                s[q].y += on ? v[w][q].y : 0.f;
                s[q].z += on ? v[w][q].z : 0.f;
                s[q].w += on ? v[w][q].w : 0.f;
            }
    }
}

// four neighbours (one row i, columns j ..) of a symmetric operand's tile to both their places
__device__ __forceinline__ void place_sums(char *A, int steps, int index, float4 s, float scale) {
    int ti, tj;
    tile_of(index >> 10, ti, tj);
    const int reg = index >> 6 & 15, ln = index & 63;
    const int i = ti * 32 + 8 * (reg >> 2) + 4 * (ln >> 5) + (reg & 3), j = tj * 32 + (ln & 31);
    const float x[4] = {s.x * scale, s.y * scale, s.z * scale, s.w * scale};
    const parts_of<4> p(x);
    if (ti != tj) {
        char *d = A + element_at(i, j, steps);
        *reinterpret_cast<halfx4 *>(d) = p.hi;
        *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        char *d = A + element_at(j + v, i, steps);
        *reinterpret_cast<_Float16 *>(d) = p.hi[v];
        *reinterpret_cast<_Float16 *>(d + kBlock) = p.lo[v];
    }
}

__global__ __launch_bounds__(256) void small_sum_kernel(const float *__restrict__ partial, int ranges, int tiles,
                                                        const float *__restrict__ scal, packed_half A) {
    const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= tiles * 1024) return;
    float4 s[1];
    sum_ranges<1, 16>(partial + i, 0, ranges, (int64_t)tiles * 1024, s);
    place_sums(A.data, A.steps, i, s[0], (scal ? scal[1] : 1.f) * 0x1p-14f);
}

// 10 us a launch at 100 x 300, of which the matrix products are under 2: the launch itself, the sums of A (data
// of the other workgroups, 200 KB each) and five waits bound it.
// One step; A from its ranges' sums, or packed where they were summed ahead (ranges = 0).
// LAST: O, else X^T packed and the next A's partial sums.  2 g waves: a 32 x 32 tile of the slice each.
template <typename T, bool LAST, int g>
__global__ __launch_bounds__(2 * g *kWave) void small_step_kernel(const float *__restrict__ sums, int ranges,
                                                                  packed_half A, packed_half Xt, int m, int n,
                                                                  const float *__restrict__ scal, packed_half out,
                                                                  float *__restrict__ partial, T *__restrict__ O,
                                                                  int64_t ldo, int tall, float scale) {
    constexpr int steps = 2 * g, waves = 2 * g, per = (tiles_of(g) + waves - 1) / waves;
    __shared__ __attribute__((aligned(16))) char LA[g * steps * 2 * kBlock];
    __shared__ __attribute__((aligned(16))) char LY[2 * steps * 2 * kBlock];
    __shared__ __attribute__((aligned(16))) char LX[LAST ? 16 : g * kSliceSteps * 2 * kBlock];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int l = lane & 31, h = lane >> 5;
    const int gi = wave >> 1, wj = wave & 1;
    const float dev = scal ? scal[0] : 1.f, f = dev * scale;
    halfx8 xh[steps], xl[steps];  // the slice's fragments, ahead of what the products wait for
    auto load = [&](int j0) {
        // (a group past the end: the last one's, not stored and zeroed where it would count)
        const char *p = Xt.data + (int64_t)min(j0 / kGroup + wj, Xt.groups - 1) * steps * (2 * kBlock) + lane * 16;
#pragma unroll
        for (int st = 0; st < steps; ++st) {
            xh[st] = *reinterpret_cast<const halfx8 *>(p + st * (2 * kBlock));
            xl[st] = *reinterpret_cast<const halfx8 *>(p + st * (2 * kBlock) + kBlock);
        }
    };
    load(blockIdx.x * kSlice);
    if (ranges > 0) {
        constexpr int items = tiles_of(g) * 256, threads = waves * kWave, each = items / threads;
        static_assert(items % threads == 0, "whole rounds");
        float4 a[each];
        sum_ranges<each, 4>(sums + threadIdx.x * 4, threads * 4, ranges, tiles_of(g) * 1024, a);
#pragma unroll
        for (int q = 0; q < each; ++q)
            place_sums(LA, steps, (threadIdx.x + q * threads) * 4, a[q], dev * dev * 0x1p-14f);
    } else {
        for (int i = threadIdx.x * 16; i < g * steps * 2 * kBlock; i += waves * kWave * 16)
            *reinterpret_cast<float4 *>(LA + i) = *reinterpret_cast<const float4 *>(A.data + i);
    }
    __syncthreads();
    floatx16 acc[per] = {}, low[per] = {};
    for (int j0 = blockIdx.x * kSlice; j0 < n; j0 += gridDim.x * kSlice) {
        const int gj = j0 / kGroup + wj;
        const bool on = gj < Xt.groups;
        const char *xt = Xt.data + (int64_t)min(gj, Xt.groups - 1) * steps * (2 * kBlock);
        floatx16 y = {}, z = {}, s = {};
#pragma unroll
        for (int st = 0; st < steps; ++st) {
            const char *p = LA + (gi * steps + st) * (2 * kBlock) + lane * 16;
            const halfx8 ah = *reinterpret_cast<const halfx8 *>(p), al = *reinterpret_cast<const halfx8 *>(p + kBlock);
            y = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, xh[st], y, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, xh[st], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, xl[st], s, 0, 0, 0);
        }
        const int mine = 2 * gi * (2 * kBlock) + l * 16 + 8 * h;  // this tile in the rows of X^T and Y^T
        halfx4 th[4], tl[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const char *p = xt + mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            th[q] = *reinterpret_cast<const halfx4 *>(p);
            tl[q] = *reinterpret_cast<const halfx4 *>(p + kBlock);
        }
        if (j0 + (int)gridDim.x * kSlice < n) load(j0 + gridDim.x * kSlice);
        y = (y + s) * 0x1p-14f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v[4] = {y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
            const parts_of<4> p(v);
            char *d = LY + wj * steps * (2 * kBlock) + mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            *reinterpret_cast<halfx4 *>(d) = p.hi;
            *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
        }
        __syncthreads();
        s = floatx16{};
#pragma unroll
        for (int st = 0; st < steps; ++st)
            product_step(LA + (gi * steps + st) * (2 * kBlock) + lane * 16,
                         LY + (wj * steps + st) * (2 * kBlock) + lane * 16, z, s);
        z = (z + s) * 0x1p-14f;
        const int j = gj * 32 + l;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int to = mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = (float)th[q][e] + (float)tl[q][e];
                v[e] = on ? f * fmaf(kC, z[4 * q + e], fmaf(kB, y[4 * q + e], kA * x)) : 0.f;
            }
            const int i = gi * 32 + 8 * q + 4 * h;
            if constexpr (LAST) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < m && j < n) O[tall ? j * ldo + i + e : (i + e) * ldo + j] = (T)v[e];
            } else {
                const parts_of<4> p(v);
                if (on) {
                    char *d = out.data + (int64_t)gj * steps * (2 * kBlock) + to;
                    *reinterpret_cast<halfx4 *>(d) = p.hi;
                    *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    char *d = LX + element_at(i + e, wj * 32 + l, kSliceSteps);
                    *reinterpret_cast<_Float16 *>(d) = p.hi[e];
                    *reinterpret_cast<_Float16 *>(d + kBlock) = p.lo[e];
                }
            }
        }
        __syncthreads();  // Y is read (and X' stored)
        if constexpr (!LAST) gram_slice<g, waves, per>(LX, wave, lane, acc, low);
    }
    if constexpr (!LAST) store_gram<g, waves, per>(partial, wave, lane, acc, low);
}

// ---------------------------------------------------------------------------
// matrices that one workgroup's LDS holds: the whole call but for the prox in one launch
// ---------------------------------------------------------------------------
//
// g x c waves, a 32 x 32 block of X each.  LDS: A, X by columns, and in turn A X by columns and X by
// rows (whose reads and writes barriers keep apart).
template <typename T, int g, int c>
__global__ __launch_bounds__(g * c * kWave) void tiny_kernel(update_src u, int tall, int m, int n, int n_steps, float eps,
                                                             T *O, int64_t ldo, float scale) {
    constexpr int waves = g * c, steps = 2 * g, wide = 2 * c;  // steps of the rows, of the columns
    __shared__ __attribute__((aligned(16))) char LA[g * steps * 2 * kBlock];
    __shared__ __attribute__((aligned(16))) char LX[c * steps * 2 * kBlock];
    __shared__ __attribute__((aligned(16))) char LY[c * steps * 2 * kBlock];
    __shared__ double lds[waves];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int l = lane & 31, h = lane >> 5, gi = wave / c, gj = wave - gi * c;
    // U along its rows; element v of a thread is (i, j) of X
    auto at = [&](int v, int &i, int &j) {
        const int f = threadIdx.x + waves * kWave * v;
        i = tall ? f % (32 * g) : f / (32 * c);
        j = tall ? f / (32 * g) : f % (32 * c);
    };
    float dev;
    {
        float x[16];
        const T *G = static_cast<const T *>(u.G);
        float gv[16], mv[16] = {};
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            int i, j;
            at(v, i, j);
            const int r = min(tall ? j : i, u.N - 1), k = min(tall ? i : j, u.K - 1);
            gv[v] = to_f32(G[(int64_t)r * u.ldg + k]);
        }
        if (u.M)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                int i, j;
                at(v, i, j);
                const int r = min(tall ? j : i, u.N - 1), k = min(tall ? i : j, u.K - 1);
                mv[v] = u.M[(int64_t)r * u.ldm + k];
            }
        double sum = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            int i, j;
            at(v, i, j);
            const bool on = i < m && j < n;
            const float m_new = fmaf(u.mu, mv[v], gv[v]);
            if (on && u.M_out) u.M_out[(int64_t)(tall ? j : i) * u.ldo + (tall ? i : j)] = m_new;
            x[v] = on ? update_at(u, gv[v], m_new) : 0.f;
            sum = fma((double)x[v], (double)x[v], sum);
        }
        const norm_scale ns(sqrt(block_sum<waves>(sum, lds)), eps);
        dev = ns.s;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            int i, j;
            at(v, i, j);
            const float y = ldexpf(x[v], kScaleX - ns.e);
            const _Float16 hi = (_Float16)y, lo = (_Float16)(y - (float)hi);
            char *a = LX + element_at(j, i, steps), *b = LY + element_at(i, j, wide);
            *reinterpret_cast<_Float16 *>(a) = hi;
            *reinterpret_cast<_Float16 *>(a + kBlock) = lo;
            *reinterpret_cast<_Float16 *>(b) = hi;
            *reinterpret_cast<_Float16 *>(b + kBlock) = lo;
        }
    }
    const int mine = (gj * steps + 2 * gi) * (2 * kBlock) + l * 16 + 8 * h;  // this block in the columns of X and A X
    for (int k = 0; k < n_steps; ++k) {
        __syncthreads();
        for (int t = wave; t < tiles_of(g); t += waves) {  // A
            int ti, tj;
            tile_of(t, ti, tj);
            floatx16 acc = {}, low = {};
#pragma unroll 4
            for (int st = 0; st < wide; ++st)
                product_step(LY + (ti * wide + st) * (2 * kBlock) + lane * 16, LY + (tj * wide + st) * (2 * kBlock) + lane * 16,
                             acc, low);
            acc = (acc + low) * (dev * dev * 0x1p-14f);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
                const parts_of<4> p(v);
                char *d = LA + (tj * steps + 2 * ti + (q >> 1)) * (2 * kBlock) + (q & 1) * 512 + l * 16 + 8 * h;
                *reinterpret_cast<halfx4 *>(d) = p.hi;
                *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
                if (ti == tj) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d = LA + element_at(ti * 32 + 8 * q + 4 * h + e, tj * 32 + l, steps);
                    *reinterpret_cast<_Float16 *>(d) = p.hi[e];
                    *reinterpret_cast<_Float16 *>(d + kBlock) = p.lo[e];
                }
            }
        }
        __syncthreads();
        floatx16 y = {}, z = {}, s = {};
#pragma unroll
        for (int st = 0; st < steps; ++st)
            product_step(LA + (gi * steps + st) * (2 * kBlock) + lane * 16, LX + (gj * steps + st) * (2 * kBlock) + lane * 16, y, s);
        y = (y + s) * 0x1p-14f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // (X by rows is read: a barrier ago)
            const float v[4] = {y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
            const parts_of<4> p(v);
            char *d = LY + mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            *reinterpret_cast<halfx4 *>(d) = p.hi;
            *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
        }
        __syncthreads();
        s = floatx16{};
#pragma unroll
        for (int st = 0; st < steps; ++st)
            product_step(LA + (gi * steps + st) * (2 * kBlock) + lane * 16, LY + (gj * steps + st) * (2 * kBlock) + lane * 16, z, s);
        z = (z + s) * 0x1p-14f;
        const bool last = k + 1 == n_steps;
        const float f = last ? dev * scale : dev;
        float v[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const char *p = LX + mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            const halfx4 hi = *reinterpret_cast<const halfx4 *>(p), lo = *reinterpret_cast<const halfx4 *>(p + kBlock);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[4 * q + e] = f * fmaf(kC, z[4 * q + e], fmaf(kB, y[4 * q + e], kA * ((float)hi[e] + (float)lo[e])));
        }
        const int j = gj * 32 + l;
        if (last) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = gi * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                if (i < m && j < n) O[tall ? j * ldo + i : i * ldo + j] = (T)v[r];
            }
            return;
        }
        dev = 1.f;
        __syncthreads();  // A X is read, and X by columns
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float w[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            const parts_of<4> p(w);
            char *d = LX + mine + (q >> 1) * (2 * kBlock) + (q & 1) * 512;
            *reinterpret_cast<halfx4 *>(d) = p.hi;
            *reinterpret_cast<halfx4 *>(d + kBlock) = p.lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                d = LY + element_at(gi * 32 + 8 * q + 4 * h + e, j, wide);
                *reinterpret_cast<_Float16 *>(d) = p.hi[e];
                *reinterpret_cast<_Float16 *>(d + kBlock) = p.lo[e];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// the products
// ---------------------------------------------------------------------------

// A workgroup's tile: WM x WN waves of TM x TN matrix instructions, WK waves
// sharing the reduction, KS steps between two barriers.
template <int TM_, int TN_, int WM_, int WN_, int WK_, int KS_>
struct tile_shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WK = WK_, KS = KS_;
    static constexpr int GA = TM * WM, GB = TN * WN;
    static constexpr int waves = WM * WN * WK, threads = waves * kWave;
};

struct product_args {
    packed_half A, B;           // D[i][j] = sum_k A[i][k] B[j][k]
    int rows, cols;             // of D
    int tiles_m, tiles_n;
    int symmetric;              // D = D^T: only tiles with a 32 x 32 block on or above the diagonal
    // v = dev (al D + be E) + ga [i == j]
    float al, be, ga;
    const float *dev;           // nullable: 1
    packed_half E;              // E[j][i] packed by rows j (data null: none)
    packed_half out_n, out_t;   // v packed with rows j, and with rows i (data null: not stored)
    void *O;                    // or v as a matrix: O[i][j], flipped: O[j][i]
    int64_t ldo;
    int flip;
    // The first `whole` of `tiles` tiles take a workgroup each, the others `ranges`:
    // partial sums [range][tile - whole][lane order], joined by a second launch.
    int tiles, whole, ranges, range_stages;
    float *partial;
};

// Tiles of a symmetric product: tile column tn has those tm with a 32 x 32 block on or above the diagonal.
template <typename S>
__host__ __device__ __forceinline__ int column_tiles(int tn, int tiles_m) {
    const int c = (tn * S::GB + S::GB - 1) / S::GA + 1;
    return c < tiles_m ? c : tiles_m;
}
template <typename S>
__host__ __device__ __forceinline__ int band_tiles(int first, int tiles_m, int tiles_n) {
    int c = 0;
    for (int tn = first; tn < first + 8 && tn < tiles_n; ++tn) c += column_tiles<S>(tn, tiles_m);
    return c;
}
// Tile number t to its place: bands of 8 tile columns (other products: rows) walked across the band.
template <typename S>
__host__ __device__ __forceinline__ void place_of(int t, int symmetric, int tiles_m, int tiles_n, int &tm, int &tn) {
    if (!symmetric) {
        const int band = t / (8 * tiles_n), r = t - band * 8 * tiles_n;
        const int h = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
        tn = r / h;
        tm = band * 8 + (r - tn * h);
        return;
    }
    int first = 0, r = t;
    for (int c = band_tiles<S>(0, tiles_m, tiles_n); r >= c; c = band_tiles<S>(first, tiles_m, tiles_n)) {
        r -= c;
        first += 8;
    }
    const int h = tiles_n - first < 8 ? tiles_n - first : 8, all = column_tiles<S>(first, tiles_m);
    if (r < all * h) {
        tm = r / h;
        tn = first + r - tm * h;
        return;
    }
    r -= all * h;
    for (tm = all;; ++tm) {  // the rows that only the band's later columns have
        int f = first;
        while (column_tiles<S>(f, tiles_m) <= tm) ++f;
        const int k = first + h - f;
        if (r < k) {
            tn = f + r;
            return;
        }
        r -= k;
    }
}

constexpr int kTurned = 32 * 33;  // floats of a turned block

// The epilogue of a 32 x 32 block.  Lane l, register 4 q + e holds row 8 q + 4 (l / 32) + e,
// column l % 32: four consecutive indices of a packed row j (8 bytes a part), so
// the matrix packed by rows j is stored from the registers, the one by rows i through LDS.
struct operand_e {  // E of a block, as stored
    halfx4 hi[4], lo[4];
    __device__ __forceinline__ operand_e(const product_args &P, int gi, int gj, int lane) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            hi[q] = lo[q] = halfx4{};
            if (P.E.data == nullptr) continue;
            const char *p = P.E.data + ((int64_t)gj * P.E.steps + 2 * gi + (q >> 1)) * (P.E.parts * kBlock) +
                            ((lane & 31) + 32 * (q & 1)) * 16 + 8 * (lane >> 5);
            hi[q] = *reinterpret_cast<const halfx4 *>(p);
            if (P.E.parts == 2) lo[q] = *reinterpret_cast<const halfx4 *>(p + kBlock);
        }
    }
};

template <typename O>
__device__ __forceinline__ void finish_block(const product_args &P, int gi, int gj, int lane, const floatx16 &acc,
                                             const operand_e &E, float *buf) {
    const float dev = P.dev ? *P.dev : 1.f;
    const int l = lane & 31, h = lane >> 5;
    const int i0 = gi * kGroup, j = gj * kGroup + l;
    float v[16];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + 8 * q + 4 * h + e;
            float x = dev * fmaf(P.al, acc[4 * q + e], P.be * ((float)E.hi[q][e] + (float)E.lo[q][e]));
            if (i == j && i < P.rows) x += P.ga;
            v[4 * q + e] = x;
        }
    }
    if (P.O) {
        O *out = static_cast<O *>(P.O);
        if (j < P.cols)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = i0 + 8 * (r >> 2) + 4 * h + (r & 3);
                if (i < P.rows) out[P.flip ? j * P.ldo + i : i * P.ldo + j] = (O)v[r];
            }
        return;
    }
    {
        const packed_half &o = P.out_n;
        char *d = o.data + ((int64_t)gj * o.steps + 2 * gi) * (o.parts * kBlock) + l * 16 + 8 * h;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float x[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            const parts_of<4> p(x);
            char *to = d + (q >> 1) * (o.parts * kBlock) + (q & 1) * 512;
            *reinterpret_cast<halfx4 *>(to) = p.hi;
            if (o.parts == 2) *reinterpret_cast<halfx4 *>(to + kBlock) = p.lo;
        }
    }
    if (P.out_t.data == nullptr || (P.symmetric && gi == gj)) return;
    const packed_half &o = P.out_t;
#pragma unroll
    for (int r = 0; r < 16; ++r) buf[(8 * (r >> 2) + 4 * h + (r & 3)) * 33 + l] = v[r];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    char *d = o.data + ((int64_t)gi * o.steps + 2 * gj) * (o.parts * kBlock) + lane * 16;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = buf[l * 33 + 16 * s + 8 * h + e];
        const parts_of<8> p(x);
        *reinterpret_cast<halfx8 *>(d + s * (o.parts * kBlock)) = p.hi;
        if (o.parts == 2) *reinterpret_cast<halfx8 *>(d + s * (o.parts * kBlock) + kBlock) = p.lo;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// (not past the operands, nor below a symmetric result's diagonal)
template <typename O>
__device__ __forceinline__ void finish_block(const product_args &P, int gi, int gj, int lane, const floatx16 &acc,
                                             float *buf) {
    if (gi >= P.A.groups || gj >= P.B.groups || (P.symmetric && gi > gj)) return;
    finish_block<O>(P, gi, gj, lane, acc, operand_e(P, gi, gj, lane), buf);
}

// One tile, or one range of its reduction.  Stages of packed blocks are copied straight into LDS, up to
// three ahead of the one in use; fragments are read in the lane's order, the next step's while this one's
// are multiplied (five steps of 4096 x 4096, read behind the barrier and ahead: two parts 3875 and 3690 us, one
// part 1632 and 1553).  With two parts a wave reads 8 fragments for 12 matrix instructions and the pipe is
// 74-77 % busy at the 1.6 GHz that the power limit leaves (4096 x 4096 x 4096: 348 us, 1.18 PFLOP/s of
// fp16); with one part 6 for 8, 56-59 % busy at 1.9 GHz, 139 us (0.99 PFLOP/s), where all workgroups
// start and end together and the result's 10 bytes an element are waited for.
template <int NP, typename S, typename O>
__global__ __launch_bounds__(S::threads, 2) void product_kernel(product_args P) {
    constexpr int PIECES = (S::GA + S::GB) * NP * S::KS;  // 1 KB blocks of a stage
    constexpr int LPW = PIECES / S::waves;
    static_assert(PIECES % S::waves == 0, "every wave issues the same number of loads");
    constexpr int SB = PIECES * kBlock;
    constexpr int TM = S::TM, TN = S::TN, GA = S::GA, GB = S::GB, KS = S::KS;
    __shared__ __attribute__((aligned(16))) char S0[SB];
    __shared__ __attribute__((aligned(16))) char S1[SB];
    __shared__ __attribute__((aligned(16))) char S2[SB];
    // Each XCD (blocks are dealt round-robin) takes one contiguous range of the whole tiles, whose
    // operand rows its L2 then holds.
    const int per = (P.whole + 7) / 8;
    int t, range = -1;
    if ((int)blockIdx.x < 8 * per) {
        t = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
        if (t >= P.whole) return;
    } else {
        const int r = (int)blockIdx.x - 8 * per;
        t = P.whole + r / P.ranges;
        range = r % P.ranges;
    }
    int tm, tn;
    place_of<S>(t, P.symmetric, P.tiles_m, P.tiles_n, tm, tn);
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wk = wave / (S::WM * S::WN), wp = wave % (S::WM * S::WN);
    const int wgm = wp / S::WN * TM, wgn = wp % S::WN * TN;  // the wave's first groups in the tile
    constexpr bool TWO = NP == 2;
    floatx16 acc[TM][TN], small[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) acc[a][b] = small[a][b] = floatx16{};

    {
        const int steps = P.A.steps;
        const int st0 = range < 0 ? 0 : range * P.range_stages;
        const int all = (steps + KS - 1) / KS;
        const int stages = range < 0 ? all : min(P.range_stages, all - st0);
        // this wave's blocks of a stage: piece p = wave + j * waves, a group's blocks side by side
        const char *src[LPW];
        int at[LPW];     // the piece's step in the stage
        int stride[LPW]; // bytes of a step
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
            const int p = wave + j * S::waves;
            const int g = p / (NP * KS), q = p - g * (NP * KS);
            const packed_half &o = g < GA ? P.A : P.B;
            const int row = g < GA ? min(tm * GA + g, P.A.groups - 1) : min(tn * GB + g - GA, P.B.groups - 1);
            at[j] = q / NP;
            stride[j] = o.parts * kBlock;
            src[j] = o.data + (int64_t)row * steps * stride[j] + (q % NP) * kBlock;
        }
        const unsigned l0 = lds_address(S0) + wave * kBlock, l1 = lds_address(S1) + wave * kBlock,
                       l2 = lds_address(S2) + wave * kBlock;
        auto load = [&](unsigned dst, int c) {
#pragma unroll
            for (int j = 0; j < LPW; ++j) {
                // (steps past the end: the last one's blocks again, not used)
                const int st = min((st0 + c) * KS + at[j], steps - 1);
                dma16(src[j], (unsigned)st * stride[j] + lane * 16, dst + j * S::waves * kBlock);
            }
        };
        // fragments of a stage's step kk of this wave, and their products
        struct fragments {
            halfx8 a[NP][TM], b[NP][TN];
        } frag[2];
        auto read = [&](const char *cur, int kk, fragments &f) {
            const int o = (kk * S::WK + wk) * NP * kBlock + lane * 16;
#pragma unroll
            for (int q = 0; q < NP; ++q) {
#pragma unroll
                for (int a = 0; a < TM; ++a)
                    f.a[q][a] = *reinterpret_cast<const halfx8 *>(cur + (wgm + a) * (NP * KS * kBlock) + o + q * kBlock);
#pragma unroll
                for (int b = 0; b < TN; ++b)
                    f.b[q][b] = *reinterpret_cast<const halfx8 *>(cur + (GA + wgn + b) * (NP * KS * kBlock) + o + q * kBlock);
            }
        };
        auto multiply = [&](const fragments &f) {
            auto term = [&](floatx16(&d)[TM][TN], int qa, int qb) {
#pragma unroll
                for (int a = 0; a < TM; ++a)
#pragma unroll
                    for (int b = 0; b < TN; ++b)
                        d[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.a[qa][a], f.b[qb][b], d[a][b], 0, 0, 0);
            };
            term(acc, 0, 0);
            if constexpr (TWO) {
                term(small, 1, 0);
                term(small, 0, 1);
            }
        };
        auto together = [&] {  // (wait_vm waits for the reads from LDS too)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        constexpr int H = KS / S::WK;  // steps of a stage that a wave takes
        // Stage c, its first fragments in frag[first]: the next ones are read while these are multiplied.  Before
        // those of stage c + 1: its blocks have landed everywhere (the loads of stage c + 2 may still be
        // out), and every wave has its last fragments of stage c, whose buffer then takes stage c + 3.
        // `inner`: stage c + 3 is known to exist (a loop without conditions, whose waits the compiler can count).
        auto stage = [&](auto inner, int c, const char *cur, const char *next, unsigned here, int first) {
#pragma unroll
            for (int kk = 0; kk < H; ++kk) {
                const fragments &now = frag[(first + kk) & 1];
                fragments &then = frag[(first + kk + 1) & 1];
                if (kk + 1 < H) {
                    read(cur, kk + 1, then);
                } else if constexpr (inner.value) {
                    asm volatile("" ::: "memory");  // no read moves behind the wait
                    wait_vm<LPW>();
                    together();
                    load(here, c + 3);
                    read(next, 0, then);
                } else {
                    asm volatile("" ::: "memory");
                    if (c + 2 < stages)
                        wait_vm<LPW>();
                    else
                        wait_vm<0>();
                    if (c + 1 < stages) {
                        together();
                        if (c + 3 < stages) load(here, c + 3);
                        read(next, 0, then);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);  // (or the reads sink to where their values are used)
                // (steps are even in number: only the last of more than two a stage can end inside one)
                if (inner.value || KS <= 2 || (st0 + c) * KS + kk * S::WK + wk < steps) multiply(now);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        load(l0, 0);
        if (stages > 1) load(l1, 1);
        if (stages > 2) load(l2, 2);
        if (stages > 2)
            wait_vm<2 * LPW>();
        else if (stages > 1)
            wait_vm<LPW>();
        else
            wait_vm<0>();
        together();
        read(S0, 0, frag[0]);
        constexpr int odd = H & 1;  // the set that the next stage begins with is the other one
        int c = 0;
        for (const std::true_type inner; c + 8 < stages; c += 6) {
            stage(inner, c, S0, S1, l0, 0);
            stage(inner, c + 1, S1, S2, l1, odd);
            stage(inner, c + 2, S2, S0, l2, 0);
            stage(inner, c + 3, S0, S1, l0, odd);
            stage(inner, c + 4, S1, S2, l1, 0);
            stage(inner, c + 5, S2, S0, l2, odd);
        }
        for (const std::false_type inner; c < stages; c += 6) {
            stage(inner, c, S0, S1, l0, 0);
            if (c + 1 < stages) stage(inner, c + 1, S1, S2, l1, odd);
            if (c + 2 < stages) stage(inner, c + 2, S2, S0, l2, 0);
            if (c + 3 < stages) stage(inner, c + 3, S0, S1, l0, odd);
            if (c + 4 < stages) stage(inner, c + 4, S1, S2, l1, 0);
            if (c + 5 < stages) stage(inner, c + 5, S2, S0, l2, odd);
        }
        if constexpr (TWO)
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b) acc[a][b] += small[a][b];
        if constexpr (S::WK > 1) {  // the waves that share a position, in their order
            constexpr int n = TM * TN * 16 * kWave;  // floats of a wave
            static_assert((S::WK - 1) * S::WM * S::WN * n * 4 <= SB, "the sums fit a stage");
            __syncthreads();
            float *buf = reinterpret_cast<float *>(S0);
            if (wk > 0)
#pragma unroll
                for (int a = 0; a < TM; ++a)
#pragma unroll
                    for (int b = 0; b < TN; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            buf[((wk - 1) * S::WM * S::WN + wp) * n + ((a * TN + b) * 16 + r) * kWave + lane] = acc[a][b][r];
            __syncthreads();
            if (wk > 0) return;
            for (int w = 0; w < S::WK - 1; ++w)
#pragma unroll
                for (int a = 0; a < TM; ++a)
#pragma unroll
                    for (int b = 0; b < TN; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            acc[a][b][r] += buf[(w * S::WM * S::WN + wp) * n + ((a * TN + b) * 16 + r) * kWave + lane];
        }
    }
    if (range >= 0) {
        float *d = P.partial + ((int64_t)range * (P.tiles - P.whole) + t - P.whole) * (GA * GB * 16 * kWave) +
                   wp * (TM * TN * 16 * kWave) + lane;
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) d[((a * TN + b) * 16 + r) * kWave] = acc[a][b][r];
        return;
    }

    float *buf = nullptr;
    if (P.out_t.data != nullptr) {
        // two positions in each of two buffers that every wave has read its last
        // fragments from (behind the barrier in front of the shared sums, if there are any)
        if constexpr (S::WK == 1) __syncthreads();
        constexpr int each = S::WM * S::WN / 2;
        static_assert(each * kTurned * 4 <= SB, "room for the turned blocks");
        const int second = wp / each;
        buf = reinterpret_cast<float *>(S::WK > 1 ? (second ? S2 : S1) : (second ? S1 : S0)) + (wp - second * each) * kTurned;
    }
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) finish_block<O>(P, tm * GA + wgm + a, tn * GB + wgn + b, lane, acc[a][b], buf);
}

// A product of few blocks: a workgroup a 32 x 32 block, its 16 waves sharing the reduction, fragments straight from
// memory (a step of them is a wave's 1 KB a part), U steps in flight.  Bound by latency: the launch, the operands
// (which other XCDs' workgroups stored), the sums of the waves and the epilogue, 5-6 us at 300 x 784.
constexpr int kBlockWaves = 16, kMostBlocks = 512, kMostBlockSteps = 256;

template <int NP, typename O>
__global__ __launch_bounds__(kBlockWaves *kWave) void block_kernel(product_args P) {
    constexpr int waves = kBlockWaves, U = 4;
    __shared__ float sums[waves][16 * kWave];
    __shared__ float turned[kTurned];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, steps = P.A.steps;
    int gi, gj;
    if (P.symmetric) {  // blocks gi <= gj by columns
        gj = (int)((sqrtf(8.f * blockIdx.x + 1.f) - 1.f) * 0.5f);
        while (gj * (gj + 1) / 2 > (int)blockIdx.x) --gj;
        while ((gj + 1) * (gj + 2) / 2 <= (int)blockIdx.x) ++gj;
        gi = blockIdx.x - gj * (gj + 1) / 2;
    } else {
        gj = blockIdx.x / P.A.groups;
        gi = blockIdx.x - gj * P.A.groups;
    }
    gi = uniform(gi);
    gj = uniform(gj);
    const char *pa = P.A.data + (int64_t)gi * steps * (P.A.parts * kBlock) + lane * 16;
    const char *pb = P.B.data + (int64_t)gj * steps * (P.B.parts * kBlock) + lane * 16;
    floatx16 acc = {}, small = {};
    for (int s0 = wave; s0 < steps; s0 += waves * U) {
        halfx8 a[U][NP], b[U][NP];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int st = min(s0 + u * waves, steps - 1);  // (past the end the last again, not used)
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                a[u][q] = *reinterpret_cast<const halfx8 *>(pa + (int64_t)st * (P.A.parts * kBlock) + q * kBlock);
                b[u][q] = *reinterpret_cast<const halfx8 *>(pb + (int64_t)st * (P.B.parts * kBlock) + q * kBlock);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * waves >= steps) break;
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][0], b[u][0], acc, 0, 0, 0);
            if constexpr (NP == 2) {
                small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][1], b[u][0], small, 0, 0, 0);
                small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][0], b[u][1], small, 0, 0, 0);
            }
        }
    }
    if constexpr (NP == 2) acc += small;
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[wave][r * kWave + lane] = acc[r];
    const operand_e E(P, gi, gj, lane);  // (for the first wave: ahead of the wait)
    __syncthreads();
    static_assert(waves == 16, "a wave a register");
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < waves; ++w) t += sums[w][wave * kWave + lane];
    sums[0][wave * kWave + lane] = t;  // (read by this wave alone)
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = sums[0][r * kWave + lane];
    finish_block<O>(P, gi, gj, lane, acc, E, turned);
}

// The blocks of the tiles that were cut: a wave adds the ranges of a 32 x 32 block and finishes it.
template <typename S, typename O>
__global__ __launch_bounds__(256) void join_kernel(product_args P) {
    constexpr int blocks = S::GA * S::GB;
    __shared__ float turned[4][kTurned];
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int id = blockIdx.x * 4 + wave;
    static_assert(blocks % 4 == 0, "whole workgroups");
    const int t = P.whole + id / blocks, n = id % blocks;
    int tm, tn;
    place_of<S>(t, P.symmetric, P.tiles_m, P.tiles_n, tm, tn);
    // block n of a tile in the order of the partial sums: position, then (a, b)
    constexpr int each = S::TM * S::TN;
    const int wp = n / each, ab = n % each;
    const int gi = tm * S::GA + wp / S::WN * S::TM + ab / S::TN, gj = tn * S::GB + wp % S::WN * S::TN + ab % S::TN;
    const float *p = P.partial + ((int64_t)(t - P.whole) * blocks + n) * (16 * kWave) + lane;
    const int64_t stride = (int64_t)(P.tiles - P.whole) * blocks * (16 * kWave);
    floatx16 sum = {};
    for (int w = 0; w < P.ranges; w += 2) {
        floatx16 x, y;
        const int64_t second = w + 1 < P.ranges ? stride : 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = p[r * kWave];
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = p[second + r * kWave];
        sum += x;
        if (second) sum += y;
        p += 2 * stride;
    }
    finish_block<O>(P, gi, gj, lane, sum, turned[wave]);
}

// Large products: 128 x 128 tiles.  Products of fewer tiles: 128 x 64, or 64 x 64 with two waves a
// position and four steps between two barriers.  One part, where they fill the CUs: 256 x 256, of eight waves.
template <int NP>
using large_tile = tile_shape<2, 2, 2, 2, 1, NP == 2 ? 1 : 2>;
using medium_tile = tile_shape<2, 1, 2, 2, 1, 2>;
using huge_tile = tile_shape<2, 4, 4, 2, 1, 2>;
using small_tile = tile_shape<1, 1, 2, 2, 2, 4>;

template <typename S>
void count_tiles(product_args &P) {
    P.tiles_m = (int)ceil_div(P.A.groups, S::GA);
    P.tiles_n = (int)ceil_div(P.B.groups, S::GB);
    P.tiles = P.tiles_m * P.tiles_n;
    if (!P.symmetric) return;
    P.tiles = 0;
    for (int first = 0; first < P.tiles_n; first += 8) P.tiles += band_tiles<S>(first, P.tiles_m, P.tiles_n);
}

constexpr int kCus = 256;
// (also twice the partial sums of a small matrix's A)
constexpr size_t kPartialBytes = (size_t)16 << 20;
static_assert(kPartialBytes >= (size_t)kCus * 128 * 128 * sizeof(float) &&
                  kPartialBytes / 2 >= (size_t)kMostRanges * tiles_of(4) * 1024 * sizeof(float), "partial sums");

// The tiles past the last whole round of the CUs are cut into up to `most` ranges that fill
// one, where that saves `least` stages of a tile: the join costs a launch of 5 us.
template <int NP, typename S, typename O>
hipError_t launch_tiles(product_args P, int most, int least, hipStream_t s) {
    count_tiles<S>(P);
    const int stages = (int)ceil_div(P.A.steps, S::KS), rest = P.tiles % kCus;
    const int ranges = rest > 0 ? std::min(std::min(kCus / rest, most), stages / 4) : 1;
    P.whole = P.tiles;
    if (ranges > 1 && stages - stages / ranges >= least) {
        P.whole = P.tiles - rest;
        P.range_stages = (int)ceil_div(stages, ranges);
        P.ranges = (int)ceil_div(stages, P.range_stages);
    }
    const int cut = (P.tiles - P.whole) * P.ranges;
    const unsigned grid = (unsigned)(ceil_div(P.whole, 8) * 8 + cut);
    product_kernel<NP, S, O><<<grid, S::threads, 0, s>>>(P);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || cut == 0) return e;
    join_kernel<S, O><<<(unsigned)((P.tiles - P.whole) * S::GA * S::GB / 4), 256, 0, s>>>(P);
    return hipGetLastError();
}

// Few blocks take a workgroup each: us for five steps with small tiles and with blocks, two parts 300 x 784 125 and 102,
// 512 x 512 137 and 109, 700 x 700 (484 blocks and 253) 155 and 126; up to 800 blocks 850 x 850 162 -> 188; one part
// 300 x 784 102 and 83, 700 x 700 119 and 107.  A long reduction wants more workgroups, ranges of small tiles:
// 200 x 9216 (28 blocks of 576 steps) 137 and 160, but one part 300 x 4096 (256 steps) 136 and 126.
// The others by the number of large tiles.  us for five steps, every product with small, medium and large tiles, two parts:
// 700 x 700 159, 217, 324; 1001 x 1777 242, 328, 353; 1500 x 1500 485, 438, 457; 2048 x 2048 895, 725, 754; 2500 x 2500 1472,
// 1177, 1124 (and 1150 as chosen: the symmetric ones, 210 large tiles, medium); 3500 x 3500 3410, 2765, 2586.  One
// part: 1001 x 1777 172, 225, 260; 1500 x 1500 247, 256, 305 (as chosen 238); 2048 x 2048 461, 369, 405 (as chosen 380);
// 4096 x 4096 2240, 1840, 1600, with huge tiles for the product with X 1556; 4096 x 16384 large 5255, huge 4900, 8192 x
// 8192 11900, 10890; not where they leave a tenth of the CUs idle (576 tiles: 4096 x 9216, where both take 3160).  With
// two parts, or four waves of 128 x 128, they were slower.  Cut tiles: 4096 x 4096 4070 -> 3645 (528 symmetric
// tiles: 16 past the second round), 3500 x 3500 2720 -> 2580, 2048 x 2048 (272 medium) 742 -> 718; one part's medium tiles
// only where more is saved (2048 x 2048 366 -> 412).
template <int NP, typename O>
hipError_t launch_product(product_args P, hipStream_t s) {
    if constexpr (NP == 1) {
        count_tiles<huge_tile>(P);
        if (!P.symmetric && P.tiles * 10 >= ceil_div(P.tiles, kCus) * kCus * 9) return launch_tiles<NP, huge_tile, O>(P, 1, 0, s);
    }
    const int64_t blocks = P.symmetric ? (int64_t)P.A.groups * (P.A.groups + 1) / 2 : (int64_t)P.A.groups * P.B.groups;
    if (blocks <= kMostBlocks && P.A.steps <= kMostBlockSteps) {
        block_kernel<NP, O><<<(unsigned)blocks, kBlockWaves * kWave, 0, s>>>(P);
        return hipGetLastError();
    }
    count_tiles<large_tile<NP>>(P);
    if (P.tiles >= kCus) return launch_tiles<NP, large_tile<NP>, O>(P, 4, 40, s);
    if (P.tiles >= kCus / (NP == 2 ? 4 : 2)) return launch_tiles<NP, medium_tile, O>(P, 4, NP == 2 ? 40 : 100, s);
    return launch_tiles<NP, small_tile, O>(P, 32, 24, s);
}

struct muon_ws {
    double *norm;
    float *scal;
    packed_half X, Xt[2], A, T, P, Q[2];
    float *partial;
    size_t bytes;
};

// parts of X and the m x m operands; X^T always has two (the residual of one part)
muon_ws carve(int N, int K, int np, void *ws) {
    const int m = N < K ? N : K, n = N < K ? K : N;
    if (m <= kSmall) np = 2;
    muon_ws w{};
    char *p = static_cast<char *>(ws);
    auto take = [&](size_t b) {
        char *q = p;
        p += (b + 255) / 256 * 256;
        return q;
    };
    auto operand = [&](int rows, int k, int parts) {
        return packed_half{take(packed_half_bytes(rows, k, parts)), (int)ceil_div(rows, kGroup), even_steps(k), parts};
    };
    w.norm = reinterpret_cast<double *>(take(sizeof(double) * kNormBlocks));
    w.scal = reinterpret_cast<float *>(take(2 * sizeof(float)));
    w.X = operand(m, n, np);
    w.Xt[0] = operand(n, m, 2);
    w.Xt[1] = operand(n, m, 2);
    w.A = operand(m, m, np);
    w.P = operand(m, m, np);
    if (np == 2) {
        w.T = operand(m, m, np);
        w.Q[0] = operand(m, m, np);
        w.Q[1] = operand(m, m, np);
    }
    w.partial = reinterpret_cast<float *>(take(kPartialBytes));
    w.bytes = (size_t)(p - static_cast<char *>(ws));
    return w;
}

float exp2i(int e) { return std::ldexp(1.f, e); }

int norm_blocks(const muon_args &a) {
    const int64_t chunks = (int64_t)a.N * ceil_div(a.K, 4);
    return (int)(chunks < kNormBlocks * 256 ? ceil_div(chunks, 256) : kNormBlocks);
}

// Steps between two products with X: the m x m products that stand for them pay where X is
// wider than square and they are not bound by their launches.  us, one step and three, two parts:
// 512 x 512 110 and 117, 300 x 784 101 and 108, 500 x 1500 131 and 129, 300 x 1200 118 and 111, 150 x 1000 93 and 95,
// 200 x 2000 128 and 112, 400 x 2000 152 and 129, 512 x 4096 196 and 157, 200 x 9216 188 and 137; 600 x 2000 161 and 148,
// 1001 x 1777 237 and 233, 2048 x 2048 699 and 779, 2048 x 4096 1053 and 929, 4096 x 9216 6877 and 5095.
int most_steps(int m, int n) {
    return 2 * (int64_t)n >= 3 * (int64_t)m && (m > 512 || n >= 3 * (int64_t)m) ? kMaxGroup : 1;
}

template <typename T, int g>
hipError_t run_small(const muon_args &a, const update_src &u, void *ws, hipStream_t s) {
    const bool tall = a.N > a.K;
    const int m = tall ? a.K : a.N, n = tall ? a.N : a.K;
    muon_ws w = carve(a.N, a.K, 2, ws);
    const int nb = norm_blocks(a), slices = (int)ceil_div(n, kSlice);
    const int ranges = slices < kMostRanges ? slices : kMostRanges;
    momentum_kernel<T><<<nb, 256, 0, s>>>(u, w.norm);
    small_pack_kernel<T, g><<<ranges, kPackWaves<g> * kWave, 0, s>>>(u, tall, w.norm, nb, a.eps, w.Xt[0], m, n, w.scal, w.partial);
    hipError_t e = hipGetLastError();
    for (int k = 0; k < a.steps && e == hipSuccess; ++k) {
        const float *scal = k == 0 ? w.scal : nullptr;
        // (a launch reads the sums of one half and writes those of the other)
        float *sums = w.partial + (k & 1) * (kPartialBytes / 8), *next = w.partial + (~k & 1) * (kPartialBytes / 8);
        if (ranges > kSumRanges)
            small_sum_kernel<<<tiles_of(g), 256, 0, s>>>(sums, ranges, tiles_of(g), scal, w.A);
        const int given = ranges > kSumRanges ? 0 : ranges;
        if (k + 1 < a.steps)
            small_step_kernel<float, false, g><<<ranges, 2 * g * kWave, 0, s>>>(
                sums, given, w.A, w.Xt[k & 1], m, n, scal, w.Xt[~k & 1], next, nullptr, 0, 0, 1.f);
        else
            small_step_kernel<T, true, g><<<slices, 2 * g * kWave, 0, s>>>(
                sums, given, w.A, w.Xt[k & 1], m, n, scal, packed_half{}, nullptr, static_cast<T *>(a.O), a.ldo, tall,
                a.scale * exp2i(-kScaleX));
        e = hipGetLastError();
    }
    return e;
}

template <typename T, int g, int c>
hipError_t run_tiny(const muon_args &a, const update_src &u, hipStream_t s) {
    tiny_kernel<T, g, c><<<1, g * c * kWave, 0, s>>>(u, a.N > a.K, std::min(a.N, a.K), std::max(a.N, a.K), a.steps, a.eps,
                                                     static_cast<T *>(a.O), a.ldo, a.scale * exp2i(-kScaleX));
    return hipGetLastError();
}

template <typename T>
hipError_t run_small(const muon_args &a, const update_src &u, void *ws, hipStream_t s) {
    const int m = std::min(a.N, a.K), n = std::max(a.N, a.K);
    // In one launch where a workgroup's waves need no more than that time of a chain of launches
    // (us, launches and one): 32 x 128 29.9 and 17.7, 32 x 256 31.0 and 24.3, 64 x 128 36.8 and 24.6, 96 x 128 45.5 and
    // 36.4; not 32 x 512 34.6 and 44.0, 64 x 256 37.7 and 41.3 (16 waves).
    if (m <= 32 && n <= 128) return run_tiny<T, 1, 4>(a, u, s);
    if (m <= 32 && n <= 256) return run_tiny<T, 1, 8>(a, u, s);
    if (m <= 64 && n <= 128) return run_tiny<T, 2, 4>(a, u, s);
    if (m <= 96 && n <= 128) return run_tiny<T, 3, 4>(a, u, s);
    if (m <= 32) return run_small<T, 1>(a, u, ws, s);
    if (m <= 64) return run_small<T, 2>(a, u, ws, s);
    if (m <= 96) return run_small<T, 3>(a, u, ws, s);
    return run_small<T, 4>(a, u, ws, s);
}

template <int NP, typename T>
hipError_t run(const muon_args &a, const update_src &u, void *ws, hipStream_t s) {
    const bool tall = a.N > a.K;
    const int m = tall ? a.K : a.N, n = tall ? a.N : a.K;
    muon_ws w = carve(a.N, a.K, NP, ws);
    const int nb = norm_blocks(a);
    momentum_kernel<T><<<nb, 256, 0, s>>>(u, w.norm);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)ceil_div(n, 64), (unsigned)ceil_div(m, 64));
    pack_update_kernel<T><<<grid, 256, 0, s>>>(u, tall, w.norm, nb, a.eps, w.X, w.Xt[0], w.scal);
    e = hipGetLastError();

    // D = A B^T over sa + sb scale bits, packed with `scale` bits into out
    auto symmetric = [&](const packed_half &A, int sa, const packed_half &B, int sb, const packed_half &out, int scale,
                         float al, float be, float ga, const packed_half &E, int se, const float *dev) {
        product_args P{};
        P.A = A; P.B = B;
        P.rows = P.cols = m;
        P.symmetric = 1;
        P.al = al * exp2i(scale - sa - sb);
        P.be = be * exp2i(scale - se);
        P.ga = ga * exp2i(scale);
        P.dev = dev;
        P.E = E;
        P.out_n = P.out_t = out;
        P.partial = w.partial;
        return launch_product<NP, float>(P, s);
    };
    const packed_half none{};
    int left = a.steps, cur = 0;
    bool first = true;
    while (left > 0 && e == hipSuccess) {
        const int g = NP == 1 ? 1 : std::min(left, most_steps(m, n));
        left -= g;
        e = symmetric(w.X, kScaleX, w.X, kScaleX, w.A, kScaleX, 1.f, 0.f, 0.f, none, 0, first ? w.scal + 1 : nullptr);
        packed_half *Q = &w.P, *Q2 = &w.Q[1];
        for (int k = 0; k < g && e == hipSuccess; ++k) {
            // (one step in a group: b A + c A^2, and a X is added to the product)
            packed_half *P = k == 0 && g > 1 ? &w.Q[0] : &w.P;
            e = symmetric(w.A, kScaleX, w.A, kScaleX, *P, kScaleP, kC, kB, g > 1 ? kA : 0.f, w.A, kScaleX, nullptr);
            if (k == 0) {
                Q = P;
            } else if (e == hipSuccess) {
                e = symmetric(*P, kScaleP, *Q, kScaleP, *Q2, kScaleP, 1.f, 0.f, 0.f, none, 0, nullptr);
                std::swap(Q, Q2);
            }
            if (k + 1 < g && e == hipSuccess) {
                e = symmetric(*P, kScaleP, w.A, kScaleX, w.T, kScaleX, 1.f, 0.f, 0.f, none, 0, nullptr);
                if (e == hipSuccess)
                    e = symmetric(w.T, kScaleX, *P, kScaleP, w.A, kScaleX, 1.f, 0.f, 0.f, none, 0, nullptr);
            }
        }
        if (e != hipSuccess) break;
        product_args P{};
        P.partial = w.partial;
        P.A = *Q;
        P.B = w.Xt[cur];
        P.rows = m; P.cols = n;
        const int scale = left > 0 ? kScaleX : 0;
        const float sc = left > 0 ? 1.f : a.scale;
        P.al = sc * exp2i(scale - kScaleP - kScaleX);
        P.dev = first ? w.scal : nullptr;
        if (g == 1) {
            P.E = w.Xt[cur];
            P.be = sc * kA * exp2i(scale - kScaleX);
        }
        if (left > 0) {
            P.out_n = w.Xt[cur ^ 1];
            P.out_t = w.X;
            e = launch_product<NP, float>(P, s);
        } else {
            P.O = a.O;
            P.ldo = a.ldo;
            P.flip = tall;
            e = launch_product<NP, T>(P, s);
        }
        cur ^= 1;
        first = false;
    }
    return e;
}

template <typename T>
hipError_t run_type(const muon_args &a, void *ws, hipStream_t s) {
    const update_src u{a.G, a.ldg, a.M, a.ldm, a.M_out, a.ldmo, a.mu, a.nesterov, a.N, a.K};
    if (std::min(a.N, a.K) <= kSmall) return run_small<T>(a, u, ws, s);
    return a.parts == 1 ? run<1, T>(a, u, ws, s) : run<2, T>(a, u, ws, s);
}

}  // namespace

// 32-bit chunk numbers, and offsets inside a packed group; grid rows
bool muon_fits(int N, int K) { return (int64_t)N * K <= INT32_MAX && N <= (1 << 22) && K <= (1 << 22); }

size_t muon_workspace_bytes(int N, int K, int parts) {
    return N > 0 && K > 0 && muon_fits(N, K) ? carve(N, K, parts, nullptr).bytes : 0;
}

hipError_t launch_muon(const muon_args &a, void *ws, hipStream_t s) {
    if (a.N == 0 || a.K == 0) return hipSuccess;
    if (a.dtype == kTypeF32) return run_type<float>(a, ws, s);
    if (a.dtype == kTypeBF16) return run_type<__bf16>(a, ws, s);
    return run_type<_Float16>(a, ws, s);
}

}  // namespace l1csr
