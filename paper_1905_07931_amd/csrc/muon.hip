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
#include <cmath>
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

__device__ __forceinline__ double block_sum(double x, double *lds) {  // 256 threads
#pragma unroll
    for (int d = kWave / 2; d >= 1; d >>= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
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

template <typename T>
__device__ __forceinline__ float update_at(const update_src &u, float g, float m_new) {
    return u.M == nullptr ? g : (u.nesterov ? fmaf(u.mu, m_new, g) : m_new);
}

// M' and the partial sums of U^2, four columns a thread; one pass at memory speed
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
            const double x = (double)update_at<T>(u, to_f32(gv[e]), mv[e]);
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
    sum = block_sum(sum, lds);
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

// 2^14 2^e U packed by rows (X) and by columns (X^T); 2^e |U|_F in [1/2, 1).
// scal[0] = s, scal[1] = s^2 with s = 1 / (2^e (|U|_F + eps)).  A workgroup takes 64 x 64 of X.
template <typename T>
__global__ __launch_bounds__(256) void pack_update_kernel(update_src u, int tall, const double *__restrict__ part,
                                                          int n_part, float eps, packed_half X, packed_half Xt,
                                                          float *__restrict__ scal) {
    constexpr int LD = 65;
    __shared__ float tile[64 * LD];
    __shared__ double lds[4];
    double sum = 0;
    for (int i = threadIdx.x; i < n_part; i += 256) sum += part[i];
    const double norm = sqrt(block_sum(sum, lds));
    int e = 0;
    double s;
    if (norm < INFINITY) {
        (void)frexp(norm, &e);
        const double d = ldexp(norm + (double)eps, -e);
        s = d > 0 ? 1 / d : 0;
    } else {
        s = NAN;  // an infinity or a NaN in U, or a norm past double: nothing to give
    }
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        scal[0] = (float)s;
        scal[1] = (float)(s * s);
    }
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;  // of X
    const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;    // of U
    const T *G = static_cast<const T *>(u.G);
    const int col = threadIdx.x & 63, q = threadIdx.x >> 6;
#pragma unroll 4
    for (int r = q; r < 64; r += 4) {
        float x = 0.f;
        if (r0 + r < u.N && c0 + col < u.K) {
            const float g = to_f32(G[(int64_t)(r0 + r) * u.ldg + c0 + col]);
            float m = 0.f;
            if (u.M)
                m = u.M_out ? u.M_out[(int64_t)(r0 + r) * u.ldo + c0 + col]
                            : fmaf(u.mu, u.M[(int64_t)(r0 + r) * u.ldm + c0 + col], g);
            x = ldexpf(update_at<T>(u, g, m), kScaleX - e);
        }
        tile[tall ? col * LD + r : r * LD + col] = x;
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, l = lane & 31, h = lane >> 5;
    for (int b = q; b < 16; b += 4) {  // blocks of X, then of X^T
        const bool t = b >= 8;
        const packed_half &o = t ? Xt : X;
        const int gg = b >> 2 & 1, ss = b & 3;
        const int g = (t ? j0 : i0) / kGroup + gg, st = (t ? i0 : j0) / kStep + ss;
        if (g >= o.groups || st >= o.steps) continue;
        float x[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int row = gg * 32 + l, k = ss * 16 + h * 8 + v;
            x[v] = t ? tile[k * LD + row] : tile[row * LD + k];
        }
        const parts_of<8> p(x);
        char *d = o.data + ((int64_t)g * o.steps + st) * (o.parts * kBlock) + lane * 16;
        *reinterpret_cast<halfx8 *>(d) = p.hi;
        if (o.parts == 2) *reinterpret_cast<halfx8 *>(d + kBlock) = p.lo;
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
    int tiles_m, tiles_n, symmetric;  // symmetric: D = D^T, tiles with tm <= tn only
    // v = dev (al D + be E) + ga [i == j]
    float al, be, ga;
    const float *dev;           // nullable: 1
    packed_half E;              // E[j][i] packed by rows j (data null: none)
    packed_half out_n, out_t;   // v packed with rows j, and with rows i (data null: not stored)
    void *O;                    // or v as a matrix: O[i][j], flipped: O[j][i]
    int64_t ldo;
    int flip;
    float *partial;             // ranges of the reduction: [range][tile][lane order]
    int ranges, range_stages;   // 1: the whole reduction
};

enum { kWhole = 0, kRange = 1, kJoin = 2 };  // one launch; the ranges' sums; their sum and the epilogue

template <int NP, typename S, int PHASE, typename O>
__global__ __launch_bounds__(S::threads, 2) void product_kernel(product_args P) {
    constexpr int PIECES = (S::GA + S::GB) * NP * S::KS;  // 1 KB blocks of a stage
    constexpr int LPW = PIECES / S::waves;
    static_assert(PIECES % S::waves == 0, "every wave issues the same number of loads");
    constexpr int SB = PIECES * kBlock;
    constexpr int TM = S::TM, TN = S::TN, GA = S::GA, GB = S::GB, KS = S::KS;
    __shared__ __attribute__((aligned(16))) char S0[SB];
    __shared__ __attribute__((aligned(16))) char S1[SB];
    __shared__ __attribute__((aligned(16))) char S2[SB];
    // Tiles in bands of 8 tile rows (symmetric: tile columns) walked across the band; each XCD (blocks
    // are dealt round-robin) takes one contiguous range, whose operand rows its L2 then holds.
    const int T = P.symmetric ? P.tiles_n * (P.tiles_n + 1) / 2 : P.tiles_m * P.tiles_n, per = (T + 7) / 8;
    const int t = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || t >= T) return;
    int tm, tn;
    if (P.symmetric) {
        int b = 0;  // bands of 8 columns: 32 b^2 + 4 b tiles lie before band b
        while (32 * (b + 1) * (b + 1) + 4 * (b + 1) <= t) ++b;
        int r = t - (32 * b * b + 4 * b);
        const int h = min(8, P.tiles_n - 8 * b);
        if (r < 8 * b * h) {
            tm = r / h;
            tn = 8 * b + r - tm * h;
        } else {
            r -= 8 * b * h;
            int x = 0;
            while (r >= h - x) r -= h - x++;
            tm = 8 * b + x;
            tn = tm + r;
        }
    } else {
        const int band = t / (8 * P.tiles_n), r = t - band * 8 * P.tiles_n;
        const int h = min(8, P.tiles_m - band * 8);
        tn = r / h;
        tm = band * 8 + (r - tn * h);
    }
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wk = wave / (S::WM * S::WN), wp = wave % (S::WM * S::WN);
    const int wgm = wp / S::WN * TM, wgn = wp % S::WN * TN;  // the wave's first groups in the tile
    constexpr bool TWO = NP == 2;
    floatx16 acc[TM][TN], small[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) acc[a][b] = small[a][b] = floatx16{};

    if constexpr (PHASE != kJoin) {
        const int steps = P.A.steps;
        const int st0 = PHASE == kRange ? (int)blockIdx.y * P.range_stages : 0;
        const int all = (steps + KS - 1) / KS;
        const int stages = PHASE == kRange ? min(P.range_stages, all - st0) : all;
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
        auto compute = [&](const char *cur, int c) {
#pragma unroll
            for (int kk = 0; kk < KS; kk += S::WK) {
                if (KS > 2 && (st0 + c) * KS + kk + wk >= steps) break;
                const int o = (kk + wk) * NP * kBlock + lane * 16;
                halfx8 af[NP][TM], bf[NP][TN];
#pragma unroll
                for (int q = 0; q < NP; ++q) {
#pragma unroll
                    for (int a = 0; a < TM; ++a)
                        af[q][a] = *reinterpret_cast<const halfx8 *>(cur + (wgm + a) * (NP * KS * kBlock) + o + q * kBlock);
#pragma unroll
                    for (int b = 0; b < TN; ++b)
                        bf[q][b] =
                            *reinterpret_cast<const halfx8 *>(cur + (GA + wgn + b) * (NP * KS * kBlock) + o + q * kBlock);
                }
                auto term = [&](floatx16(&d)[TM][TN], int qa, int qb) {
#pragma unroll
                    for (int a = 0; a < TM; ++a)
#pragma unroll
                        for (int b = 0; b < TN; ++b)
                            d[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(af[qa][a], bf[qb][b], d[a][b], 0, 0, 0);
                };
                term(acc, 0, 0);
                if constexpr (TWO) {
                    term(small, 1, 0);
                    term(small, 0, 1);
                }
            }
        };
        // stage c: its blocks have landed everywhere (the loads of stage c + 1 may
        // still be out), and the buffer that the loads of stage c + 2 fill was
        // last read in stage c - 1, whose reads every wave has finished here
        auto stage = [&](int c, const char *cur, unsigned nxt2) {
            if (c + 1 < stages)
                wait_vm<LPW>();
            else
                wait_vm<0>();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (c + 2 < stages) load(nxt2, c + 2);
            compute(cur, c);
        };
        load(l0, 0);
        if (stages > 1) load(l1, 1);
        for (int c = 0; c < stages; c += 3) {
            stage(c, S0, l2);
            if (c + 1 < stages) stage(c + 1, S1, l0);
            if (c + 2 < stages) stage(c + 2, S2, l1);
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
    } else if (wk > 0) {
        return;
    }
    if constexpr (PHASE != kWhole) {
        constexpr int n = TM * TN * 16 * kWave, per_tile = S::WM * S::WN * n;
        float *d = P.partial + (int64_t)t * per_tile + wp * n + lane;
        const int64_t range = (int64_t)T * per_tile;
        if constexpr (PHASE == kRange) {
            d += blockIdx.y * range;
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) d[((a * TN + b) * 16 + r) * kWave] = acc[a][b][r];
            return;
        }
        for (int w = 0; w < P.ranges; ++w, d += range)
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[a][b][r] += d[((a * TN + b) * 16 + r) * kWave];
    }

    // The epilogue.  Lane l, register 4 q + e of a 32 x 32 tile holds row 8 q + 4 (l / 32) + e,
    // column l % 32: four consecutive indices of a packed row j (8 bytes a part), so
    // the matrix packed by rows j is stored from the registers, the one by rows i through LDS.
    const float dev = P.dev ? *P.dev : 1.f;
    const int l = lane & 31, h = lane >> 5;
    const bool both = P.out_t.data != nullptr && !(P.symmetric && tm == tn);
    float *buf = nullptr;
    if (both) {
        // two positions in each of two buffers that every wave has read its last
        // fragments from (behind the barrier in front of the shared sums, if there are any)
        if constexpr (S::WK == 1) __syncthreads();
        static_assert(S::WM * S::WN <= 4 && 2 * 32 * 33 * 4 <= SB, "room for the turned tiles");
        buf = reinterpret_cast<float *>(S::WK > 1 ? (wp < 2 ? S1 : S2) : (wp < 2 ? S0 : S1)) + (wp & 1) * (32 * 33);
    }
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) {
            const int gi = tm * GA + wgm + a, gj = tn * GB + wgn + b;
            if (gi >= P.A.groups || gj >= P.B.groups) continue;
            const int i0 = gi * kGroup, j = gj * kGroup + l;
            float v[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float e4[4] = {0.f, 0.f, 0.f, 0.f};
                if (P.E.data) {
                    const char *p = P.E.data + ((int64_t)gj * P.E.steps + 2 * gi + (q >> 1)) * (P.E.parts * kBlock) +
                                    (l + 32 * (q & 1)) * 16 + 8 * h;
                    const halfx4 hi = *reinterpret_cast<const halfx4 *>(p);
                    halfx4 lo = {};
                    if (P.E.parts == 2) lo = *reinterpret_cast<const halfx4 *>(p + kBlock);
#pragma unroll
                    for (int e = 0; e < 4; ++e) e4[e] = (float)hi[e] + (float)lo[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = i0 + 8 * q + 4 * h + e;
                    float x = dev * fmaf(P.al, acc[a][b][4 * q + e], P.be * e4[e]);
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
                continue;
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
            if (both) {
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
        }
}

// Large products: 128 x 128 tiles.  Products of few tiles: 64 x 64, two waves a
// position, four steps between two barriers.
template <int NP>
using large_tile = tile_shape<2, 2, 2, 2, 1, NP == 2 ? 1 : 2>;
using small_tile = tile_shape<1, 1, 2, 2, 2, 4>;

template <typename S>
int64_t tile_count(const product_args &P, int *tm, int *tn) {
    *tm = (int)ceil_div(P.A.groups, S::GA);
    *tn = (int)ceil_div(P.B.groups, S::GB);
    return P.symmetric ? (int64_t)*tn * (*tn + 1) / 2 : (int64_t)*tm * *tn;
}

constexpr int kRangeTiles = 512;  // most (tile, range) pairs of a product cut into ranges
constexpr size_t kPartialBytes = (size_t)kRangeTiles * 64 * 64 * sizeof(float);

template <int NP, typename O>
hipError_t launch_product(product_args P, hipStream_t s) {
    int tm, tn;
    int64_t T = tile_count<large_tile<NP>>(P, &tm, &tn);
    if (T >= 256) {
        P.tiles_m = tm;
        P.tiles_n = tn;
        product_kernel<NP, large_tile<NP>, kWhole, O><<<(unsigned)(ceil_div(T, 8) * 8), large_tile<NP>::threads, 0, s>>>(P);
        return hipGetLastError();
    }
    T = tile_count<small_tile>(P, &tm, &tn);
    P.tiles_m = tm;
    P.tiles_n = tn;
    const unsigned grid = (unsigned)(ceil_div(T, 8) * 8);
    const int stages = (int)ceil_div(P.A.steps, small_tile::KS);
    int ranges = P.partial ? (int)(kRangeTiles / 2 / T) : 1;
    if (ranges > stages / 4) ranges = stages / 4;
    if (ranges < 2) {
        product_kernel<NP, small_tile, kWhole, O><<<grid, small_tile::threads, 0, s>>>(P);
        return hipGetLastError();
    }
    if constexpr (sizeof(O) == sizeof(float)) {
        P.range_stages = (int)ceil_div(stages, ranges);
        P.ranges = (int)ceil_div(stages, P.range_stages);
        product_kernel<NP, small_tile, kRange, float><<<dim3(grid, (unsigned)P.ranges), small_tile::threads, 0, s>>>(P);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        product_kernel<NP, small_tile, kJoin, float><<<grid, small_tile::threads, 0, s>>>(P);
        return hipGetLastError();
    }
    return hipErrorInvalidValue;
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

template <int NP, typename T>
hipError_t run(const muon_args &a, const update_src &u, void *ws, hipStream_t s) {
    const bool tall = a.N > a.K;
    const int m = tall ? a.K : a.N, n = tall ? a.N : a.K;
    muon_ws w = carve(a.N, a.K, NP, ws);
    const int64_t chunks = (int64_t)a.N * ceil_div(a.K, 4);
    const int nb = (int)(chunks < kNormBlocks * 256 ? ceil_div(chunks, 256) : kNormBlocks);
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
        const int g = NP == 1 ? 1 : (left < kMaxGroup ? left : kMaxGroup);
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
    return a.parts == 1 ? run<1, T>(a, u, ws, s) : run<2, T>(a, u, ws, s);
}

}  // namespace

size_t muon_workspace_bytes(int N, int K, int parts) {
    return N > 0 && K > 0 ? carve(N, K, parts, nullptr).bytes : 0;
}

hipError_t launch_muon(const muon_args &a, void *ws, hipStream_t s) {
    if (a.N == 0 || a.K == 0) return hipSuccess;
    if (a.dtype == kTypeF32) return run_type<float>(a, ws, s);
    if (a.dtype == kTypeBF16) return run_type<__bf16>(a, ws, s);
    return run_type<_Float16>(a, ws, s);
}

}  // namespace l1csr
