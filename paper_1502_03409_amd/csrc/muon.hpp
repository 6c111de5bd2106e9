// A step of gradient descent whose update is the momentum with its singular values brought near one.
//
//   m' = mu m + g;  u = g + mu m' (looking ahead) or m';  X = u / |u|;  steps times  X <- a X + b (X X^T) X + c (X X^T)^2 X;
//   w' = (1 - decay) w - rate X.
//
// With A = X X^T (or X^T X, whichever is smaller) and S = A + b / (2 c) I the polynomial is P = c S S + (a - b^2 / (4 c)) I, and a step X <- P X:
// products, and nothing to add but on a diagonal.  A, S and P are symmetric: tiles below the diagonal are formed and stored twice.
//
// Products with the longer side are the long ones, so up to three steps go by on the short side alone: all of their A and P are polynomials of the
// first A and commute, the next A is (P A) P, and X takes the product Q of the group's P at once.  No more than three, because a rounding of the
// first A, r of |A| at most, grows with the square of what Q does to it: r 3.4445^4 by the third step, where it meets singular values of 0.08 and
// more of the largest, and 3.4445^8 by the fifth.  What a group's later A is off by counts where it brings singular values near one, which start at
// about one over the root of the short side: within three steps of few and not before the fourth of thousands, so short groups come first on short
// sides and last on long ones (fp32, 41 x 1280 0.46 and 0.1 10^-5 off with groups of 3, 2 and of 2, 3; bf16, 8192 x 4096 0.19 % and 0.28 %).
//
// Between products X, A, S, P and Q are held in fp16, times powers of two.  Singular values of X lie in [0, 1.203] throughout, because |u| bounds
// the largest and a s + b s^3 + c s^5 maps [0, 1.203] into itself, so no value of X, A, S, P exceeds 1.203, 1.447, 1.176, 3.445 in magnitude, nor
// one of Q a power of 3.445, and the powers of two put all of them at the upper end of fp16's range: what a rounding costs is 2^-12 of values that
// count, an eighth of bf16's, and small ones lose nothing below 2^-24 of the largest.  For bf16 weights one fp16 value is held; for fp32 weights two, a value and what its rounding leaves, 22 bits,
// and three products of them are formed.  Sums, norms and the momentum are fp32 and more.
#pragma once
#include "head_planes.hpp"
#include "head_gemm.hpp"

namespace lc {
namespace head {

constexpr float kMuonA = 3.4445f, kMuonB = -4.7750f, kMuonC = 2.0315f;
constexpr float kShift = kMuonB / (2.f * kMuonC), kRest = (float)(3.4445 - 4.7750 * 4.7750 / (4 * 2.0315));
constexpr float kScaleX = 0x1p14f, kScaleA = 0x1p14f;                 // 1.203 and 1.447 times these, and 3.4445, 3.4445^2, 3.4445^3 times
constexpr float kScaleQ[4] = {0.f, 0x1p13f, 0x1p12f, 0x1p10f};        // those, stay below 2^16 (P is the first Q)
constexpr int kGroupSteps = 3, kLateSide = 1024;
constexpr int kMostSums = 1024;   // partial sums of a matrix's squares

typedef _Float16 half_t;
__device__ __forceinline__ bf16_t half_bits(float v) { return __builtin_bit_cast(bf16_t, (half_t)v); }

template <typename T> struct MuonFormat;
template <> struct MuonFormat<bf16_t> { static constexpr int PL = HALF, N = 1; };
template <> struct MuonFormat<float> { static constexpr int PL = HALF2, N = 2; };

// momentum and what is orthogonalised of one value
__device__ __forceinline__ float next_momentum(float m, float g, float mu) { return __builtin_fmaf(mu, m, g); }
__device__ __forceinline__ float looked_ahead(float m, float g, float mu, bool ahead) { return ahead ? __builtin_fmaf(mu, m, g) : m; }

__device__ __forceinline__ double workgroup_sum(double s) {
    __shared__ double part[4];
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

// eight floats at any alignment, n of them
__device__ __forceinline__ void store8(float *p, const float (&v)[8], int n) {
    if (n >= 8) {
        __builtin_memcpy(p, v, 32);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = v[e];
    }
}

// m' and the partial sums of u's squares, `parts` workgroups a matrix of n values; bound by HBM (841 of 2048 x 128 in fp32, 2.6 GB, 0.47 ms).
template <typename T>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const T *g, const float *m, float *m_out, double *partial, long long n, int parts, float mu,
                                                            int ahead) {
    const long long item = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    g += item * n, m += item * n, m_out += item * n;
    double s = 0.0;
    const auto some = [&](long long i, int left, float (&a)[8], float (&b)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            b[e] = next_momentum(b[e], a[e], mu);
            const double u = looked_ahead(b[e], a[e], mu, ahead);
            if (e < left) s += u * u;
        }
        store8(m_out + i, b, left);
    };
    const long long step = parts * 2048LL;
    long long i = (part * 256LL + threadIdx.x) * 8;
    for (; i + step + 8 <= n; i += 2 * step) {   // two at a time
        float a[2][8], b[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            load8(g + i + k * step, 0, 8, a[k]);
            load8(m + i + k * step, 0, 8, b[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) some(i + k * step, 8, a[k], b[k]);
    }
    for (; i < n; i += step) {
        const int left = (int)min(n - i, 8LL);
        float a[8], b[8];
        load8(g + i, 0, left, a);
        load8(m + i, 0, left, b);
        some(i, left, a, b);
    }
    s = workgroup_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// planes of eight fp16 values each
template <int PLANES>
__device__ __forceinline__ void put_halves(bf16_t *to, long long plane, const float (&v)[8]) {
    u32x4 w[PLANES];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const half_t a = (half_t)v[2 * e], b = (half_t)v[2 * e + 1];
        w[0][e] = (unsigned)__builtin_bit_cast(bf16_t, a) | (unsigned)__builtin_bit_cast(bf16_t, b) << 16;
        if constexpr (PLANES == 2)
            w[1][e] = (unsigned)half_bits(v[2 * e] - (float)a) | (unsigned)half_bits(v[2 * e + 1] - (float)b) << 16;
    }
#pragma unroll
    for (int q = 0; q < PLANES; ++q) *(u32x4 *)(to + q * plane) = w[q];
}

// Bound by HBM as well (the same, 2.6 GB, 0.47 ms); doing both passes over 128 MB at a time, for the second to find the first one's in the cache
// behind the L2 caches, took 0.05 ms from it and added 0.1 to the first.
constexpr int kStartPieces = 2;   // of eight values, a thread
// X = u / |u| as planes [item][rows][ld], zeros behind a row.  A matrix of zeros stays one; one with an infinite or NaN value becomes NaN.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void muon_start_kernel(const T *g, const float *m, const double *partial, bf16_t *x, long long plane, int rows, int cols,
                                                         int ld, int parts, int groups, float mu, int ahead) {
    const long long item = blockIdx.x / groups, n = (long long)rows * cols;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += partial[item * parts + i];
    s = sqrt(workgroup_sum(s));
    const double f = !__builtin_isfinite(s) ? __builtin_nan("") : s > 0.0 ? (double)kScaleX / s : 0.0;
    const int pieces = ld / 8;
    const long long all = (long long)rows * pieces, from = (blockIdx.x - item * groups) * (256LL * kStartPieces) + threadIdx.x;
    const T *const gi = g + item * n;
    const float *const mi = m + item * n;
    float a[kStartPieces][8], b[kStartPieces][8];
    int r[kStartPieces], c[kStartPieces];
#pragma unroll
    for (int k = 0; k < kStartPieces; ++k) {
        const long long at = min(from + 256 * k, all - 1);
        r[k] = (int)(at / pieces), c[k] = (int)(at - (long long)r[k] * pieces) * 8;
        load8(gi + (long long)r[k] * cols, c[k], cols, a[k]);
        load8(mi + (long long)r[k] * cols, c[k], cols, b[k]);
    }
#pragma unroll
    for (int k = 0; k < kStartPieces; ++k) {
        if (from + 256 * k >= all) break;
#pragma unroll
        for (int e = 0; e < 8; ++e)   // 1 / |u| may be beyond fp32
            b[k][e] = c[k] + e < cols ? (float)((double)looked_ahead(b[k][e], a[k][e], mu, ahead) * f) : 0.f;
        put_halves<PLANES>(x + (item * rows + r[k]) * ld + c[k], plane, b[k]);
    }
}

// A product as planes of fp16: times `factor`, `diag` added on the diagonal; zeros in the columns behind the last one up to ld.  MIRROR: the
// result is symmetric, tiles beside the diagonal go to their mirrored place as well; and where there is a second place, all goes there too, with
// `diag2` added on the diagonal.
template <int PLANES, bool MIRROR>
struct PlaneEpi {
    bf16_t *out, *out2;
    long long plane, each;
    int ld;
    float factor, diag, diag2;
    __device__ __forceinline__ void item(int i) {
        out += i * each;
        if (MIRROR && out2) out2 += i * each;
    }
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int Nn, int, char *lds) const {
        const int h = lane >> 5, l32 = lane & 31;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int m = m0 + 32 * i + l32, n = n0 + 32 * j + 8 * (e >> 2) + 4 * h + (e & 3);
                    const float v = acc[i][j][e] * factor + (m == n ? diag : 0.f);
                    acc[i][j][e] = n < Nn && m < M ? v : 0.f;
                }
        send(acc, m0, n0, lane, M, Nn, out, lds);
        if (MIRROR && out2) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int m = m0 + 32 * i + l32, n = n0 + 32 * j + 8 * (e >> 2) + 4 * h + (e & 3);
                        if (m == n && m < M) acc[i][j][e] += diag2 - diag;
                    }
            send(acc, m0, n0, lane, M, Nn, out2, lds);
        }
    }
    template <int MT, int NT>
    __device__ __forceinline__ void send(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int Nn, bf16_t *to, char *lds) const {
        const int h = lane >> 5, l32 = lane & 31;
        const RowStage<bf16_t, NT * 32> stage = {lds, lane};
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16_t v[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = part(acc[i][j][4 * q + r], p);
                        stage.put(32 * j + 8 * q + 4 * h, v);
                    }
                stage.take([&](int r, int c, const u32x4 &w) {
                    const int m = m0 + 32 * i + r;
                    if (m < M && n0 + c < ld) *(u32x4 *)(to + p * plane + (long long)m * ld + n0 + c) = w;
                });
            }
        });
        // On the diagonal the tile has both places itself, and other waves store what would be the mirrored ones.  Symmetric tiles are square and two
        // waves wide, whether two or four waves share their height.
        constexpr int SIDE = NT * 64;
        if (!MIRROR || m0 / SIDE == n0 / SIDE) return;
        typedef RowStage<bf16_t, MT * 32> Across;
        const Across across = {lds, lane};
        for_blocks<NT>([&](auto block) __attribute__((always_inline)) {
            constexpr int j = decltype(block)::value;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        *(bf16_t *)(lds + (8 * (e >> 2) + 4 * h + (e & 3)) * Across::PITCH + (32 * i + l32) * 2) = part(acc[i][j][e], p);
                across.take([&](int r, int c, const u32x4 &w) {
                    const int n = n0 + 32 * j + r;
                    if (n < Nn && m0 + c < ld) *(u32x4 *)(to + p * plane + (long long)n * ld + m0 + c) = w;
                });
            }
        });
    }
    static __device__ __forceinline__ bf16_t part(float v, int p) {
        const half_t a = (half_t)v;
        return p == 0 ? __builtin_bit_cast(bf16_t, a) : half_bits(v - (float)a);
    }
    static constexpr bool SYM = MIRROR;
    __device__ __forceinline__ float result(float v, int m, int n) const { return v * factor + (m == n ? diag : 0.f); }
    // four columns k .. k + 3 of row m, of n rows
    __device__ __forceinline__ void put4(int m, int k, float (&v)[4], int n) const {
        put4_at(out, m, k, v, n);
        if (!MIRROR || !out2) return;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (m == k + e) v[e] += diag2 - diag;
        put4_at(out2, m, k, v, n);
    }
    __device__ __forceinline__ void put4_at(bf16_t *to, int m, int k, const float (&v)[4], int n) const {
        typedef bf16_t V4 __attribute__((ext_vector_type(4)));
        if (m >= n || k >= ld) return;
#pragma unroll
        for (int p = 0; p < PLANES; ++p) *(V4 *)(to + p * plane + (long long)m * ld + k) = (V4){part(v[0], p), part(v[1], p), part(v[2], p), part(v[3], p)};
    }
};

// The last product: w' = keep w - rate X.
template <typename T>
struct UpdateEpi {
    const T *w;
    T *w_out;
    long long each;
    int cols;
    float keep, rate;   // rate: times what the product's factor is
    __device__ __forceinline__ void item(int i) { w += i * each, w_out += i * each; }
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int, int, char *lds) const {
        typedef RowStage<float, NT * 32> Stage;
        const Stage stage = {lds, lane};
        constexpr int TAKES = 32 * Stage::PIECES / 64;
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value;
            float old[TAKES][4];   // all before the first store: a load behind a store waits until that has reached memory
#pragma unroll
            for (int t = 0; t < TAKES; ++t) {
                const int at = t * 64 + lane, m = m0 + 32 * i + at / Stage::PIECES, n = n0 + at % Stage::PIECES * 4;
                const T *p = w + (long long)min(m, M - 1) * cols;
                if (n + 4 <= cols) {
                    T v[4];
                    __builtin_memcpy(v, p + n, sizeof(v));
#pragma unroll
                    for (int r = 0; r < 4; ++r) old[t][r] = widen<T>(v[r]);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) old[t][r] = widen<T>(p[min(n + r, cols - 1)]);
                }
            }
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    stage.put(32 * j + 8 * q + 4 * (lane >> 5), v);
                }
            int t = 0;
            stage.take([&](int r, int c, const u32x4 &x) {
                const int m = m0 + 32 * i + r, n = n0 + c;
                T o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned u = x[e];
                    o[e] = narrow<T>(keep * old[t][e] - rate * __builtin_bit_cast(float, u));
                }
                ++t;
                if (m >= M) return;
                T *p = w_out + (long long)m * cols;
                if (n + 4 <= cols) {
                    __builtin_memcpy(p + n, o, sizeof(o));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + e < cols) p[n + e] = o[e];
                }
            });
        });
    }
    static constexpr bool SYM = false;
    __device__ __forceinline__ float result(float v, int, int) const { return v; }
    __device__ __forceinline__ void put4(int m, int k, float (&v)[4], int n) const {
        if (m >= n) return;
        const T *const p = w + (long long)m * cols + k;
        T *const to = w_out + (long long)m * cols + k;
        T o[4];
        if (k + 4 <= cols) {
            __builtin_memcpy(o, p, sizeof(o));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = narrow<T>(keep * widen<T>(o[e]) - rate * v[e]);
            __builtin_memcpy(to, o, sizeof(o));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k + e < cols) to[e] = narrow<T>(keep * widen<T>(p[e]) - rate * v[e]);
        }
    }
};

// The sums of a part, as PartEpi stores them: [item][part][M][ld].
struct StackPartEpi : PartEpi {
    int at;
    __device__ __forceinline__ void item(int i) { at = i; }
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int live_rows, int nn, int, char *lds) const {
        PartEpi::run(acc, m0, n0, lane, live_rows, nn, at, lds);
    }
};

// Adds up the parts of a symmetric product, tiles of 64 x 64 on and below the diagonal, and stores them as PlaneEpi does.  Bound by the parts.
template <int PLANES>
__global__ __launch_bounds__(256) void muon_join_kernel(const float *part, int splits, int n, int ldp, PlaneEpi<PLANES, true> epi) {
    __shared__ float tile[64][65];
    const Shape sh = {n, n, 0, nullptr, 0, nullptr, 0, 1, 1, 1};
    int tm, tn, item;
    tile_in_stack(sh, blockIdx.x, (n + 63) / 64, 0, 1, &tm, &tn, &item);
    epi.item(item);
    const int r0 = threadIdx.x / 16, c = threadIdx.x % 16 * 4;
    f32x4 s[4] = {};
    for (int p = 0; p < splits; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = min(tm * 64 + r0 + 16 * i, n - 1), at = min(tn * 64 + c, ldp - 4);
            s[i] += *(const f32x4 *)(part + (((long long)item * splits + p) * n + m) * ldp + at);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = tm * 64 + r0 + 16 * i;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = tn * 64 + c + e;
            v[e] = m < n && k < n ? s[i][e] * epi.factor + (m == k ? epi.diag : 0.f) : 0.f;
            tile[r0 + 16 * i][c + e] = v[e];
        }
        epi.put4(m, tn * 64 + c, v, n);
    }
    if (tm == tn) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = tile[c + e][r0 + 16 * i];
        epi.put4(tn * 64 + r0 + 16 * i, tm * 64 + c, v, n);
    }
}

// A product with a short side and a short contraction, a tile of 32 x 32 a workgroup: each wave takes 64 of every 256 indices, from memory straight to
// registers, all at once for up to 512, and the waves' sums are added up in LDS.  What the product before has just written comes from beyond this
// XCD's L2 cache, and a compute unit has only so many lines on their way at a time: neither more buffers nor earlier reads of LDS make tiles of 64 x
// 64 faster, more and smaller workgroups do.  Two of 256 x 256 times their like in fp32 10.8 us and 6.4, times 256 x 400 8.7 us and 6.5, a step of
// two of 256 x 400 155 us and 101.
//
// FB COL: what lies by columns takes its turn through LDS of the wave's own, to be read by the transposing load.
template <int PL, int PLANES, int FB, typename Epi>
__global__ __launch_bounds__(256) void muon_block_kernel(Operand A, Operand B, Shape sh, Epi epi) {
    constexpr int STEP = 64 * 32 * 2;   // bytes of 64 indices of 32 columns
    __shared__ __attribute__((aligned(16))) float sums[4][32][36];
    __shared__ __attribute__((aligned(1024))) char turned[FB == COL ? 4 * PLANES * STEP : 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5, K = (int)A.ld;   // zeros from sh.K on
    int tm, tn, item;
    tile_in_stack(sh, blockIdx.x, (sh.M + 31) / 32, (sh.Nn + 31) / 32, 1, &tm, &tn, &item);
    epi.item(item);
    const bf16_t *const a = A.p0 + item * A.each + min(tm * 32 + l32, sh.M - 1) * A.ld, *const b0 = B.p0 + item * B.each;
    const int col = tn * 32 + lane % 4 * 8;
    u32x4 va[2][PLANES][4], vb[2][PLANES][4];
    const auto load = [&](auto slot, int k0) __attribute__((always_inline)) {
        constexpr int s = decltype(slot)::value;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int k = k0 + 16 * c + 8 * h, r = k0 + 16 * c + lane / 4;
            const bool in = FB == COL ? r < sh.K && col < B.ld : k < K;
            const bf16_t *const b = FB == COL ? b0 + r * B.ld + col : b0 + min(tn * 32 + l32, sh.Nn - 1) * B.ld + k;
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                va[s][p][c] = vb[s][p][c] = (u32x4){0, 0, 0, 0};
                if (k < K) va[s][p][c] = *(const u32x4 *)(a + p * A.plane + k);
                if (in) vb[s][p][c] = *(const u32x4 *)(b + p * B.plane);
            }
        }
    };
    char *const mine = turned + (FB == COL ? wave * PLANES * STEP : 0);
    Reader<COL, 32, 1> reader;
    if constexpr (FB == COL) {
        reader.init((unsigned)(size_t)(__attribute__((address_space(3))) char *)mine, 0, lane);
        reader.turn(0);
    }
    f32x16 acc = {};
    const auto multiply = [&](auto slot) __attribute__((always_inline)) {
        constexpr int s = decltype(slot)::value;
        if constexpr (FB == COL) {   // a wave's LDS accesses are done in their order
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int c = 0; c < 4; ++c) *(u32x4 *)(mine + p * STEP + c * 1024 + lane * 16) = vb[s][p][c];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                Reader<COL, 32, 1> at = reader;
                at.at[0] += p * STEP;
#pragma unroll
                for (int c = 0; c < 4; ++c) vb[s][p][c] = at.read(c, 0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < Format<PL>::PAIRS; ++t)
                acc = Format<PL>::mul(vb[s][Format<PL>::B >> (4 * t) & 1][c], va[s][Format<PL>::A >> (4 * t) & 1][c], acc);
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int k = wave * 64;
    load(even, k);
    for (; k < K; k += 512) {
        load(odd, k + 256);
        multiply(even);
        load(even, k + 512);
        multiply(odd);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) *(f32x4 *)&sums[wave][l32][8 * q + 4 * h] = (f32x4){acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    const int r = threadIdx.x / 8, c = threadIdx.x % 8 * 4, m = tm * 32 + r;
    f32x4 *const own = (f32x4 *)&sums[0][r][c];   // of all waves' sums a thread has four places to itself
    f32x4 s = *own;
#pragma unroll
    for (int w = 1; w < 4; ++w) s += *(const f32x4 *)&sums[w][r][c];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = v[e] = m < sh.M && tn * 32 + c + e < sh.Nn ? epi.result(s[e], m, tn * 32 + c + e) : 0.f;
    if constexpr (Epi::SYM) *own = s;
    epi.put4(m, tn * 32 + c, v, sh.M);
    if constexpr (Epi::SYM) {
        if (tm == tn) return;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sums[0][c + e][r];
        epi.put4(tn * 32 + r, tm * 32 + c, v, sh.M);
    }
}

template <int PL, int FB, typename Epi>
int launch_block(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    const int mt = ceil_div(sh.M, 32), nt = ceil_div(sh.Nn, 32);
    const long long wgs = tiles_in(sh, mt, nt) * sh.stack;
    const LaunchPlan p = make_plan(name, {PL, ROW, FB, 32, 32}, {sh.M, sh.Nn, sh.K, 1, sh.stack, sh.sym}, dim3((unsigned)wgs), 256, 0);
    LC_PLAN_REQUIRE(p, wgs <= 0x7fffffffLL && sh.stack >= 1 && sh.sym == (int)Epi::SYM && (!sh.sym || (sh.M == sh.Nn && mt <= 4096)));
    LC_PLAN_REQUIRE(p, A.ld % 8 == 0 && A.ld >= sh.K && A.ld < sh.K + 8 && B.ld % 8 == 0 && (FB == COL ? B.ld >= sh.Nn : B.ld == A.ld));
    LC_PLAN_REQUIRE(p, A.plane % 8 == 0 && B.plane % 8 == 0 && A.each % 8 == 0 && B.each % 8 == 0 && A.rows >= sh.M && B.rows >= sh.Nn);
    LC_PLAN_REQUIRE(p, ptr_aligned16(A.p0) && ptr_aligned16(B.p0));
    LC_LAUNCH(p, name, (muon_block_kernel<PL, PL == HALF2 ? 2 : 1, FB, Epi>), s, A, B, sh, epi);
    return LC_OK;
}

// How products of a stack are cut: into tiles of 256, 192, 128, 64 or 32, their contraction into parts.
struct StackCut {
    int tile, splits;
    double us;   // by the estimate
};
// The cut that takes least by an estimate in microseconds from measured times: what begins and ends a tile, and for each 64 indices and pair of
// planes a step of the tiles that share the fullest compute unit.  fp16, n x n times its like, the half below the diagonal, tiles of 64 / 128 /
// 192 / 256: n = 256 4.9 / 7.0 / 12.4 / 12.0 us, 1024 9.0 / 12.7 / 21.9 / 27, 2048 21.9 / 24.4 / 34.8 / 45, 4096 149 / 99 / 77 / 92, two of 4096
// 260 / 167 / 150 / 188, 5120 295 / 168 / 159 / 128; two of 8192 x 4096 times 4096 x 4096 with tiles of 128 / 256 563 / 473, with the update 621 / 547.
// Two planes: 4096 367 / 283 / 212 / 296, 5120 671 / 420 / 454 / 392, four of 2048 177 / 151 / 203 / 191; what tiles of 256 lose there is not in the
// estimate (191 us taken for 139): their epilogue keeps 203 registers of a lane in scratch.  Parts cost a kernel and
// their bytes: 1021 x 20011 times its transpose 152 us whole and 33 + 7 in 14.  Tiles of 192 read rows only.
//
// Products whose workgroups of 32 x 32 hardly share compute units take those (five steps in fp32, symmetric products in tiles of 32 and of 64:
// 512 x 512 154 and 181 us, 768 x 768 260 and 253, eight of 256 x 400 123 and 149, 32 of 256 x 256 199 and 166; 256 x 4000 with A so 258, with A in
// parts of tiles of 64 134; products with X in tiles of 32 and of 64: 512 x 512 131 and 157, 400 x 700 138 and 157, 256 x 2000 the same).
inline double stack_tiles(const Shape &sh, int tile) { return (double)tiles_in(sh, ceil_div(sh.M, tile), ceil_div(sh.Nn, tile)) * sh.stack; }
constexpr double kSplitTiles = 512;   // no product of more tiles of 128 is cut along its contraction
enum { ROWS_ONLY = 1, MAY_SPLIT = 2, BLOCKS = 4 };   // ROWS_ONLY: both operands by rows; BLOCKS: the first is, tiles of 32 may be
constexpr int kBlockSide = 512, kBlockLong = 1024;   // of products in tiles of 32
inline StackCut choose_stack_cut(const Shape &sh, int pairs, int how) {
    const int steps = ceil_div(sh.K, kStep);
    if ((how & BLOCKS) && std::min(sh.M, sh.Nn) <= kBlockSide && sh.K <= kBlockLong && stack_tiles(sh, 32) <= 2 * kComputeUnits)
        return {32, 1, 3 + 0.4 * steps * (pairs > 1 ? 2 : 1)};
    StackCut best = {128, 1, 1e30};
    const bool may_split = (how & MAY_SPLIT) && stack_tiles(sh, 128) <= kSplitTiles;
    const long long result = sh.M * round_up(sh.Nn, 4) * sh.stack;
    for (int s = 1; s == 1 || (may_split && s <= kMostSplits && s <= steps / 2 && s * result <= kMostParts); ++s)
        for (const int tile : {64, 128, 192, 256}) {
            if (tile == 192 && !(how & ROWS_ONLY)) continue;
            const double load = stack_tiles(sh, tile) * s / kComputeUnits, most = std::ceil(load);
            double ends, step;
            if (tile == 64) ends = 3.4, step = std::max(0.5, 0.28 * load);
            else if (tile == 128) ends = 4.5, step = most <= 1 ? 0.57 : most <= 2 ? 0.92 : 0.55 * most;
            else if (tile == 192) ends = 9, step = load <= 0.5 ? 0.9 : 1.15 * most;
            else ends = 14, step = most <= 1 ? 1.3 : most <= 2 ? 3.0 : 1.8 * most;
            const double us = ends + (double)ceil_div(steps, s) * pairs * step + (s > 1 ? 6 + 4e-6 * s * (double)result / 4 : 0);
            if (us < best.us) best = {tile, s, us};
        }
    return best;
}

template <int PL, int FA, int FB, typename Epi>
int launch_stack(const char *name, const Operand &A, const Operand &B, const Shape &sh, const StackCut &c, const Epi &epi, hipStream_t s) {
    // Two planes from operands of one are the first A of a short side up to kChain, one tile of 128 or larger: larger ones begin, end and step
    // longer, so the estimate takes none.
    constexpr bool LARGE = !(PL == HALF && std::is_same<Epi, PlaneEpi<2, true>>::value);
    if constexpr (FA == ROW && !std::is_same<Epi, StackPartEpi>::value)
        if (c.tile == 32) return launch_block<PL, FB>(name, A, B, sh, epi, s);
    if constexpr (LARGE)
        if (c.tile == 256) return launch_tiles<PL, FA, FB, 256, 256, 3, 2, 8>(name, A, B, sh, c.splits, epi, s);
    if constexpr (LARGE && FA == ROW && FB == ROW)
        if (c.tile == 192) return launch_tiles<PL, FA, FB, 192, 192, 3, 2>(name, A, B, sh, c.splits, epi, s);
    if (c.tile == 64) return launch_tiles<PL, FA, FB, 64, 64, 3, 2>(name, A, B, sh, c.splits, epi, s);
    return launch_tiles<PL, FA, FB, 128, 128, 3, 2>(name, A, B, sh, c.splits, epi, s);
}

// A symmetric product of a stack.
template <int PL, int FA, int FB, int PLANES>
int launch_symmetric(const char *name, const Operand &A, const Operand &B, const Shape &sh, const PlaneEpi<PLANES, true> &epi, const Parts &part,
                     hipStream_t s) {
    const StackCut c = choose_stack_cut(sh, Format<PL>::PAIRS, (FA == ROW && FB == ROW ? ROWS_ONLY | BLOCKS : 0) | MAY_SPLIT);
    if (c.splits == 1) return launch_stack<PL, FA, FB>(name, A, B, sh, c, epi, s);
    const int ldp = (int)round_up(sh.Nn, 4);
    const long long wgs = (long long)stack_tiles(sh, 64);
    const LaunchPlan p = make_plan("muon_join", {PLANES}, {sh.M, c.splits, sh.stack}, dim3((unsigned)wgs), 256, 0);
    LC_PLAN_REQUIRE(p, wgs <= 0x7fffffffLL && (long long)c.splits * sh.stack * sh.M * ldp <= part.floats && ldp >= 4);
    if (int rc = launch_stack<PL, FA, FB>(name, A, B, sh, c, StackPartEpi{{part.at, ldp, sh.M}, 0}, s)) return rc;
    LC_LAUNCH(p, name, (muon_join_kernel<PLANES>), s, part.at, c.splits, sh.M, ldp, epi);
    return LC_OK;
}

// ---------------------------------------------------------------------------------------------------------------------------
// A group's steps on the short side where that is at most kChain: one workgroup a matrix, everything in LDS and registers.  A and Q stay in fp32
// between products, in the layout of the accumulators; operands go through two places of LDS as planes, which the fragments are read from as
// in a tile of the other products.  2 x 2 waves, each B / 2 x B / 2.  Two planes inside whatever the weights' type: on a short side singular values
// are near one after few steps, where one plane of A showed (64 x 1408 in bf16: off by 0.57 % with one, 0.18 % with two, of which the weights' own
// rounding is 0.17 %), and all of it costs little.
//
// 841 matrices of 128 x 128: two and three steps 124 us and 204, 35 us for each of 14 products with kernels of their own.  The matrix unit is busy
// 22 % of the cycles: a workgroup has a compute unit for itself, and nothing overlaps what lies between products.
constexpr int kChain = 128;
template <int B>
struct Chain {
    static constexpr int PL = HALF2, PLANES = 2, MT = B / 64, PLANE = B * B * 2;   // bytes of a plane
    static constexpr int PLACE = PLANES * PLANE;
    typedef f32x16 Square[MT][MT];
    char *lds;
    int lane, m0, n0;
    // where four values from column n on of row m lie in a plane: steps of 64 columns, rows of 128 bytes whose 16-byte pieces are exchanged by the row
    static __device__ __forceinline__ int at(int m, int n) { return (n / 64 * B + m) * 128 + ((((n & 63) / 8) ^ ((m >> 1) & 7)) * 16) + (n & 7) * 2; }
    // fn(block row, block column, component, row, column of the component's four)
    template <typename Fn>
    __device__ __forceinline__ void each4(const Fn &fn) const {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) fn(i, j, 4 * q, m0 + 32 * i + (lane & 31), n0 + 32 * j + 8 * q + 4 * (lane >> 5));
    }
    __device__ __forceinline__ void put(int place, const Square &v) const {   // as planes
        each4([&](int i, int j, int e, int m, int n) __attribute__((always_inline)) {
            typedef bf16_t V4 __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                V4 w;
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = PlaneEpi<PLANES, true>::part(v[i][j][e + r], p);
                *(V4 *)(lds + place * PLACE + p * PLANE + at(m, n)) = w;
            }
        });
    }
    // left times right, which is symmetric: rows of both
    __device__ __forceinline__ void multiply(int left, int right, Square &acc) const {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = (f32x16){};
#pragma unroll
        for (int k = 0; k < B; k += 16) {
            u32x4 a[PLANES][MT], b[PLANES][MT];
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    a[p][i] = *(const u32x4 *)(lds + left * PLACE + p * PLANE + at(m0 + 32 * i + (lane & 31), k + 8 * (lane >> 5)));
                    b[p][i] = *(const u32x4 *)(lds + right * PLACE + p * PLANE + at(n0 + 32 * i + (lane & 31), k + 8 * (lane >> 5)));
                }
#pragma unroll
            for (int q = 0; q < Format<PL>::PAIRS; ++q)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < MT; ++j)
                        acc[i][j] = Format<PL>::mul(b[Format<PL>::B >> (4 * q) & 1][j], a[Format<PL>::A >> (4 * q) & 1][i], acc[i][j]);
        }
    }
};

template <int OUT, int B>
__global__ __launch_bounds__(256) void muon_chain_kernel(const bf16_t *a, bf16_t *out, long long plane, long long each, int n, int ld, int len) {
    typedef Chain<B> C;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int wave = threadIdx.x >> 6;
    const C c = {smem, (int)threadIdx.x & 63, wave / 2 * (B / 2), wave % 2 * (B / 2)};
    a += blockIdx.x * each, out += blockIdx.x * each;
    typename C::Square held, q, acc;   // A, Q
    c.each4([&](int i, int j, int e, int m, int k) __attribute__((always_inline)) {
        typedef bf16_t V4 __attribute__((ext_vector_type(4)));
        const bool in = m < n && k < ld;   // columns up to ld are zeros behind the last one
#pragma unroll
        for (int r = 0; r < 4; ++r) held[i][j][e + r] = 0.f;
#pragma unroll
        for (int p = 0; p < C::PLANES; ++p) {
            V4 w = {0, 0, 0, 0};
            if (in) w = *(const V4 *)(a + p * plane + (long long)m * ld + k);
            *(V4 *)(smem + p * C::PLANE + C::at(m, k)) = w;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bf16_t h = w[r];
                held[i][j][e + r] += (float)__builtin_bit_cast(half_t, h);
            }
        }
    });
    __syncthreads();
    for (int step = 0; step < len; ++step) {
        // place 0 holds A
        c.multiply(0, 0, acc);
        c.each4([&](int i, int j, int e, int m, int k) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                acc[i][j][e + r] = acc[i][j][e + r] * (kMuonC * kScaleQ[1] / (kScaleA * kScaleA)) + held[i][j][e + r] * (kMuonB * kScaleQ[1] / kScaleA) +
                                   (m == k + r && m < n ? kMuonA * kScaleQ[1] : 0.f);
        });
        const bool more = step + 1 < len;
        if (step || more) c.put(1, acc);   // P
        if (step == 0)
#pragma unroll
            for (int i = 0; i < C::MT; ++i)
#pragma unroll
                for (int j = 0; j < C::MT; ++j) q[i][j] = acc[i][j];
        __syncthreads();
        if (more) {
            c.multiply(1, 0, acc);   // P A
#pragma unroll
            for (int i = 0; i < C::MT; ++i)
#pragma unroll
                for (int j = 0; j < C::MT; ++j) acc[i][j] *= 1.f / kScaleQ[1];
            __syncthreads();
            c.put(0, acc);
            __syncthreads();
            c.multiply(0, 1, held);   // P A P
#pragma unroll
            for (int i = 0; i < C::MT; ++i)
#pragma unroll
                for (int j = 0; j < C::MT; ++j) held[i][j] *= 1.f / kScaleQ[1];
            __syncthreads();
        }
        if (step) {   // Q
            c.put(0, q);
            __syncthreads();
            c.multiply(1, 0, q);
            const float f = step == 1 ? kScaleQ[2] / (kScaleQ[1] * kScaleQ[1]) : kScaleQ[3] / (kScaleQ[1] * kScaleQ[2]);
#pragma unroll
            for (int i = 0; i < C::MT; ++i)
#pragma unroll
                for (int j = 0; j < C::MT; ++j) q[i][j] *= f;
            __syncthreads();
        }
        if (more) {
            c.put(0, held);
            __syncthreads();
        }
    }
    c.each4([&](int i, int j, int e, int m, int k) __attribute__((always_inline)) {
        typedef bf16_t V4 __attribute__((ext_vector_type(4)));
        if (m >= n || k >= ld) return;
#pragma unroll
        for (int p = 0; p < OUT; ++p) {
            V4 w;
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = PlaneEpi<OUT, true>::part(q[i][j][e + r], p);
            *(V4 *)(out + p * plane + (long long)m * ld + k) = w;
        }
    });
}

template <int OUT, int B>
int launch_chain(const bf16_t *a, bf16_t *q, long long plane, long long each, int n, int ld, int len, int items, hipStream_t s) {
    const LaunchPlan p = make_plan("muon_chain", {OUT, B}, {n, ld, len, items}, dim3((unsigned)items), 256, 2 * Chain<B>::PLACE);
    LC_PLAN_REQUIRE(p, n <= B && ld % 8 == 0 && ld >= n && ld < n + 8 && len >= 1 && len <= kGroupSteps);
    LC_LAUNCH(p, "muon_step (Q)", (muon_chain_kernel<OUT, B>), s, a, q, plane, each, n, ld, len);
    return LC_OK;
}

// ---------------------------------------------------------------------------------------------------------------------------
// X Q where rows are short, at most kShort values: a wave keeps Q and lets rows of X stream by, 32 at a time, from memory to registers and back.  Tiles
// through LDS begin and end once for each 64 rows and are wide for nobody (3249 of 768 x 16 in fp32: 198 us, and 298 where w is
// updated; 1485 of 5248 x 19 in bf16 506 and 1893).  Tall matrices only: few rows of many columns take tiles (1485 of 19 x 5248 in bf16 2.17 ms a step, 1.41
// lying the other way).
constexpr int kShort = 64, kShortBlocks = 4;   // blocks of 32 rows a wave
template <typename T, int PL, int PLANES, int NT, bool UPDATE>
__global__ __launch_bounds__(256) void muon_short_kernel(const bf16_t *x, long long plane, const bf16_t *q, long long qplane, int rows, int cols, int ld,
                                                         int groups, PlaneEpi<PLANES, false> to, UpdateEpi<T> up) {
    constexpr int KC = NT * 2;   // steps of 16 values of a row
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
    const long long item = blockIdx.x / groups;
    const int first = ((int)(blockIdx.x - item * groups) * 4 + wave) * (32 * kShortBlocks);
    x += item * rows * ld, q += item * cols * ld;
    if constexpr (UPDATE) up.item((int)item);
    else to.item((int)item);
    const u32x4 none = {0, 0, 0, 0};
    u32x4 b[PLANES][KC][NT];
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int n = 32 * j + l32, k = 16 * c + 8 * h;
                b[p][c][j] = n < cols && k < ld ? *(const u32x4 *)(q + p * qplane + n * ld + k) : none;
            }
#pragma unroll 2
    for (int i = 0; i < kShortBlocks; ++i) {
        const int m = first + 32 * i + l32;
        if (first + 32 * i >= rows) break;
        const long long row = min(m, rows - 1);
        u32x4 a[PLANES][KC];
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const int k = 16 * c + 8 * h;
                a[p][c] = k < ld ? *(const u32x4 *)(x + p * plane + row * ld + k) : none;
            }
        float old[NT][4][4];
        if constexpr (UPDATE) {
            const T *const w = up.w + row * cols;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int n = 32 * j + 8 * e + 4 * h;
                    T v[4];
                    if (n + 4 <= cols) {
                        __builtin_memcpy(v, w + n, sizeof(v));
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = w[min(n + r, cols - 1)];
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) old[j][e][r] = widen<T>(v[r]);
                }
        }
        f32x16 acc[NT] = {};
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int t = 0; t < Format<PL>::PAIRS; ++t)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[j] = Format<PL>::mul(b[Format<PL>::B >> (4 * t) & 1][c][j], a[Format<PL>::A >> (4 * t) & 1][c], acc[j]);
        if (m >= rows) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = 32 * j + 8 * e + 4 * h;
                if constexpr (UPDATE) {
                    T *const w = up.w_out + row * cols;
                    T o[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] = narrow<T>(up.keep * old[j][e][r] - up.rate * acc[j][4 * e + r]);
                    if (n + 4 <= cols) {
                        __builtin_memcpy(w + n, o, sizeof(o));
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n + r < cols) w[n + r] = o[r];
                    }
                } else if (n < ld) {   // zeros behind the last column: Q has none there
                    typedef bf16_t V4 __attribute__((ext_vector_type(4)));
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
                        V4 w;
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[r] = to.part(acc[j][4 * e + r] * to.factor, p);
                        *(V4 *)(to.out + p * to.plane + row * ld + n) = w;
                    }
                }
            }
    }
}

template <typename T, int PL, bool UPDATE, int PLANES>
int launch_short(const Operand &X, const Operand &Q, int rows, int cols, int items, const PlaneEpi<PLANES, false> &to, const UpdateEpi<T> &up, hipStream_t s) {
    const int groups = ceil_div(rows, 4 * 32 * kShortBlocks);
    const LaunchPlan p = make_plan("muon_short", {PL, UPDATE}, {rows, cols, (int)X.ld, items}, dim3((unsigned)((long long)items * groups)), 256, 0);
    LC_PLAN_REQUIRE(p, cols <= kShort && X.ld == Q.ld && X.ld % 8 == 0 && X.ld >= cols && X.ld < cols + 8 && (long long)items * groups <= 0x7fffffffLL);
    if (cols <= 32)
        LC_LAUNCH(p, "muon_step (X)", (muon_short_kernel<T, PL, PLANES, 1, UPDATE>), s, X.p0, X.plane, Q.p0, Q.plane, rows, cols, (int)X.ld, groups, to, up);
    else
        LC_LAUNCH(p, "muon_step (X)", (muon_short_kernel<T, PL, PLANES, 2, UPDATE>), s, X.p0, X.plane, Q.p0, Q.plane, rows, cols, (int)X.ld, groups, to, up);
    return LC_OK;
}

constexpr long long kStackBytes = 1LL << 30;   // of X's planes at a time
constexpr long long kScratchBytes = 4LL << 30, kRestBytes = 4 * kMostParts + 4096;   // of all that several matrices take; of parts, and of what rounds pieces up

// Products of `items` matrices: short sides, the long side, the update of X.
struct MuonShapes {
    Shape sq, sx, up;
    MuonShapes(int items, int rows, int cols) {
        const int small = std::min(rows, cols);
        sq = sx = Shape{small, small, small, nullptr, 0, nullptr, 0, 1, items, 1};
        sx.K = std::max(rows, cols);
        up = {rows, cols, small, nullptr, 0, nullptr, 0, 1, items, 0};
    }
};
// Steps that go by on the short side at a time: kGroupSteps, or one where the products with the long side cost no more by the estimate (no
// less than their bytes at 4.5 TB/s).  Both: 841 of 2048 x 128 in fp32 4.4 ms with one and 2.9 with three, two of 8192 x 4096 in bf16 5.3 and 4.2,
// 256 x 2000 in fp32 153 us and 134; two of 256 x 400 would take as many launches either way.  Square matrices have no longer side: as many products either way, and single steps round less.
inline double stack_us(const Shape &sh, int planes, int pairs, int how) {
    const double bytes = 2.0 * planes * sh.stack * ((double)sh.M * sh.K + (sh.sym ? 0.0 : (double)sh.Nn * sh.K) + (double)sh.M * sh.Nn);
    return std::max(choose_stack_cut(sh, pairs, how).us, bytes / 4.5e6);
}
inline int group_of(int items, int rows, int cols, int planes, int pairs) {
    if (std::min(rows, cols) <= kChain) return kGroupSteps;
    if (rows == cols) return 1;
    const MuonShapes k(items, rows, cols);
    const int by_rows = rows > cols ? 0 : ROWS_ONLY | BLOCKS;
    const double sq = stack_us(k.sq, planes, pairs, ROWS_ONLY | BLOCKS | MAY_SPLIT), sx = stack_us(k.sx, planes, pairs, by_rows | MAY_SPLIT),
                 up = stack_us(k.up, planes, pairs, rows > cols ? ROWS_ONLY | BLOCKS : BLOCKS);
    return sx + up > 3 * sq ? kGroupSteps : 1;
}

template <typename T>
struct MuonScratch {
    static constexpr int PLANES = MuonFormat<T>::N;
    int small, ld, lds, most, parts, group;   // the smaller side; values of a row of X, of what is small x small; items at a time; partial sums of a matrix
    double *partial;
    bf16_t *x[2], *s, *a = nullptr, *t = nullptr, *q[3] = {};
    Parts part = {};
    MuonScratch(Scratch &sc, int count, int rows, int cols) {
        small = std::min(rows, cols);
        ld = (int)round_up(cols, 8), lds = (int)round_up(small, 8);
        const long long values = (long long)rows * ld, each = (long long)small * lds;
        const bool chain = small <= kChain, grouped = !chain && rows != cols;   // whatever group_of says of a stack of this length
        parts = (int)std::min<long long>(kMostSums, ((long long)rows * cols + 8191) / 8192);
        const long long bytes = 8 * parts + 2 * (PLANES * (2 * values + (grouped ? 6 : 2) * each) + (chain ? 2 * each : 0));
        most = (int)std::max<long long>(1, std::min<long long>({count, kMostGroups, kStackBytes / (2 * PLANES * values), (kScratchBytes - kRestBytes) / bytes}));
        partial = sc.take<double>((long long)most * parts);
        for (auto &p : x) p = sc.take<bf16_t>(PLANES * most * values);
        const long long square = PLANES * most * each;
        s = sc.take<bf16_t>(square);
        q[0] = sc.take<bf16_t>(square);
        group = group_of(most, rows, cols, PLANES, Format<MuonFormat<T>::PL>::PAIRS);
        if (chain) a = sc.take<bf16_t>(2 * most * each);
        if (grouped)
            for (bf16_t **p : {&a, &t, &q[1], &q[2]}) *p = sc.take<bf16_t>(square);
        // of as many matrices as are cut along the contraction; a shorter stack may be cut into more parts
        const long long cut = std::min<long long>(most, (long long)(kSplitTiles / stack_tiles(MuonShapes(1, rows, cols).sx, 128)));
        part.floats = std::min(kMostParts, kMostSplits * cut * small * round_up(small, 4));
        part.at = sc.take<float>(part.floats);
    }
};

template <typename T>
int muon(const T *w, const T *g, const float *m, T *w_out, float *m_out, int count, int rows, int cols, float rate, float decay, float mu, bool ahead,
         int steps, void *ws, hipStream_t st) {
    constexpr int PL = MuonFormat<T>::PL, PLANES = MuonFormat<T>::N, PAIRS = Format<PL>::PAIRS;
    Scratch sc(ws);
    const MuonScratch<T> k(sc, count, rows, cols);
    const bool tall = rows > cols;
    const long long n = (long long)rows * cols, each = (long long)k.small * k.lds;
    const int groups = ceil_div(steps, k.group);
    for (int first = 0; first < count; first += k.most) {
        const int items = std::min(k.most, count - first);
        const long long skip = first * n, plane = (long long)k.most * rows * k.ld, splane = k.most * each;
        const LaunchPlan pm = make_plan("muon_momentum", {(int)sizeof(T)}, {items, rows, cols, k.parts}, dim3((unsigned)((long long)items * k.parts)), 256, 0);
        LC_PLAN_REQUIRE(pm, (long long)items * k.parts <= 0x7fffffffLL && (k.group == 1 || (k.group <= kGroupSteps && k.a)));
        LC_LAUNCH(pm, "muon_step (momentum)", (muon_momentum_kernel<T>), st, g + skip, m + skip, m_out + skip, k.partial, n, k.parts, mu, (int)ahead);
        const long long wgs = ((long long)rows * (k.ld / 8) + 256 * kStartPieces - 1) / (256 * kStartPieces);
        const LaunchPlan ps = make_plan("muon_start", {(int)sizeof(T)}, {items, rows, cols, k.ld}, dim3((unsigned)(items * wgs)), 256, 0);
        LC_PLAN_REQUIRE(ps, items * wgs <= 0x7fffffffLL);
        LC_LAUNCH(ps, "muon_step (start)", (muon_start_kernel<T, PLANES>), st, g + skip, m_out + skip, k.partial, k.x[0], plane, rows, cols, k.ld, k.parts,
                  (int)wgs, mu, (int)ahead);
        const auto square = [&](const bf16_t *p) { return Operand{p, p, k.lds, splane, k.small, 0, 0, each}; };
        const MuonShapes of(items, rows, cols);
        // `to` = left right / (scales of both), at the scale `scale`
        const auto multiply = [&](const char *name, const bf16_t *left, const bf16_t *right, bf16_t *to, bf16_t *to2, float factor, float diag, float diag2) {
            return launch_symmetric<PL, ROW, ROW>(name, square(left), square(right), of.sq, PlaneEpi<PLANES, true>{to, to2, splane, each, k.lds, factor, diag, diag2},
                                                  k.part, st);
        };
        int at = 0, rc;   // X's place
        for (int group = 0, done = 0; group < groups; ++group) {
            const int len = k.small > kLateSide ? ceil_div(steps - done, groups - group) : (steps - done) / (groups - group);
            const Operand X = {k.x[at], k.x[at], k.ld, plane, rows, 0, 0, (long long)rows * k.ld};
            Operand Xc = X;
            Xc.rows = k.ld;   // by columns
            const float fa = kScaleA / (kScaleX * kScaleX), fs = kShift * kScaleA;
            const bool chain = k.small <= kChain;
            const PlaneEpi<PLANES, true> ea = {len > 1 ? k.a : k.s, len > 1 ? k.s : nullptr, splane, each, k.lds, fa, len > 1 ? 0.f : fs, fs};
            const auto gram = [&](const auto &epi) {
                return tall ? launch_symmetric<PL, COL, COL>("muon_step (A)", Xc, Xc, of.sx, epi, k.part, st)
                            : launch_symmetric<PL, ROW, ROW>("muon_step (A)", X, X, of.sx, epi, k.part, st);
            };
            rc = chain ? gram(PlaneEpi<2, true>{k.a, nullptr, splane, each, k.lds, fa, 0.f, 0.f}) : gram(ea);
            if (rc) return rc;
            int q = 0;   // place of Q, the product of the group's P
            if (chain) {
                rc = k.small <= 64 ? launch_chain<PLANES, 64>(k.a, k.q[0], splane, each, k.small, k.lds, len, items, st)
                                   : launch_chain<PLANES, 128>(k.a, k.q[0], splane, each, k.small, k.lds, len, items, st);
                if (rc) return rc;
            }
            for (int i = 0; i < len && !chain; ++i) {
                const int p = i ? (q + 1) % 3 : 0;
                if ((rc = multiply("muon_step (P)", k.s, k.s, k.q[p], nullptr, kMuonC * kScaleQ[1] / (kScaleA * kScaleA), kRest * kScaleQ[1], 0.f))) return rc;
                if (i + 1 < len) {
                    if ((rc = multiply("muon_step (P A)", k.q[p], k.a, k.t, nullptr, 1.f / kScaleQ[1], 0.f, 0.f))) return rc;
                    if ((rc = multiply("muon_step (P A P)", k.t, k.q[p], k.a, k.s, 1.f / kScaleQ[1], 0.f, fs))) return rc;
                }
                if (i) {
                    const int to = (q + 2) % 3;
                    if ((rc = multiply("muon_step (Q)", k.q[p], k.q[q], k.q[to], nullptr, kScaleQ[i + 1] / (kScaleQ[1] * kScaleQ[i]), 0.f, 0.f))) return rc;
                    q = to;
                }
            }
            done += len;
            const Operand Q = square(k.q[q]);
            const PlaneEpi<PLANES, false> next = {k.x[1 - at], nullptr, plane, X.each, k.ld, 1.f / kScaleQ[len], 0.f, 0.f};
            const UpdateEpi<T> update = {w + skip, w_out + skip, n, cols, 1.f - decay, rate / (kScaleQ[len] * kScaleX)};
            const auto apply = [&](const auto &epi) {
                const StackCut cut = choose_stack_cut(of.up, PAIRS, tall ? ROWS_ONLY | BLOCKS : BLOCKS);
                return tall ? launch_stack<PL, ROW, ROW>("muon_step (X)", X, Q, of.up, cut, epi, st)
                            : launch_stack<PL, ROW, COL>("muon_step (X)", Q, Xc, of.up, cut, epi, st);
            };
            const bool last = done == steps;
            if (tall && cols <= kShort)
                rc = last ? launch_short<T, PL, true>(X, Q, rows, cols, items, next, update, st) : launch_short<T, PL, false>(X, Q, rows, cols, items, next, update, st);
            else
                rc = last ? apply(update) : apply(next);
            if (rc) return rc;
            at = 1 - at;
        }
    }
    return LC_OK;
}

template <typename T>
size_t muon_scratch(int count, int rows, int cols) {
    Scratch sc(nullptr);
    (void)MuonScratch<T>(sc, count, rows, cols);
    return sc.used;
}

}  // namespace head
}  // namespace lc
