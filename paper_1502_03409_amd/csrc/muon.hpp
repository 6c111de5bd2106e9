// A step of gradient descent whose update is the momentum with its singular values brought near one.
//
//   m' = mu m + g;  u = g + mu m' (looking ahead) or m';  X = u / |u|;  steps times  X <- a X + b (X X^T) X + c (X X^T)^2 X;
//   w' = (1 - decay) w - rate X.
//
// With S = X X^T + b / (2 c) I (or X^T X, whichever is smaller) the polynomial is P = c S S + (a - b^2 / (4 c)) I, and a step X <- P X:
// three products and nothing to add but on a diagonal.  S and P are symmetric: tiles below the diagonal are formed and stored twice.
//
// Between products X, S and P are held in fp16, times powers of two.  Singular values of X lie in [0, 1.203] throughout, because |u| bounds the
// largest and a s + b s^3 + c s^5 maps [0, 1.203] into itself, so no value of X, S, P exceeds 1.203, 1.176, 3.445 in magnitude and the powers
// put all of them at the upper end of fp16's range: what a rounding costs is 2^-12 of values that count, an eighth of bf16's, and small ones lose
// nothing below 2^-24 of the largest.  For bf16 weights one fp16 value is held; for fp32 weights two, a value and what its rounding leaves, 22 bits,
// and three products of them are formed.  Sums, norms and the momentum are fp32 and more.
#pragma once
#include "head_planes.hpp"
#include "head_gemm.hpp"

namespace lc {
namespace head {

constexpr float kMuonA = 3.4445f, kMuonB = -4.7750f, kMuonC = 2.0315f;
constexpr float kShift = kMuonB / (2.f * kMuonC), kRest = (float)(3.4445 - 4.7750 * 4.7750 / (4 * 2.0315));
constexpr float kScaleX = 0x1p14f, kScaleS = 0x1p14f, kScaleP = 0x1p13f;   // 1.203, 1.176 and 3.445 times these stay below 2^15
constexpr int kMostParts256 = 256;   // partial sums of a matrix's squares

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

// m' and the partial sums of u's squares, `parts` workgroups a matrix of n values; bound by HBM.
template <typename T>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const T *g, const float *m, float *m_out, double *partial, long long n, int parts, float mu,
                                                            int ahead) {
    const long long item = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    g += item * n, m += item * n, m_out += item * n;
    double s = 0.0;
    for (long long i = (part * 256LL + threadIdx.x) * 8; i < n; i += parts * 2048LL) {
        const int left = (int)min(n - i, 8LL);
        float a[8], b[8];
        load8(g + i, 0, left, a);
        load8(m + i, 0, left, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            b[e] = next_momentum(b[e], a[e], mu);
            const double u = looked_ahead(b[e], a[e], mu, ahead);
            if (e < left) s += u * u;
        }
        store8(m_out + i, b, left);
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
    const long long at = (blockIdx.x - item * groups) * 256LL + threadIdx.x;
    const int r = (int)(at / pieces), c = (int)(at - (long long)r * pieces) * 8;
    if (r >= rows) return;
    float a[8], b[8];
    load8(g + item * n + (long long)r * cols, c, cols, a);
    load8(m + item * n + (long long)r * cols, c, cols, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        b[e] = c + e < cols ? (float)((double)looked_ahead(b[e], a[e], mu, ahead) * f) : 0.f;   // 1 / |u| may be beyond fp32
    }
    put_halves<PLANES>(x + (item * rows + r) * ld + c, plane, b);
}

// A product as planes of fp16: times `factor`, `diag` added on the diagonal; zeros in the columns behind the last one up to ld.  MIRROR: the
// result is symmetric, tiles beside the diagonal go to their mirrored place as well.
template <int PLANES, bool MIRROR>
struct PlaneEpi {
    bf16_t *out;
    long long plane, each;
    int ld;
    float factor, diag;
    __device__ __forceinline__ void item(int i) { out += i * each; }
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
                    if (m < M && n0 + c < ld) *(u32x4 *)(out + p * plane + (long long)m * ld + n0 + c) = w;
                });
            }
        });
        if (!MIRROR || m0 / (MT * 64) == n0 / (NT * 64)) return;
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
                    if (n < Nn && m0 + c < ld) *(u32x4 *)(out + p * plane + (long long)n * ld + m0 + c) = w;
                });
            }
        });
    }
    static __device__ __forceinline__ bf16_t part(float v, int p) {
        const half_t a = (half_t)v;
        return p == 0 ? __builtin_bit_cast(bf16_t, a) : half_bits(v - (float)a);
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
};

constexpr long long kStackBytes = 1LL << 30;   // of X's planes at a time

template <typename T>
struct MuonScratch {
    static constexpr int PLANES = MuonFormat<T>::N;
    int small, ld, lds, most, parts;   // the smaller side; values of a row of X, of S and P; items at a time; partial sums of a matrix
    double *partial;
    bf16_t *x[2], *s, *p;
    MuonScratch(Scratch &sc, int count, int rows, int cols) {
        small = std::min(rows, cols);
        ld = (int)round_up(cols, 8), lds = (int)round_up(small, 8);
        const long long values = (long long)rows * ld;
        most = (int)std::max<long long>(1, std::min<long long>(count, kStackBytes / (2 * PLANES * values)));
        parts = (int)std::min<long long>(kMostParts256, ((long long)rows * cols + 8191) / 8192);
        partial = sc.take<double>((long long)most * parts);
        for (int i = 0; i < 2; ++i) x[i] = sc.take<bf16_t>(PLANES * most * values);
        s = sc.take<bf16_t>(PLANES * most * (long long)small * lds);
        p = sc.take<bf16_t>(PLANES * most * (long long)small * lds);
    }
};

template <typename T>
int muon(const T *w, const T *g, const float *m, T *w_out, float *m_out, int count, int rows, int cols, float rate, float decay, float mu, bool ahead,
         int steps, void *ws, hipStream_t st) {
    constexpr int PL = MuonFormat<T>::PL, PLANES = MuonFormat<T>::N;
    Scratch sc(ws);
    const MuonScratch<T> k(sc, count, rows, cols);
    const bool tall = rows > cols;
    const long long n = (long long)rows * cols;
    for (int first = 0; first < count; first += k.most) {
        const int items = std::min(k.most, count - first);
        const long long skip = first * n, plane = (long long)k.most * rows * k.ld, splane = (long long)k.most * k.small * k.lds;
        const LaunchPlan pm = make_plan("muon_momentum", {(int)sizeof(T)}, {items, rows, cols, k.parts}, dim3((unsigned)((long long)items * k.parts)), 256, 0);
        LC_PLAN_REQUIRE(pm, (long long)items * k.parts <= 0x7fffffffLL);
        LC_LAUNCH(pm, "muon_step (momentum)", (muon_momentum_kernel<T>), st, g + skip, m + skip, m_out + skip, k.partial, n, k.parts, mu, (int)ahead);
        const long long groups = ((long long)rows * (k.ld / 8) + 255) / 256;
        const LaunchPlan ps = make_plan("muon_start", {(int)sizeof(T)}, {items, rows, cols, k.ld}, dim3((unsigned)(items * groups)), 256, 0);
        LC_PLAN_REQUIRE(ps, items * groups <= 0x7fffffffLL);
        LC_LAUNCH(ps, "muon_step (start)", (muon_start_kernel<T, PLANES>), st, g + skip, m_out + skip, k.partial, k.x[0], plane, rows, cols, k.ld, k.parts,
                  (int)groups, mu, (int)ahead);
        const auto cut = [&](const Shape &sh) { return choose_cut(sh.M, sh.Nn, sh.K, Format<PL>::PAIRS, false, sh.stack, sh.sym); };
        const Operand S = {k.s, k.s, k.lds, splane, k.small, 0, 0, (long long)k.small * k.lds};
        const Operand P = {k.p, k.p, k.lds, splane, k.small, 0, 0, (long long)k.small * k.lds};
        const Shape sq = {k.small, k.small, k.small, nullptr, 0, nullptr, 0, 1, items, 1};
        Shape sx = sq;
        sx.K = tall ? rows : cols;
        Shape up = {rows, cols, k.small, nullptr, 0, nullptr, 0, 1, items, 0};
        for (int i = 0; i < steps; ++i) {
            const Operand X = {k.x[i & 1], k.x[i & 1], k.ld, plane, rows, 0, 0, (long long)rows * k.ld};
            Operand Xc = X;
            Xc.rows = k.ld;   // by columns
            const PlaneEpi<PLANES, true> es = {k.s, splane, S.each, k.lds, kScaleS / (kScaleX * kScaleX), kShift * kScaleS};
            const PlaneEpi<PLANES, true> ep = {k.p, splane, P.each, k.lds, kMuonC * kScaleP / (kScaleS * kScaleS), kRest * kScaleP};
            int rc = tall ? launch_cut<PL, COL, COL>("muon_step (S)", Xc, Xc, sx, cut(sx), es, st) : launch_cut<PL, ROW, ROW>("muon_step (S)", X, X, sx, cut(sx), es, st);
            if (rc) return rc;
            if ((rc = launch_cut<PL, ROW, ROW>("muon_step (P)", S, S, sq, cut(sq), ep, st))) return rc;
            const auto apply = [&](const auto &epi) {
                return tall ? launch_cut<PL, ROW, ROW>("muon_step (X)", X, P, up, cut(up), epi, st) : launch_cut<PL, ROW, COL>("muon_step (X)", P, Xc, up, cut(up), epi, st);
            };
            if (i + 1 < steps)
                rc = apply(PlaneEpi<PLANES, false>{k.x[~i & 1], plane, X.each, k.ld, 1.f / kScaleP, 0.f});
            else
                rc = apply(UpdateEpi<T>{w + skip, w_out + skip, n, cols, 1.f - decay, rate / (kScaleP * kScaleX)});
            if (rc) return rc;
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
