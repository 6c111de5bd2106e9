// Products with 8-bit weights: y[n][f] = sx[n] sw[f] sum_d qx[n][d] qw[f][d], and the gated layer formed so.
//
// A row of values x becomes whole numbers q = x / s to nearest, ties to even, with s = max |x| / 127 (no less than 2^-126, so that it has all
// its bits).  Rows of q take whole blocks of 128 bytes, zeros behind the last value, so no product has a rest to look after.  Products of whole
// numbers and their sums are exact (32 bits hold 2^17 products of 127 x 127); the sums become fp32 and take both scales before what
// follows the product, and are rounded once.
//
// The matrix instruction multiplies twice as many 8-bit as 16-bit numbers in the same time and from the same bytes.  8192 rows of 4096 -> 8192, gated,
// bf16: 36 us for the rows (100 MB) and 0.46 to 0.5 ms for the products, 2.2 to 2.4 POP/s, with the matrix unit busy 64 % of the cycles at 1.65 GHz.
// 192 rows over 100003 words: 153 us, where the weights' bytes take 88 and the products about 75; loads are waited for while tiles begin and end.
//
// Up to kFewRows rows: single blocks of 32 columns a workgroup, which fill the compute units more evenly than pairs and wait for more loads at
// once (1 x 4096 times 8192 16.5 us with two blocks, 14.9 with one; times 50000 60 and 47; gated, 4096 -> 20011, 47 and 37).
#pragma once
#include "glu.hpp"

namespace lc {
namespace head {

constexpr int kQ8Block = 128;              // bytes
constexpr int kQ8Most = 1 << 17;           // values of a row
inline int q8_ld(int D) { return (int)round_up(D, kQ8Block); }

// x / s to the nearest whole number, ties to even.  The first guess is off by one at most, and only next to a half; what the guess leaves of
// x is exact (a multiple of half a unit of s's last place, less than 2^24 of them), so the comparison with s / 2 decides as the quotient itself would.
__device__ __forceinline__ int nearest_whole(float x, float s, float inv) {
    float r = rintf(x * inv);
    const float rest = __builtin_fmaf(-r, s, x), half = 0.5f * s;
    const bool odd = (int)r & 1;
    if (rest > half || (odd && rest == half)) r += 1.f;
    if (rest < -half || (odd && rest == -half)) r -= 1.f;
    return (int)fminf(fmaxf(r, -127.f), 127.f);
}

// A workgroup a row, twice over its values, the second time from the caches.  Bound by HBM for many rows, by latency for few.
template <typename T>
__global__ __launch_bounds__(256) void q8_rows_kernel(const T *x, int8_t *q, float *scale, int D, int ld) {
    const long long n = blockIdx.x;
    const T *row = x + n * D;
    unsigned most = 0;   // of the magnitudes as whole numbers: infinities and NaN are larger than all others
    for (int c = threadIdx.x * 8; c < D; c += 2048) {
        float v[8];
        load8(row, c, D, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(unsigned, v[e]) & 0x7fffffffu);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, (unsigned)__shfl_xor((int)most, d));
    __shared__ unsigned tops[4];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    const bool fine = most < 0x7f800000u;
    const float s = fmaxf(__builtin_bit_cast(float, most) / 127.f, 0x1p-126f), inv = 1.f / s;
    if (threadIdx.x == 0) scale[n] = fine ? s : __builtin_nanf("");
    for (int c = threadIdx.x * 8; c < ld; c += 2048) {
        float v[8];
        load8(row, c, D, v);
        u32x2 w = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= (unsigned)((fine ? nearest_whole(v[e], s, inv) : 0) & 0xff) << (8 * (e & 3));
        *(u32x2 *)(q + n * ld + c) = w;
    }
}

template <typename T>
int q8_rows(const T *x, int8_t *q, float *scale, int N, int D, hipStream_t s) {
    const int ld = q8_ld(D);
    for (long long first = 0; first < N; first += kMostGroups) {
        const int some = (int)std::min(N - first, kMostGroups);
        const LaunchPlan p = make_plan("q8_rows", {(int)sizeof(T)}, {some, D, ld}, dim3(some), 256, 0);
        LC_LAUNCH(p, "q8_rows", (q8_rows_kernel<T>), s, x + first * D, q + first * ld, scale + first, D, ld);
    }
    return LC_OK;
}

// The sums times both scales, then what the inner epilogue does with the result.  EACH: 0, or the outputs of each of two matrices that a
// product's columns take in turn.
template <typename Inner, int EACH>
struct ScaledEpi {
    Inner inner;
    const float *sx, *sw0, *sw1;
    int F;
    template <int MT, int NT>
    __device__ __forceinline__ void run(i32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int Nn, int split, char *lds) const {
        f32x16 out[MT][NT];
        float row[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) row[i] = sx[min(m0 + 32 * i + (lane & 31), M - 1)];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                int f = n0 + 32 * j + 8 * q + 4 * (lane >> 5), second = 0;
                if constexpr (EACH != 0) f = pair_row(f, EACH, &second);
                const float *const sw = second ? sw1 : sw0;
                float s[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = sw[min(f + r, F - 1)];
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[i][j][4 * q + r] = (float)acc[i][j][4 * q + r] * s[r] * row[i];
            }
        inner.template run<MT, NT>(out, m0, n0, lane, M, Nn, split, lds);
    }
};

template <typename T>
struct Q8Scratch {
    int8_t *q;
    float *scale;
    Q8Scratch(Scratch &sc, int N, int D) {
        q = sc.take<int8_t>((long long)N * q8_ld(D));
        scale = sc.take<float>(N);
    }
};

inline Operand bytes_operand(const int8_t *p0, const int8_t *p1, int ld, int rows) {
    return {(const bf16_t *)p0, (const bf16_t *)p1, ld / 2, 0, rows, 0, 0};
}

template <typename T>
int q8_matmul(const T *x, const int8_t *qw, const float *sw, T *y, int N, int D, int F, void *ws, hipStream_t s) {
    Scratch sc(ws);
    const Q8Scratch<T> g(sc, N, D);
    const int ld = q8_ld(D);
    if (int rc = q8_rows<T>(x, g.q, g.scale, N, D, s)) return rc;
    const ScaledEpi<StoreEpi<T>, 0> epi = {StoreEpi<T>{y, nullptr, 0x7fffffff, N, 0, F, nullptr, nullptr, nullptr}, g.scale, sw, sw, F};
    if (N <= kFewRows)
        return launch_blocks<int8_t, ROW, 1>("q8_matmul (few rows)", FewOperand<int8_t>{g.q, g.q, ld, N, nullptr}, FewOperand<int8_t>{qw, qw, ld, F, nullptr}, N,
                                       nullptr, F, ld, epi, s);
    const Shape sh = {N, F, ld / 2, nullptr, 0, nullptr, 0};
    const Operand X = bytes_operand(g.q, g.q, ld, N), W = bytes_operand(qw, qw, ld, F);
    if (N <= 64) return launch_narrow<BYTES, ROW, 64>("q8_matmul", X, W, sh, epi, s);
    if (N <= kNarrow) return launch_narrow<BYTES, ROW, 128>("q8_matmul", X, W, sh, epi, s);
    return launch_gemm<BYTES, ROW, ROW, 8>("q8_matmul", X, W, sh, epi, s);
}

template <typename T, int ACT>
int q8_glu(const T *x, const int8_t *qg, const float *sg, const int8_t *qu, const float *su, T *h, int N, int D, int F, void *ws, hipStream_t s) {
    Scratch sc(ws);
    const Q8Scratch<T> g(sc, N, D);
    const int ld = q8_ld(D);
    if (int rc = q8_rows<T>(x, g.q, g.scale, N, D, s)) return rc;
    if (N <= kFewRows)
        return launch_blocks<int8_t, PAIR, 1>("q8_glu_fwd (few rows)", FewOperand<int8_t>{g.q, g.q, ld, N, nullptr}, FewOperand<int8_t>{qg, qu, ld, F, nullptr}, N,
                                        nullptr, 2 * (int)round_up(F, 16), ld,
                                        ScaledEpi<GluEpi<T, ACT, 16>, 16>{GluEpi<T, ACT, 16>{h, nullptr, F}, g.scale, sg, su, F}, s);
    const Shape sh = {N, 2 * (int)round_up(F, 32), ld / 2, nullptr, 0, nullptr, 0};
    const Operand X = bytes_operand(g.q, g.q, ld, N), W = bytes_operand(qg, qu, ld, F);
    const ScaledEpi<GluEpi<T, ACT>, 32> epi = {GluEpi<T, ACT>{h, nullptr, F}, g.scale, sg, su, F};
    if (N <= kNarrow) return launch_narrow<BYTES, PAIR, 128>("q8_glu_fwd", X, W, sh, epi, s);
    return launch_gemm<BYTES, ROW, PAIR, 8>("q8_glu_fwd", X, W, sh, epi, s);
}
template <typename T>
int q8_glu(int act, const T *x, const int8_t *qg, const float *sg, const int8_t *qu, const float *su, T *h, int N, int D, int F, void *ws,
           hipStream_t s) {
    return by_act(act, [&](auto a) { return q8_glu<T, a>(x, qg, sg, qu, su, h, N, D, F, ws, s); });
}

template <typename T>
size_t q8_scratch(int N, int D) {
    Scratch sc(nullptr);
    (void)Q8Scratch<T>(sc, N, D);
    return sc.used;
}

}  // namespace head
}  // namespace lc
