// Gated hidden layer: h = act(x wg^T) * (x wu^T) in one product kernel, and its gradients.
//
// Forward: a tile of the product covers the same outputs of both weight matrices (blocks of 32 rows of wg and wu alternate), so
// the activation and the product happen on the accumulators.  Backward: one pass over dh and the saved g, u leaves both
// gradients side by side, [N][2F], and two products finish: dx = [dg du] [wg; wu] and [dwg; dwu] = [dg du]^T x.  bf16 operands: rounded to bf16,
// up to kFewRows rows in two parts (as in xent.hpp; 1 row of 64 -> 64 was off by 0.26 %, where the results' own rounding is 0.17 %).
//
// 8192 x 4096 -> 8192 in bf16: forward 0.93 to 0.95 ms, the gradients' pass 0.12, dx 0.87 to 0.94, dw 0.97 to 0.99; each product is 1.1 TFLOP,
// bound as large products are.  192 rows: 40 us, the 134 MB of weights come at 3.4 TB/s.  1537 x 1021 -> 2055 in fp32: 0.37 ms for all.
#pragma once
#include "head_few.hpp"
#include "head_planes.hpp"

namespace lc {
namespace head {

// 1 / (1 + e^-g).  bf16 results: by the hardware's exponential and reciprocal, whose errors of 2^-22 vanish in the rounding.
template <typename T>
__device__ __forceinline__ float sigmoid(float g) {
    if constexpr (sizeof(T) == 4) return 1.f / (1.f + expf(-g));
    else return __builtin_amdgcn_rcpf(1.f + __expf(-g));
}
// 1 / (1 + e^-g) and 1 / (1 + e^g), which 1 minus the first would lose where a gate is open wide
template <typename T>
__device__ __forceinline__ void sigmoid_both(float g, float &s, float &rest) {
    const float e = sizeof(T) == 4 ? expf(-fabsf(g)) : __expf(-fabsf(g));
    const float more = sizeof(T) == 4 ? 1.f / (1.f + e) : __builtin_amdgcn_rcpf(1.f + e), less = e * more;
    s = g < 0.f ? less : more;
    rest = g < 0.f ? more : less;
}
template <typename T, int ACT>
__device__ __forceinline__ float act_value(float g) {
    if constexpr (ACT == LC_ACT_GELU) return 0.5f * g * erfcf(-0.70710678118654752f * g);
    const float sg = sigmoid<T>(g);
    return ACT == LC_ACT_SIGMOID ? sg : g * sg;
}
// act(g) and act'(g)
template <typename T, int ACT>
__device__ __forceinline__ void act_both(float g, float &a, float &da) {
    if constexpr (ACT == LC_ACT_GELU) {
        const float phi = 0.5f * erfcf(-0.70710678118654752f * g);
        a = g * phi;
        da = phi + g * (0.39894228040143268f * expf(-0.5f * g * g));
    } else {
        float sg, rest;
        sigmoid_both<T>(g, sg, rest);
        a = ACT == LC_ACT_SIGMOID ? sg : g * sg;
        da = ACT == LC_ACT_SIGMOID ? sg * rest : sg * (1.f + g * rest);
    }
}

// What the forward pass leaves of g and u for the backward pass.  fp32 operands: the values.  bf16 operands: 16 bits each, of which
// the first two are the sign and a mark: 0, five bits of exponent and nine of fraction for magnitudes from 2^-16 up to 2^16; 1, the eight
// bits of the fp32 exponent and six of fraction for all others, zero, infinities and NaN among them.  bf16's eight significant bits
// would show in the gradients (each would be rounded four times in all instead of twice); these ten do not.
__device__ __forceinline__ float saved_value(float v) { return v; }
__device__ __forceinline__ float saved_value(bf16_t c) {
    const unsigned sign = (unsigned)(c & 0x8000u) << 16;
    const unsigned near = ((unsigned)(c & 0x3fffu) << 14) + (111u << 23), far = (unsigned)(c & 0x3fffu) << 17;
    return __builtin_bit_cast(float, sign | ((c & 0x4000u) ? far : near));
}
template <typename T> __device__ __forceinline__ T save_value(float v);
template <> __device__ __forceinline__ bf16_t save_value<bf16_t>(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v), sign = (u >> 16) & 0x8000u, mag = u & 0x7fffffffu;
    const unsigned near = (mag + 0x1fffu + ((mag >> 14) & 1u)) >> 14;   // nearest, ties to even; a carry moves to the next exponent
    if (near >= (111u << 9) && near < (143u << 9)) return (bf16_t)(sign | (near - (111u << 9)));
    const unsigned far = mag > 0x7f800000u    ? (mag >> 17) | 0x20u          // NaN
                         : mag == 0x7f800000u ? mag >> 17
                                              : min((mag + 0xffffu + ((mag >> 17) & 1u)) >> 17, 0x3fbfu);   // what is finite stays so
    return (bf16_t)(sign | 0x4000u | far);
}
// Four at a time: the marked form is rare, and a wave passes it by where no lane has it (8192 rows of 4096 -> 8192: 0.94 ms, 1.02 with both
// forms made for every value and one taken).
__device__ __forceinline__ void save_values(const float (&v)[4], float (&o)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = v[r];
}
__device__ __forceinline__ void save_values(const float (&v)[4], bf16_t (&o)[4]) {
    unsigned most = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const unsigned u = __builtin_bit_cast(unsigned, v[r]), mag = u & 0x7fffffffu;
        const unsigned near = ((mag + 0x1fffu + ((mag >> 14) & 1u)) >> 14) - (111u << 9);
        most = max(most, near);
        o[r] = (bf16_t)((u >> 16 & 0x8000u) | near);
    }
    if (__builtin_expect(most >= 32u << 9, 0))
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = save_value<bf16_t>(v[r]);
}
// EACH 32: blocks j = 0, 2, .. of a wave are g, blocks 1, 3, .. the u of the same outputs; 16: every block holds both of 16 outputs.
template <typename T, int ACT, int EACH = 32>
struct GluEpi {
    T *h, *gu;   // gu may be null
    int F;
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int, int, char *lds) const {
        static_assert(EACH == 16 || NT % 2 == 0, "g and u of an output sit in neighbouring blocks or in one");
        const RowStage<T, NT * 16> stage = {lds, lane};
        const int f0 = n0 / 2;
        // what: 0 h, 1 g, 2 u
        auto send = [&](auto block, auto what, T *out, int ld) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value, W = decltype(what)::value;
#pragma unroll
            for (int j = 0; j < NT; j += EACH / 16)
#pragma unroll
                for (int q = 0; q < EACH / 8; ++q) {
                    T v[4];
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float g = acc[i][j][4 * q + r];
                        const float u = EACH == 16 ? acc[i][j][(8 + 4 * q + r) & 15] : acc[i][j + EACH / 32][4 * q + r];
                        if constexpr (W == 0) v[r] = narrow<T>(act_value<T, ACT>(g) * u);
                        else x[r] = W == 1 ? g : u;
                    }
                    if constexpr (W != 0) save_values(x, v);
                    stage.put(16 * j + 8 * q + 4 * (lane >> 5), v);
                }
            stage.take([&](int r, int c, const u32x4 &w) {
                const int m = m0 + 32 * i + r;
                if (m < M) store_piece(out + (long long)m * ld, f0 + c, F, w);
            });
        };
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            send(block, std::integral_constant<int, 0>(), h, F);
            if (gu) {
                send(block, std::integral_constant<int, 1>(), gu, 2 * F);
                send(block, std::integral_constant<int, 2>(), gu + F, 2 * F);
            }
        });
    }
};

// dg = dh u act'(g) and du = dh act(g), for the rows of both.  Bound by HBM: 8192 x 8192 in bf16 reads 403 MB and writes 268 MB in 0.12 ms.
template <typename T, int ACT>
struct GluGrad {
    const T *dh, *gu;
    int F, N;
    __device__ long long rows() const { return N; }
    __device__ void beside() const {}
    __device__ bool skip(int) const { return false; }
    __device__ void operator()(int r, int c, float (&v)[2][8]) const {
        float d[8], g[8], u[8];
        load8(dh + (long long)r * F, c, F, d);
        const T *p = gu + (long long)r * 2 * F;
        if (sizeof(T) == 2 && c + 8 <= F) {
            typedef u32x4 any __attribute__((aligned(2)));
            const u32x4 a = *(const any *)(p + c), b = *(const any *)(p + F + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = saved_value((bf16_t)(a[e >> 1] >> (16 * (e & 1))));
                u[e] = saved_value((bf16_t)(b[e >> 1] >> (16 * (e & 1))));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = c + e < F ? saved_value(p[c + e]) : 0.f;
                u[e] = c + e < F ? saved_value(p[F + c + e]) : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a, da;
            act_both<T, ACT>(g[e], a, da);
            v[0][e] = d[e] * u[e] * da;
            v[1][e] = d[e] * a;
        }
    }
};

template <typename T>
__global__ __launch_bounds__(256) void fill_zero_kernel(T *p, long long n) {
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) p[i] = 0;
}
template <typename T>
int launch_fill_zero(T *p, long long n, hipStream_t s) {
    const LaunchPlan pl = make_plan("glu_fill", {}, {}, dim3((unsigned)std::min<long long>((n + 255) / 256, 4096)), 256, 0);
    LC_LAUNCH(pl, "glu_bwd (no rows)", (fill_zero_kernel<T>), s, p, n);
    return LC_OK;
}

// the rows of x, wg and wu, one below the other
template <typename T>
struct Stacked {
    const T *x, *wg, *wu;
    int N, F, D;
    __device__ void beside() const {}
    __device__ bool skip(int) const { return false; }
    __device__ void operator()(int r, int c, float (&v)[1][8]) const {
        const T *p = r < N ? x + (long long)r * D : r - N < F ? wg + (long long)(r - N) * D : wu + (long long)(r - N - F) * D;
        load8(p, c, D, v[0]);
    }
};

template <typename T>
struct GluScratch {
    static constexpr int PL = Planes<T>::N;
    int Dp, Fp;
    bool direct;   // x and the weights are used where they are
    bf16_t *x, *w, *d;
    Parts part = {};   // one product at a time
    GluScratch(Scratch &sc, int N, int D, int F, bool backward) {
        Dp = (int)round_up(D, 8), Fp = (int)round_up(F, kStep);
        direct = PL == 1 && D == Dp;
        // few rows: the forward pass takes everything where it is
        x = sc.take<bf16_t>(direct || (N <= kFewRows && !backward) ? 8 : PL * ((long long)N + 2LL * F) * Dp);
        w = x ? x + (long long)N * Dp : nullptr;   // behind x in each plane, so that one launch lays all three out
        // rows of the gradients' two parts, for any number of rows up to N
        const int twice = PL == 1 && backward ? 2 * std::min(N, kFewRows) : 0;
        d = backward ? sc.take<bf16_t>(2LL * Fp * std::max(PL * N, twice)) : nullptr;
        if (!backward) return;
        part.floats = std::max({part_floats(std::max(N, twice), D, Fp + F), part_floats(2 * Fp, D, N), twice * round_up(D, 4)});
        part.at = sc.take<float>(part.floats);
    }
    // x and both weights as operands: laid out first unless they are where they can be used
    int operands(const T *xs, const T *wg, const T *wu, int N, int D, int F, Operand *X, Operand *W, hipStream_t s) const {
        if (direct) {
            *X = {(const bf16_t *)xs, (const bf16_t *)xs, D, 0, N, 0, 0};
            *W = {(const bf16_t *)wg, (const bf16_t *)wu, D, 0, F, 0, 0};
            return LC_OK;
        }
        const long long plane = ((long long)N + 2LL * F) * Dp;
        *X = {x, x, Dp, plane, N, 0, 0};
        *W = {w, w + (long long)F * Dp, Dp, plane, F, 0, 0};
        return launch_planes<PL, 1>("glu (x, w)", Stacked<T>{xs, wg, wu, N, F, D}, x, Dp, plane, N + 2 * F, Dp, 0, s);
    }
};

template <typename T, int ACT>
int glu_forward(const T *x, const T *wg, const T *wu, T *h, T *gu, int N, int D, int F, void *ws, hipStream_t s) {
    constexpr int PL = Planes<T>::N;
    if (N <= kFewRows)
        return launch_few<T, PAIR>("glu_fwd (few rows)", FewOperand<T>{x, x, D, N, nullptr}, FewOperand<T>{wg, wu, D, F, nullptr}, N, nullptr,
                                   2 * (int)round_up(F, 16), D, GluEpi<T, ACT, 16>{h, gu, F}, s);
    Scratch sc(ws);
    const GluScratch<T> g(sc, N, D, F, false);
    Operand X, W;
    if (int rc = g.operands(x, wg, wu, N, D, F, &X, &W, s)) return rc;
    const Shape sh = {N, 2 * (int)round_up(F, 32), D, nullptr, 0, nullptr, 0};
    return launch_gemm<PL, ROW, PAIR>("glu_fwd", X, W, sh, GluEpi<T, ACT>{h, gu, F}, s);
}

template <typename T, int ACT>
int glu_backward(const T *x, const T *wg, const T *wu, const T *gu, const T *dh, T *dx, T *dwg, T *dwu, int N, int D, int F,
                 void *ws, hipStream_t s) {
    constexpr int PL = Planes<T>::N;
    if (N == 0) {
        if (int rc = launch_fill_zero(dwg, (long long)F * D, s)) return rc;
        return launch_fill_zero(dwu, (long long)F * D, s);
    }
    Scratch sc(ws);
    const GluScratch<T> g(sc, N, D, F, true);
    Operand X, W;
    if (int rc = g.operands(x, wg, wu, N, D, F, &X, &W, s)) return rc;
    const int F2 = 2 * g.Fp;
    const long long pd = (long long)N * F2;
    if constexpr (PL == 1)
        if (N <= kFewRows) {
            const int two = 2 * N;
            if (int rc = launch_planes<2, 2>("glu_bwd (gradients)", GluGrad<T, ACT>{dh, gu, F, N}, g.d, F2, 0, N, g.Fp, g.Fp, s)) return rc;
            Operand d = {g.d, g.d, F2, 0, two, 0, 0};
            if (dx) {
                W.depth = F, W.half = g.Fp, W.rows = g.Dp;
                const Shape sh = {two, D, g.Fp + F, nullptr, 0, nullptr, 0};
                if (int rc = launch_product<PL, ROW, COLPAIR, true>("glu_bwd (dx)", d, W, sh,
                                                                    StoreEpi<T>{dx, nullptr, 0x7fffffff, N, 0, D, nullptr, nullptr, nullptr}, g.part, s))
                    return rc;
            }
            d.rows = F2, X.rows = g.Dp;
            const Shape sh = {F2, D, two, nullptr, 0, nullptr, 0};
            return launch_gemm<2, COL, COL>("glu_bwd (dw)", d, X, sh, StoreEpi<T>{dwg, dwu, g.Fp, F, F, D, nullptr, nullptr, nullptr}, s);
        }
    const Operand dgu = {g.d, g.d, F2, pd, N, 0, 0};
    if (int rc = launch_planes<PL, 2>("glu_bwd (gradients)", GluGrad<T, ACT>{dh, gu, F, N}, g.d, F2, pd, N, g.Fp, g.Fp, s)) return rc;
    if (dx) {
        W.depth = F, W.half = g.Fp, W.rows = g.Dp;
        const Shape sh = {N, D, g.Fp + F, nullptr, 0, nullptr, 0};
        if (int rc = launch_product<PL, ROW, COLPAIR>("glu_bwd (dx)", dgu, W, sh,
                                                   StoreEpi<T>{dx, nullptr, 0x7fffffff, N, 0, D, nullptr, nullptr, nullptr}, g.part, s))
            return rc;
    }
    Operand dT = dgu;
    dT.rows = F2, X.rows = g.Dp;
    const Shape sh = {F2, D, N, nullptr, 0, nullptr, 0};
    return launch_product<PL, COL, COL>("glu_bwd (dw)", dT, X, sh, StoreEpi<T>{dwg, dwu, g.Fp, F, F, D, nullptr, nullptr, nullptr}, g.part, s);
}

// The two operators for one type; instantiated in a source file each.
template <typename Fn>
int by_act(int act, const Fn &fn) {
    switch (act) {
        case LC_ACT_SIGMOID: return fn(std::integral_constant<int, LC_ACT_SIGMOID>());
        case LC_ACT_SILU: return fn(std::integral_constant<int, LC_ACT_SILU>());
        default: return fn(std::integral_constant<int, LC_ACT_GELU>());
    }
}

template <typename T>
int glu_forward(int act, const T *x, const T *wg, const T *wu, T *h, T *gu, int N, int D, int F, void *ws, hipStream_t s) {
    return by_act(act, [&](auto a) { return glu_forward<T, a>(x, wg, wu, h, gu, N, D, F, ws, s); });
}
template <typename T>
int glu_backward(int act, const T *x, const T *wg, const T *wu, const T *gu, const T *dh, T *dx, T *dwg, T *dwu, int N, int D, int F,
                 void *ws, hipStream_t s) {
    return by_act(act, [&](auto a) { return glu_backward<T, a>(x, wg, wu, gu, dh, dx, dwg, dwu, N, D, F, ws, s); });
}
template <typename T>
size_t glu_scratch(int N, int D, int F, bool backward) {
    Scratch sc(nullptr);
    (void)GluScratch<T>(sc, N, D, F, backward);
    return sc.used;
}

}  // namespace head
}  // namespace lc
