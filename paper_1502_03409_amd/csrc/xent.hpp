// Softmax cross entropy over a vocabulary, projection included, with its gradients.
//
// The scores l = x w^T are never stored as such: each tile of the product leaves, per row, its largest score and the sum of
// the exponentials below it, and a small kernel joins the tiles.  The target's own score is kept out of both and apart: with z the
// logarithm of the other words' sum minus the target's score, loss = log(1 + e^z) and p(target) - 1 = -1 / (1 + e^-z), neither of
// which cancels in rows that are already learned.  With gradients a tile also leaves the
// exponentials themselves (bf16 operands: relative to the tile's largest score, in 16 bits, ten of them significant, over the whole range of
// fp32: a quarter of the rounding to bf16 that follows, and no word is too rare; fp32: the scores), for a bounded number of rows at a
// time; one pass turns them into d[n][v] = s[n] (p[n][v] - [v = t]) in place, and two products give dx = d w and dw = d^T x.
//
// 8192 rows of 4096 over 128000 words in bf16, a tenth masked: scores 6.5 to 6.7 ms, statistics 0.03, d 0.76, dx 6.3 to 6.5, dw 6.6 to 6.8;
// three products of 7.7 TFLOP each, bound as large products are.
//
// Masked rows take no part: the rows that count are gathered first, and every kernel runs over as many as there are.
//
// d meets bf16 operands as bf16, one rounding more than the sums in fp32 would have.  Over many rows that is the rounding of as many numbers;
// of few rows a few weights of rows decide what is lost (6 rows with weights of their own: 0.28 % of dx and dw, where their own rounding is
// 0.17 %).  Up to kFewRows rows are therefore kept in two bf16 parts, sixteen bits, all second parts behind all first ones: as twice
// the rows of dx's product, which its tiles of 128 have room for and whose halves are added up with its parts, and as twice the indices
// of dw's, which its steps of 64 have room for.
#pragma once
#include "head_few.hpp"
#include "head_planes.hpp"

namespace lc {
namespace head {

constexpr long long kBlockBytes = 2LL << 30;   // exponentials kept at a time

struct Rows {
    int *count;
    int *place;            // of every row: its position among those that count, or -1
    int *index, *target;   // by position
    float *scale, *tl;     // weight in the cost, but for the factor *unit; the target's score
    float *unit;           // 1 / count for the mean, else 1: the results' factor, so that d = p - [v = t] is what is rounded
    // p = exp((l - base) - log_sum): the largest score, and the logarithm of the sum of the exponentials relative to it.  As one number
    // their sum would be rounded at the scores' size, and all of a row's probabilities with it.
    float *base, *log_sum;
    float *dt, *loss;      // p(target) - 1; loss
};

// Positions of the rows that count, in order; loss 0 where masked.  One workgroup: a scan over 1024 rows at a time
// (2 us, a launch's latency, up to that many).
static __global__ __launch_bounds__(1024) void rows_kernel(const int64_t *target, const float *scale, float *loss, int N, int V, Rows o) {
    __shared__ int part[16];
    __shared__ int total;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    for (int n0 = 0; n0 < N; n0 += 1024) {
        const int n = n0 + threadIdx.x;
        const long long t = n < N ? target[n] : -1;
        const bool in = t >= 0;
        const unsigned long long mask = __ballot(in);
        if (lane == 0) part[wave] = __popcll(mask);
        __syncthreads();
        int at = total;
        for (int w = 0; w < wave; ++w) at += part[w];
        at += __popcll(mask & ((1ull << lane) - 1));
        if (n < N) o.place[n] = in ? at : -1;
        if (in) {
            o.index[at] = n;
            o.target[at] = t < V ? (int)t : -1;
            o.tl[at] = __builtin_nanf("");      // stays where no column is the target
            o.scale[at] = t >= V ? __builtin_nanf("") : scale ? scale[n] : 1.f;
        } else if (n < N) {
            loss[n] = 0.f;
        }
        __syncthreads();
        if (threadIdx.x == 0)
            for (int w = 0; w < 16; ++w) total += part[w];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *o.count = total;
        *o.unit = scale ? 1.f : 1.f / (float)max(total, 1);
    }
}

template <typename T> struct Kept;   // what a tile leaves for the gradient
template <> struct Kept<float> { typedef float V; };
template <> struct Kept<bf16_t> { typedef unsigned short V; };
__device__ __forceinline__ float kept(float, float l, float) { return l; }                                     // score l
// exponential e, 0 to 1: sign and first bit of fp32's exponent are zero, the next sixteen are kept, to nearest (NaN: the row's statistics
// have it)
__device__ __forceinline__ unsigned short kept(unsigned short, float, float e) {
    return (unsigned short)((__builtin_bit_cast(unsigned, e) + 0x2000u) >> 14);
}

// Per wave and row: the largest score, the sum of exponentials (both without the target), the target's score, and with KEEP what
// the gradient needs.
template <typename T, bool KEEP>
struct XentEpi {
    float2 *stats;       // [wave's columns][stats_ld]
    long long stats_ld;
    const int *target;
    float *tl;
    typename Kept<T>::V *keep;   // [M][ld], ld a multiple of 64 that holds all columns: exponentials (bf16) or scores (fp32)
    long long ld;
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int V, int, char *lds) const {
        typedef typename Kept<T>::V K;
        const RowStage<K, NT * 32> stage = {lds, lane};
        const int h = lane >> 5;
        int targets[MT];   // all before the first store: a load behind a store waits until that has reached memory
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = m0 + 32 * i + (lane & 31);
            targets[i] = m < M ? target[m] : -1;
        }
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value;
            const int m = m0 + 32 * i + (lane & 31);
            // columns of this wave that exist, and the target's, as this lane counts: 0 .. 3, 8 .. 11, ..
            int end = V - n0 - 4 * h, at = targets[i] - n0 - 4 * h;
            asm volatile("" : "+v"(end), "+v"(at));   // compared anew for every block of rows: the masks of all would not fit
            // the target and what lies beyond the vocabulary are taken out, where there is any of it
            if (__any(end < NT * 32 || (at >= 0 && at < NT * 32))) {
                float own = 0.f;
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int c = 32 * j + 8 * (e >> 2) + (e & 3);
                        const float l = acc[i][j][e];
                        own = c == at ? l : own;
                        acc[i][j][e] = c == at || c >= end ? -__builtin_inff() : l;
                    }
                if (m < M && at >= 0 && at < NT * 32 && (at & 4) == 0) tl[m] = own;
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -__builtin_inff() ? 0.f : top;   // all scores -inf: exponentials of 0, not of NaN
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    K v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float l = acc[i][j][4 * q + r];
                        const float e = sizeof(T) == 4 ? expf(l - base) : __builtin_amdgcn_exp2f((l - base) * 1.44269504f);
                        sum += e;
                        v[r] = kept(K(), l, e);
                    }
                    if (KEEP) stage.put(32 * j + 8 * q + 4 * h, v);
                }
            if (KEEP)
                stage.take([&](int r, int c, const u32x4 &w) {
                    const int to = m0 + 32 * i + r;
                    if (to < M && n0 + c < ld) *(u32x4 *)(keep + to * ld + n0 + c) = w;
                });
            sum += __shfl_xor(sum, 32);
            if (m < M && h == 0) stats[(n0 / (NT * 32)) * stats_ld + m] = make_float2(top, sum);
        });
    }
};

// Joins the tiles of R rows: 256 / R threads a row, each over its share of the tiles, in a fixed order.  16 rows read whole lines of
// the statistics; with few rows the share of a thread matters more (one row of 1563 tiles: 4 instead of 38 us).  Bound by latency: 5 us for
// 192 rows of 313 tiles, 25 for 8192 rows of 1000.
template <int R>
static __global__ __launch_bounds__(256) void lse_kernel(const float2 *stats, long long stats_ld, int tiles, Rows o, int first, int most,
                                                  float *loss) {
    constexpr int P = 256 / R;
    const int M = live(most, o.count, first);
    const int row = threadIdx.x % R, part = threadIdx.x / R, m = blockIdx.x * R + row;
    __shared__ float tops[P][R + 1], sums[P][R + 1];
    float top = -__builtin_inff(), sum = 0.f;
    auto join = [&](float t, float s) {
        if (t > top) {
            sum = sum * expf(top - t) + s;
            top = t;
        } else if (t != -__builtin_inff()) {
            sum += s * expf(t - top);
        } else {
            sum += s * 0.f;   // nothing, unless it is NaN
        }
    };
    if (m < M)
        for (int t = part; t < tiles; t += 4 * P) {   // four loads in flight
            float2 s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = stats[min(t + k * P, tiles - 1) * stats_ld + m];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (t + k * P < tiles) join(s[k].x, s[k].y);
        }
    tops[part][row] = top;
    sums[part][row] = sum;
    for (int w = P / 2; w; w >>= 1) {
        __syncthreads();
        if (part < w) {
            join(tops[part + w][row], sums[part + w][row]);
            tops[part][row] = top;
            sums[part][row] = sum;
        }
    }
    if (part == 0 && m < M) {
        const float tl = o.tl[first + m];
        const float z = (top - tl) + logf(sum);   // -inf where there is no other word, NaN where the target's score is -inf as well
        const float e = expf(-fabsf(z));
        float v = fmaxf(z, 0.f) + log1pf(e), dt = -(z > 0.f ? 1.f : e) / (1.f + e);
        if (!(z == z) || !(tl < __builtin_inff())) v = dt = __builtin_nanf("");   // as in inf - inf
        const float base = fmaxf(top, tl);
        o.base[first + m] = base;
        o.log_sum[first + m] = logf(sum * expf(top - base) + expf(tl - base));
        o.dt[first + m] = dt;
        o.loss[first + m] = v;
        loss[o.index[first + m]] = v;
    }
}

// The cost, by 256 threads in a fixed order.
__device__ __forceinline__ void write_cost(const Rows &o, float *cost) {
    __shared__ double part[256];
    double s = 0.0;
    const int n = *o.count;
    for (int m = threadIdx.x; m < n; m += 256) s += (double)o.scale[m] * (double)o.loss[m];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int w = 128; w; w >>= 1) {
        if (threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) *cost = (float)(part[0] * (double)*o.unit);
}
static __global__ __launch_bounds__(256) void cost_kernel(Rows o, float *cost) { write_cost(o, cost); }

// The rows that count, gathered as planes; zeros in the masked rows of dx (nullable).  Eight columns a thread; bound by
// HBM: 8192 rows of 4096 in bf16, 134 MB, 25 us.
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(const T *x, bf16_t *dst, T *dx, Rows o, int N, int D, int pieces, long long from) {
    constexpr int PL = Planes<T>::N;
    const long long at = from + blockIdx.x * 256LL + threadIdx.x;
    const int n = (int)(at / pieces), c = (int)(at - (long long)n * pieces) * 8;
    if (n >= N) return;
    const int to = o.place[n];
    if (to >= 0) {
        float v[8];
        load8(x + (long long)n * D, c, D, v);
        put_planes<PL>(dst + (long long)to * pieces * 8 + c, (long long)N * pieces * 8, v);
    } else if (dx) {
        T *row = dx + (long long)n * D + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < D) row[e] = 0;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T *p, long long n, float *cost) {
    if (cost && blockIdx.x == 0 && threadIdx.x == 0) *cost = 0.f;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) p[i] = 0;
}

// d[m][v] of the rows first .. of the block (bf16: over the exponentials themselves).  Bound by HBM: 7400 x 128000 in bf16 move 3.8 GB in
// 0.76 ms.
template <typename T>
struct XentGrad {
    const typename Kept<T>::V *keep;
    long long ld;
    const float2 *stats;
    long long stats_ld;
    Rows o;
    int first, most, V, wave_cols;
    float *cost;   // the last launch of a call brings it along (null: not this one)
    __device__ void beside() const {
        if (cost) write_cost(o, cost);
    }
    __device__ bool skip(int m) const { return m >= live(most, o.count, first); }
    __device__ long long rows() const { return live(most, o.count, first); }
    __device__ void operator()(int m, int c, float (&v)[1][8]) const {
        const int r = first + m, t = o.target[r];
        const float base = o.base[r], log_sum = o.log_sum[r], s = o.scale[r];
        if constexpr (sizeof(T) == 4) {
            const f32x4 *k = (const f32x4 *)(keep + m * ld + c);
            const f32x4 a = k[0], b = k[1];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] = s * expf(((e < 4 ? a[e & 3] : b[e & 3]) - base) - log_sum);
        } else {
            const u32x4 k = *(const u32x4 *)(keep + m * ld + c);
            const float f = __expf((stats[(c / wave_cols) * stats_ld + m].x - base) - log_sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] = s * (__builtin_bit_cast(float, ((e & 1) ? k[e >> 1] >> 2 : k[e >> 1] << 14) & 0x3fffc000u) * f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (c + e == t) v[0][e] = s * o.dt[r];
            if (c + e >= V) v[0][e] = 0.f;
        }
    }
};

template <typename T>
struct XentScratch {
    static constexpr int PL = Planes<T>::N;
    int Dp, Vp, block, blocks;   // rows of a block, number of blocks
    int wave_cols, tiles;        // columns that share an entry of the statistics; entries of a row
    bool direct;                            // w is used where it is
    Rows rows;
    bf16_t *x, *w, *d;
    float2 *stats;
    float *scores, *sum;
    Parts part = {};
    XentScratch(Scratch &sc, int N, int D, int V, bool grads) {
        Dp = (int)round_up(D, 8), Vp = (int)round_up(V, 64);
        direct = PL == 1 && D == Dp;
        block = (int)round_up(N, 8);
        if (grads) block = (int)std::min<long long>(block, std::max<long long>(kStep, kBlockBytes / ((long long)Vp * sizeof(T)) / 256 * 256));
        blocks = N ? (N + block - 1) / block : 0;
        wave_cols = N <= kFewRows ? 64 : product_wave_cols(block, V, D, Planes<T>::PAIRS);
        tiles = (V + wave_cols - 1) / wave_cols;
        rows.count = sc.take<int>(1);
        rows.unit = sc.take<float>(1);
        rows.place = sc.take<int>(N);
        rows.index = sc.take<int>(N);
        rows.target = sc.take<int>(N);
        rows.scale = sc.take<float>(N);
        rows.tl = sc.take<float>(N);
        rows.base = sc.take<float>(N);
        rows.log_sum = sc.take<float>(N);
        rows.dt = sc.take<float>(N);
        rows.loss = sc.take<float>(N);
        const bool laid_out = grads || N > kFewRows;   // the scores of few rows need neither x nor w as planes
        // rows of d's two parts, for any number of rows up to N
        const int twice = PL == 1 && grads ? 2 * std::min(N, kFewRows) : 0;
        x = laid_out ? sc.take<bf16_t>((long long)PL * N * Dp) : nullptr;
        w = direct || !laid_out ? nullptr : sc.take<bf16_t>((long long)PL * V * Dp);
        stats = sc.take<float2>((V + 63) / 64 * (long long)block);   // as for the smaller tiles that fewer rows may take
        if (!grads) return;
        d = sc.take<bf16_t>((long long)Vp * std::max(PL * block, twice));
        scores = PL == 3 ? sc.take<float>((long long)block * Vp) : nullptr;
        part.floats = std::max({part_floats(std::max(block, twice), D, V), part_floats(V, D, block), twice * round_up(D, 4)});
        part.at = sc.take<float>(part.floats);
        sum = blocks > 1 ? sc.take<float>((long long)V * D) : nullptr;
    }
};

// The operator for one type; instantiated in a source file each.
template <typename T>
int xent(const T *x, const T *w, const int64_t *target, const float *scale, float *loss, float *cost, T *dx, T *dw, int N, int D, int V,
         bool grads, void *ws, hipStream_t s) {
    constexpr int PL = Planes<T>::N;
    Scratch sc(ws);
    const XentScratch<T> g(sc, N, D, V, grads);
    if (N == 0) {
        const long long n = grads ? (long long)V * D : 0;
        const LaunchPlan p = make_plan("xent_zero", {}, {}, dim3((unsigned)std::min<long long>((n + 256) / 256, 4096)), 256, 0);
        LC_LAUNCH(p, "xent (no rows)", (zero_kernel<T>), s, dw, n, cost);
        return LC_OK;
    }
    const LaunchPlan one = make_plan("xent_rows", {}, {N}, dim3(1), 1024, 0);
    LC_LAUNCH(one, "xent (rows)", rows_kernel, s, target, scale, loss, N, V, g.rows);
    const long long px = (long long)N * g.Dp, pw = (long long)V * g.Dp;
    const bool few = N <= kFewRows;   // the scores of few rows need neither x nor w laid out
    const bool fine = few && grads && PL == 1;   // d in two parts
    if (!few || grads) {
        const int pieces = g.Dp / 8;
        const int rc = in_launches((long long)N * pieces, [&](long long from, unsigned n) -> int {
            const LaunchPlan p = make_plan("xent_gather", {PL}, {N, D}, dim3(n), 256, 0);
            LC_LAUNCH(p, "xent (x)", (gather_kernel<T>), s, x, g.x, grads ? dx : nullptr, g.rows, N, D, pieces, from);
            return LC_OK;
        });
        if (rc) return rc;
    }
    if (!g.direct && (!few || grads))
        if (int rc = launch_planes<PL, 1>("xent (w)", Stored<T>{w, V, D}, g.w, g.Dp, pw, V, g.Dp, 0, s)) return rc;
    const Operand W = g.direct ? Operand{(const bf16_t *)w, (const bf16_t *)w, D, 0, V, 0, 0} : Operand{g.w, g.w, g.Dp, pw, V, 0, 0};
    for (int b = 0; b < g.blocks; ++b) {
        const int first = b * g.block, most = std::min(g.block, N - first);
        Operand X = {g.x + (long long)first * g.Dp, g.x, g.Dp, px, most, 0, 0}, Wc = W;
        const Shape sh = {most, V, D, g.rows.count, first, nullptr, 0};
        typename Kept<T>::V *keep = (typename Kept<T>::V *)(PL == 3 ? (void *)g.scores : (void *)g.d);
        int rc;
        auto scores = [&](auto epi) {
            if (few)
                return launch_few<T, ROW>("xent (few rows)", FewOperand<T>{x, x, D, N, g.rows.index}, FewOperand<T>{w, w, D, V, nullptr}, N,
                                          g.rows.count, V, D, epi, s);
            return launch_cut<PL, ROW, ROW>("xent", X, W, sh, choose_cut(g.block, V, D, Planes<T>::PAIRS, false), epi, s);
        };
        if (!grads)
            rc = scores(XentEpi<T, false>{g.stats, g.block, g.rows.target + first, g.rows.tl + first, nullptr, 0});
        else
            rc = scores(XentEpi<T, true>{g.stats, g.block, g.rows.target + first, g.rows.tl + first, keep, g.Vp});
        if (rc) return rc;
        if (most >= 2048) {
            const LaunchPlan p = make_plan("xent_lse", {16}, {most}, dim3((most + 15) / 16), 256, 0);
            LC_LAUNCH(p, "xent (logsumexp)", lse_kernel<16>, s, g.stats, (long long)g.block, g.tiles, g.rows, first, most, loss);
        } else {
            const LaunchPlan p = make_plan("xent_lse", {1}, {most}, dim3(most), 256, 0);
            LC_LAUNCH(p, "xent (logsumexp)", lse_kernel<1>, s, g.stats, (long long)g.block, g.tiles, g.rows, first, most, loss);
        }
        if (!grads) continue;
        if constexpr (PL == 1)
            if (fine) {   // one block
                const int two = 2 * N;
                if ((rc = launch_planes<2, 1>("xent (d)", XentGrad<T>{keep, g.Vp, g.stats, g.block, g.rows, 0, N, V, g.wave_cols, cost}, g.d, g.Vp, 0, N, g.Vp,
                                              0, s)))
                    return rc;
                Operand d = {g.d, g.d, g.Vp, 0, two, 0, 0};
                Wc.rows = X.rows = g.Dp;
                if (dx) {
                    const Shape shx = {two, D, V, g.rows.count, 0, nullptr, 0, 2};
                    if ((rc = launch_product<PL, ROW, COL, true>("xent (dx)", d, Wc, shx,
                                                                 StoreEpi<T>{dx, nullptr, 0x7fffffff, N, 0, D, g.rows.index, nullptr, g.rows.unit}, g.part, s)))
                        return rc;
                }
                const Shape shw = {V, D, two, nullptr, 0, g.rows.count, 0, 2};
                d.rows = g.Vp;
                return launch_gemm<2, COL, COL>("xent (dw)", d, X, shw, StoreEpi<T>{dw, nullptr, 0x7fffffff, V, 0, D, nullptr, nullptr, g.rows.unit}, s);
            }
        const long long pd = (long long)g.block * g.Vp;
        if ((rc = launch_planes<PL, 1>("xent (d)", XentGrad<T>{keep, g.Vp, g.stats, g.block, g.rows, first, most, V, g.wave_cols,
                                                          b + 1 == g.blocks ? cost : nullptr},
                                      g.d, g.Vp, pd, most, g.Vp, 0, s)))
            return rc;
        Operand d = {g.d, g.d, g.Vp, pd, most, 0, 0};
        Wc.rows = X.rows = g.Dp;
        if (dx) {
            const Shape shx = {most, D, V, g.rows.count, first, nullptr, 0};
            if ((rc = launch_product<PL, ROW, COL>("xent (dx)", d, Wc, shx,
                                                StoreEpi<T>{dx, nullptr, 0x7fffffff, most, 0, D, g.rows.index + first, nullptr, g.rows.unit}, g.part, s)))
                return rc;
        }
        const Shape shw = {V, D, most, nullptr, 0, g.rows.count, first};
        d.rows = g.Vp;
        const float *add = b ? g.sum : nullptr;
        if (b + 1 < g.blocks)
            rc = launch_product<PL, COL, COL>("xent (dw)", d, X, shw, StoreEpi<float>{g.sum, nullptr, 0x7fffffff, V, 0, D, nullptr, add, nullptr}, g.part, s);
        else
            rc = launch_product<PL, COL, COL>("xent (dw)", d, X, shw, StoreEpi<T>{dw, nullptr, 0x7fffffff, V, 0, D, nullptr, add, g.rows.unit}, g.part, s);
        if (rc) return rc;
    }
    if (grads) return LC_OK;
    const LaunchPlan p = make_plan("xent_cost", {}, {N}, dim3(1), 256, 0);
    LC_LAUNCH(p, "xent (cost)", cost_kernel, s, g.rows, cost);
    return LC_OK;
}

template <typename T>
size_t xent_scratch(int N, int D, int V, bool grads) {
    Scratch sc(nullptr);
    (void)XentScratch<T>(sc, N, D, V, grads);
    return sc.used;
}

}  // namespace head
}  // namespace lc
