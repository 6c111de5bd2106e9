// The matrix products of the supervised head: C[m][n] = sum_k A[m][k] B[n][k] over operand planes, with what follows the
// product done on the accumulators (an epilogue functor).
//
// The matrix instruction gets B's rows as its first operand, so a lane holds four consecutive n of one m: in block (i, j) of a
// wave, component 4 q + r of lane l is m = m0 + 32 i + l % 32, n = n0 + 32 j + 8 q + 4 (l / 32) + r.
//
// fp32 operands come as three bf16 planes each.  Six of the nine products of planes are formed (the others are below 2^-24 of
// the result), all into the same fp32 accumulators.  A wave whose accumulators are not all finite (an
// operand is infinite or NaN, or a sum overflowed on the way) forms its tile again with the fp32 instruction: planes add up to the
// operand exactly.
#pragma once
#include "head_common.hpp"

namespace lc {
namespace head {

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// What a product needs besides its operands.  rows_dev (nullable): the rows of A that count, minus first_row, at most M.
// k_dev (nullable): the same for the contraction.  Both are read on the device.
struct Shape {
    int M, Nn, K;
    const int *rows_dev;
    int rows_first;
    const int *k_dev;
    int k_first;
};
__device__ __forceinline__ int live(int most, const int *dev, int first) {
    return dev ? max(0, min(most, *dev - first)) : most;
}

// Adds the exact products of a wave's rows with the fp32 matrix instruction: lane l brings eight consecutive k of its row.
template <int MT, int NT, int FA, int FB>
__device__ __forceinline__ void product_exact(const Operand &A, const Operand &B, int m0, int n0, int K, int lane,
                                           f32x16 (&acc)[MT][NT]) {
    const int l32 = lane & 31, h = lane >> 5;
    auto whole = [&](const Operand &o, auto form, int r, int k, float (&v)[8]) {
        constexpr int FORM = decltype(form)::value;
        for (int e = 0; e < 8; ++e) {
            const bf16_t *p;
            bool in = k + e < K;
            if constexpr (FORM == PAIR) {
                int second;
                const int f = min(pair_row(r, &second), o.rows - 1);
                p = (second ? o.p1 : o.p0) + f * o.ld + k + e;
            } else if constexpr (FORM == ROW) {
                p = o.p0 + min(r, o.rows - 1) * o.ld + k + e;
            } else {
                const bool second = FORM == COLPAIR && k + e >= o.half;
                const int d = k + e - (second ? o.half : 0);
                if (FORM == COLPAIR) in &= d < o.depth;
                p = (second ? o.p1 : o.p0) + d * o.ld + min(r, o.rows - 1);
            }
            float s = 0.f;
            for (int q = 2; q >= 0; --q)
                if (in) s += from_bf16(p[q * o.plane]);
            v[e] = s;
        }
    };
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {   // one block at a time: this is rare, and must not take registers from the rest
            f32x16 c = {};
#pragma unroll 1
            for (int k = 0; k < K; k += 16) {
                float a[8], b[8];
                whole(A, std::integral_constant<int, FA>(), m0 + 32 * i + l32, k + 8 * h, a);
                whole(B, std::integral_constant<int, FB>(), n0 + 32 * j + l32, k + 8 * h, b);
#pragma unroll
                for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(b[e], a[e], c, 0, 0, 0);
            }
            acc[i][j] = c;
        }
}

template <int MT, int NT>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[MT][NT]) {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) ok &= __builtin_isfinite(acc[i][j][e]);
    return __all(ok);
}

// Tile order: groups of kGroup tiles along m share their tiles along n, and an XCD walks a contiguous range, so that the
// workgroups that run at once on one XCD share operand rows in its L2.
constexpr int kGroup = 8;
__device__ __forceinline__ void tile_of(int wg, int mt, int nt, int *tm, int *tn) {
    const int id = remap_xcd(wg, mt * nt);
    const int group = id / (kGroup * nt), first = group * kGroup, size = min(kGroup, mt - first);
    const int in = id - group * kGroup * nt;
    *tm = first + in % size;
    *tn = in / size;
}

// ---------------------------------------------------------------------------------------------------------------------------
// The tiled product.  BM x BN of the result per workgroup, WM x WN waves, steps of 64 along the contraction through two LDS
// buffers that are filled by loads which go straight there; one barrier a step: behind it the other buffer is free (every wave
// has read it) and this one is full (every wave has waited for its loads), so a step's loads have a whole step to arrive.
//
// An operand's tile is kept as it lies in memory.  By rows (ROW, PAIR): 128 bytes a row, its eight 16-byte pieces exchanged by
// the row's low bits so that the 32 rows a fragment reads fall on all banks.  By columns (COL, COLPAIR): 64 rows of
// BM or BN values, 64-byte pieces exchanged by the row's bits, read with the transposing LDS load, which hands lane i of 16 the
// four k of column i from four rows of 32 bytes.
template <int N>
__device__ __forceinline__ int col_swizzle(int k) {   // N columns: N / 32 pieces of 64 bytes
    return ((k & 3) | ((k >> 3) & 1) << 2) & (N / 32 - 1);
}

template <int FORM, int N, int NW>
struct Stager {
    static constexpr bool COLS = FORM == COL || FORM == COLPAIR;
    static constexpr int Q = N / 8 / NW;   // load instructions of a wave a step, 1024 bytes each
    unsigned off[Q];
    gbyte_ptr base[FORM == PAIR ? Q : FORM == COLPAIR ? 2 : 1];
    long long ld2, plane2;                 // bytes
    int wave, lane, depth, half;
    __device__ __forceinline__ void init(const Operand &o, int r0, int wave_, int lane_) {
        wave = wave_, lane = lane_;
        ld2 = o.ld * 2, plane2 = o.plane * 2;
        depth = o.depth, half = o.half;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int g = q * NW + wave;   // this kilobyte of the tile
            if constexpr (COLS) {
                const int pc = lane % (N / 8);
                const int c = ((pc / 4) ^ col_swizzle<N>(first_k(q))) * 4 + pc % 4;
                off[q] = (unsigned)((long long)first_k(q) * ld2) + (unsigned)(min(r0 + 8 * c, o.rows - 8) - r0) * 2;
            } else {
                int f0 = r0 + 8 * g, second = 0;
                if constexpr (FORM == PAIR) f0 = pair_row(f0, &second);
                const int top = min(f0, o.rows - 1);
                const int rel = min(f0 + lane / 8, o.rows - 1) - (FORM == PAIR ? top : r0);
                if constexpr (FORM == PAIR) base[q] = (gbyte_ptr)((second ? o.p1 : o.p0) + (long long)top * o.ld);
                off[q] = (unsigned)((long long)rel * ld2) + first_k(q) * 2;
            }
        }
        if constexpr (FORM == ROW) base[0] = (gbyte_ptr)(o.p0 + (long long)r0 * o.ld);
        if constexpr (COLS) base[0] = (gbyte_ptr)(o.p0 + r0);
        if constexpr (FORM == COLPAIR) base[1] = (gbyte_ptr)(o.p1 + r0);
    }
    // the index within the step of the first value (by columns: of all values) of this lane's 16 bytes of load q
    __device__ __forceinline__ int first_k(int q) const {
        if constexpr (COLS) return (q * NW + wave) * (512 / N) + lane / (N / 8);
        else return ((lane % 8) ^ (lane / 8)) * 8;
    }
    // indices from k0 on that exist, of K in all (by rows: in whole 16-byte pieces)
    __device__ __forceinline__ int left(int k0, int K) const {
        if constexpr (FORM == COLPAIR) return depth - (k0 >= half ? k0 - half : k0);
        else return COLS ? K - k0 : (K - k0 + 7) & ~7;
    }
    // The step from k0 on into LDS.  Where less than a step is left, lanes beyond it read its start; clear() follows.
    __device__ __forceinline__ void load(unsigned lds, int k0, int K, int pl) const {
        const int n = left(k0, K);
        const bool second = FORM == COLPAIR && k0 >= half;
        const int k1 = second ? k0 - half : k0;
        const long long at = (COLS ? k1 * ld2 : k1 * 2LL) + pl * plane2;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            unsigned o = off[q];
            if (n < kStep && first_k(q) >= n) o -= COLS ? (unsigned)((long long)first_k(q) * ld2) : first_k(q) * 2;
            load_lds16((FORM == PAIR ? base[q] : FORM == COLPAIR ? (second ? base[1] : base[0]) : base[0]) + at, o,
                       lds + (q * NW + wave) * 1024);
        }
    }
    // zeros for what is beyond the `n` indices left of this step (the same bytes this lane brought)
    __device__ __forceinline__ void clear(char *lds, int n) const {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (first_k(q) >= n) *(u32x4 *)(lds + (q * NW + wave) * 1024 + lane * 16) = (u32x4){0, 0, 0, 0};
    }
};

// The fragments of a wave's T blocks of 32 rows from r0 of a tile of N.
template <int FORM, int N, int T>
struct Reader {
    static constexpr bool COLS = FORM == COL || FORM == COLPAIR;
    unsigned at[COLS ? T : 4];
    __device__ __forceinline__ void init(int r0, int lane) {
        if constexpr (COLS) {
            const int s = lane % 16, g = lane / 16;
            const int k = 8 * (g >> 1) + s / 4;
#pragma unroll
            for (int i = 0; i < T; ++i)
                at[i] = k * (2 * N) + (((r0 / 32 + i) ^ col_swizzle<N>(k)) * 64) + (g & 1) * 32 + (s % 4) * 8;
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) at[c] = (r0 + (lane & 31)) * 128 + (((2 * c + (lane >> 5)) ^ (lane & 7)) * 16);
        }
    }
    __device__ __forceinline__ u32x4 read(unsigned lds, int c, int i) const {
        typedef __attribute__((address_space(3))) u32x4 *p4;
        if constexpr (COLS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 *p2;
            const unsigned a = lds + at[i] + c * (16 * 2 * N);
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p2)(size_t)a));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p2)(size_t)(a + 4 * 2 * N)));
            return (u32x4){lo[0], lo[1], hi[0], hi[1]};
        } else {
            return *(p4)(size_t)(lds + at[c] + i * (32 * 128));
        }
    }
};

template <int PL, int FA, int FB, int BM, int BN, int WM, int WN, typename Epi>
__global__ __launch_bounds__(64 * WM * WN, 2) void gemm_kernel(Operand A, Operand B, Shape sh, int mt, int nt, Epi epi) {
    constexpr int NW = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32, PAIRS = PL == 3 ? 6 : 1;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tm, tn;
    tile_of(blockIdx.x, mt, nt, &tm, &tn);
    const int M = live(sh.M, sh.rows_dev, sh.rows_first);
    const int K = live(sh.K, sh.k_dev, sh.k_first);
    if (tm * BM >= M) return;
    Stager<FA, BM, NW> sa;
    Stager<FB, BN, NW> sb;
    sa.init(A, tm * BM, wave, lane);
    sb.init(B, tn * BN, wave, lane);
    Reader<FA, BM, MT> ra;
    Reader<FB, BN, NT> rb;
    const int wm = wave / WN, wn = wave % WN;
    ra.init(wm * MT * 32, lane);
    rb.init(wn * NT * 32, lane);
    constexpr unsigned ABYTES = BM * 128, STAGE = (BM + BN) * 128;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char *)smem;
    f32x16 acc[MT][NT] = {};
    const int steps = (K + kStep - 1) / kStep * PAIRS;
    auto stage = [&](int st) {
        const int kt = PAIRS == 1 ? st : st / PAIRS, s = PAIRS == 1 ? 0 : st - kt * PAIRS;
        const unsigned l = lds0 + (st & 1) * STAGE;
        // planes of A and B in the six products: 00 10 01 11 02 20
        const int pa = PL == 1 ? 0 : (0x010102 >> (4 * (5 - s))) & 0xf, pb = PL == 1 ? 0 : (0x001120 >> (4 * (5 - s))) & 0xf;
        sa.load(l, kt * kStep, K, pa);
        sb.load(l + ABYTES, kt * kStep, K, pb);
    };
    if (steps) stage(0);
    for (int st = 0; st < steps; ++st) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (st + 1 < steps) stage(st + 1);
        const unsigned l = lds0 + (st & 1) * STAGE;
        {
            const int k0 = (PAIRS == 1 ? st : st / PAIRS) * kStep;
            const int la = sa.left(k0, K), lb = sb.left(k0, K);
            if (la < kStep || lb < kStep) {
                sa.clear(smem + (st & 1) * STAGE, la);
                sb.clear(smem + (st & 1) * STAGE + ABYTES, lb);
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
        }
        u32x4 a[2][MT], b[2][NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) a[0][i] = ra.read(l, 0, i);
#pragma unroll
        for (int j = 0; j < NT; ++j) b[0][j] = rb.read(l + ABYTES, 0, j);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c < 3) {
#pragma unroll
                for (int i = 0; i < MT; ++i) a[(c + 1) & 1][i] = ra.read(l, c + 1, i);
#pragma unroll
                for (int j = 0; j < NT; ++j) b[(c + 1) & 1][j] = rb.read(l + ABYTES, c + 1, j);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mfma32(b[c & 1][j], a[c & 1][i], acc[i][j]);
        }
    }
    const int m0 = tm * BM + wm * MT * 32, n0 = tn * BN + wn * NT * 32;
    if (m0 >= M || n0 >= sh.Nn) return;
    if constexpr (PL == 3) {
        if (!all_finite(acc)) product_exact<MT, NT, FA, FB>(A, B, m0, n0, K, lane, acc);
    }
    epi.run(acc, m0, n0, lane, M, sh.Nn);
}

template <int PL, int FA, int FB, int BM, int BN, int WM, int WN, typename Epi>
int launch_tiles(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    const int mt = ceil_div(sh.M, BM), nt = ceil_div(sh.Nn, BN);
    const LaunchPlan p = make_plan(name, {PL, FA, FB, BM, BN}, {sh.M, sh.Nn, sh.K}, dim3((unsigned)((long long)mt * nt)), 64 * WM * WN,
                                   2 * (BM + BN) * 128);
    LC_PLAN_REQUIRE(p, (long long)mt * nt <= 0x7fffffffLL);
    LC_PLAN_REQUIRE(p, A.ld % 8 == 0 && B.ld % 8 == 0 && A.plane % 8 == 0 && B.plane % 8 == 0);
    constexpr bool CA = FA == COL || FA == COLPAIR, CB = FB == COL || FB == COLPAIR;
    LC_PLAN_REQUIRE(p, CA ? A.rows % 8 == 0 && A.ld >= A.rows && A.rows >= sh.M : A.rows >= sh.M && A.ld >= sh.K);
    LC_PLAN_REQUIRE(p, CB ? B.rows % 8 == 0 && B.ld >= B.rows && B.rows >= sh.Nn : B.rows >= (FB == PAIR ? 1 : sh.Nn) && B.ld >= sh.K);
    LC_PLAN_REQUIRE(p, FA != PAIR && FA != COLPAIR && (FB != PAIR || sh.Nn == 64 * ceil_div(B.rows, 32)));
    LC_PLAN_REQUIRE(p, FB != COLPAIR || (B.half % kStep == 0 && B.depth >= 1 && B.depth <= B.half && sh.K == B.half + B.depth));
    LC_PLAN_REQUIRE(p, A.ld <= (1 << 22) && B.ld <= (1 << 22));   // 256 rows' offsets stay below 2^31 bytes
    LC_PLAN_REQUIRE(p, ptr_aligned16(A.p0) && ptr_aligned16(B.p0) && ptr_aligned16(B.p1));
    LC_LAUNCH(p, name, (gemm_kernel<PL, FA, FB, BM, BN, WM, WN, Epi>), s, A, B, sh, mt, nt, epi);
    return LC_OK;
}

// A workgroup per 256 x 256 of the result where that fills the chip, per 128 x 128 (two at a time on a compute unit) where not.
template <int PL, int FA, int FB, typename Epi>
int launch_gemm(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    if (sh.M == 0 || sh.Nn == 0) return LC_OK;
    if ((long long)ceil_div(sh.M, 256) * ceil_div(sh.Nn, 256) >= kComputeUnits)
        return launch_tiles<PL, FA, FB, 256, 256, 2, 4>(name, A, B, sh, epi, s);
    return launch_tiles<PL, FA, FB, 128, 128, 2, 2>(name, A, B, sh, epi, s);
}

// four consecutive values of one row; n counts from the row's start and may run past its end at `width`
template <typename T>
__device__ __forceinline__ void store4(T *row, int n, int width, bool vec, const float (&v)[4]) {
    if (vec && n + 3 < width) {
        if constexpr (sizeof(T) == 4) {
            *(f32x4 *)(row + n) = (f32x4){v[0], v[1], v[2], v[3]};
        } else {
            *(u16x4 *)(row + n) = (u16x4){to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]), to_bf16(v[3])};
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (n + r < width) row[n + r] = narrow<T>(v[r]);
    }
}

// The product itself, into one or two matrices of `width` columns: rows from `second` on go to out1.  index (nullable): row m
// goes to row index[m].  add (nullable): fp32 [M][width], added; factor (nullable): times *factor; then rounded.
template <typename T>
struct StoreEpi {
    T *out0, *out1;
    int second, width0rows, width1rows;   // rows that exist of each
    int width;
    const int *index;
    const float *add, *factor;
    template <int MT, int NT>
    __device__ __forceinline__ void run(const f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int Nn) const {
        const bool vec = width % 4 == 0;
        const float f = factor ? *factor : 1.f;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = m0 + 32 * i + (lane & 31);
            if (m >= M) continue;
            const bool up = m >= second;
            const int row = up ? m - second : m;
            if (row >= (up ? width1rows : width0rows)) continue;
            T *o = (up ? out1 : out0) + (long long)(index ? index[row] : row) * width;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int n = n0 + 32 * j + 8 * q + 4 * (lane >> 5);
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[r] = acc[i][j][4 * q + r];
                        if (add && n + r < width) v[r] += add[(long long)m * width + n + r];
                        v[r] *= f;
                    }
                    store4(o, n, width, vec, v);
                }
        }
    }
};

}  // namespace head
}  // namespace lc
