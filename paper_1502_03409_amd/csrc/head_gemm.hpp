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

// planes of A and B in the product of pair s
__device__ __host__ constexpr int pair_a(int s) { return s == 1 || s == 3 ? 1 : s == 5 ? 2 : 0; }
__device__ __host__ constexpr int pair_b(int s) { return s == 2 || s == 3 ? 1 : s == 4 ? 2 : 0; }

// What a product needs besides its operands.  rows_dev (nullable): the rows of A that count, minus first_row, at most M.
// k_dev (nullable): the same for the contraction.  Both are read on the device.
struct Shape {
    int M, Nn, K;   // K: padded length of the contraction
    const int *rows_dev;
    int rows_first;
    const int *k_dev;
    int k_first;
};
__device__ __forceinline__ int live(int most, const int *dev, int first) {
    return dev ? max(0, min(most, *dev - first)) : most;
}

// Adds the exact products of a wave's rows with the fp32 matrix instruction: lane l brings eight consecutive k of its row.
template <int MT, int NT, bool PAIR>
__device__ __forceinline__ void product_exact(const Operand &A, const Operand &B, int m0, int n0, int K, int lane,
                                           f32x16 (&acc)[MT][NT]) {
    const f32x16 zero = {};
    for (int i = 0; i < MT; ++i)
        for (int j = 0; j < NT; ++j) acc[i][j] = zero;
    const int l32 = lane & 31, h = lane >> 5;
    auto whole = [](const bf16_t *row, long long plane, float (&v)[8]) {
        u32x4 p[3];
        for (int q = 0; q < 3; ++q) p[q] = *(const u32x4 *)(row + q * plane);
        for (int e = 0; e < 8; ++e) {
            float s = 0.f;
            for (int q = 2; q >= 0; --q) s += (e & 1) ? bf16_hi(p[q][e >> 1]) : bf16_lo(p[q][e >> 1]);
            v[e] = s;
        }
    };
    for (int k = 0; k < K; k += 16) {
        float a[MT][8], b[NT][8];
#pragma unroll
        for (int i = 0; i < MT; ++i) whole(operand_row<false>(A, m0 + 32 * i + l32) + k + 8 * h, A.plane, a[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) whole(operand_row<PAIR>(B, n0 + 32 * j + l32) + k + 8 * h, B.plane, b[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j][e], a[i][e], acc[i][j], 0, 0, 0);
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

// Both operands straight from global memory: a workgroup of 2 x 2 waves of 64 x 64.
template <int PL, bool PAIR, typename Epi>
__global__ __launch_bounds__(256) void gemm_kernel(Operand A, Operand B, Shape sh, int mt, int nt, Epi epi) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int tm, tn;
    tile_of(blockIdx.x, mt, nt, &tm, &tn);
    const int M = live(sh.M, sh.rows_dev, sh.rows_first);
    const int K = (live(sh.K, sh.k_dev, sh.k_first) + kStep - 1) / kStep * kStep;
    const int m0 = tm * 128 + (wave >> 1) * 64, n0 = tn * 128 + (wave & 1) * 64;
    if (m0 >= M || n0 >= sh.Nn) return;
    f32x16 acc[2][2] = {};
    const bf16_t *a[2], *b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        a[i] = operand_row<false>(A, m0 + 32 * i + (lane & 31)) + 8 * (lane >> 5);
        b[i] = operand_row<PAIR>(B, n0 + 32 * i + (lane & 31)) + 8 * (lane >> 5);
    }
    for (int k = 0; k < K; k += 32) {
#pragma unroll
        for (int s = 0; s < (PL == 3 ? 6 : 1); ++s) {
            const long long qa = pair_a(s) * A.plane, qb = pair_b(s) * B.plane;
            u32x4 av[2][2], bv[2][2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    av[c][i] = *(const u32x4 *)(a[i] + qa + k + 16 * c);
                    bv[c][i] = *(const u32x4 *)(b[i] + qb + k + 16 * c);
                }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mfma32(bv[c][j], av[c][i], acc[i][j]);
        }
    }
    if constexpr (PL == 3) {
        if (!all_finite(acc)) product_exact<2, 2, PAIR>(A, B, m0, n0, K, lane, acc);
    }
    epi.run(acc, m0, n0, lane, M, sh.Nn);
}

template <int PL, bool PAIR, typename Epi>
int launch_gemm(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    if (sh.M == 0 || sh.Nn == 0) return LC_OK;
    const int mt = ceil_div(sh.M, 128), nt = ceil_div(sh.Nn, 128);
    const LaunchPlan p = make_plan(name, {PL, PAIR}, {sh.M, sh.Nn, sh.K}, dim3((unsigned)((long long)mt * nt)), 256, 0);
    LC_PLAN_REQUIRE(p, (long long)mt * nt <= 0x7fffffffLL);
    LC_PLAN_REQUIRE(p, sh.K % kStep == 0 && A.ld % 8 == 0 && B.ld % 8 == 0 && A.plane % 8 == 0 && B.plane % 8 == 0);
    LC_PLAN_REQUIRE(p, A.ld >= sh.K && B.ld >= sh.K && A.rows >= 1 && B.rows >= 1);
    LC_PLAN_REQUIRE(p, ptr_aligned16(A.p0) && ptr_aligned16(B.p0) && ptr_aligned16(B.p1));
    LC_LAUNCH(p, name, (gemm_kernel<PL, PAIR, Epi>), s, A, B, sh, mt, nt, epi);
    return LC_OK;
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
