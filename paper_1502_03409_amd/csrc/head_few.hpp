// Products with at most 32 rows on the left (answers for a few images): the weights stream by once, from HBM to registers.
//
// Two kernels.  Where rows begin at 16-byte boundaries the weights pass through LDS, because whole lines can go there directly; rows
// of any other alignment go straight to registers.  In both, a workgroup owns NB blocks of 32 columns of the result; its four waves take
// turns along the contraction, 64 indices (whole lines of the weights) at a time, and add up through LDS.  Bound by HBM: what matters is how many loads are in flight, so each wave asks for its next
// 16 vectors of weights before it uses the last ones.  A pair of matrices shares a block, 16 rows of each in turn, so that a
// small layer can be cut into single blocks.  fp32 operands meet the fp32 matrix instruction, as they are: it keeps up with
// HBM here, and needs no planes.
#pragma once
#include "head_gemm.hpp"

namespace lc {
namespace head {

constexpr int kFewRows = 32;

template <typename T>
struct FewOperand {   // row r at p + r * ld
    const T *p0, *p1;   // PAIR: two matrices, 16 rows of each in turn
    long long ld;
    int rows;
    const int *index;   // nullable: row r is row index[r]
};

// 8 values of a row as the matrix instructions take them; rows have any alignment
template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
    static constexpr int SET = 8;   // vectors of a block a wave asks for at a time
    u32x4 v;
    __device__ __forceinline__ void load(const bf16_t *p) {
        typedef u32x4 any __attribute__((aligned(2)));
        v = *(const any *)p;
    }
    __device__ __forceinline__ void keep(bool in) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = in ? v[e] : 0u;
    }
    __device__ __forceinline__ void load_first(const bf16_t *p, int n) {   // n < 8 of them, zeros behind
        v = (u32x4){0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) v[e >> 1] |= (unsigned)p[e] << (16 * (e & 1));
    }
    static __device__ __forceinline__ f32x16 mul(const Frag &b, const Frag &a, f32x16 c) { return mfma32(b.v, a.v, c); }
};
template <> struct Frag<float> {
    static constexpr int SET = 4;
    f32x4 v[2];
    __device__ __forceinline__ void load(const float *p) {
        typedef f32x4 any __attribute__((aligned(4)));
        v[0] = *(const any *)p;
        v[1] = *(const any *)(p + 4);
    }
    __device__ __forceinline__ void keep(bool in) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = in ? v[e >> 2][e & 3] : 0.f;
    }
    __device__ __forceinline__ void load_first(const float *p, int n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = e < n ? p[e] : 0.f;
    }
    static __device__ __forceinline__ f32x16 mul(const Frag &b, const Frag &a, f32x16 c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(b.v[e >> 2][e & 3], a.v[e >> 2][e & 3], c, 0, 0, 0);
        return c;
    }
};

template <typename T, int FB, int NB, typename Epi>
__global__ __launch_bounds__(256, 2) void few_kernel(FewOperand<T> A, FewOperand<T> B, int M, const int *rows_dev, int Nn, int K, Epi epi) {
    constexpr int C = Frag<T>::SET;   // vectors of 16 indices; the four waves take turns of 64 indices
    constexpr int SUMS = 3 * NB * 64;
    __shared__ f32x16 sums[SUMS * 64 > kEpiBytes<NB> ? SUMS : (kEpiBytes<NB> + 63) / 64];   // of waves 1 to 3; then the epilogue's
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    M = live(M, rows_dev, 0);
    if (M == 0) return;
    const int m = min(l32, M - 1), n0 = blockIdx.x * (32 * NB);
    const T *a = A.p0 + (long long)(A.index ? A.index[m] : m) * A.ld, *b[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        int f = n0 + 32 * j + l32, second = 0;
        if (FB == PAIR) f = pair_row(f, 16, &second);
        b[j] = (second ? B.p1 : B.p0) + (long long)min(f, B.rows - 1) * B.ld;
    }
    f32x16 acc[1][NB] = {};
    Frag<T> fa[2][C], fb[2][C][NB];
    const int whole = K / (64 * C), k_end = K / 8 * 8;
    auto load = [&](int s, int set, auto full) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int k = ((s * (C / 4) + c / 4) * 4 + wave) * 64 + c % 4 * 16 + 8 * h;
            const bool in = decltype(full)::value || k < k_end;
            const int at = in ? k : 0;
            fa[set][c].load(a + at);
#pragma unroll
            for (int j = 0; j < NB; ++j) fb[set][c][j].load(b[j] + at);
            if (!decltype(full)::value) {   // beyond the end: zeros (of both, so that no infinity of another place shows)
                fa[set][c].keep(in);
#pragma unroll
                for (int j = 0; j < NB; ++j) fb[set][c][j].keep(in);
            }
        }
    };
    auto use = [&](int set) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[0][j] = Frag<T>::mul(fb[set][c][j], fa[set][c], acc[0][j]);
    };
    const std::true_type yes;
    if (whole) load(0, 0, yes);
    for (int s = 0; s < whole; s += 2) {
        if (s + 1 < whole) load(s + 1, 1, yes);
        use(0);
        if (s + 2 < whole) load(s + 2, 0, yes);
        if (s + 1 < whole) use(1);
    }
    if (whole * 64 * C < k_end) {
        load(whole, 0, std::false_type());
        use(0);
    }
    if (wave == 0 && k_end < K) {   // up to seven values
        Frag<T> r, w;
        r.load_first(a + k_end, h ? 0 : K - k_end);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            w.load_first(b[j] + k_end, h ? 0 : K - k_end);
            acc[0][j] = Frag<T>::mul(w, r, acc[0][j]);
        }
    }
    if (wave) {
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[((wave - 1) * NB + j) * 64 + lane] = acc[0][j];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[0][j] += sums[(w * NB + j) * 64 + lane];
    epi.run(acc, 0, n0, lane, M, Nn, 0, (char *)sums);
}

// The number format of an operand that comes in 16-byte pieces of one plane; 8-bit whole numbers (int8_t) only through LDS
template <typename T> struct FewFormat : Format<1> {};
template <> struct FewFormat<int8_t> : Format<BYTES> {};

// The same through LDS: each wave has a ring of ST steps of its own and waits for nobody.  A load instruction brings whole lines, eight
// rows of 128 bytes; from registers' loads 32 rows of 32 bytes, lines stay in the vector cache until their other parts are asked for, and
// that cache, not HBM, bounds what is in flight (5 rows against 100003 x 4096 in bf16: 4.2 TB/s through registers).
// XQ: load instructions for x a step, eight rows each.
constexpr int ring_bytes(int NB, int XQ, int ST) { return kWaves * ST * (NB * 4 + XQ) * 1024; }
template <typename T, int FB, int NB, int XQ, int ST, typename Epi>
__global__ __launch_bounds__(256, ring_bytes(NB, XQ, ST) > 81920 ? 1 : 2) void few_ring_kernel(FewOperand<T> A, FewOperand<T> B, int M,
                                                                                              const int *rows_dev, int Nn, int K, Epi epi) {
    constexpr int Q = NB * 4, LOADS = Q + XQ, STAGE = LOADS * 1024, EACH = 128 / (int)sizeof(T), PIECE = 16 / (int)sizeof(T);
    static_assert(ring_bytes(NB, XQ, ST) >= 3 * NB * 64 * 64 && ring_bytes(NB, XQ, ST) >= kEpiBytes<NB>, "the waves' sums and the epilogue go there too");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    M = live(M, rows_dev, 0);
    if (M == 0) return;
    const int n0 = blockIdx.x * (32 * NB);
    // load q of the weights: rows 8 q .. 8 q + 7, 16 bytes a lane; the eight pieces of a row exchanged by bits of the row
    const unsigned ld = (unsigned)(B.ld * sizeof(T));
    int second;
    const int top = min(FB == PAIR ? pair_row(n0, 16, &second) : n0, B.rows - 1);
    gbyte_ptr p0 = (gbyte_ptr)(B.p0 + (long long)top * B.ld), p1 = (gbyte_ptr)(B.p1 + (long long)top * B.ld), px = (gbyte_ptr)A.p0;
    unsigned off[Q], xoff[XQ];
    auto piece_of = [&](int q) { return (lane % 8) ^ ((4 * (q & 1) + lane / 16) & 7); };   // of the row, in this lane's place
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        int f = n0 + 8 * q + lane / 8;
        if (FB == PAIR) f = pair_row(f, 16, &second);
        off[q] = (unsigned)(min(f, B.rows - 1) - top) * ld + piece_of(q) * 16;
    }
#pragma unroll
    for (int q = 0; q < XQ; ++q) {
        const int m = min(8 * q + lane / 8, M - 1);
        xoff[q] = (unsigned)((A.index ? A.index[m] : m) * A.ld * sizeof(T)) + piece_of(q) * 16;
    }
    const unsigned ring = (unsigned)(size_t)(__attribute__((address_space(3))) char *)smem + wave * (ST * STAGE);
    char *const mine = smem + wave * (ST * STAGE);
    const int steps = (K + EACH - 1) / EACH, own = steps > wave ? (steps - wave + 3) / 4 : 0;   // steps wave, wave + 4, ..
    auto load = [&](int s) {
        const int k0 = (4 * s + wave) * EACH, left = (K - k0) / PIECE;   // whole pieces that exist
        const unsigned l = ring + (unsigned)(s % ST) * STAGE;
        const long long at = (long long)(4 * s + wave) * 128;
#pragma unroll
        for (int q = 0; q < Q; ++q)   // lanes beyond the end read the step's start
            load_lds16((FB == PAIR && (q & 2) ? p1 : p0) + at, piece_of(q) < left ? off[q] : off[q] - piece_of(q) * 16, l + q * 1024);
#pragma unroll
        for (int q = 0; q < XQ; ++q)
            load_lds16(px + at, piece_of(q) < left ? xoff[q] : xoff[q] - piece_of(q) * 16, l + (Q + q) * 1024);
    };
    typedef typename FewFormat<T>::Acc Acc;
    Acc acc[1][NB] = {};
#pragma unroll
    for (int s = 0; s < ST - 1; ++s)
        if (s < own) load(s);
#pragma unroll 1
    for (int s = 0; s < own; ++s) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the step before has been read: its place is free
        if (s + ST - 1 < own) {
            load(s + ST - 1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 1) * LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        char *const l = mine + (s % ST) * STAGE;
        const int left = (K - (4 * s + wave) * EACH) / PIECE;
        if (left < 8) {   // what is beyond the end: zeros, of both operands
#pragma unroll
            for (int q = 0; q < LOADS; ++q)
                if (piece_of(q < Q ? q : q - Q) >= left) *(u32x4 *)(l + q * 1024 + lane * 16) = (u32x4){0, 0, 0, 0};
        }
        // rows beyond those of x that were brought take the last one's place; their sums are dropped
        const int xr = min(l32, 8 * XQ - 1), xswap = (xr >> 1) & 7, wswap = (l32 >> 1) & 7;
        if constexpr (sizeof(T) <= 2) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const u32x4 x = *(const u32x4 *)(l + Q * 1024 + xr * 128 + (((2 * c + h) ^ xswap) * 16));
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    acc[0][j] = FewFormat<T>::mul(*(const u32x4 *)(l + j * 4096 + l32 * 128 + (((2 * c + h) ^ wswap) * 16)), x, acc[0][j]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) {   // eight values: a lane brings four of them, so a product takes values e and 4 + e
                const f32x4 x = *(const f32x4 *)(l + Q * 1024 + xr * 128 + (((2 * c + h) ^ xswap) * 16));
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const f32x4 w = *(const f32x4 *)(l + j * 4096 + l32 * 128 + (((2 * c + h) ^ wswap) * 16));
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[e], x[e], acc[0][j], 0, 0, 0);
                }
            }
        }
    }
    __syncthreads();   // all rings are free
    Acc *const sums = (Acc *)smem;
    if (wave) {
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[((wave - 1) * NB + j) * 64 + lane] = acc[0][j];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[0][j] += sums[(w * NB + j) * 64 + lane];
    epi.run(acc, 0, n0, lane, M, Nn, 0, smem);
}

// Two blocks a workgroup where that leaves one for every compute unit (x is then read half as often), single ones where not: 8192 x 4096
// weights in bf16 37 against 44 us, 2603 x 1000 in fp32 20 against 15 (both through registers).
template <typename T, int FB, int NB, typename Epi>
int launch_blocks(const char *name, const FewOperand<T> &A, const FewOperand<T> &B, int M, const int *rows_dev, int Nn, int K,
                  const Epi &epi, hipStream_t s) {
    const bool ring = A.ld * sizeof(T) % 16 == 0 && B.ld * sizeof(T) % 16 == 0 && K * sizeof(T) % 16 == 0;
    const LaunchPlan p = make_plan(name, {(int)sizeof(T), FB, NB, ring}, {M, Nn, K}, dim3(ceil_div(Nn, 32 * NB)), 256,
                                   !ring ? 0 : M <= 8 ? ring_bytes(NB, 1, 4) : ring_bytes(NB, 4, 3));
    LC_PLAN_REQUIRE(p, M >= 1 && M <= kFewRows && A.rows >= M && A.ld >= K && B.ld >= K && B.rows >= 1);
    LC_PLAN_REQUIRE(p, FB == PAIR ? Nn == 32 * ceil_div(B.rows, 16) : B.rows >= Nn);
    LC_PLAN_REQUIRE(p, A.ld <= (1 << 20) && B.ld <= (1 << 20));   // 64 rows' offsets stay below 2^31 bytes
    LC_PLAN_REQUIRE(p, ptr_aligned16(A.p0) && ptr_aligned16(B.p0) && ptr_aligned16(B.p1));
    if constexpr (sizeof(T) == 1) LC_PLAN_REQUIRE(p, ring);
    else if (!ring) {
        LC_LAUNCH(p, name, (few_kernel<T, FB, NB, Epi>), s, A, B, M, rows_dev, Nn, K, epi);
        return LC_OK;
    }
    if (M <= 8) LC_LAUNCH(p, name, (few_ring_kernel<T, FB, NB, 1, 4, Epi>), s, A, B, M, rows_dev, Nn, K, epi);
    else LC_LAUNCH(p, name, (few_ring_kernel<T, FB, NB, 4, 3, Epi>), s, A, B, M, rows_dev, Nn, K, epi);
    return LC_OK;
}
template <typename T, int FB, typename Epi>
int launch_few(const char *name, const FewOperand<T> &A, const FewOperand<T> &B, int M, const int *rows_dev, int Nn, int K, const Epi &epi,
               hipStream_t s) {
    if constexpr (FB == PAIR)
        if (ceil_div(Nn, 64) < kComputeUnits) return launch_blocks<T, FB, 1>(name, A, B, M, rows_dev, Nn, K, epi, s);
    return launch_blocks<T, FB, 2>(name, A, B, M, rows_dev, Nn, K, epi, s);
}

}  // namespace head
}  // namespace lc
