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
//
// PL 2: one plane each, but A, by columns, is the second part of each value behind all first ones, along the contraction, and B's indices come
// twice; all of it within one step.
//
// Large products are bound by the matrix unit, by waits for the operand with two buffers and by the clock that the chip's power allows:
// 1.13 to 1.23 PFLOP/s in the three of 7373 x 128000 x 4096, with the unit busy 62 to 67 % of the cycles at 1.7 to 1.8 GHz and waves waiting
// in 20 to 24 % (the library's plain products of these sizes reach 1.3 to 1.6).  What follows a 256 x 256 tile's loop overlaps nothing, as its
// workgroup is alone on its compute unit, and is long: the gated forward kernels have 103 to 140 KB of code, beyond the instruction cache, and
// those that store bf16 gradients keep 208 registers in scratch memory on the way.  The loops themselves have no spills.
// In fp32 six products make one: 143 TFLOP/s of fp32 in 700 x 30011 x 768, where the unit of 128 x 128 tiles is busy 46 % and waves wait in
// 30 % of the cycles; an order of the six that takes seven tiles from the L2 caches, not twelve, gained 4 % in a loop over all six and lost
// 30 % to that loop's length.
#pragma once
#include "head_common.hpp"

namespace lc {
namespace head {

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Number formats of a product, the first template parameter of what follows.  1, 2, 3: bf16 planes, as above.  HALF: one fp16 plane.  HALF2:
// two fp16 planes, a value and what its rounding to the first leaves, of which three products of four are formed (the fourth is below 2^-22
// of the result).  BYTES: 8-bit whole numbers, two in the place of one 16-bit value, sums in 32-bit whole numbers: the matrix instruction
// takes the same 16 bytes of a row as those for 16-bit values, so nothing else changes, and sizes along the contraction count pairs.
enum { HALF = 4, HALF2 = 5, BYTES = 6 };
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
// PAIRS: products of planes; A, B: the plane of each operand in them, four bits a product.  STACK: products of a stack of matrices.
template <int PL> struct Format {
    typedef f32x16 Acc;
    static constexpr int PAIRS = 1;
    static constexpr unsigned A = 0, B = 0;
    static constexpr bool STACK = false;
    static __device__ __forceinline__ Acc mul(u32x4 a, u32x4 b, Acc c) { return mfma32(a, b, c); }
};
template <> struct Format<3> : Format<1> {   // 00 10 01 11 02 20
    static constexpr int PAIRS = 6;
    static constexpr unsigned A = 0x201010, B = 0x021100;
};
template <> struct Format<HALF> : Format<1> {
    static constexpr bool STACK = true;
    static __device__ __forceinline__ Acc mul(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
template <> struct Format<HALF2> : Format<HALF> {   // 00 10 01
    static constexpr int PAIRS = 3;
    static constexpr unsigned A = 0x010, B = 0x100;
};
template <> struct Format<BYTES> : Format<1> {
    typedef i32x16 Acc;
    static __device__ __forceinline__ Acc mul(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};

// fn(0), fn(1), .. with the numbers as types: the accumulators may only be indexed by constants, however long fn is
template <int N, int I = 0, typename Fn>
__device__ __forceinline__ void for_blocks(const Fn &fn) {
    if constexpr (I < N) {
        fn(std::integral_constant<int, I>());
        for_blocks<N, I + 1>(fn);
    }
}

// What a product needs besides its operands.  rows_dev (nullable): the rows of A that count, minus first_row, at most M.
// k_dev (nullable): the same for the contraction.  Both are read on the device, and count `times` times.
struct Shape {
    int M, Nn, K;
    const int *rows_dev;
    int rows_first;
    const int *k_dev;
    int k_first;
    int times = 1;
    int stack = 1;      // products of this shape, one item of a stack each
    int sym = 0;        // the result is symmetric: only tiles on and below the diagonal are formed
};
__device__ __forceinline__ int live(int most, const int *dev, int first, int times = 1) {
    return dev ? max(0, min(most, times * (*dev - first))) : most;
}

// Value k of row r of an operand: its planes added up; 0 from k_end on.
template <int FORM>
__device__ __forceinline__ float whole_value(const Operand &o, int r, int k, int k_end) {
    const bf16_t *p;
    bool in = k < k_end;
    if constexpr (FORM == PAIR) {
        int second;
        const int f = min(pair_row(r, 32, &second), o.rows - 1);
        p = (second ? o.p1 : o.p0) + f * o.ld + k;
    } else if constexpr (FORM == ROW) {
        p = o.p0 + min(r, o.rows - 1) * o.ld + k;
    } else {
        const bool second = FORM == COLPAIR && k >= o.half;
        const int d = k - (second ? o.half : 0);
        if (FORM == COLPAIR) in &= d < o.depth;
        p = (second ? o.p1 : o.p0) + d * o.ld + min(r, o.rows - 1);
    }
    return in ? from_bf16(p[2 * o.plane]) + from_bf16(p[o.plane]) + from_bf16(p[0]) : 0.f;
}

// The products of a wave's rows with the fp32 matrix instruction.  Rare, so one block and one value at a time: it must not take
// registers from the rest.
template <int MT, int NT, int FA, int FB>
__device__ __forceinline__ void product_exact(const Operand &A, const Operand &B, int m0, int n0, int k_first, int k_end, int lane,
                                              f32x16 (&acc)[MT][NT]) {
    const int l32 = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            f32x16 c = {};
#pragma unroll 1
            for (int k = k_first; k < k_end; k += 2)
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(whole_value<FB>(B, n0 + 32 * j + l32, k + h, k_end),
                                                         whole_value<FA>(A, m0 + 32 * i + l32, k + h, k_end), c, 0, 0, 0);
            acc[i][j] = c;
        }
}

// whether the sums of all rows that count are finite (operands may hold anything in rows behind them)
template <int MT, int NT>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[MT][NT], int rows, int lane) {
    bool ok = true;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        bool fine = true;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) fine &= __builtin_isfinite(acc[i][j][e]);
        ok &= fine || 32 * i + (lane & 31) >= rows;
    }
    return __all(ok);
}

// Tile order: rows that do not count have no tiles (their workgroups are the last ones); groups of kGroup tiles along m share their tiles
// along n, and an XCD walks a contiguous range, so that the workgroups that run at once on one XCD share operand rows in its L2.
constexpr int kGroup = 8;
__device__ __forceinline__ bool tile_of(int wg, int mt, int nt, int splits, int *tm, int *tn, int *split) {
    if (wg >= mt * nt * splits) return false;
    int id = remap_xcd(wg, mt * nt * splits);
    *split = id / (mt * nt);
    id -= *split * (mt * nt);
    const int group = id / (kGroup * nt), first = group * kGroup, size = min(kGroup, mt - first);
    const int in = id - group * kGroup * nt;
    *tm = first + in % size;
    *tn = in / size;
    return true;
}

// Tiles of one product of a shape, and in a stack: all tiles of a part of an item one after the other, so that an XCD has few items at a time;
// of a symmetric result row by row.  item: of the stack, times the parts, plus the part.
__device__ __host__ __forceinline__ long long tiles_in(const Shape &sh, int mt, int nt) { return sh.sym ? (long long)mt * (mt + 1) / 2 : (long long)mt * nt; }
__device__ __forceinline__ void tile_in_stack(const Shape &sh, int wg, int mt, int nt, int splits, int *tm, int *tn, int *item) {
    const int tiles = (int)tiles_in(sh, mt, nt), id = remap_xcd(wg, gridDim.x);
    *item = id / tiles;
    const int t = id - *item * tiles;
    if (sh.sym) {
        int r = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        r -= r * (r + 1) / 2 > t;
        r += (r + 1) * (r + 2) / 2 <= t;
        *tm = r, *tn = t - r * (r + 1) / 2;
    } else {
        const int group = t / (kGroup * nt), first = group * kGroup, size = min(kGroup, mt - first), in = t - group * kGroup * nt;
        *tm = first + in % size, *tn = in / size;
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// The tiled product.  BM x BN of the result per workgroup of 2 x 2 waves, or 4 x 2 (W 8) where tiles are large: two waves on a SIMD wait for
// different things (8192 x 4096 times 128000 6.97 ms with four, 6.65 with eight, the same bits; the matrix unit is busy 69 to 72 % of the cycles
// then, at the 1.54 to 1.6 GHz that power allows), steps of 64 along the contraction, through LDS buffers that
// are filled by loads which go straight there: NA for A, NB for B (three and two are all 160 KB for 256 x 256).  A long contraction over
// few tiles is cut into `splits` parts, whose sums are added up by a kernel of their own.
//
// An operand's tile is kept as it lies in memory.  By rows (ROW, PAIR): 128 bytes a row (whole lines: half lines at a time come at half the
// rate, 15 against 25 TB/s from the L2 caches), whose eight 16-byte pieces are exchanged by bits of the row so that 16 rows read at
// once fall on all 64 banks.  By columns (COL, COLPAIR): 64 rows of BM or BN values, 64-byte pieces exchanged by the row's bits, read with
// the transposing LDS load, which hands lane i of 16 the four k of column i from four rows of 32 bytes.
//
// Order of a step: its quarters of 16 indices; while one is multiplied, the fragments of the next are read, between the matrix
// instructions.  In the last quarter, after the first few products have been issued, comes the step's one barrier: behind it the next
// step is there for everybody (each wave has waited for its own loads) and this step's buffers are free (each wave has read them).
// Loads go out evenly: the address unit takes one every 18 clocks, and a wave that waits for it cannot issue matrix instructions.  Behind
// a barrier comes first the B whose buffer it has freed, still in the last quarter, then, over the second and third quarter that follow,
// such an A; with three and two buffers that A may stay in flight across the next barrier, with five of each all of three steps.
template <int N>
__device__ __forceinline__ int col_swizzle(int k) {   // N columns: N / 32 pieces of 64 bytes
    return ((k & 3) | ((k >> 3) & 1) << 2) & (N / 32 - 1);
}

constexpr int kWaves = 4;

// Brings an operand's tile of N rows, one step after the other.  A wave can issue about six other instructions per matrix instruction, so
// what a step needs is kept running: one base for all of a wave's loads, which moves along, and one offset per load.
template <int FORM, int N, int PL, int W = kWaves>
struct Stager {
    static constexpr bool COLS = FORM == COL || FORM == COLPAIR;
    static constexpr int Q = N / 8 / W;   // load instructions of a wave a step, 1024 bytes each
    static constexpr int PAIRS = Format<PL>::PAIRS;
    unsigned off[Q];
    gbyte_ptr base, base2;                     // of the current kStep indices; the second matrix (PAIR: of these indices, COLPAIR: its start)
    long long move, plane, at;                 // bytes: to the next kStep indices, to the next plane, to the current plane
    unsigned ld2, planes;                      // planes of the six products, the next one's lowest
    int wave, lane, K, depth, half, kt, pair;
    bool trimmed;
    // again: 0, or the indices that are there, which come twice within the one step (by columns)
    __device__ __forceinline__ void init(const Operand &o, int r0, int kt_, int K_, unsigned planes_, int wave_, int lane_, int again = 0) {
        wave = wave_, lane = lane_, K = K_, kt = kt_, pair = 0, planes = planes_, at = 0;
        const long long ld = o.ld * 2;
        ld2 = (unsigned)ld, plane = o.plane * 2;
        depth = o.depth, half = o.half;
        move = COLS ? kStep * ld : kStep * 2;
        // load q of this wave brings rows 8 (q W + wave) on: of a pair, with four waves, those of the first matrix for even q; with eight, those
        // of one matrix
        int second;
        const int top = min(FORM == PAIR ? pair_row(r0, 32, &second) : r0, o.rows - 1);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if constexpr (COLS) {
                const int pc = lane % (N / 8);
                const int c = ((pc / 4) ^ col_swizzle<N>(first_k(q))) * 4 + pc % 4;
                const int k = first_k(q) >= again && first_k(q) < 2 * again ? first_k(q) - again : first_k(q);
                off[q] = (unsigned)k * ld2 + (unsigned)(min(r0 + 8 * c, o.rows - 8) - r0) * 2;
            } else {
                int f = r0 + 8 * (q * W + wave), s;
                if constexpr (FORM == PAIR) f = pair_row(f, 32, &s);
                off[q] = (unsigned)(min(f + lane / 8, o.rows - 1) - top) * ld2 + first_k(q) * 2;
            }
        }
        if constexpr (COLS) base = (gbyte_ptr)(o.p0 + r0), base2 = (gbyte_ptr)(o.p1 + r0);
        else base = (gbyte_ptr)(o.p0 + (long long)top * o.ld), base2 = (gbyte_ptr)(o.p1 + (long long)top * o.ld);
        if (FORM == PAIR && W == 8 && wave >= 4) base = base2;
        if (FORM == COLPAIR && kt * kStep >= half) base = base2, base += (kt - half / kStep) * move;
        else base += kt * move;
        if (FORM == PAIR) base2 += kt * move;
        trimmed = false;
        trim();
    }
    // the index within the step of the first value (by columns: of all values) of this lane's 16 bytes of load q
    __device__ __forceinline__ int first_k(int q) const {
        if constexpr (COLS) return (q * W + wave) * (512 / N) + lane / (N / 8);
        else return ((lane % 8) ^ (4 * (wave & 1) + lane / 16)) * 8;
    }
    // indices from this step on that exist (by rows: in whole 16-byte pieces)
    __device__ __forceinline__ int left(int step) const {
        const int k0 = step * kStep;
        if constexpr (FORM == COLPAIR) return depth - (k0 >= half ? k0 - half : k0);
        else return COLS ? K - k0 : (K - k0 + 7) & ~7;
    }
    // Where less than a step is left, lanes beyond it read its start; clear() follows.
    __device__ __forceinline__ void trim() {
        const int n = left(kt);
        if (trimmed || n < kStep) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const unsigned by = first_k(q) * (COLS ? ld2 : 2u);
                const int was = FORM == COLPAIR ? depth % kStep : 0;   // only the end of the first matrix has something behind it
                if (trimmed && first_k(q) >= was) off[q] += by;
                if (n < kStep && first_k(q) >= n) off[q] -= by;
            }
            trimmed = n < kStep;
        }
    }
    __device__ __forceinline__ void next() {   // on to the next step: the next pair of planes, or the next indices
        if constexpr (PAIRS > 1) {
            if (++pair < PAIRS) {
                const unsigned q = planes >> (4 * pair);
                at = q & 1 ? plane : q & 2 ? 2 * plane : 0;
                return;
            }
            pair = 0, at = 0;
        }
        ++kt;
        base += move;
        if (FORM == PAIR) base2 += move;
        if (FORM == COLPAIR && kt * kStep == half) base = base2;
        if (kt * kStep < K) trim();
    }
    template <int q>
    __device__ __forceinline__ void load(unsigned lds) const {
        const gbyte_ptr p = FORM == PAIR && W == 4 && q % 2 ? base2 : base;
        load_lds16(PAIRS == 1 && PL != 2 ? p : p + at, off[q], lds + q * W * 1024);
    }
    // zeros for what is beyond the `n` indices left of a step (the same bytes this lane brought)
    __device__ __forceinline__ void clear(char *lds, int n) const {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (first_k(q) >= n) *(u32x4 *)(lds + (q * W + wave) * 1024 + lane * 16) = (u32x4){0, 0, 0, 0};
    }
};

// The fragments of a wave's T blocks of 32 rows from r0 of a tile of N.
template <int FORM, int N, int T>
struct Reader {
    static constexpr bool COLS = FORM == COL || FORM == COLPAIR;
    unsigned first[COLS ? T : 4], at[COLS ? T : 4];   // in the first buffer, in the current one
    __device__ __forceinline__ void init(unsigned lds, int r0, int lane) {
        if constexpr (COLS) {
            const int s = lane % 16, g = lane / 16;
            const int k = 8 * (g >> 1) + s / 4;
#pragma unroll
            for (int i = 0; i < T; ++i)
                first[i] = lds + k * (2 * N) + (((r0 / 32 + i) ^ col_swizzle<N>(k)) * 64) + (g & 1) * 32 + (s % 4) * 8;
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) first[c] = lds + (r0 + (lane & 31)) * 128 + (((2 * c + (lane >> 5)) ^ ((lane >> 1) & 7)) * 16);
        }
    }
    __device__ __forceinline__ void turn(unsigned buffer) {
#pragma unroll
        for (int i = 0; i < (COLS ? T : 4); ++i) {
            at[i] = first[i] + buffer;
            asm volatile("" : "+v"(at[i]));   // held, not formed anew for every read
        }
    }
    __device__ __forceinline__ u32x4 read(int c, int i) const {
        typedef const __attribute__((address_space(3))) char *p1;
        typedef __attribute__((address_space(3))) u32x4 *p4;
        const p1 p = (p1)(size_t)at[COLS ? i : c];
        if constexpr (COLS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 *p2;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p2)(p + c * (16 * 2 * N))));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((p2)(p + c * (16 * 2 * N) + 4 * 2 * N)));
            return (u32x4){lo[0], lo[1], hi[0], hi[1]};
        } else {
            return *(p4)(p + i * (32 * 128));
        }
    }
};

// LDS of a wave's epilogue: one block of 32 rows on its way to whole 16-byte pieces.
template <int NT> constexpr int kEpiBytes = 32 * (NT * 32 * 4 + 16);

template <int PL, int FA, int FB, int BM, int BN, int NA, int NB, int W, typename Epi>
__global__ __launch_bounds__(64 * W, W > kWaves || (NA * BM + NB * BN) * 128 <= 81920 ? 2 : 1) void gemm_kernel(Operand A, Operand B, Shape sh, int nt, int splits, Epi epi) {
    constexpr int MT = BM / (16 * W), NT = BN / 64, PAIRS = Format<PL>::PAIRS;
    static_assert(NA >= 3 && NB >= 2 && NB <= NA, "what may stay in flight at a step's barrier is counted for these");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int M = live(sh.M, sh.rows_dev, sh.rows_first, sh.times);
    const int K = live(sh.K, sh.k_dev, sh.k_first, sh.times);
    int tm, tn, split;
    if constexpr (Format<PL>::STACK) {
        int item;
        tile_in_stack(sh, blockIdx.x, (M + BM - 1) / BM, nt, splits, &tm, &tn, &item);
        split = item % splits;
        A.p0 += item / splits * A.each, B.p0 += item / splits * B.each;
        epi.item(item);
    } else {
        if (!tile_of(blockIdx.x, (M + BM - 1) / BM, nt, splits, &tm, &tn, &split)) return;
    }
    const int wm = wave / 2, wn = wave % 2;
    constexpr unsigned ABYTES = BM * 128, BBYTES = BN * 128, B0 = NA * ABYTES;   // A's buffers, then B's
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) char *)smem;
    Reader<FA, BM, MT> ra;
    Reader<FB, BN, NT> rb;
    ra.init(lds0, wm * MT * 32, lane);
    rb.init(lds0 + B0, wn * NT * 32, lane);
    typename Format<PL>::Acc acc[MT][NT] = {};
    // parts are whole steps of the contraction at its longest; what is beyond its actual end is left out
    const int per = ((sh.K + kStep - 1) / kStep + splits - 1) / splits;
    const int kt0 = split * per, kt1 = min((K + kStep - 1) / kStep, kt0 + per), steps = max(0, kt1 - kt0) * PAIRS;
    Stager<FA, BM, PL, W> sa;
    Stager<FB, BN, PL, W> sb;
    sa.init(A, tm * BM, kt0, K, Format<PL>::A, wave, lane);
    sb.init(B, tn * BN, kt0, K, Format<PL>::B, wave, lane, PL == 2 ? K / 2 : 0);
    constexpr int QA = Stager<FA, BM, PL, W>::Q, QB = Stager<FB, BN, PL, W>::Q;
    const unsigned lds_wave = lds0 + wave * 1024;
    auto load_a = [&](unsigned buffer, auto number) __attribute__((always_inline)) { sa.template load<decltype(number)::value>(lds_wave + buffer); };
    auto load_b = [&](unsigned buffer, auto number) __attribute__((always_inline)) { sb.template load<decltype(number)::value>(lds_wave + B0 + buffer); };
    // buffers of this step, of the next, and A's of the one before, which is free
    unsigned ao = 0, aprev = (NA - 1) * ABYTES, anext = ABYTES, bo = 0, bnext = BBYTES;
    int akt = kt0, as = 0;   // the step that arrives next
    // The step in these buffers is there and everybody may read it: its loads have landed (`ahead` that were issued later stay in flight),
    // all waves have read what they need of the step before, and what lies beyond the contraction is zero.
    auto arrive = [&](unsigned a_at, unsigned b_at, auto ahead) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(ahead)::value) : "memory");
        const int la = sa.left(akt), lb = sb.left(akt);
        if (__builtin_expect(min(la, lb) < kStep, 0)) {
            sa.clear(smem + a_at, la);
            sb.clear(smem + B0 + b_at, lb);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if (PAIRS == 1 || ++as == PAIRS) as = 0, ++akt;
    };
    u32x4 a[2][MT], b[2][NT];
    auto fetch = [&](int c, int r) __attribute__((always_inline)) {   // read r of the MT + NT of quarter c, as the products need them
        if (r == 0) a[c & 1][0] = ra.read(c, 0);
        else if (r <= NT) b[c & 1][r - 1] = rb.read(c, r - 1);
        else a[c & 1][r - NT] = ra.read(c, r - NT);
    };
    constexpr int P = MT * NT, R = MT + NT;
    constexpr int BAR = P / 4;   // products of the last quarter in front of the barrier
    constexpr int FAR = NA - 1 > NB ? NA - 1 : NB, BEHIND = (NA - 2) * QA + (NB - 2) * QB;
    // One step.  left: steps from this one on; FULL: more than FAR.
    auto step = [&](auto full, int left) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        const bool has_next = FULL || left > 1;
        for_blocks<4>([&](auto quarter) __attribute__((always_inline)) {
            constexpr int c = decltype(quarter)::value;
            for_blocks<P>([&](auto product) __attribute__((always_inline)) {
                constexpr int p = decltype(product)::value;
                if constexpr (c == 3 && p == BAR) {
                    if (has_next) {
                        if (FULL || left > FAR) arrive(anext, bnext, std::integral_constant<int, BEHIND>());
                        else arrive(anext, bnext, std::integral_constant<int, 0>());
                        ra.turn(anext);
                        rb.turn(bnext);
                    }
                }
                acc[p / NT][p % NT] = Format<PL>::mul(b[c & 1][p % NT], a[c & 1][p / NT], acc[p / NT][p % NT]);
                if constexpr (c < 3) {
#pragma unroll
                    for (int r = p * R / P; r < (p + 1) * R / P; ++r) fetch(c + 1, r);
                } else if constexpr (p >= BAR) {
                    constexpr int S = P - BAR;
                    if (has_next) {
#pragma unroll
                        for (int r = (p - BAR) * R / S; r < (p - BAR + 1) * R / S; ++r) fetch(0, r);
                    }
                    if (FULL || left > NB)   // a B, into this step's buffer
                        for_blocks<(p - BAR + 1) * QB / S - (p - BAR) * QB / S>([&](auto k) __attribute__((always_inline)) {
                            load_b(bo, std::integral_constant<int, (p - BAR) * QB / S + decltype(k)::value>());
                        });
                    if (p == P - 1 && (FULL || left > NB)) sb.next();
                }
                if constexpr (c == 1 || c == 2) {   // an A, into the buffer of the step before
                    if (FULL || left > NA - 1)
                        for_blocks<(p + 1) * (QA / 2) / P - p * (QA / 2) / P>([&](auto k) __attribute__((always_inline)) {
                            load_a(aprev, std::integral_constant<int, (c - 1) * (QA / 2) + p * (QA / 2) / P + decltype(k)::value>());
                        });
                    if (c == 2 && p == P - 1 && (FULL || left > NA - 1)) sa.next();
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        aprev = ao, ao = anext, anext = anext == (NA - 1) * ABYTES ? 0 : anext + ABYTES;
        bo = bnext, bnext = bnext == (NB - 1) * BBYTES ? 0 : bnext + BBYTES;
    };
    if (steps) {   // what earlier steps would have sent for
        for_blocks<(NA - 1 > NB ? NA - 1 : NB)>([&](auto s) __attribute__((always_inline)) {
            constexpr int at = decltype(s)::value;
            if (at < steps) {
                if constexpr (at < NA - 1) {
                    for_blocks<QA>([&](auto q) __attribute__((always_inline)) { load_a(at * ABYTES, q); });
                    sa.next();
                }
                if constexpr (at < NB) {
                    for_blocks<QB>([&](auto q) __attribute__((always_inline)) { load_b(at * BBYTES, q); });
                    sb.next();
                }
            }
        });
        if (steps > FAR) arrive(0, 0, std::integral_constant<int, BEHIND + QB>());
        else arrive(0, 0, std::integral_constant<int, 0>());
        ra.turn(0);
        rb.turn(0);
#pragma unroll
        for (int r = 0; r < R; ++r) fetch(0, r);
    }
    int left = steps;
#pragma unroll 1
    for (; left > FAR; --left) step(std::true_type(), 0);
#pragma unroll 1
    for (; left > 0; --left) step(std::false_type(), left);
    const int m0 = tm * BM + wm * MT * 32, n0 = tn * BN + wn * NT * 32;
    if constexpr (PL == 3) {
        if (m0 < M && n0 < sh.Nn && !all_finite(acc, M - m0, lane))
            product_exact<MT, NT, FA, FB>(A, B, m0, n0, kt0 * kStep, min(K, kt1 * kStep), lane, acc);
    }
    __syncthreads();   // the buffers are free for the epilogue
    if (m0 >= M || n0 >= sh.Nn) return;
    epi.run(acc, m0, n0, lane, M, sh.Nn, split, smem + wave * kEpiBytes<NT>);
}

template <int PL, int FA, int FB, int BM, int BN, int NA, int NB, int W = kWaves, typename Epi>
int launch_tiles(const char *name, const Operand &A, const Operand &B, const Shape &sh, int splits, const Epi &epi, hipStream_t s) {
    const int mt = ceil_div(sh.M, BM), nt = ceil_div(sh.Nn, BN);
    constexpr int LDS = (NA * BM + NB * BN) * 128;
    static_assert(W * kEpiBytes<BN / 64> <= LDS, "the epilogue's LDS is that of the buffers");
    const long long wgs = tiles_in(sh, mt, nt) * splits * sh.stack;
    const LaunchPlan p = make_plan(name, {PL, FA, FB, BM, BN, NA, NB, W}, {sh.M, sh.Nn, sh.K, splits, sh.stack, sh.sym}, dim3((unsigned)wgs), 64 * W, LDS);
    LC_PLAN_REQUIRE(p, wgs <= 0x7fffffffLL && splits >= 1);
    LC_PLAN_REQUIRE(p, Format<PL>::STACK ? sh.stack >= 1 && !sh.rows_dev && !sh.k_dev && (!sh.sym || (BM == BN && sh.M == sh.Nn && mt <= 4096))
                                         : sh.stack == 1 && !sh.sym);
    LC_PLAN_REQUIRE(p, A.ld % 8 == 0 && B.ld % 8 == 0 && A.plane % 8 == 0 && B.plane % 8 == 0);
    constexpr bool CA = FA == COL || FA == COLPAIR, CB = FB == COL || FB == COLPAIR;
    LC_PLAN_REQUIRE(p, CA ? A.rows % 8 == 0 && A.ld >= A.rows && A.rows >= sh.M : A.rows >= sh.M && A.ld >= sh.K);
    LC_PLAN_REQUIRE(p, CB ? B.rows % 8 == 0 && B.ld >= B.rows && B.rows >= sh.Nn : B.rows >= (FB == PAIR ? 1 : sh.Nn) && B.ld >= sh.K);
    LC_PLAN_REQUIRE(p, PL != 2 || (FA == COL && FB == COL && splits == 1 && sh.K <= kStep && sh.K % 2 == 0));
    LC_PLAN_REQUIRE(p, FA != PAIR && FA != COLPAIR && (FB != PAIR || sh.Nn == 64 * ceil_div(B.rows, 32)));
    LC_PLAN_REQUIRE(p, FB != COLPAIR || (B.half % kStep == 0 && B.depth >= 1 && B.half - B.depth < kStep && B.depth <= B.half &&
                                         sh.K == B.half + B.depth));
    LC_PLAN_REQUIRE(p, A.ld <= (1 << 22) && B.ld <= (1 << 22));   // 256 rows' offsets stay below 2^31 bytes
    LC_PLAN_REQUIRE(p, ptr_aligned16(A.p0) && ptr_aligned16(B.p0) && ptr_aligned16(B.p1));
    LC_LAUNCH(p, name, (gemm_kernel<PL, FA, FB, BM, BN, NA, NB, W, Epi>), s, A, B, sh, nt, splits, epi);
    return LC_OK;
}

// ---------------------------------------------------------------------------------------------------------------------------
// Epilogues.  A lane's values of one row lie 32 columns apart, four at a time; through LDS they become whole 16-byte pieces of rows, so
// that a wave's store covers lines.

// 32 rows of COLS values of type V on their way; the pitch spreads rows over the banks.
template <typename V, int COLS>
struct RowStage {
    static constexpr int PITCH = COLS * (int)sizeof(V) + 16, PIECES = COLS * (int)sizeof(V) / 16, EACH = 16 / (int)sizeof(V);
    char *lds;
    int lane;
    // four values of this lane's row from column c on
    __device__ __forceinline__ void put(int c, const V (&v)[4]) const {
        typedef V V4 __attribute__((ext_vector_type(4)));
        *(V4 *)(lds + (lane & 31) * PITCH + c * (int)sizeof(V)) = (V4){v[0], v[1], v[2], v[3]};
    }
    // each(row, column, piece) for all pieces; LDS serves a wave in order
    template <typename Each>
    __device__ __forceinline__ void take(const Each &each) const {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < 32 * PIECES / 64; ++p) {
            const int at = p * 64 + lane, row = at / PIECES, piece = at % PIECES;
            each(row, piece * EACH, *(const u32x4 *)(lds + row * PITCH + piece * 16));
        }
        __builtin_amdgcn_wave_barrier();
    }
};

// a piece of a row of `width` values from column n on, at any alignment
template <typename V>
__device__ __forceinline__ void store_piece(V *row, int n, int width, const u32x4 &w) {
    constexpr int EACH = 16 / sizeof(V);
    if (n + EACH <= width) {
        __builtin_memcpy(row + n, &w, 16);
    } else {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (n + e < width) {
                const unsigned x = w[e * sizeof(V) / 4];
                if constexpr (sizeof(V) == 4) ((unsigned *)row)[n + e] = x;
                else ((unsigned short *)row)[n + e] = (unsigned short)(x >> (16 * (e & 1)));
            }
    }
}

// The product itself, into one or two matrices of `width` columns: rows from `second` on go to out1.  index (nullable): row m
// goes to row index[m].  add (nullable): fp32 [M][width], added; factor (nullable): times *factor; then rounded.
template <typename T>
struct StoreEpi {
    T *out0, *out1;
    int second, rows0, rows1;   // rows that exist of each
    int width;
    const int *index;
    const float *add, *factor;
    // which row of its matrix row m goes to; -1: nowhere
    __device__ __forceinline__ int place(int m) const {
        const bool up = m >= second;
        const int r = up ? m - second : m;
        return r >= (up ? rows1 : rows0) ? -1 : index ? index[r] : r;
    }
    __device__ __forceinline__ T *row(int m, int place) const { return (m >= second ? out1 : out0) + (long long)place * width; }
    __device__ __forceinline__ void finish(int m, int n, float f, float (&v)[4], T (&o)[4]) const {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (add && n + r < width) v[r] += add[(long long)m * width + n + r];
            o[r] = narrow<T>(v[r] * f);
        }
    }
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int, int, char *lds) const {
        const RowStage<T, NT * 32> stage = {lds, lane};
        const float f = factor ? *factor : 1.f;
        // by the lane of the row in its block, all before the first store: a load behind a store waits until that has reached memory
        int places[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = m0 + 32 * i + (lane & 31);
            places[i] = m < M ? place(m) : -1;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = m0 + 32 * i + (lane & 31);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = 32 * j + 8 * q + 4 * (lane >> 5);
                    float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    T o[4];
                    finish(min(m, M - 1), n0 + c, f, v, o);
                    stage.put(c, o);
                }
            stage.take([&](int r, int c, const u32x4 &w) {
                const int to = m0 + 32 * i + r;
                const int at = __shfl(places[i], r);
                if (at >= 0) store_piece(row(to, at), n0 + c, width, w);
            });
        }
    }
};

// The sums of one part of the contraction, as they are: [split][M][ld] floats, ld a multiple of 4.
struct PartEpi {
    float *part;
    long long ld;
    int M;
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int live_rows, int, int split, char *lds) const {
        const RowStage<float, NT * 32> stage = {lds, lane};
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    stage.put(32 * j + 8 * q + 4 * (lane >> 5), v);
                }
            stage.take([&](int r, int c, const u32x4 &w) {
                const int m = m0 + 32 * i + r;
                if (m < live_rows && n0 + c < ld) *(u32x4 *)(part + ((long long)split * M + m) * ld + n0 + c) = w;
            });
        }
    }
};

// Adds the parts up in their order and stores the sums, four columns a thread.  Bound by the latency of the loads where the result
// is small, so kJoin parts are in flight at a time: 16 parts of 192 x 1024 3.9 us, 6.8 one after the other.  FOLD: the product's rows
// are the first and then the second parts of half as many.
constexpr int kJoin = 8;
template <typename T, bool FOLD>
__global__ __launch_bounds__(256) void join_parts_kernel(const float *part, long long ld, int splits, Shape sh, StoreEpi<T> epi) {
    const long long id = blockIdx.x * 256LL + threadIdx.x, quads = ld / 4;
    const int m = (int)(id / quads), n = (int)(id - m * quads) * 4;
    const int rows = live(sh.M, sh.rows_dev, sh.rows_first, sh.times) / (FOLD ? 2 : 1);
    if (m >= rows) return;
    const auto sum = [&](int row) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, p[kJoin];
        for (int i = 0; i < splits; i += kJoin) {
#pragma unroll
            for (int k = 0; k < kJoin; ++k) p[k] = *(const f32x4 *)(part + ((long long)min(i + k, splits - 1) * sh.M + row) * ld + n);
#pragma unroll
            for (int k = 0; k < kJoin; ++k)
                if (i + k < splits) s += p[k];
        }
        return s;
    };
    f32x4 s = sum(m);
    if constexpr (FOLD) s += sum(rows + m);
    const int at = epi.place(m);
    if (at < 0) return;
    T *const row = epi.row(m, at);
    float v[4] = {s[0], s[1], s[2], s[3]};
    T o[4];
    epi.finish(m, n, epi.factor ? *epi.factor : 1.f, v, o);
    if (n + 4 <= epi.width) {
        __builtin_memcpy(row + n, o, sizeof(o));
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (n + r < epi.width) row[n + r] = o[r];
    }
}

// How a product is cut: into tiles of 256 x 256, one on a compute unit, or of 128 x 128, two on one or, with more buffers, one; and its
// contraction into parts.
struct Cut {
    enum Tile { LARGE, SMALL, DEEP } tile;
    int splits;
};
// The cut that takes least by an estimate in microseconds from measured times: a step of a large tile 1.7, of two small ones that share
// a compute unit 0.82, of one that has it for itself and so five buffers 0.5 (192 rows of 4096 with weights from HBM: 44 us, 55 with the
// usual buffers), and what begins and ends a tile; joining parts moves 8 bytes a value at 4 TB/s.
// From four rounds of large tiles on these are taken in any case: they bring half the bytes into LDS per product, and the chip runs
// at the clock its power allows (8192 x 128000 x 4096 6.8 against 8.0 ms).  Both cuts at other sizes: 192 x 16384 x 4096 85 us large
// and 40 small; 1000 x 768 x 30011 in fp32 3330 and 1572, in 16 parts 256 and 265.
// Parts take no more than kMostParts floats, as many as the largest result that is cut at all: of 19000 products drawn from the ranges of
// gradients of up to 8192 rows two lose by it, 0.1 % by the estimate.
constexpr int kMostSplits = 32;
constexpr long long kMostParts = 1LL << 26;
inline Cut choose_cut(int M, int Nn, int K, int pairs, bool may_split) {
    const double large = (double)ceil_div(M, 256) * ceil_div(Nn, 256), small = (double)ceil_div(M, 128) * ceil_div(Nn, 128);
    if (large >= 4 * kComputeUnits) return Cut{Cut::LARGE, 1};
    const int steps = ceil_div(K, kStep);
    Cut best = {Cut::SMALL, 1};
    double least = 1e30;
    const long long result = M * round_up(Nn, 4);
    for (int s = 1; s == 1 || (may_split && s <= kMostSplits && s <= steps / 2 && s * result <= kMostParts); ++s) {
        const double part = (double)ceil_div(steps, s) * pairs;
        const double join = s > 1 ? 4 + 8e-6 * s * (double)M * Nn / 4 : 0;
        const double rounds = std::ceil(large * s / kComputeUnits), wgs = small * s;
        const double tl = rounds * (part * 1.7 + 15) + join;
        const bool deep = wgs <= kComputeUnits;
        const double ts = (deep ? part * 0.5 + 4 : std::max(1.0, wgs / (2 * kComputeUnits) + 0.25) * (part * 0.82 + 6)) + join;
        if (tl < least) best = {Cut::LARGE, s}, least = tl;
        if (ts < least) best = {deep ? Cut::DEEP : Cut::SMALL, s}, least = ts;
    }
    return best;
}

// W: waves of a large tile.
template <int PL, int FA, int FB, int W = kWaves, typename Epi>
int launch_cut(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Cut &c, const Epi &epi, hipStream_t s) {
    if (c.tile == Cut::LARGE) return launch_tiles<PL, FA, FB, 256, 256, 3, 2, W>(name, A, B, sh, c.splits, epi, s);
    if (c.tile == Cut::SMALL) return launch_tiles<PL, FA, FB, 128, 128, 3, 2>(name, A, B, sh, c.splits, epi, s);
    return launch_tiles<PL, FA, FB, 128, 128, 5, 5>(name, A, B, sh, c.splits, epi, s);
}

// columns of a wave in such a product
inline int product_wave_cols(int M, int Nn, int K, int pairs) { return choose_cut(M, Nn, K, pairs, false).tile == Cut::LARGE ? 128 : 64; }

// A product whose epilogue needs whole sums.
template <int PL, int FA, int FB, int W = kWaves, typename Epi>
int launch_gemm(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    if (sh.M == 0 || sh.Nn == 0) return LC_OK;
    return launch_cut<PL, FA, FB, W>(name, A, B, sh, choose_cut(sh.M, sh.Nn, sh.K, PL == 3 ? 6 : 1, false), epi, s);
}

// A product of up to kNarrow rows, as mini-batches that are answered have, with tiles of 64 rows: what waits for weights from HBM is more
// workgroups, and no row is padded to 128 (8-bit, 4096 long, tiles of 64 x 128 and 128 x 128: 192 rows times 8192 26 and 37 us, in fewer steps at a
// time 30, times 100003 158 and 173; 64 rows times 100003 107 and 113, 101 with 64 x 64).  A fourth tile ends what is gained: 8-bit, 192, 193 and 256
// rows times 100003 145, 168 and 181 us so and 153, 154 and 163 in the others, bf16, 1024 long, times 20011 14.5, 21.8 and 22.0 so and 18.6, 18.6 and
// 18.9 in the others; short of that only bf16 times 100003 loses (192 rows 263 and 247), and times 8192 up to 256 rows would gain (29 and 35).
constexpr int kNarrow = 192;
template <int PL, int FB, int BN, typename Epi>
int launch_narrow(const char *name, const Operand &A, const Operand &B, const Shape &sh, const Epi &epi, hipStream_t s) {
    constexpr int NB = BN == 64 ? 4 : 3;
    return launch_tiles<PL, ROW, FB, 64, BN, NB, NB>(name, A, B, sh, 1, epi, s);
}

// Floats that are enough for the parts of any product of up to M rows and up to K indices that is cut: a shorter product may be cut into more
// parts.
inline long long part_floats(int M, int Nn, int K) {
    const int most = std::min(kMostSplits, ceil_div(K, kStep) / 2);
    return most > 1 ? std::min(kMostParts, most * M * round_up(Nn, 4)) : 0;
}

// Scratch for the sums of parts: as many floats as were set aside.
struct Parts {
    float *at;
    long long floats;
};

// A product that is stored, cut along its contraction where that helps; FOLD: always through its parts.
template <int PL, int FA, int FB, bool FOLD = false, int W = kWaves, typename T>
int launch_product(const char *name, const Operand &A, const Operand &B, const Shape &sh, const StoreEpi<T> &epi, const Parts &part, hipStream_t s) {
    if (sh.M == 0 || sh.Nn == 0) return LC_OK;
    const Cut c = choose_cut(sh.M, sh.Nn, sh.K, PL == 3 ? 6 : 1, true);
    if (!FOLD && c.splits == 1) return launch_cut<PL, FA, FB, W>(name, A, B, sh, c, epi, s);
    const long long ld = round_up(sh.Nn, 4);
    const long long blocks = ((long long)(FOLD ? sh.M / 2 : sh.M) * (ld / 4) + 255) / 256;
    const LaunchPlan p = make_plan(name, {}, {sh.M, sh.Nn, c.splits}, dim3((unsigned)blocks), 256, 0);
    LC_PLAN_REQUIRE(p, blocks <= 0x7fffffffLL && part.at && c.splits * sh.M * ld <= part.floats);
    if (int rc = launch_cut<PL, FA, FB, W>(name, A, B, sh, c, PartEpi{part.at, ld, sh.M}, s)) return rc;
    LC_LAUNCH(p, name, (join_parts_kernel<T, FOLD>), s, part.at, ld, c.splits, sh, epi);
    return LC_OK;
}

}  // namespace head
}  // namespace lc
