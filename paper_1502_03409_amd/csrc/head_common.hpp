// What the kernels of the supervised head share: operand planes, bf16 conversion, workspaces, host checks.
#pragma once
#include "../../include/lc_head.h"
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lc_common.hpp"

namespace lc {
namespace head {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bf16_t to_bf16(float v) { return __builtin_bit_cast(bf16_t, (__bf16)v); }   // nearest, ties to even
__device__ __forceinline__ float from_bf16(bf16_t v) { return bf16_lo(v); }
template <typename T> __device__ __forceinline__ float widen(T v);
template <> __device__ __forceinline__ float widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen<bf16_t>(bf16_t v) { return from_bf16(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t narrow<bf16_t>(float v) { return to_bf16(v); }

// The three bf16 parts of an fp32 value: v = p[0] + p[1] + p[2] exactly, down to bits of 2^-133, the smallest that bf16 has.  Each part is the
// nearest bf16 to what remains, so the remainders have eight bits less each time; the first part of a value that would round to infinity is
// cut instead.  An infinity or NaN is its own first part, the others zero.
__device__ __forceinline__ void split3(float v, bf16_t (&p)[3]) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    if ((u & 0x7f800000u) == 0x7f800000u) {
        p[0] = (bf16_t)((u >> 16) | ((u & 0xffffu) ? 0x40u : 0u));   // a NaN whose payload lies in the low half stays one
        p[1] = p[2] = 0;
        return;
    }
    p[0] = to_bf16(v);
    if ((p[0] & 0x7f80u) == 0x7f80u) p[0] = (bf16_t)(u >> 16);
    float r = v - from_bf16(p[0]);
    p[1] = to_bf16(r);
    r -= from_bf16(p[1]);
    p[2] = to_bf16(r);
}

// Two bf16 parts of an fp32 value, sixteen bits.  Both have its sign and neither is zero unless the value is (the second is 2^-24 of a
// value that the first has whole), so that times infinity they add up to infinity and not to NaN.
__device__ __forceinline__ void split2(float v, bf16_t (&p)[3]) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    p[0] = (bf16_t)(u >> 16);
    const float r = v - from_bf16(p[0]);
    p[1] = to_bf16(r != 0.f ? r : v * 0x1p-24f);
    if ((u & 0x7f800000u) == 0x7f800000u) p[0] = p[1] = (bf16_t)((u >> 16) | ((u & 0xffffu) ? 0x40u : 0u));   // a NaN stays one
}

// Number of bf16 planes that hold an operand of storage type T, and of plane pairs whose products count.
template <typename T> struct Planes;
template <> struct Planes<bf16_t> { static constexpr int N = 1, PAIRS = 1; };
template <> struct Planes<float> { static constexpr int N = 3, PAIRS = 6; };

// An operand of a product, as bf16 planes: plane q starts at p0 + q * plane.  How the matrix lies (FORM):
//   ROW      row r of the operand at r * ld, contiguous along the contraction
//   PAIR     two such matrices (p0, p1) of `rows` rows each, blocks of 32 rows taken from them in turn, so that any tile of 64 rows
//            or more holds both values of every output it covers
//   COL      index k of the contraction at k * ld, contiguous along the operand's rows
//   COLPAIR  two such matrices one after the other along the contraction: `depth` indices of the first from 0 on, as many of the
//            second from `half` (a multiple of kStep) on
enum { ROW = 0, PAIR = 1, COL = 2, COLPAIR = 3 };
constexpr int kStep = 64;   // indices of the contraction a step
struct Operand {
    const bf16_t *p0, *p1;
    long long ld, plane;
    int rows;          // rows that exist, COL: in whole 16-byte pieces
    int depth, half;   // COLPAIR
};
__device__ __host__ __forceinline__ int pair_row(int v, int each, int *second) {   // each: rows taken in turn
    *second = v / each & 1;
    return v / (2 * each) * each + v % each;
}

inline long long round_up(long long a, long long b) { return (a + b - 1) / b * b; }

// Hands out 256-byte aligned pieces of a workspace; with a null base it only counts.
struct Scratch {
    char *base;
    size_t used = 0;
    explicit Scratch(void *ws) : base((char *)ws) {}
    template <typename T>
    T *take(long long n) {
        T *p = base ? (T *)(base + used) : nullptr;
        used += ((size_t)n * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

// Sizes of a head's matrices: widths 1 .. 2^20, rows 0 .. 2^24, so that every index within a row or a tile has 31 bits and
// every product of two sizes is formed in 64.
inline bool head_width(long long v) { return v >= 1 && v <= (1 << 20); }
inline bool head_rows(long long v) { return v >= 0 && v <= (1 << 24); }

}  // namespace head
}  // namespace lc
