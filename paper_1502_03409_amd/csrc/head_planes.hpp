// Laying out operands: a matrix given by a functor becomes rows of bf16 planes, padded with zeros to whole 16-byte pieces.  Read
// once, written once, 16 bytes a thread and plane; bound by HBM: 30011 x 768 fp32 values into three planes, 230 MB, 36 us.  The one
// rounding here is that of a single plane to bf16, or of two to sixteen bits, for gradients that meet bf16 operands in the matrix unit; three
// planes lose nothing.
#pragma once
#include "head_common.hpp"

namespace lc {
namespace head {

// eight values as planes at p: 16 bytes each
template <int PL>
__device__ __forceinline__ void put_planes(bf16_t *to, long long plane, const float (&v)[8]) {
    bf16_t p[8][3];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (PL == 3) split3(v[e], p[e]);
        else if constexpr (PL == 2) split2(v[e], p[e]);
        else p[e][0] = to_bf16(v[e]);
    }
#pragma unroll
    for (int q = 0; q < PL; ++q) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (unsigned)p[2 * e][q] | (unsigned)p[2 * e + 1][q] << 16;
        *(u32x4 *)(to + q * plane) = w;
    }
}

// get(r, c, v): v[o][0..7] are columns c .. c + 7 of row r of output o (0 outside the matrix); output o lies `apart` * o columns to
// the right.  skip(r): rows that nobody reads.  beside(): something small that the first workgroup does as well.  Two planes: the second
// lies get.rows() rows behind the first, a number that the device may know alone.
template <int PL, int OUT, typename Get>
__global__ __launch_bounds__(256) void planes_kernel(Get get, bf16_t *dst, long long ld, long long plane, int rows, int pieces, int apart, long long from) {
    if (blockIdx.x == 0 && from == 0) get.beside();
    const long long at = from + blockIdx.x * 256LL + threadIdx.x;
    const int r = (int)(at / pieces), c = (int)(at - (long long)r * pieces) * 8;
    if (r >= rows || get.skip(r)) return;
    if constexpr (PL == 2) plane = get.rows() * ld;
    float v[OUT][8];
    get(r, c, v);
#pragma unroll
    for (int o = 0; o < OUT; ++o) put_planes<PL>(dst + (long long)r * ld + c + (long long)o * apart, plane, v[o]);
}

// eight consecutive values of a row from column c on (any alignment), zeros from column C on
template <typename T>
__device__ __forceinline__ void load8(const T *row, int c, int C, float (&v)[8]) {
    if (c + 8 <= C) {
        if constexpr (sizeof(T) == 4) {
            typedef f32x4 any __attribute__((aligned(4)));
            const f32x4 a = *(const any *)(row + c), b = *(const any *)(row + c + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
        } else {
            typedef u32x4 any __attribute__((aligned(2)));
            const u32x4 a = *(const any *)(row + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (e & 1) ? bf16_hi(a[e >> 1]) : bf16_lo(a[e >> 1]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < C ? widen<T>(row[c + e]) : 0.f;
    }
}

// A stored matrix of R rows
template <typename T>
struct Stored {
    const T *p;
    int R, C;
    __device__ void beside() const {}
    __device__ bool skip(int) const { return false; }
    __device__ void operator()(int r, int c, float (&v)[1][8]) const { load8(p + (long long)r * C, c, C, v[0]); }
};

// rows x cols (cols: of one output, padded to whole pieces) at dst
template <int PL, int OUT, typename Get>
int launch_planes(const char *name, const Get &get, bf16_t *dst, long long ld, long long plane, int rows, int cols, int apart, hipStream_t s) {
    const long long pieces = cols / 8;
    return in_launches(rows * pieces, [&](long long from, unsigned n) -> int {
        const LaunchPlan p = make_plan(name, {PL, OUT}, {rows, cols, apart}, dim3(n), 256, 0);
        LC_PLAN_REQUIRE(p, cols % 8 == 0 && ld % 8 == 0 && plane % 8 == 0 && apart % 8 == 0);
        LC_PLAN_REQUIRE(p, (long long)apart * (OUT - 1) + cols <= ld);
        LC_LAUNCH(p, name, (planes_kernel<PL, OUT, Get>), s, get, dst, ld, plane, rows, (int)pieces, apart, from);
        return LC_OK;
    });
}

}  // namespace head
}  // namespace lc
