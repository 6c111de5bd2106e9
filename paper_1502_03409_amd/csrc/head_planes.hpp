// Laying out operands: a matrix given by a functor becomes bf16 planes, by rows and / or transposed, padded with zeros to
// whole steps of the contraction.  Read once, written once; bound by HBM.
#pragma once
#include "head_common.hpp"

namespace lc {
namespace head {

// Where planes go: rows [..][ld] with ld the padded number of columns, and / or the transpose [..][ldT].
struct PlanesOut {
    bf16_t *rows = nullptr;    // may be null
    long long ld = 0, plane = 0;
    bf16_t *cols = nullptr;    // transposed; may be null
    long long ldT = 0, planeT = 0;
};

// One workgroup per 64 x 64 block, blocks along the columns fastest.  get(r, c) is the value or 0 outside the matrix; the
// transposed side has cols_out rows (those beyond are not written) and the row side rows_out.
template <int PL, typename Get>
__global__ __launch_bounds__(256) void planes_kernel(Get get, PlanesOut o, int rows_out, int cols_out, int cblocks) {
    __shared__ bf16_t t[PL][64][66];
    const int r0 = blockIdx.x / cblocks * 64, c0 = blockIdx.x % cblocks * 64;
    const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    if (get.idle(r0)) return;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int r = ty + 4 * i;
        const float v = get(r0 + r, c0 + tx);
        bf16_t p[3];
        if constexpr (PL == 3) split3(v, p);
        else p[0] = to_bf16(v);
#pragma unroll
        for (int q = 0; q < PL; ++q) {
            t[q][r][tx] = p[q];
            if (o.rows && r0 + r < rows_out) o.rows[q * o.plane + (long long)(r0 + r) * o.ld + c0 + tx] = p[q];
        }
    }
    if (!o.cols) return;
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int c = ty + 4 * i;
        if (c0 + c < cols_out)
#pragma unroll
            for (int q = 0; q < PL; ++q) o.cols[q * o.planeT + (long long)(c0 + c) * o.ldT + r0 + tx] = t[q][tx][c];
    }
}

// A stored matrix of R rows; `index` (nullable): row r is row index[r] of it, for r < *count
template <typename T>
struct Stored {
    const T *p;
    long long ld;
    int R, C;
    const int *index, *count;
    __device__ bool idle(int) const { return false; }
    __device__ float operator()(int r, int c) const {
        if (c >= C || r >= (index ? *count : R)) return 0.f;
        return widen<T>(p[(long long)(index ? index[r] : r) * ld + c]);
    }
};

template <int PL, typename Get>
int launch_planes(const char *name, const Get &get, const PlanesOut &o, int rows, int cols, int rows_out, int cols_out,
                  hipStream_t s) {
    const long long rb = (rows + 63) / 64, cb = (cols + 63) / 64;
    if (rb * cb == 0) return LC_OK;
    const LaunchPlan p = make_plan(name, {PL}, {rows, cols, rows_out, cols_out}, dim3((unsigned)(rb * cb)), 256, 0);
    LC_PLAN_REQUIRE(p, rb * cb <= 0x7fffffffLL);
    LC_PLAN_REQUIRE(p, !o.rows || o.ld >= cb * 64);
    LC_PLAN_REQUIRE(p, !o.cols || o.ldT >= rb * 64);
    LC_LAUNCH(p, name, (planes_kernel<PL, Get>), s, get, o, rows_out, cols_out, (int)cb);
    return LC_OK;
}

}  // namespace head
}  // namespace lc
