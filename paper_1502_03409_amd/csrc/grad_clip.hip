// Global 2-norm of a list of tensors, and the tensors scaled by min(1, max_norm / norm).
//
// Two passes over the values, 16 bytes a lane and load; bound by HBM beyond the caches (the second pass walks backwards, so that it
// starts with what the first has left in them), by the two launches for short lists.  The list travels in the kernel arguments, as
// many tensors a launch as fit, cut into chunks; a workgroup finds the tensor of each of its chunks by bisection.  Squares are summed in
// 64 bits, whose rate is far above what memory brings, so nothing over- or underflows on the way; every workgroup leaves one partial
// sum, and each workgroup of the second pass adds all of them up again in the same order instead of waiting for a kernel that does it
// once.
//
// 10^5 values in three tensors 13 us, two launches; 5 10^7 in 60 tensors of both types, 172 MB, most of which the second pass finds in the
// 256 MB behind the L2 caches, 107 us; 10^9 values, which move 11.7 GB over both passes, 2.1 ms: 5.6 TB/s.
#include "head_common.hpp"

namespace lc {
namespace head {
namespace {

constexpr int kBatch = 128;              // tensors a launch
constexpr int kChunk = 4096;             // values of one tensor that a workgroup takes at a time
constexpr int kMostGroups = 2048;        // workgroups a launch: eight a compute unit
constexpr long long kMostValues = 1LL << 40;

struct Batch {
    const void *src[kBatch];
    void *dst[kBatch];
    int first[kBatch];                   // first chunk of each tensor
    unsigned char bf16[kBatch];
    long long n[kBatch];
    int count, chunks;
};

// The batch's tensor that chunk b belongs to.
__device__ __forceinline__ int tensor_of(const Batch &t, int b) {
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= b) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double part[4];
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

// Values src[0 .. n), n <= kChunk, through one(value's index) where no 16-byte vector fits and vec(index of its first value) for whole
// vectors of W values; the first `head` values come before the first aligned vector.
template <int W, typename One, typename Vec>
__device__ __forceinline__ void walk(int n, int head, const One &one, const Vec &vec) {
    head = min(head, n);
    const int vectors = (n - head) / W, tail = head + vectors * W;
    if ((int)threadIdx.x < head) one(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kChunk / W / 256; ++i) {
        const int v = i * 256 + threadIdx.x;
        if (v < vectors) vec(head + v * W);
    }
    if (tail + (int)threadIdx.x < n) one(tail + threadIdx.x);
}
template <typename T>
__device__ __forceinline__ int head_of(const T *p) { return (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T); }

template <typename T>
__device__ __forceinline__ double squares(const T *p, int n) {
    constexpr int W = 16 / sizeof(T);
    double s = 0.0;
    walk<W>(
        n, head_of(p), [&](int i) { const double v = widen<T>(p[i]); s += v * v; },
        [&](int i) {
            const u32x4 a = *(const u32x4 *)(p + i);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const unsigned w = W == 4 ? a[e & 3] : a[(e >> 1) & 3];
                const float v = W == 4 ? __builtin_bit_cast(float, w) : (e & 1) ? bf16_hi(w) : bf16_lo(w);
                s += (double)v * (double)v;
            }
        });
    return s;
}

__global__ __launch_bounds__(256) void squares_kernel(Batch t, double *partial) {
    double s = 0.0;
    for (int b = blockIdx.x; b < t.chunks; b += gridDim.x) {
        const int k = tensor_of(t, b);
        const long long i0 = (long long)(b - t.first[k]) * kChunk;
        const int n = (int)min((long long)kChunk, t.n[k] - i0);
        s += t.bf16[k] ? squares((const bf16_t *)t.src[k] + i0, n) : squares((const float *)t.src[k] + i0, n);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double whole_sum(const double *partial, int groups) {
    double s = 0.0;
    for (int i = threadIdx.x; i < groups; i += 256) s += partial[i];
    return block_sum(s);
}

__global__ __launch_bounds__(256) void norm_kernel(const double *partial, int groups, float *norm) {
    const double s = whole_sum(partial, groups);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// A factor of 1 copies: an infinity or NaN stays as it is, bit for bit.  Factors below 2^-100, which fp32 would hold with fewer bits or
// not at all, multiply in 64 bits.
struct Factor {
    double whole;
    float c;
    bool tiny;
    __device__ __forceinline__ explicit Factor(double f) : whole(f), c((float)f), tiny(f < 0x1p-100) {}
    __device__ __forceinline__ float times(float v) const { return tiny ? (float)((double)v * whole) : v * c; }
};
template <typename T>
__device__ __forceinline__ void scale(const T *p, T *o, int n, const Factor &f) {
    constexpr int W = 16 / sizeof(T);
    const bool copies = f.c == 1.f;
    const auto one = [&](int i) { o[i] = copies ? p[i] : narrow<T>(f.times(widen<T>(p[i]))); };
    if (((uintptr_t)p ^ (uintptr_t)o) & 15) {   // no vector is aligned on both sides
        for (int i = threadIdx.x; i < n; i += 256) one(i);
        return;
    }
    walk<W>(n, head_of(p), one, [&](int i) {
        u32x4 a = *(const u32x4 *)(p + i);
        if (!copies)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned w = a[e];
                if constexpr (W == 4) a[e] = __builtin_bit_cast(unsigned, f.times(__builtin_bit_cast(float, w)));
                else a[e] = (unsigned)to_bf16(f.times(bf16_lo(w))) | (unsigned)to_bf16(f.times(bf16_hi(w))) << 16;
            }
        *(u32x4 *)(o + i) = a;
    });
}

__global__ __launch_bounds__(256) void scale_kernel(Batch t, const double *partial, int groups, float max_norm, float *norm_out) {
    const double norm = sqrt(whole_sum(partial, groups));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const bool clips = __builtin_isfinite(norm) && norm > (double)max_norm;
    const Factor f(clips ? (double)max_norm / norm : 1.0);
    for (int b = t.chunks - 1 - (int)blockIdx.x; b >= 0; b -= gridDim.x) {
        const int k = tensor_of(t, b);
        if (!clips && t.src[k] == t.dst[k]) continue;
        const long long i0 = (long long)(b - t.first[k]) * kChunk;
        const int n = (int)min((long long)kChunk, t.n[k] - i0);
        if (t.bf16[k]) scale((const bf16_t *)t.src[k] + i0, (bf16_t *)t.dst[k] + i0, n, f);
        else scale((const float *)t.src[k] + i0, (float *)t.dst[k] + i0, n, f);
    }
}

// Workgroups of one launch: all batches together leave about kMostGroups partial sums.
int most_groups(int32_t count) { return std::max(32, kMostGroups / std::max(1, (count + kBatch - 1) / kBatch)); }

long long chunks_of(long long n) { return (n + kChunk - 1) / kChunk; }

bool list_ok(const lc_tensor_t *list, int32_t count) {
    if (count < 0) return false;
    long long values = 0;
    for (int i = 0; i < count; ++i) {
        if (list[i].n < 0 || list[i].n > kMostValues - values || (list[i].dtype != LC_F32 && list[i].dtype != LC_BF16)) return false;
        values += list[i].n;
    }
    return values / kChunk + count <= 0x7fffffffLL;
}

// calls fn(batch, workgroups, index of the first workgroup's partial sum) until all tensors have had their turn; *groups: in all
template <typename Fn>
int for_batches(const lc_tensor_t *list, int32_t count, int *groups, const Fn &fn) {
    Batch t;
    t.count = t.chunks = 0;
    *groups = 0;
    for (int i = 0; i < count; ++i) {
        if (list[i].n) {
            t.src[t.count] = list[i].src;
            t.dst[t.count] = list[i].dst;
            t.n[t.count] = list[i].n;
            t.bf16[t.count] = list[i].dtype == LC_BF16;
            t.first[t.count++] = t.chunks;
            t.chunks += (int)chunks_of(list[i].n);
        }
        if (t.count && (t.count == kBatch || i + 1 == count)) {
            const int n = std::min(t.chunks, most_groups(count));
            if (int rc = fn(t, (unsigned)n, *groups)) return rc;
            *groups += n;
            t.count = t.chunks = 0;
        }
    }
    return LC_OK;
}

int clip(const lc_tensor_t *list, int32_t count, bool scales, float max_norm, float *norm, void *ws, size_t ws_bytes, hipStream_t s) {
    if (!norm || (count > 0 && !list)) return LC_ENULL;
    if (!list_ok(list, count) || (scales && !(max_norm > 0.f))) return LC_EINVAL;
    if ((uintptr_t)norm & 3u || !ptr_aligned16(ws)) return LC_EALIGN;
    for (int i = 0; i < count; ++i) {
        if (!list[i].n) continue;
        if (!list[i].src || (scales && !list[i].dst)) return LC_ENULL;
        const uintptr_t low = list[i].dtype == LC_F32 ? 3u : 1u;
        if (((uintptr_t)list[i].src & low) || (scales && ((uintptr_t)list[i].dst & low))) return LC_EALIGN;
    }
    double *partial = (double *)ws;
    int groups = 0, again = 0;
    int rc = for_batches(list, count, &groups, [](const Batch &, unsigned, int) { return (int)LC_OK; });
    if (!ws || ws_bytes < 8 * (size_t)std::max(1, groups)) return LC_EWORKSPACE;
    rc = for_batches(list, count, &groups, [&](const Batch &t, unsigned n, int at) -> int {
        const LaunchPlan p = make_plan("grad_squares", {}, {t.count, t.chunks}, dim3(n), 256, 0);
        LC_LAUNCH(p, "grad_norm", squares_kernel, s, t, partial + at);
        return LC_OK;
    });
    if (rc) return rc;
    if (!scales || groups == 0) {
        const LaunchPlan p = make_plan("grad_norm", {}, {}, dim3(1), 256, 0);
        LC_LAUNCH(p, "grad_norm (sum)", norm_kernel, s, partial, groups, norm);
        return LC_OK;
    }
    return for_batches(list, count, &again, [&](const Batch &t, unsigned n, int at) -> int {
        const LaunchPlan q = make_plan("grad_scale", {}, {t.count, t.chunks}, dim3(n), 256, 0);
        LC_LAUNCH(q, "grad_clip", scale_kernel, s, t, partial, groups, max_norm, at == 0 ? norm : nullptr);
        return LC_OK;
    });
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

size_t grad_clip_workspace_bytes(int64_t values, int32_t count) {
    if (values < 0 || count < 0 || values > kMostValues) return 0;
    // a partial sum a workgroup; each tensor ends in at most one chunk that is not full
    return 8 * (size_t)std::min<long long>(values / kChunk + count + 1, (long long)most_groups(count) * (count / kBatch + 1));
}

int grad_norm(const lc_tensor_t *list, int32_t count, float *norm, void *ws, size_t ws_bytes, void *hip_stream) {
    return clip(list, count, false, 0.f, norm, ws, ws_bytes, (hipStream_t)hip_stream);
}

int grad_clip(const lc_tensor_t *list, int32_t count, float max_norm, float *norm, void *ws, size_t ws_bytes, void *hip_stream) {
    return clip(list, count, true, max_norm, norm, ws, ws_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
