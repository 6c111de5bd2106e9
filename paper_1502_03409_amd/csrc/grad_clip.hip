// Global 2-norm of a list of tensors, and the tensors scaled by min(1, max_norm / norm).
//
// Two passes over the values.  The list travels in the kernel arguments, as many tensors a launch as fit; a workgroup finds the
// tensor its block of values belongs to by bisection.  Squares are summed in 64 bits, whose rate is far above what memory brings,
// so nothing over- or underflows on the way; every block leaves one partial sum, and each workgroup of the second pass adds all of
// them up again in the same order instead of waiting for a kernel that does it once.
#include "head_common.hpp"

namespace lc {
namespace head {
namespace {

constexpr int kBatch = 128;                 // tensors a launch
constexpr long long kBlockValues = 16384;   // values a workgroup
constexpr long long kMostValues = 1LL << 40;

struct Batch {
    const void *src[kBatch];
    void *dst[kBatch];
    int first[kBatch];                      // first workgroup of each tensor
    unsigned char bf16[kBatch];
    long long n[kBatch];
    int count;
};

// The batch's tensor that workgroup b works on.
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

__device__ __forceinline__ float load_value(const void *p, bool bf16, long long i) {
    return bf16 ? from_bf16(((const bf16_t *)p)[i]) : ((const float *)p)[i];
}

__global__ __launch_bounds__(256) void squares_kernel(Batch t, double *partial) {
    const int k = tensor_of(t, blockIdx.x);
    const long long i0 = (long long)(blockIdx.x - t.first[k]) * kBlockValues, i1 = min(t.n[k], i0 + kBlockValues);
    double s = 0.0;
    for (long long i = i0 + threadIdx.x; i < i1; i += 256) {
        const double v = load_value(t.src[k], t.bf16[k], i);
        s += v * v;
    }
    s = block_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double whole_sum(const double *partial, long long blocks) {
    double s = 0.0;
    for (long long i = threadIdx.x; i < blocks; i += 256) s += partial[i];
    return block_sum(s);
}

__global__ __launch_bounds__(256) void norm_kernel(const double *partial, long long blocks, float *norm) {
    const double s = whole_sum(partial, blocks);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

__global__ __launch_bounds__(256) void scale_kernel(Batch t, const double *partial, long long blocks, float max_norm) {
    const double norm = sqrt(whole_sum(partial, blocks));
    const bool clips = __builtin_isfinite(norm) && norm > (double)max_norm;
    const float c = clips ? (float)((double)max_norm / norm) : 1.f;
    const int k = tensor_of(t, blockIdx.x);
    if (!clips && t.src[k] == t.dst[k]) return;
    const long long i0 = (long long)(blockIdx.x - t.first[k]) * kBlockValues, i1 = min(t.n[k], i0 + kBlockValues);
    for (long long i = i0 + threadIdx.x; i < i1; i += 256) {
        if (t.bf16[k]) ((bf16_t *)t.dst[k])[i] = clips ? to_bf16(from_bf16(((const bf16_t *)t.src[k])[i]) * c) : ((const bf16_t *)t.src[k])[i];
        else ((float *)t.dst[k])[i] = ((const float *)t.src[k])[i] * c;
    }
}

long long blocks_of(const lc_tensor_t *list, int32_t count) {
    long long b = 0;
    for (int i = 0; i < count; ++i) b += (list[i].n + kBlockValues - 1) / kBlockValues;
    return b;
}

bool list_ok(const lc_tensor_t *list, int32_t count) {
    if (count < 0) return false;
    long long values = 0;
    for (int i = 0; i < count; ++i) {
        if (list[i].n < 0 || list[i].n > kMostValues - values || (list[i].dtype != LC_F32 && list[i].dtype != LC_BF16)) return false;
        values += list[i].n;
    }
    return values / kBlockValues + count <= 0x7fffffffLL;
}

// calls fn(batch, workgroups, index of the first workgroup's partial sum) until all tensors have had their turn
template <typename Fn>
int for_batches(const lc_tensor_t *list, int32_t count, const Fn &fn) {
    long long done = 0;
    Batch t;
    t.count = 0;
    long long blocks = 0;
    for (int i = 0; i < count; ++i) {
        if (list[i].n) {
            t.src[t.count] = list[i].src;
            t.dst[t.count] = list[i].dst;
            t.n[t.count] = list[i].n;
            t.bf16[t.count] = list[i].dtype == LC_BF16;
            t.first[t.count++] = (int)blocks;
            blocks += (list[i].n + kBlockValues - 1) / kBlockValues;
        }
        if (t.count && (t.count == kBatch || i + 1 == count)) {
            if (int rc = fn(t, (unsigned)blocks, done)) return rc;
            done += blocks;
            blocks = 0;
            t.count = 0;
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
    const long long blocks = blocks_of(list, count);
    if (!ws || ws_bytes < 8 * (size_t)std::max(1LL, blocks)) return LC_EWORKSPACE;
    double *partial = (double *)ws;
    int rc = for_batches(list, count, [&](const Batch &t, unsigned n, long long at) -> int {
        const LaunchPlan p = make_plan("grad_squares", {}, {t.count}, dim3(n), 256, 0);
        LC_LAUNCH(p, "grad_norm", squares_kernel, s, t, partial + at);
        return LC_OK;
    });
    if (rc) return rc;
    const LaunchPlan p = make_plan("grad_norm", {}, {}, dim3(1), 256, 0);
    LC_LAUNCH(p, "grad_norm (sum)", norm_kernel, s, partial, blocks, norm);
    if (!scales) return LC_OK;
    return for_batches(list, count, [&](const Batch &t, unsigned n, long long) -> int {
        const LaunchPlan q = make_plan("grad_scale", {}, {t.count}, dim3(n), 256, 0);
        LC_LAUNCH(q, "grad_clip", scale_kernel, s, t, partial, blocks, max_norm);
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
    return 8 * (size_t)(values / kBlockValues + count + 1);   // each tensor ends in at most one workgroup that is not full
}

int grad_norm(const lc_tensor_t *list, int32_t count, float *norm, void *ws, size_t ws_bytes, void *hip_stream) {
    return clip(list, count, false, 0.f, norm, ws, ws_bytes, (hipStream_t)hip_stream);
}

int grad_clip(const lc_tensor_t *list, int32_t count, float max_norm, float *norm, void *ws, size_t ws_bytes, void *hip_stream) {
    return clip(list, count, true, max_norm, norm, ws, ws_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
