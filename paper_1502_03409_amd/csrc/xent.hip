// C ABI of the softmax cross entropy: arguments are checked on the host, then the operator for the operands' type runs (xent.hpp).
#include "head_common.hpp"

namespace lc {
namespace head {

template <typename T>
int xent(const T *x, const T *w, const int64_t *target, const float *scale, float *loss, float *cost, T *dx, T *dw, int N, int D, int V,
         bool grads, void *ws, hipStream_t s);
template <typename T>
size_t xent_scratch(int N, int D, int V, bool grads);

namespace {

bool xent_sizes(int32_t N, int32_t D, int32_t V, int dtype) {
    return head_rows(N) && head_width(D) && head_width(V) && (dtype == LC_F32 || dtype == LC_BF16);
}

int xent_checked(const void *x, const void *w, const int64_t *target, const float *scale, float *loss, float *cost, void *dx, void *dw,
                 int32_t N, int32_t D, int32_t V, int dtype, bool grads, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!xent_sizes(N, D, V, dtype)) return LC_EINVAL;
    if (!w || !cost || (grads && !dw) || (N && (!x || !target || !loss))) return LC_ENULL;
    for (const void *p : {x, w, (const void *)dx, (const void *)dw, (const void *)ws, (const void *)scale, (const void *)loss,
                          (const void *)cost})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if ((uintptr_t)target & 7u) return LC_EALIGN;   // read one at a time: a batch may start at any row of a list
    if (!ws || ws_bytes < xent_workspace_bytes(N, D, V, dtype, grads)) return LC_EWORKSPACE;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16)
        return xent<bf16_t>((const bf16_t *)x, (const bf16_t *)w, target, scale, loss, cost, (bf16_t *)dx, (bf16_t *)dw, N, D, V, grads, ws, s);
    return xent<float>((const float *)x, (const float *)w, target, scale, loss, cost, (float *)dx, (float *)dw, N, D, V, grads, ws, s);
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

size_t xent_workspace_bytes(int32_t N, int32_t D, int32_t V, int dtype, int grads) {
    if (!xent_sizes(N, D, V, dtype)) return 0;
    return dtype == LC_BF16 ? xent_scratch<bf16_t>(N, D, V, grads != 0) : xent_scratch<float>(N, D, V, grads != 0);
}

int xent_fwd(const void *x, const void *w, const int64_t *target, const float *scale, float *loss, float *cost, int32_t N, int32_t D,
             int32_t V, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    return xent_checked(x, w, target, scale, loss, cost, nullptr, nullptr, N, D, V, dtype, false, ws, ws_bytes, hip_stream);
}

int xent_fwd_bwd(const void *x, const void *w, const int64_t *target, const float *scale, float *loss, float *cost, void *dx, void *dw,
                 int32_t N, int32_t D, int32_t V, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    return xent_checked(x, w, target, scale, loss, cost, dx, dw, N, D, V, dtype, true, ws, ws_bytes, hip_stream);
}

}  // extern "C"
