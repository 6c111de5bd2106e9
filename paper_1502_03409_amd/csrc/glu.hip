// C ABI of the gated layer: arguments are checked on the host, then the operator for the operands' type runs (glu.hpp).
#include "head_common.hpp"

namespace lc {
namespace head {

template <typename T>
int glu_forward(int act, const T *x, const T *wg, const T *wu, T *h, T *gu, int N, int D, int F, void *ws, hipStream_t s);
template <typename T>
int glu_backward(int act, const T *x, const T *wg, const T *wu, const T *gu, const T *dh, T *dx, T *dwg, T *dwu, int N, int D, int F,
                 void *ws, hipStream_t s);
template <typename T>
size_t glu_scratch(int N, int D, int F, bool backward);

namespace {

bool glu_sizes(int32_t N, int32_t D, int32_t F, int dtype) {
    return head_rows(N) && head_width(D) && head_width(F) && (dtype == LC_F32 || dtype == LC_BF16);
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

size_t glu_workspace_bytes(int32_t N, int32_t D, int32_t F, int dtype, int backward) {
    if (!glu_sizes(N, D, F, dtype)) return 0;
    return dtype == LC_BF16 ? glu_scratch<bf16_t>(N, D, F, backward != 0) : glu_scratch<float>(N, D, F, backward != 0);
}

int glu_fwd(const void *x, const void *wg, const void *wu, void *h, void *gu, int32_t N, int32_t D, int32_t F, int act,
            int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!glu_sizes(N, D, F, dtype) || act < LC_ACT_SIGMOID || act > LC_ACT_GELU) return LC_EINVAL;
    if (!wg || !wu || (N && (!x || !h))) return LC_ENULL;
    for (const void *p : {x, wg, wu, (const void *)h, (const void *)gu, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if (!ws || ws_bytes < glu_workspace_bytes(N, D, F, dtype, 0)) return LC_EWORKSPACE;
    if (N == 0) return LC_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16)
        return glu_forward<bf16_t>(act, (const bf16_t *)x, (const bf16_t *)wg, (const bf16_t *)wu, (bf16_t *)h, (bf16_t *)gu, N, D, F, ws, s);
    return glu_forward<float>(act, (const float *)x, (const float *)wg, (const float *)wu, (float *)h, (float *)gu, N, D, F, ws, s);
}

int glu_bwd(const void *x, const void *wg, const void *wu, const void *gu, const void *dh, void *dx, void *dwg, void *dwu,
            int32_t N, int32_t D, int32_t F, int act, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!glu_sizes(N, D, F, dtype) || act < LC_ACT_SIGMOID || act > LC_ACT_GELU) return LC_EINVAL;
    if (!wg || !wu || !dwg || !dwu || (N && (!x || !gu || !dh))) return LC_ENULL;
    for (const void *p : {x, wg, wu, gu, dh, (const void *)dx, (const void *)dwg, (const void *)dwu, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if (!ws || ws_bytes < glu_workspace_bytes(N, D, F, dtype, 1)) return LC_EWORKSPACE;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16)
        return glu_backward<bf16_t>(act, (const bf16_t *)x, (const bf16_t *)wg, (const bf16_t *)wu, (const bf16_t *)gu, (const bf16_t *)dh,
                                    (bf16_t *)dx, (bf16_t *)dwg, (bf16_t *)dwu, N, D, F, ws, s);
    return glu_backward<float>(act, (const float *)x, (const float *)wg, (const float *)wu, (const float *)gu, (const float *)dh, (float *)dx,
                               (float *)dwg, (float *)dwu, N, D, F, ws, s);
}

}  // extern "C"
