// C ABI of the softmax's answers: arguments are checked on the host, then the operator for the operands' type runs (logp.hpp).
#include "head_common.hpp"

namespace lc {
namespace head {

template <typename T>
int logp_forward(const T *x, const T *w, const int64_t *tags, const LogpOut &out, int N, int D, int V, void *ws, hipStream_t s);
template <typename T>
int logp_backward(const T *x, const T *w, const int64_t *tags, const float *logp, const float *state, const float *dlogp, const float *dentropy, T *dx,
                  T *dw, int N, int D, int V, int T_, void *ws, hipStream_t s);
template <typename T>
size_t logp_scratch(int N, int D, int V, int K, bool given, bool grads);

namespace {

bool logp_sizes(int32_t N, int32_t D, int32_t V, int32_t T, int32_t K, int dtype) {
    return head_rows(N) && head_width(D) && head_width(V) && T >= 0 && T <= 64 && K >= 0 && K <= 64 && K <= V && (dtype == LC_F32 || dtype == LC_BF16);
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

size_t logp_workspace_bytes(int32_t N, int32_t D, int32_t V, int32_t T, int32_t K, int dtype, int grads) {
    if (!logp_sizes(N, D, V, T, K, dtype)) return 0;
    const auto bytes = [&](int k, bool g) { return dtype == LC_BF16 ? logp_scratch<bf16_t>(N, D, V, k, T > 0, g) : logp_scratch<float>(N, D, V, k, T > 0, g); };
    const size_t forward = std::max(bytes(K, false), bytes(0, false));   // fewer words may be looked for in another way
    return grads ? std::max(forward, bytes(0, true)) : forward;
}

int logp_fwd(const void *x, const void *w, const int64_t *tags, float *logp, float *entropy, int64_t *top, float *top_logp, float *state, int32_t N,
             int32_t D, int32_t V, int32_t T, int32_t K, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!logp_sizes(N, D, V, T, K, dtype)) return LC_EINVAL;
    if (!w || (N && (!x || (T && (!tags || !logp)) || (K && (!top || !top_logp))))) return LC_ENULL;
    for (const void *p : {x, w, (const void *)logp, (const void *)entropy, (const void *)top, (const void *)top_logp, (const void *)state,
                          (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if ((uintptr_t)tags & 7u) return LC_EALIGN;   // read one at a time: a batch may start at any row of a list
    if (!ws || ws_bytes < logp_workspace_bytes(N, D, V, T, K, dtype, 0)) return LC_EWORKSPACE;
    const LogpOut out = {logp, entropy, top, top_logp, state, T, K};
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16) return logp_forward<bf16_t>((const bf16_t *)x, (const bf16_t *)w, tags, out, N, D, V, ws, s);
    return logp_forward<float>((const float *)x, (const float *)w, tags, out, N, D, V, ws, s);
}

int logp_bwd(const void *x, const void *w, const int64_t *tags, const float *logp, const float *state, const float *dlogp, const float *dentropy,
             void *dx, void *dw, int32_t N, int32_t D, int32_t V, int32_t T, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!logp_sizes(N, D, V, T, 0, dtype)) return LC_EINVAL;
    if (!w || !dw || (N && (!x || !state || (T && (!tags || !logp || !dlogp))))) return LC_ENULL;
    for (const void *p : {x, w, (const void *)logp, (const void *)state, (const void *)dlogp, (const void *)dentropy, (const void *)dx,
                          (const void *)dw, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if ((uintptr_t)tags & 7u) return LC_EALIGN;
    if (!ws || ws_bytes < logp_workspace_bytes(N, D, V, T, 0, dtype, 1)) return LC_EWORKSPACE;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16)
        return logp_backward<bf16_t>((const bf16_t *)x, (const bf16_t *)w, tags, logp, state, dlogp, dentropy, (bf16_t *)dx, (bf16_t *)dw, N, D, V, T, ws, s);
    return logp_backward<float>((const float *)x, (const float *)w, tags, logp, state, dlogp, dentropy, (float *)dx, (float *)dw, N, D, V, T, ws, s);
}

}  // extern "C"
