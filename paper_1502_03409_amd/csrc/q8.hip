// C ABI of the products with 8-bit weights: arguments are checked on the host, then the operator for the rows' type runs (q8.hpp).
#include "head_common.hpp"

namespace lc {
namespace head {

template <typename T>
int q8_rows(const T *x, int8_t *q, float *scale, int N, int D, hipStream_t s);
template <typename T>
int q8_matmul(const T *x, const int8_t *qw, const float *sw, T *y, int N, int D, int F, void *ws, hipStream_t s);
template <typename T>
int q8_glu(int act, const T *x, const int8_t *qg, const float *sg, const int8_t *qu, const float *su, T *h, int N, int D, int F, void *ws,
           hipStream_t s);

namespace {

// 2^17 products of two numbers up to 127 stay below 2^31
bool q8_sizes(int32_t N, int32_t D, int32_t F, int dtype) {
    return head_rows(N) && head_width(D) && D <= (1 << 17) && head_width(F) && (dtype == LC_F32 || dtype == LC_BF16);
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

int q8_row_bytes(int32_t D) { return q8_sizes(0, D, 1, LC_F32) ? (int32_t)round_up(D, 128) : 0; }

size_t q8_workspace_bytes(int32_t N, int32_t D, int32_t F, int dtype) {
    if (!q8_sizes(N, D, F, dtype)) return 0;
    Scratch sc(nullptr);
    (void)sc.take<int8_t>((long long)N * q8_row_bytes(D));
    (void)sc.take<float>(N);
    return std::max<size_t>(sc.used, 256);
}

int q8_rows(const void *x, int8_t *q, float *scale, int32_t N, int32_t D, int dtype, void *hip_stream) {
    if (!q8_sizes(N, D, 1, dtype)) return LC_EINVAL;
    if (N == 0) return LC_OK;
    if (!x || !q || !scale) return LC_ENULL;
    for (const void *p : {x, (const void *)q, (const void *)scale})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    hipStream_t s = (hipStream_t)hip_stream;
    return dtype == LC_BF16 ? q8_rows<bf16_t>((const bf16_t *)x, q, scale, N, D, s) : q8_rows<float>((const float *)x, q, scale, N, D, s);
}

int q8_matmul(const void *x, const int8_t *q, const float *scale, void *y, int32_t N, int32_t D, int32_t F, int dtype, void *ws,
              size_t ws_bytes, void *hip_stream) {
    if (!q8_sizes(N, D, F, dtype)) return LC_EINVAL;
    if (!q || !scale || (N && (!x || !y))) return LC_ENULL;
    for (const void *p : {x, (const void *)q, (const void *)scale, (const void *)y, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if (!ws || ws_bytes < q8_workspace_bytes(N, D, F, dtype)) return LC_EWORKSPACE;
    if (N == 0) return LC_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16) return q8_matmul<bf16_t>((const bf16_t *)x, q, scale, (bf16_t *)y, N, D, F, ws, s);
    return q8_matmul<float>((const float *)x, q, scale, (float *)y, N, D, F, ws, s);
}

int q8_glu_fwd(const void *x, const int8_t *qg, const float *sg, const int8_t *qu, const float *su, void *h, int32_t N, int32_t D, int32_t F,
               int act, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!q8_sizes(N, D, F, dtype) || act < LC_ACT_SIGMOID || act > LC_ACT_GELU) return LC_EINVAL;
    if (!qg || !sg || !qu || !su || (N && (!x || !h))) return LC_ENULL;
    for (const void *p : {x, (const void *)qg, (const void *)sg, (const void *)qu, (const void *)su, (const void *)h, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if (!ws || ws_bytes < q8_workspace_bytes(N, D, F, dtype)) return LC_EWORKSPACE;
    if (N == 0) return LC_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16) return q8_glu<bf16_t>(act, (const bf16_t *)x, qg, sg, qu, su, (bf16_t *)h, N, D, F, ws, s);
    return q8_glu<float>(act, (const float *)x, qg, sg, qu, su, (float *)h, N, D, F, ws, s);
}

}  // extern "C"
