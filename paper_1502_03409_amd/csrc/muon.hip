// C ABI of the orthogonalised step: arguments are checked on the host, then the operator for the weights' type runs (muon.hpp).
#include "head_common.hpp"

namespace lc {
namespace head {

template <typename T>
int muon(const T *w, const T *g, const float *m, T *w_out, float *m_out, int count, int rows, int cols, float rate, float decay, float mu, bool ahead,
         int steps, void *ws, hipStream_t s);
template <typename T>
size_t muon_scratch(int count, int rows, int cols);

namespace {

bool muon_sizes(int32_t count, int32_t rows, int32_t cols, int dtype) {
    return head_rows(count) && head_width(rows) && head_width(cols) && std::min(rows, cols) <= (1 << 15) &&
           (long long)rows * cols <= (1LL << 40) / std::max(1, count) && (dtype == LC_F32 || dtype == LC_BF16);
}

}  // namespace
}  // namespace head
}  // namespace lc

using namespace lc;
using namespace lc::head;

extern "C" {

size_t muon_workspace_bytes(int32_t count, int32_t rows, int32_t cols, int dtype) {
    if (!muon_sizes(count, rows, cols, dtype)) return 0;
    return dtype == LC_BF16 ? muon_scratch<bf16_t>(count, rows, cols) : muon_scratch<float>(count, rows, cols);
}

int muon_step(const void *w, const void *g, const float *m, void *w_out, float *m_out, int32_t count, int32_t rows, int32_t cols, float rate,
              float decay, float momentum, int nesterov, int32_t steps, int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!muon_sizes(count, rows, cols, dtype) || steps < 1 || steps > 32) return LC_EINVAL;
    if (!std::isfinite(rate) || !std::isfinite(decay) || !std::isfinite(momentum)) return LC_EINVAL;
    if (count && (!w || !g || !m || !w_out || !m_out)) return LC_ENULL;
    for (const void *p : {w, g, (const void *)m, (const void *)w_out, (const void *)m_out, (const void *)ws})
        if (!ptr_aligned16(p)) return LC_EALIGN;
    if (!ws || ws_bytes < muon_workspace_bytes(count, rows, cols, dtype)) return LC_EWORKSPACE;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == LC_BF16)
        return muon<bf16_t>((const bf16_t *)w, (const bf16_t *)g, m, (bf16_t *)w_out, m_out, count, rows, cols, rate, decay, momentum, nesterov != 0,
                            steps, ws, s);
    return muon<float>((const float *)w, (const float *)g, m, (float *)w_out, m_out, count, rows, cols, rate, decay, momentum, nesterov != 0, steps, ws, s);
}

}  // extern "C"
