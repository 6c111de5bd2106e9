// Log probabilities, entropies and likeliest words for bf16 operands (logp.hpp).
#include "logp.hpp"

namespace lc {
namespace head {

template int logp_forward<bf16_t>(const bf16_t *, const bf16_t *, const int64_t *, const LogpOut &, int, int, int, void *, hipStream_t);
template int logp_backward<bf16_t>(const bf16_t *, const bf16_t *, const int64_t *, const float *, const float *, const float *, const float *, bf16_t *, bf16_t *, int, int,
                               int, int, void *, hipStream_t);
template size_t logp_scratch<bf16_t>(int, int, int, int, bool, bool);

}  // namespace head
}  // namespace lc
