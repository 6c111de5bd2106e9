// Log probabilities, entropies and likeliest words for fp32 operands (logp.hpp).
#include "logp.hpp"

namespace lc {
namespace head {

template int logp_forward<float>(const float *, const float *, const int64_t *, const LogpOut &, int, int, int, void *, hipStream_t);
template int logp_backward<float>(const float *, const float *, const int64_t *, const float *, const float *, const float *, const float *, float *, float *, int, int,
                               int, int, void *, hipStream_t);
template size_t logp_scratch<float>(int, int, int, int, bool, bool);

}  // namespace head
}  // namespace lc
