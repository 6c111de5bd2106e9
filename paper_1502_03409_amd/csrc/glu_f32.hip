// The gated layer for fp32 operands (glu.hpp).
#include "glu.hpp"

namespace lc {
namespace head {

template int glu_forward<float>(int, const float *, const float *, const float *, float *, float *, int, int, int, void *, hipStream_t);
template int glu_backward<float>(int, const float *, const float *, const float *, const float *, const float *, float *, float *, float *, int,
                                int, int, void *, hipStream_t);
template size_t glu_scratch<float>(int, int, int, bool);

}  // namespace head
}  // namespace lc
