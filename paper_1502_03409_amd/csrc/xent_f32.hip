// The softmax cross entropy for fp32 operands (xent.hpp).
#include "xent.hpp"

namespace lc {
namespace head {

template int xent<float>(const float *, const float *, const int64_t *, const float *, float *, float *, float *, float *, int, int, int, bool, void *,
                        hipStream_t);
template size_t xent_scratch<float>(int, int, int, bool);

}  // namespace head
}  // namespace lc
