// The softmax cross entropy for bf16 operands (xent.hpp).
#include "xent.hpp"

namespace lc {
namespace head {

template int xent<bf16_t>(const bf16_t *, const bf16_t *, const int64_t *, const float *, float *, float *, bf16_t *, bf16_t *, int, int, int, bool, void *,
                        hipStream_t);
template size_t xent_scratch<bf16_t>(int, int, int, bool);

}  // namespace head
}  // namespace lc
