// The gated layer for bf16 operands (glu.hpp).
#include "glu.hpp"

namespace lc {
namespace head {

template int glu_forward<bf16_t>(int, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, bf16_t *, int, int, int, void *, hipStream_t);
template int glu_backward<bf16_t>(int, const bf16_t *, const bf16_t *, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, bf16_t *, bf16_t *, int,
                                int, int, void *, hipStream_t);
template size_t glu_scratch<bf16_t>(int, int, int, bool);

}  // namespace head
}  // namespace lc
