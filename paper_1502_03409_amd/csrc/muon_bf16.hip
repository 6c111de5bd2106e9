// The orthogonalised step for bf16 weights (muon.hpp).
#include "muon.hpp"

namespace lc {
namespace head {

template int muon<bf16_t>(const bf16_t *, const bf16_t *, const float *, bf16_t *, float *, int, int, int, float, float, float, bool, int, void *, hipStream_t);
template size_t muon_scratch<bf16_t>(int, int, int);

}  // namespace head
}  // namespace lc
