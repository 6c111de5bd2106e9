// The orthogonalised step for fp32 weights (muon.hpp).
#include "muon.hpp"

namespace lc {
namespace head {

template int muon<float>(const float *, const float *, const float *, float *, float *, int, int, int, float, float, float, bool, int, void *, hipStream_t);
template size_t muon_scratch<float>(int, int, int);

}  // namespace head
}  // namespace lc
