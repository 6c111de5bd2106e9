// Products with 8-bit weights for fp32 rows (q8.hpp).
#include "q8.hpp"

namespace lc {
namespace head {

template int q8_rows<float>(const float *, int8_t *, float *, int, int, hipStream_t);
template int q8_matmul<float>(const float *, const int8_t *, const float *, float *, int, int, int, void *, hipStream_t);
template int q8_glu<float>(int, const float *, const int8_t *, const float *, const int8_t *, const float *, float *, int, int, int, void *, hipStream_t);

}  // namespace head
}  // namespace lc
