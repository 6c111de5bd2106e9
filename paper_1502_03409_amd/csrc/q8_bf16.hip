// Products with 8-bit weights for bf16 rows (q8.hpp).
#include "q8.hpp"

namespace lc {
namespace head {

template int q8_rows<bf16_t>(const bf16_t *, int8_t *, float *, int, int, hipStream_t);
template int q8_matmul<bf16_t>(const bf16_t *, const int8_t *, const float *, bf16_t *, int, int, int, void *, hipStream_t);
template int q8_glu<bf16_t>(int, const bf16_t *, const int8_t *, const float *, const int8_t *, const float *, bf16_t *, int, int, int, void *, hipStream_t);

}  // namespace head
}  // namespace lc
