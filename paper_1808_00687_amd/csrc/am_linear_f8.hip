// The matrix products of 8-bit operands (forward only).
#include "am_linear.h"

namespace wfd {

template <>
void am_product_forward<f8>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    am_product<f8, false, false>(p, tile, st);
}

}  // namespace wfd
