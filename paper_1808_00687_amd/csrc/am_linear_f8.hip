// The matrix products of 8-bit operands (forward only).
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_forward<f8>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<f8>(p, st);
    else am_product<f8, false, false>(p, tile, st);
}

}  // namespace wfd
