// The products of gated layers with 8-bit operands (forward).
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_gated<f8>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<f8, true>(p, st);
    else am_gated_product<f8>(p, tile, st);
}

}  // namespace wfd
