// The products of gated layers with f16 operands (forward).
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_gated<f16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<f16, true>(p, st);
    else am_gated_product<f16>(p, tile, st);
}

}  // namespace wfd
