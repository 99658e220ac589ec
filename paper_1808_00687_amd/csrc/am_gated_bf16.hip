// The products of gated layers with bf16 operands (forward).
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_gated<bf16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<bf16, true>(p, st);
    else am_gated_product<bf16>(p, tile, st);
}

}  // namespace wfd
