// The matrix products of f16 operands.
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_forward<f16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<f16>(p, st);
    else am_product<f16, false, false>(p, tile, st);
}

template <>
void am_product_dx<f16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    am_product<f16, false, true>(p, tile, st);
}

template <>
void am_product_dw<f16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    am_product<f16, true, true>(p, tile, st);
}

}  // namespace wfd
