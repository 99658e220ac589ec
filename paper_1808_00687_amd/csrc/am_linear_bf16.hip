// The matrix products of bf16 operands.
#include "am_linear.h"
#include "am_thin.h"

namespace wfd {

template <>
void am_product_forward<bf16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (tile == 0) am_thin<bf16>(p, st);
    else am_product<bf16, false, false>(p, tile, st);
}

template <>
void am_product_dx<bf16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    am_product<bf16, false, true>(p, tile, st);
}

template <>
void am_product_dw<bf16>(const AmProduct &p, int32_t tile, hipStream_t st)
{
    am_product<bf16, true, true>(p, tile, st);
}

}  // namespace wfd
