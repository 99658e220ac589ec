// The matrix products of f16 operands.
#include "am_linear.h"

namespace wfd {

template <>
void am_product_forward<f16>(const AmProduct &p, hipStream_t st)
{
    am_product<f16, false, false>(p, st);
}

template <>
void am_product_dx<f16>(const AmProduct &p, hipStream_t st)
{
    am_product<f16, false, true>(p, st);
}

template <>
void am_product_dw<f16>(const AmProduct &p, hipStream_t st)
{
    am_product<f16, true, true>(p, st);
}

}  // namespace wfd
