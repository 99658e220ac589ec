// The matrix products of bf16 operands.
#include "am_linear.h"

namespace wfd {

template <>
void am_product_forward<bf16>(const AmProduct &p, hipStream_t st)
{
    am_product<bf16, false, false>(p, st);
}

template <>
void am_product_dx<bf16>(const AmProduct &p, hipStream_t st)
{
    am_product<bf16, false, true>(p, st);
}

template <>
void am_product_dw<bf16>(const AmProduct &p, hipStream_t st)
{
    am_product<bf16, true, true>(p, st);
}

}  // namespace wfd
