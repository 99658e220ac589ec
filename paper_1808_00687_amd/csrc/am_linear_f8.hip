// The matrix products of 8-bit operands (forward only).
#include "am_linear.h"

namespace wfd {

template <>
void am_product_forward<f8>(const AmProduct &p, hipStream_t st)
{
    am_product<f8, false, false>(p, st);
}

}  // namespace wfd
