// product_f16.hip -- the products of product.hpp on 16-bit IEEE operands.
#include "layer_util.hpp"
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f16(ProductForm form, ProductGroups groups, ProductArgs g, hipStream_t s)
{
    return product_launch<_Float16>(form, groups, g, s);
}
}  // namespace gett
