// product_f32.hip -- the products of product.hpp on 32-bit operands.
#include "layer_util.hpp"
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f32(ProductForm form, ProductGroups groups, ProductArgs g, hipStream_t s)
{
    return product_launch<float>(form, groups, g, s);
}
}  // namespace gett
