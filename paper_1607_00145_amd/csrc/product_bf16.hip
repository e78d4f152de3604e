// product_bf16.hip -- the products of product.hpp on bfloat16 operands.
#include "layer_util.hpp"
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_bf16(ProductForm form, ProductGroups groups, ProductArgs g, hipStream_t s)
{
    return product_launch<bf16>(form, groups, g, s);
}
}  // namespace gett
