// product_bf16.hip -- the products of product.hpp on bfloat16 operands.
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_bf16(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s)
{
    return product_launch<bf16>(form, groups, g, p, s);
}
}  // namespace gett
