// product_f32.hip -- the products of product.hpp on 32-bit operands.
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f32(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s)
{
    return product_launch<float>(form, groups, g, p, s);
}
}  // namespace gett
