// product_f16.hip -- the products of product.hpp on 16-bit IEEE operands.
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f16(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s)
{
    return product_launch<_Float16>(form, groups, g, p, s);
}
}  // namespace gett
