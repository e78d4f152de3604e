// product_f16.hip -- the products of product.hpp on 16-bit IEEE operands.
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f16(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s)
{
    return product_launch<_Float16>(form, groups, g, p, s);
}
gett_status_t product_pair_f16(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                             const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                             hipStream_t s)
{
    return product_launch_pair<_Float16>(x, groupsX, px, w, groupsW, pw, s);
}
}  // namespace gett
