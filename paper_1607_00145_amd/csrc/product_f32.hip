// product_f32.hip -- the products of product.hpp on 32-bit operands.
#include "product_launch.hpp"

namespace gett {
gett_status_t product_launch_f32(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s)
{
    return product_launch<float>(form, groups, g, p, s);
}
gett_status_t product_pair_f32(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                             const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                             hipStream_t s)
{
    return product_launch_pair<float>(x, groupsX, px, w, groupsW, pw, s);
}
}  // namespace gett
