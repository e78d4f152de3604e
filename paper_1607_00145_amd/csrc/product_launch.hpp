// product_launch.hpp -- which tiles a product of product.hpp takes, and its
// launch; included by one .hip file per element type.
#pragma once
#include "launch.hpp"
#include "product.hpp"

namespace gett {


template <typename T, ProductForm FORM, typename S>
gett_status_t product_tiles(ProductGroups groups, ProductArgs g, hipStream_t s)
{
    int64_t tm = (g.m + S::BM - 1) / S::BM;
    const int64_t tn = (g.n + S::BN - 1) / S::BN;
    g.tilesM = (int)tm;
    g.tilesMInv = recip(tm);
    if (groups == kByRows) tm = g.m / S::BM + g.experts + 1;
    if (groups == kByK) tm *= g.experts;
    if (!fits_launch(tm * tn, S::THREADS)) return GETT_ERROR_NOT_SUPPORTED;
    g.tilesN = (int)tn;
    g.tilesNInv = recip(tn);
    constexpr auto kernel = product_kernel<T, FORM, S>;
    if (allow_dynamic_lds<kernel>(S::LDS) != hipSuccess) return GETT_ERROR_HIP;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tm * tn)), dim3(S::THREADS), S::LDS, s, g, (int)groups);
    return launched(hipGetLastError());
}

typedef ProductShape<2, 2, 2, 2, 2> ProductMid;

template <typename T, ProductForm FORM>
gett_status_t product_form(ProductGroups groups, const ProductArgs &g, hipStream_t s)
{
    return product_tiles<T, FORM, ProductMid>(groups, g, s);
}

template <typename T>
gett_status_t product_launch(ProductForm form, ProductGroups groups, const ProductArgs &g, hipStream_t s)
{
    if (form == kRowsRows) return product_form<T, kRowsRows>(groups, g, s);
    if (form == kRowsColumns) return product_form<T, kRowsColumns>(groups, g, s);
    return product_form<T, kColumnsColumns>(groups, g, s);
}

}  // namespace gett
