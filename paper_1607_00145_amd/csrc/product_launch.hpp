// product_launch.hpp -- the launch of a product of product.hpp; included by one .hip
// file per element type.
#pragma once
#include "launch.hpp"
#include "layer_util.hpp"
#include "product_few.hpp"

namespace gett {

// Fills in a product's tiles; false where there are too many.
template <typename T> bool product_fill(ProductArgs &g, const ProductPlan &p)
{
    // (ids are below 2^31 with a grid's stride added)
    if (p.units >= INT32_MAX / 2 || p.tiles >= INT32_MAX / 2 || 4 * p.tilesN >= INT32_MAX ||
        p.slices * ((int64_t)g.k * (int)sizeof(T) / 128 + 1) >= INT32_MAX)
        return false;
    g.tiles = (int)p.tiles;
    g.tilesM = (int)p.tilesM;
    g.tilesN = (int)p.tilesN;
    g.bandRows = (int)p.bandRows;
    g.tilesMInv = recip(p.tilesM);
    g.bandInv = recip(4 * p.tilesN);
    g.full = (int)p.full;
    g.slices = (int)p.slices;
    g.slicesInv = recip(p.slices);
    g.units = (int)p.units;
    return true;
}

template <typename T, ProductForm FORM, typename S>
gett_status_t product_tiles(ProductGroups groups, ProductArgs g, const ProductPlan &p, hipStream_t s)
{
    if (!product_fill<T>(g, p)) return GETT_ERROR_NOT_SUPPORTED;
    constexpr auto kernel = product_kernel<T, FORM, S>;
    if (allow_dynamic_lds<kernel>(S::LDS) != hipSuccess) return GETT_ERROR_HIP;
    const unsigned blocks = persistent_grid<kernel>(S::THREADS, (unsigned)g.units, S::LDS);
    if (blocks == 0) return GETT_ERROR_HIP;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(S::THREADS), S::LDS, s, g, (int)groups);
    return launched(hipGetLastError());
}

template <typename T, typename S>
gett_status_t product_pair(ProductArgs x, ProductGroups groupsX, const ProductPlan &px, ProductArgs w,
                           ProductGroups groupsW, const ProductPlan &pw, hipStream_t s)
{
    if (!product_fill<T>(x, px) || !product_fill<T>(w, pw)) return GETT_ERROR_NOT_SUPPORTED;
    constexpr auto kernel = product_pair_kernel<T, S>;
    if (allow_dynamic_lds<kernel>(S::LDS) != hipSuccess) return GETT_ERROR_HIP;
    const unsigned first = persistent_grid<kernel>(S::THREADS, (unsigned)x.units, S::LDS);
    const unsigned second = persistent_grid<kernel>(S::THREADS, (unsigned)w.units, S::LDS);
    if (first == 0 || second == 0) return GETT_ERROR_HIP;
    hipLaunchKernelGGL(kernel, dim3(first + second), dim3(S::THREADS), S::LDS, s, x, (int)groupsX, (int)first,
                       w, (int)groupsW);
    return launched(hipGetLastError());
}

// Eight wavefronts of 128 x 64 (one workgroup a CU: its LDS); four of 64 x 64 and of
// 32 x 32 (two a CU).
typedef ProductShape<4, 2, 2, 4, 2> ProductBig;
typedef ProductShape<2, 2, 2, 2, 2> ProductMid;
typedef ProductShape<1, 1, 2, 2, 4> ProductSmall;
// The same, one a CU: of few tiles each is alone on its CU and may have all of the
// LDS, with more panels on their way (the small ones with two for each barrier: 200 x
// 4096 x 4096 in bf16 18.3 -> 16.9 us).
typedef ProductShape<2, 2, 2, 2, 4> ProductMidDeep;
typedef ProductShape<1, 1, 2, 2, 4, 2> ProductSmallDeep;

// Few rows: a workgroup for 32 columns and, of experts, for each row that may be an
// expert's first.
template <typename T>
gett_status_t product_few(ProductGroups groups, ProductArgs g, hipStream_t s)
{
    const int m = g.m;
    const int64_t tn = ((int64_t)g.n + kFewCols - 1) / kFewCols;
    const int64_t blocks = tn * (groups == kByRows ? g.m : 1);
    if (!fits_launch(blocks, 1024)) return GETT_ERROR_NOT_SUPPORTED;
    g.tilesN = (int)tn;
    g.bandInv = recip(tn);
    auto launch = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, g, (int)groups);
        return launched(hipGetLastError());
    };
    // (experts: rows that share one read its weights once each, from the XCD's cache)
    if (groups == kByRows && m <= 2 * g.experts) return launch(product_row_kernel<T, 1>, 64 * kRowWaves);
    if (groups == kWhole && m == 1) return launch(product_row_kernel<T, 1>, 64 * kRowWaves);
    if (groups == kWhole && m == 2) return launch(product_row_kernel<T, 2>, 64 * kRowWaves);
    if (groups == kWhole && m <= 4) return launch(product_row_kernel<T, 4>, 64 * kRowWaves);
    return launch(product_few_kernel<T>, 64 * kFewWaves);
}

template <typename T, ProductForm FORM>
gett_status_t product_slabs_one(ProductGroups groups, ProductArgs g, const ProductPlan &p, hipStream_t s)
{
    typedef ProductSlabs S;
    if (!product_fill<T>(g, p) || !fits_launch(p.units, S::THREADS)) return GETT_ERROR_NOT_SUPPORTED;
    hipLaunchKernelGGL((product_slabs_kernel<T, FORM, S>), dim3((unsigned)g.units), dim3(S::THREADS), S::LDS, s,
                       g, (int)groups);
    return launched(hipGetLastError());
}

template <typename T, ProductForm FORM>
gett_status_t product_form(ProductGroups groups, const ProductArgs &g, const ProductPlan &p, hipStream_t s)
{
    if (p.shape == kSlabs) return product_slabs_one<T, FORM>(groups, g, p, s);
    if constexpr (sizeof(T) == 2)   // (in 32 bits the middle ones are bound by the instructions)
        if (p.shape == 0) return product_tiles<T, FORM, ProductBig>(groups, g, p, s);
    const bool deep = p.units <= kProductCus;
    if (p.shape == 1 && deep) return product_tiles<T, FORM, ProductMidDeep>(groups, g, p, s);
    if (p.shape == 1) return product_tiles<T, FORM, ProductMid>(groups, g, p, s);
    if (deep) return product_tiles<T, FORM, ProductSmallDeep>(groups, g, p, s);
    return product_tiles<T, FORM, ProductSmall>(groups, g, p, s);
}

template <typename T>
gett_status_t product_launch(ProductForm form, ProductGroups groups, const ProductArgs &g,
                             const ProductPlan &p, hipStream_t s)
{
    if (p.shape == kFewRows)
        return product_few<T>(groups, g, s);
    if (form == kRowsRows) return product_form<T, kRowsRows>(groups, g, p, s);
    if (form == kRowsColumns) return product_form<T, kRowsColumns>(groups, g, p, s);
    return product_form<T, kColumnsColumns>(groups, g, p, s);
}

// Both products of a backward pass, of the same tiles.
template <typename T>
gett_status_t product_launch_pair(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                                  const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                                  hipStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (px.shape == 0) return product_pair<T, ProductBig>(x, groupsX, px, w, groupsW, pw, s);
    if (px.shape == kSlabs) {
        typedef ProductSlabs S;
        ProductArgs gx = x, gw = w;
        if (!product_fill<T>(gx, px) || !product_fill<T>(gw, pw) || !fits_launch(px.units + pw.units, S::THREADS))
            return GETT_ERROR_NOT_SUPPORTED;
        hipLaunchKernelGGL((product_slabs_pair_kernel<T, S>), dim3((unsigned)(gx.units + gw.units)),
                           dim3(S::THREADS), S::LDS, s, gx, (int)groupsX, gx.units, gw, (int)groupsW);
        return launched(hipGetLastError());
    }
    const bool deep = px.units + pw.units <= kProductCus;
    if (px.shape == 1)
        return deep ? product_pair<T, ProductMidDeep>(x, groupsX, px, w, groupsW, pw, s)
                    : product_pair<T, ProductMid>(x, groupsX, px, w, groupsW, pw, s);
    return deep ? product_pair<T, ProductSmallDeep>(x, groupsX, px, w, groupsW, pw, s)
                : product_pair<T, ProductSmall>(x, groupsX, px, w, groupsW, pw, s);
}

}  // namespace gett
