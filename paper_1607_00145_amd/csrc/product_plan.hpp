// product_plan.hpp -- the shapes of product.hpp's tiles, and a product's plan.
#pragma once
#include <stdint.h>

#include "gett_layers.h"

namespace gett {

enum ProductForm { kRowsRows, kRowsColumns, kColumnsColumns };
enum ProductGroups { kWhole, kByRows, kByK };

constexpr int kFewRows = 3;   // product_few.hpp
constexpr int64_t kProductCus = 256;

bool product_is_few(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t k);

struct ProductPlan {
    int shape;                                  // tiles of 256 >> shape, or kFewRows
    int64_t tilesM, tilesN, bandRows, tiles;    // bandRows: rows of tiles of all experts
    int64_t full, slices, units;                // tiles from `full` on: `slices` workgroups
    int64_t counters, slotBytes;                // of the workspace
};
ProductPlan product_plan(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t k,
                         int64_t experts);

}  // namespace gett

// Which tiles a product takes (as gett_mx_tiles): for tests.
extern "C" void gett_product_tiles(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k,
                                   struct gett_tiles *out);
