// product_plan.hpp -- the shapes of product.hpp's tiles, and a product's plan.
#pragma once
#include <stdint.h>

#include "gett_layers.h"

namespace gett {

enum ProductForm { kRowsRows, kRowsColumns, kColumnsColumns };
enum ProductGroups { kWhole, kByRows, kByK };

constexpr int kSlabs = 3, kFewRows = 4;   // ProductSlabs; product_few.hpp
constexpr int64_t kProductCus = 256;

// grid: the columns' operand lies on the 16-byte grid
bool product_is_few(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t experts,
                    bool grid);

struct ProductPlan {
    int shape;                                  // tiles of 256 >> shape (of 32: kSlabs), or kFewRows
    int64_t tilesM, tilesN, bandRows, tiles;    // bandRows: rows of tiles of all experts
    int64_t full, slices, units;                // tiles from `full` on: `slices` workgroups
    int64_t counters, slotBytes;                // of the workspace
    double us;                                  // estimate
};
// only: the shape to take (-1: the best)
ProductPlan product_plan(gett_dtype_t dtype, ProductForm form, ProductGroups groups, int64_t m, int64_t n,
                         int64_t k, int64_t experts, int only = -1);

}  // namespace gett

// Which tiles a product takes (as gett_mx_tiles): for tests.
extern "C" void gett_product_tiles(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k,
                                   struct gett_tiles *out);
