// product_plan.cpp -- which tiles a product of product.hpp takes, and how many
// workgroups share one.
//
// A launch lasts as many rounds as its tiles fill the workgroups that are resident
// at once, each as long as its panels and a fixed part (first loads, results).  Tiles
// of a last, incomplete round may be cut along K so that their slices fill it, which
// costs a trip of the partial sums through memory.  The smallest estimate wins.
//
// us per panel with the CUs full and with one workgroup each, per tile, and for a
// join of s slices, measured: the products of 8192 x 8192 x 4096, 1023 x 515 x 1000 and
// 200 x 4096 x 4096.
#include "product_plan.hpp"

#include "layers.hpp"

namespace gett {

namespace {

struct ShapeCost {
    int edge;          // rows and columns of a tile
    int perCu;         // workgroups resident
    double full, alone, tile, join, joinEach;
};
constexpr ShapeCost kCost16[3] = {{256, 1, 1.50, 1.20, 9.0, 15.0, 6.0},
                                  {128, 2, 1.00, 0.50, 4.0, 9.0, 2.5},
                                  {64, 2, 0.42, 0.27, 2.5, 3.5, 0.5}};
constexpr ShapeCost kCost32[3] = {{},   // (none: the middle ones are bound by the instructions)
                                  {128, 2, 3.90, 2.05, 4.0, 9.0, 2.5},
                                  {64, 2, 1.05, 0.60, 2.5, 3.5, 0.5}};
constexpr int64_t kCus = kProductCus;

}  // namespace

// y = x w^T of up to 32 rows (and of up to 64 rows of experts in all), unless a long sum
// of few columns leaves most CUs without work: tiles share it.  us, few rows against
// tiles, of 32 rows: 8192 x 4096 bf16 21.8, 18.1 (16 rows 19.0, 17.8; 5 rows 17.9,
// 17.7), fp32 35.8, 42.6; 4096 x 1024 7.2, 8.1; 512 x 4096 17.6, 10.2; of 64 rows 8192 x
// 4096 30.7, 18.1.
bool product_is_few(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t k)
{
    if (groups == kByRows) return m <= 64;
    return m <= 4 || (m <= 32 && (n > 1024 || k * type_size(dtype) <= 4096));
}

ProductPlan product_plan(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t k,
                         int64_t experts)
{
    const int64_t KP = 128 / type_size(dtype);
    ProductPlan best = {};
    double least = 1e300;
    for (int shape = 0; shape < 3; ++shape) {
        if (dtype == GETT_FLOAT32 && shape == 0) continue;
        const ShapeCost &c = dtype == GETT_FLOAT32 ? kCost32[shape] : kCost16[shape];
        ProductPlan p = {};
        p.shape = shape;
        p.tilesM = (m + c.edge - 1) / c.edge;
        p.tilesN = (n + c.edge - 1) / c.edge;
        p.bandRows = p.tilesM;
        int64_t panels = (k + KP - 1) / KP;
        double tiles = (double)(p.tilesM * p.tilesN);
        if (groups == kByRows) {
            // as many tiles as any split among the experts needs; about so many of them
            // hold rows
            p.bandRows = m / c.edge + experts + 1;
            const double used = (double)(experts < m ? experts : m);
            tiles = (double)m / c.edge + used / 2;
            tiles = (tiles > used ? tiles : used) * (double)p.tilesN;
        } else if (groups == kByK) {
            p.bandRows = p.tilesM * experts;
            tiles *= (double)experts;
            panels = (panels + experts - 1) / experts;
        }
        p.tiles = p.full = p.units = p.bandRows * p.tilesN;
        p.slices = 1;
        const double slots = (double)(kCus * c.perCu);
        if (groups != kWhole) {
            const double rounds = tiles / slots;
            const double part = tiles <= kCus ? c.alone : c.full;
            // (the experts' tiles differ and even out over the rounds)
            const double us = (rounds < 1 ? 1 : rounds) * ((double)panels * part + c.tile);
            if (us < least) {
                least = us;
                best = p;
            }
            continue;
        }
        const int64_t all = kCus * c.perCu, rounds = p.tiles / all, rest = p.tiles % all;
        for (int64_t s = 1; s <= 16; ++s) {
            if (s > 1 && (rest == 0 || rest * s > all || panels < 2 * s)) break;
            double us = (double)rounds * ((double)panels * c.full + c.tile);
            if (rest)
                us += (double)((panels + s - 1) / s) * (rest * s <= kCus ? c.alone : c.full) + c.tile;
            if (s > 1) us += c.join + c.joinEach * (double)s;
            if (us >= least) continue;
            least = us;
            best = p;
            best.slices = s;
            best.full = s > 1 ? p.tiles - rest : p.tiles;
            best.units = best.full + (s > 1 ? rest * s : 0);
            best.counters = s > 1 ? rest : 0;
            best.slotBytes = s > 1 ? rest * s * c.edge * c.edge * 4 : 0;
        }
    }
    return best;
}

}  // namespace gett

extern "C" void gett_product_tiles(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k,
                                   struct gett_tiles *out)
{
    if (gett::product_is_few(dtype, gett::kWhole, m, n, k)) {
        *out = {0, 1, 0, (n + 31) / 32};
        return;
    }
    const gett::ProductPlan p = gett::product_plan(dtype, gett::kWhole, m, n, k, 0);
    out->edge = 256 >> p.shape;
    out->slices = p.slices;
    out->shared = p.counters;
    out->workgroups = p.units;
}
