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
// 200 x 4096 x 4096; of blocks of 32 those of 2048 x 1024 x 1024, 128 x 2048 x 2048, 512 x
// 512 x 4096 and 2048 x 2048 x 128.
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
                                  {64, 2, 0.42, 0.22, 2.5, 3.5, 0.5}};
constexpr ShapeCost kCost32[3] = {{},   // (none: the middle ones are bound by the instructions)
                                  {128, 2, 3.90, 2.05, 4.0, 9.0, 2.5},
                                  {64, 2, 1.05, 0.60, 2.5, 3.5, 0.5}};
// Blocks of 32 x 32 by the form (a k of 32 columns of 16 bits is half a line).  us, tiles of
// 64 against blocks: 128 x 2048 x 2048 bf16 11.5, 5.9 and fp32 19.5, 13.6; 1024 x 512 x 1000
// fp32 20.5, 13.5; 2048 x 1024 x 1024 bf16 11.8, 14.0, dw 10.8, 22.0.
constexpr ShapeCost kBlocks16[3] = {{32, 3, 0.25, 0.065, 1.5, 0, 0},
                                    {32, 3, 0.32, 0.090, 1.5, 0, 0},
                                    {32, 3, 0.45, 0.140, 1.5, 0, 0}};
constexpr ShapeCost kBlocks32 = {32, 3, 0.44, 0.165, 1.4, 0, 0};
constexpr int64_t kCus = kProductCus;
// A block is a workgroup of 256 threads, and a launch has fewer than 2^32 threads also
// where it takes two products; the other shapes' workgroups take tile after tile.
constexpr int64_t kMostBlocks = (int64_t)1 << 22;

// a panel's time with so many workgroups at once
double panel_us(const ShapeCost &c, int64_t units)
{
    const double us = c.full * (double)((units + kCus - 1) / kCus) / c.perCu;
    return us < c.alone ? c.alone : us > c.full ? c.full : us;
}

}  // namespace

// y = x w^T of so few rows that a wavefront takes rows of w whole: up to 2 in 16 bits,
// unless the blocks of 32 columns keep every CU busy, and up to 4 in 32 bits; of experts
// up to two rows each.  us, rows of w against blocks: 1 row with 2048 x 2048 bf16 4.7, 6.4,
// 8192 x 4096 14.2, 11.9; 3 rows with 2048 x 2048 bf16 7.4, 6.5, fp32 9.5, 14.5; 16 and 64
// rows of 64 experts of 1024 x 2048 bf16 11.8, 19.4 and 40.7, 31.4, fp32 21.5, 72.4 and 74,
// 88.  Where w would have to be copied onto the 16-byte grid, up to 32 rows (of experts
// 64) take it as it lies: 18 rows of 12 experts of 333 x 500 bf16 4.8, 11.6.
bool product_is_few(gett_dtype_t dtype, ProductGroups groups, int64_t m, int64_t n, int64_t experts,
                    bool grid)
{
    const bool half = type_size(dtype) == 2;
    if (!grid) return m <= (groups == kByRows ? 64 : 32);
    if (groups == kByRows) return m <= 2 * experts && m <= (half ? 32 : 64);
    return half ? m <= 2 && n < 32 * kCus : m <= 4;
}

ProductPlan product_plan(gett_dtype_t dtype, ProductForm form, ProductGroups groups, int64_t m, int64_t n,
                         int64_t k, int64_t experts, int only)
{
    const int64_t KP = 128 / type_size(dtype);
    ProductPlan best = {};
    best.us = 1e300;
    for (int shape = 0; shape <= kSlabs; ++shape) {
        if (dtype == GETT_FLOAT32 && shape == 0) continue;
        if (only >= 0 && shape != only) continue;
        const ShapeCost &c = dtype == GETT_FLOAT32 ? (shape == kSlabs ? kBlocks32 : kCost32[shape])
                                                   : (shape == kSlabs ? kBlocks16[form] : kCost16[shape]);
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
        if (shape == kSlabs && p.units > kMostBlocks) continue;
        const int64_t all = kCus * c.perCu;
        if (groups != kWhole) {
            const double rounds = tiles / (double)all;
            // (the experts' tiles differ and even out over the rounds)
            p.us = (rounds < 1 ? 1 : rounds) * ((double)panels * panel_us(c, (int64_t)tiles) + c.tile);
            if (p.us < best.us) best = p;
            continue;
        }
        const int64_t rounds = p.tiles / all, rest = p.tiles % all;
        for (int64_t s = 1; s <= 16; ++s) {
            if (s > 1 && (shape == kSlabs || rest == 0 || rest * s > all || panels < 2 * s)) break;
            p.us = (double)rounds * ((double)panels * c.full + c.tile);
            if (rest) p.us += (double)((panels + s - 1) / s) * panel_us(c, rest * s) + c.tile;
            if (s > 1) p.us += c.join + c.joinEach * (double)s;
            if (p.us >= best.us) continue;
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
    if (gett::product_is_few(dtype, gett::kWhole, m, n, 0, true)) {
        *out = {0, 1, 0, (n + 31) / 32};
        return;
    }
    const gett::ProductPlan p = gett::product_plan(dtype, gett::kRowsRows, gett::kWhole, m, n, k, 0);
    out->edge = 256 >> p.shape;
    out->slices = p.slices;
    out->shared = p.counters;
    out->workgroups = p.units;
}
