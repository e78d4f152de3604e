// layer_util.hpp -- jobs of layer_util.hip's passes.
#pragma once
#include "product.hpp"

namespace gett {

// rows x cols numbers -> a copy on the 16-byte grid, `pieces` pieces a row
struct CopyJob {
    const void *src;
    void *dst;
    int64_t ld;              // of the source, elements
    int rows, cols, pieces;
    Recip piecesInv;
    const int32_t *order;    // rows by expert of `choices` rows a token, or nullptr
    int choices;
    Recip choicesInv;
    int perMatrix;           // rows of one of several matrices `step` apart (0: one matrix)
    Recip perMatrixInv;
    int64_t step;
};
gett_status_t copy_launch(gett_dtype_t t, const CopyJob &j, hipStream_t s);

// dZ (or nullptr) and, per workgroup row (slot), the sums of its columns (or nullptr)
struct SlopeJob {
    const void *dY, *Z;
    void *dZ;
    float *sums;
    int64_t ldy, ldz, ldd;
    int m, n;
    int activation;
    Drop drop;
    const int32_t *offsets;  // rows by expert, or nullptr
    int experts;
    int across, shift;       // workgroups along the columns, rows of one (set by the launch)
    Recip acrossInv;
};
int64_t slope_slots(int64_t m, int64_t n, int experts);   // experts 0: no offsets
gett_status_t slope_launch(gett_dtype_t t, SlopeJob j, hipStream_t s);
gett_status_t sums_launch(gett_dtype_t t, SlopeJob j, void *out, hipStream_t s);

struct CombineJob {
    const void *H, *weights, *residual;
    void *Y;
    const int32_t *place;
    int64_t ldh, ldr, ldy;
    int tokens, k, cols, runs;   // runs of eight columns
    Recip runsInv;
};
gett_status_t combine_launch(gett_dtype_t t, gett_dtype_t tH, gett_dtype_t tw, const CombineJob &j,
                             hipStream_t s);

struct CombineGradJob {
    const void *dY, *H, *weights;
    void *dH, *dweights;
    const int32_t *place, *offsets;
    int64_t ldy, ldh, ldd;
    int tokens, k, cols, experts;
};
gett_status_t combine_grad_launch(gett_dtype_t t, gett_dtype_t tw, const CombineGradJob &j, hipStream_t s);

gett_status_t product_launch_f32(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                 const ProductPlan &p, hipStream_t s);
gett_status_t product_launch_bf16(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                  const ProductPlan &p, hipStream_t s);
gett_status_t product_launch_f16(ProductForm form, ProductGroups groups, const ProductArgs &g,
                                 const ProductPlan &p, hipStream_t s);
gett_status_t product_pair_f32(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                               const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                               hipStream_t s);
gett_status_t product_pair_bf16(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                                const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                                hipStream_t s);
gett_status_t product_pair_f16(const ProductArgs &x, ProductGroups groupsX, const ProductPlan &px,
                               const ProductArgs &w, ProductGroups groupsW, const ProductPlan &pw,
                               hipStream_t s);
inline gett_status_t product_launch_one(gett_dtype_t t, ProductForm form, ProductGroups groups,
                                        const ProductArgs &g, const ProductPlan &p, hipStream_t s)
{
    if (t == GETT_FLOAT32) return product_launch_f32(form, groups, g, p, s);
    return t == GETT_BFLOAT16 ? product_launch_bf16(form, groups, g, p, s)
                              : product_launch_f16(form, groups, g, p, s);
}
// Slots of a shared sum begin at `slots` of the workspace.
inline gett_status_t product_launch_of(gett_dtype_t t, ProductForm form, ProductGroups groups,
                                       ProductArgs g, const ProductPlan &p, const Partials &hold,
                                       int64_t slots, hipStream_t s)
{
    if (p.slices > 1) {
        g.slots = reinterpret_cast<float *>(static_cast<char *>(hold.tiles) + slots);
        g.counters = hold.counters;
    }
    return product_launch_one(t, form, groups, g, p, s);
}

// The products dX = dz w and dW = dz^T x of a backward pass, one or both.  Of tiles of
// the same size they are one launch.
struct BackwardProducts {
    ProductArgs x = {}, w = {};
    ProductGroups groupsX = kWhole, groupsW = kWhole;
    ProductPlan px = {}, pw = {};
    bool wantX = false, wantW = false;
    // dX is m x k and sums over n, dW n x k and over m.  A launch of one for both saves 2.5
    // us, which may outweigh the better tiles for one of them.  (Both are planned also
    // where one is wanted, and shared sums are cut alike however many panels a stage has:
    // a gradient does not depend on what else is.)
    void plan(gett_dtype_t t, int64_t m, int64_t n, int64_t k, int64_t experts)
    {
        auto of_x = [&](int only) { return product_plan(t, kRowsColumns, groupsX, m, k, n, experts, only); };
        auto of_w = [&](int only) { return product_plan(t, kColumnsColumns, groupsW, n, k, m, experts, only); };
        px = of_x(-1);
        pw = of_w(-1);
        if (px.shape == pw.shape) return;
        double least = px.us + pw.us + 2.5;
        for (int shape = 0; shape <= kSlabs; ++shape) {
            const ProductPlan x1 = of_x(shape), w1 = of_w(shape);
            if (x1.us + w1.us >= least) continue;
            least = x1.us + w1.us;
            px = x1;
            pw = w1;
        }
    }
    int64_t slotsX() const { return wantX ? px.slotBytes : 0; }
    int64_t slotBytes() const { return slotsX() + (wantW ? pw.slotBytes : 0); }
    int64_t countersX() const { return wantX ? px.counters : 0; }
    uint64_t counters() const { return (uint64_t)(countersX() + (wantW ? pw.counters : 0)); }
    gett_status_t launch(gett_dtype_t t, const Partials &hold, int64_t slots, hipStream_t s)
    {
        auto share = [&](ProductArgs &g, const ProductPlan &p, int64_t at, int64_t counter) {
            if (p.slices <= 1) return;
            g.slots = reinterpret_cast<float *>(static_cast<char *>(hold.tiles) + slots + at);
            g.counters = hold.counters + counter;
        };
        share(x, px, 0, 0);
        share(w, pw, slotsX(), countersX());
        if (wantX && wantW && px.shape == pw.shape) {
            if (t == GETT_FLOAT32) return product_pair_f32(x, groupsX, px, w, groupsW, pw, s);
            return t == GETT_BFLOAT16 ? product_pair_bf16(x, groupsX, px, w, groupsW, pw, s)
                                      : product_pair_f16(x, groupsX, px, w, groupsW, pw, s);
        }
        gett_status_t st = GETT_SUCCESS;
        if (wantX) st = product_launch_one(t, kRowsColumns, groupsX, x, px, s);
        if (wantW && st == GETT_SUCCESS) st = product_launch_one(t, kColumnsColumns, groupsW, w, pw, s);
        return st;
    }
};

// ----------------------------------------------------------- host helpers ---

// Parts of a stream's workspace, each on the 256-byte grid.
struct Arena {
    uint64_t bytes = 0;
    int64_t take(int64_t n)
    {
        const int64_t at = (int64_t)bytes;
        bytes += (uint64_t)round_up(n, 256);
        return at;
    }
};

// A matrix as an operand of a product: as it lies, or copied onto the 16-byte grid
// with rows of `width` numbers, zeros behind the last column.
struct Operand {
    const char *p;
    int64_t ld;        // bytes
    int width;         // numbers of a row that may be read
    int64_t copyAt;    // in the workspace, -1: not copied
};
inline int64_t piece_numbers(gett_dtype_t t) { return 16 / type_size(t); }
// A tile's rows are reached by 32-bit offsets: 256 rows 16 MB apart at most.
constexpr int64_t kDirectStride = (int64_t)1 << 24;
inline bool on_grid(gett_dtype_t t, int64_t rows, int64_t cols, const void *p, int64_t stride)
{
    const int64_t item = type_size(t);
    return (uintptr_t)p % 16 == 0 && cols % piece_numbers(t) == 0 &&
           (rows <= 1 || (stride * item % 16 == 0 && stride * item < kDirectStride));
}
inline Operand operand_of(gett_dtype_t t, int64_t rows, int64_t cols, const void *p, int64_t stride,
                          bool direct, Arena &a, int64_t copyRows)
{
    const int64_t item = type_size(t), width = round_up(cols, piece_numbers(t));
    if (rows == 0 || cols == 0) return {nullptr, 16, 0, -1};
    if (direct)
        return {static_cast<const char *>(p), (rows > 1 ? stride : cols) * item, (int)cols, -1};
    return {nullptr, width * item, (int)width, a.take(copyRows * width * item)};
}

// Enqueues the copy of an operand that is not on the grid, into its workspace.
inline gett_status_t place_copy(gett_dtype_t t, Operand &o, const Partials &hold, int64_t rows,
                                int64_t cols, const void *p, int64_t stride, hipStream_t s,
                                const int32_t *order = nullptr, int choices = 1, int64_t perMatrix = 0,
                                int64_t step = 0)
{
    if (o.copyAt < 0) return GETT_SUCCESS;
    char *to = static_cast<char *>(hold.tiles) + o.copyAt;
    o.p = to;
    const int64_t pieces = o.width / piece_numbers(t);
    const CopyJob j = {p, to, rows > 1 ? stride : cols, (int)rows, (int)cols, (int)pieces,
                       recip(pieces), order, choices, recip(choices), (int)perMatrix,
                       recip(perMatrix > 0 ? perMatrix : 1), step};
    return copy_launch(t, j, s);
}

// A product's operands and sizes; its form and result are the caller's to fill in.
inline ProductArgs product_args(const Operand &M, const Operand &N, int64_t m, int64_t n, int64_t k)
{
    ProductArgs g = {};
    g.M = M.p;
    g.N = N.p;
    g.ldm = M.ld;
    g.ldn = N.ld;
    g.m = (int)m;
    g.n = (int)n;
    g.k = (int)k;
    return g;
}

}  // namespace gett
