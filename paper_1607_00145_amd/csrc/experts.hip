// experts.hip -- the experts' products of gett_layers.h and the sum of their rows.
//
// A list of products of different numbers of rows, which the device alone knows:
// the launch has as many tiles as any split of the rows among the experts could
// need (rows / tile + experts + 1), a workgroup finds its expert from the offsets,
// and those left over end at once.  8192 tokens of 4 among 32 experts, 2048 x 1536 in
// bf16: 283 us forwards (206 GFLOP: 0.73 PFLOP/s with the gather and the SiLU), 530
// for both gradients of a product (0.78); half a tile an expert, 1/8 of the work, is empty.
#include "layer_util.hpp"

namespace gett {

namespace {

struct ExpertSizes {
    int64_t tokens, rows, n, width;
    int k, experts;
};

gett_status_t sizes_ok(gett_dtype_t dtype, int64_t tokens, int k, int experts)
{
    if (!float_type(dtype) || tokens < 0 || k < 1 || experts < 1) return GETT_ERROR_INVALID_VALUE;
    if (tokens >= kLayerRows || experts > kMostExperts || k > kMostChoices || tokens * k >= kLayerRows)
        return GETT_ERROR_NOT_SUPPORTED;
    return GETT_SUCCESS;
}

// The experts' weights: experts x n x width.
gett_status_t weights_ok(gett_dtype_t dtype, int64_t experts, int64_t n, int64_t width, const void *W,
                         int64_t stride, int64_t step, Extent &e)
{
    e = {nullptr, 0};
    const gett_status_t st = layer_matrix(dtype, n, width, W, stride, e);
    if (st != GETT_SUCCESS || !e.bytes) return st;
    const __int128 all = (__int128)(experts - 1) * step * type_size(dtype) + e.bytes;
    if (experts > 1 && step < 0) return GETT_ERROR_INVALID_VALUE;
    if (all >= (__int128)1 << 62 || experts * n >= INT32_MAX) return GETT_ERROR_NOT_SUPPORTED;
    e.bytes = (int64_t)all;
    return GETT_SUCCESS;
}

struct WeightsOperand {
    Operand o;
    int64_t step;   // bytes
};
WeightsOperand weights_operand(gett_dtype_t t, int64_t experts, int64_t n, int64_t width, const void *W,
                               int64_t stride, int64_t step, bool anywhere, Arena &a)
{
    const int64_t item = type_size(t);
    const bool direct = anywhere || (on_grid(t, n, width, W, stride) &&
                                     (experts == 1 || step * item % 16 == 0));
    WeightsOperand w = {operand_of(t, n, width, W, stride, direct, a, experts * n), 0};
    w.step = w.o.copyAt >= 0 ? n * w.o.ld : step * item;
    return w;
}
gett_status_t place_weights(gett_dtype_t t, WeightsOperand &w, const Partials &hold, int64_t experts,
                            int64_t n, int64_t width, const void *W, int64_t stride, int64_t step,
                            hipStream_t s)
{
    return place_copy(t, w.o, hold, experts * n, width, W, stride, s, nullptr, 1, n, step);
}

}  // namespace

}  // namespace gett

extern "C" {

gett_status_t gett_experts(gett_dtype_t dtype, int64_t tokens, int k, int experts, int64_t n,
                           int64_t width, const void *X, int64_t stride_x, int gather,
                           const void *W, int64_t stride_w, int64_t stride_we, const void *bias,
                           int activation, const int32_t *order, const int32_t *offsets, void *Z,
                           int64_t stride_z, void *Y, int64_t stride_y, void *stream)
{
    using namespace gett;
    gett_status_t st = sizes_ok(dtype, tokens, k, experts);
    if (st != GETT_SUCCESS) return st;
    if (!activation_ok(activation)) return GETT_ERROR_INVALID_VALUE;
    const int64_t rows = tokens * k;
    Extent x, w, b = {}, z = {}, y, eo = {}, ef;
    st = layer_matrix(dtype, gather ? tokens : rows, width, X, stride_x, x);
    if (st == GETT_SUCCESS) st = weights_ok(dtype, experts, n, width, W, stride_w, stride_we, w);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, rows, n, Y, stride_y, y);
    if (st == GETT_SUCCESS && bias) st = layer_list((int64_t)experts * n, type_size(dtype), bias, b);
    if (st == GETT_SUCCESS && Z) st = layer_matrix(dtype, rows, n, Z, stride_z, z);
    if (st == GETT_SUCCESS && gather) st = layer_list(rows, 4, order, eo);
    if (st == GETT_SUCCESS) st = layer_list(rows ? experts + 1 : 0, 4, offsets, ef);
    if (st != GETT_SUCCESS || !y.bytes) return st;
    const Extent in[5] = {x, w, b, eo, ef};
    for (const Extent &e : in)
        if (!apart(y, e) || !apart(z, e)) return GETT_ERROR_INVALID_VALUE;
    if (!apart(y, z)) return GETT_ERROR_INVALID_VALUE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // rows that are gathered in the product are reached by 32-bit offsets
    const int64_t reach = tokens > 1 ? tokens * stride_x * type_size(dtype) : 0;
    // few rows are taken at any address
    const bool direct = on_grid(dtype, n, width, W, stride_w) &&
                        (experts == 1 || stride_we * type_size(dtype) % 16 == 0);
    const bool few = product_is_few(dtype, kByRows, rows, n, experts, direct);
    const bool gridX = few || (on_grid(dtype, gather ? tokens : rows, width, X, stride_x) &&
                               (!gather || reach < 0xffff0000ll));
    Arena arena;
    Operand ox = operand_of(dtype, gather ? tokens : rows, width, X, stride_x, gridX, arena, rows);
    WeightsOperand ow = weights_operand(dtype, experts, n, width, W, stride_w, stride_we, few, arena);
    Partials hold;
    if (arena.bytes) {
        st = stream_workspace(s, 0, arena.bytes, hold);
        if (st != GETT_SUCCESS) return st;
        st = place_copy(dtype, ox, hold, rows, width, X, stride_x, s, gather ? order : nullptr, k);
        if (st == GETT_SUCCESS)
            st = place_weights(dtype, ow, hold, experts, n, width, W, stride_w, stride_we, s);
        if (st != GETT_SUCCESS) return st;
    }
    ProductArgs g = product_args(ox, ow.o, rows, n, width);
    g.kM = ox.width;
    g.kN = ow.o.width;
    g.stepN = ow.step;
    g.experts = experts;
    g.offsets = offsets;
    if (gather && ox.copyAt < 0) {
        g.order = order;
        g.choices = k;
        g.choicesInv = recip(k);
    }
    g.out = {static_cast<const char *>(bias), nullptr, static_cast<char *>(Z), static_cast<char *>(Y), 0,
             stride_z, stride_y, activation, 0, {}};
    ProductPlan plan = {};
    if (few) plan.shape = kFewRows;
    else plan = product_plan(dtype, kRowsRows, kByRows, rows, n, width, experts);
    return product_launch_of(dtype, kRowsRows, kByRows, g, plan, hold, 0, s);
}

gett_status_t gett_experts_grad(gett_dtype_t dtype, int64_t tokens, int k, int experts, int64_t n,
                                int64_t width, const void *dY, int64_t stride_dy, const void *Z,
                                int64_t stride_z, const void *X, int64_t stride_x, int gather,
                                const void *W, int64_t stride_w, int64_t stride_we, int activation,
                                const int32_t *order, const int32_t *offsets, const int32_t *place,
                                void *dX, int64_t stride_dx, void *dW, void *dbias, void *stream)
{
    using namespace gett;
    gett_status_t st = sizes_ok(dtype, tokens, k, experts);
    if (st != GETT_SUCCESS) return st;
    if (!activation_ok(activation)) return GETT_ERROR_INVALID_VALUE;
    const int64_t rows = tokens * k, item = type_size(dtype);
    const bool active = activation != GETT_ACTIVATION_NONE;
    Extent y, z = {}, x = {}, w = {}, ex = {}, ew = {}, eb = {}, eo = {}, ep = {}, ef;
    st = layer_matrix(dtype, rows, n, dY, stride_dy, y);
    if (st == GETT_SUCCESS && active) st = layer_matrix(dtype, rows, n, Z, stride_z, z);
    if (st == GETT_SUCCESS && (width < 0 || width >= kLayerCols))
        st = width < 0 ? GETT_ERROR_INVALID_VALUE : GETT_ERROR_NOT_SUPPORTED;
    if (st == GETT_SUCCESS && experts * n >= INT32_MAX) st = GETT_ERROR_NOT_SUPPORTED;
    if (st == GETT_SUCCESS && dW) st = layer_matrix(dtype, gather ? tokens : rows, width, X, stride_x, x);
    if (st == GETT_SUCCESS && dX) st = weights_ok(dtype, experts, n, width, W, stride_w, stride_we, w);
    if (st == GETT_SUCCESS && dX) st = layer_matrix(dtype, gather ? tokens : rows, width, dX, stride_dx, ex);
    if (st == GETT_SUCCESS && dW) st = layer_list((int64_t)experts * n * width, item, dW, ew);
    if (st == GETT_SUCCESS && dbias) st = layer_list((int64_t)experts * n, item, dbias, eb);
    if (st == GETT_SUCCESS && gather && dW) st = layer_list(rows, 4, order, eo);
    if (st == GETT_SUCCESS && gather && dX) st = layer_list(rows, 4, place, ep);
    const bool wanted = ex.bytes || ew.bytes || eb.bytes;
    if (st == GETT_SUCCESS) st = layer_list(wanted ? experts + 1 : 0, 4, offsets, ef);
    if (st != GETT_SUCCESS || !wanted) return st;
    const Extent in[7] = {y, z, x, w, eo, ep, ef}, out[3] = {ex, ew, eb};
    for (int i = 0; i < 3; ++i) {
        for (const Extent &e : in)
            if (!apart(out[i], e)) return GETT_ERROR_INVALID_VALUE;
        for (int j = i + 1; j < 3; ++j)
            if (!apart(out[i], out[j])) return GETT_ERROR_INVALID_VALUE;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool products = ex.bytes || ew.bytes, sum = eb.bytes;
    const bool direct = !active && on_grid(dtype, rows, n, dY, stride_dy);
    Arena arena;
    Operand oz = operand_of(dtype, rows, n, dY, stride_dy, direct || !products, arena, rows);
    Operand ox = {nullptr, 16, 0, -1};
    WeightsOperand ow = {ox, 0};
    if (ew.bytes)
        ox = operand_of(dtype, rows, width, X, stride_x,
                        !gather && on_grid(dtype, rows, width, X, stride_x), arena, rows);
    if (ex.bytes) ow = weights_operand(dtype, experts, n, width, W, stride_w, stride_we, false, arena);
    const int64_t sumsAt = sum ? arena.take(slope_slots(rows, n, experts) * n * 4) : -1;
    // the rows' gradients, which a token sums in 32 bits
    const int64_t partsAt = ex.bytes && gather ? arena.take(rows * width * 4) : -1;
    BackwardProducts both;
    both.wantX = ex.bytes;
    both.wantW = ew.bytes;
    both.groupsX = kByRows;
    both.groupsW = kByK;
    both.plan(dtype, rows, n, width, experts);
    Partials hold;
    if (arena.bytes) {
        st = stream_workspace(s, 0, arena.bytes, hold);
        if (st != GETT_SUCCESS) return st;
    }
    char *ws = static_cast<char *>(hold.tiles);
    SlopeJob j = {dY, Z, nullptr, sum ? reinterpret_cast<float *>(ws + sumsAt) : nullptr, stride_dy,
                  stride_z, 0, (int)rows, (int)n, activation, {}, offsets, experts, 0, 0, {}};
    if (oz.copyAt >= 0) {
        oz.p = ws + oz.copyAt;
        j.dZ = ws + oz.copyAt;
        j.ldd = oz.width;
    }
    if (j.dZ || j.sums) st = slope_launch(dtype, j, s);
    if (st == GETT_SUCCESS && sum) st = sums_launch(dtype, j, dbias, s);
    if (st == GETT_SUCCESS)
        st = place_copy(dtype, ox, hold, rows, width, X, stride_x, s, gather ? order : nullptr, k);
    if (st == GETT_SUCCESS)
        st = place_weights(dtype, ow, hold, experts, n, width, W, stride_w, stride_we, s);
    if (st != GETT_SUCCESS) return st;
    ProductArgs &gx = both.x, &gw = both.w;
    gx = product_args(oz, ow.o, rows, width, n);
    gx.kM = oz.width;
    gx.fullN = ow.o.width;
    gx.stepN = ow.step;
    gx.out.Y = gather ? ws + partsAt : static_cast<char *>(dX);
    gx.out.ldy = gather ? width : stride_dx;
    gx.out.wide = gather ? 1 : 0;
    gw = product_args(oz, ox, n, width, rows);
    gw.fullM = oz.width;
    gw.fullN = ox.width;
    gw.stepN = n * width;
    gw.out.Y = static_cast<char *>(dW);
    gw.out.ldy = width;
    gx.experts = gw.experts = experts;
    gx.offsets = gw.offsets = offsets;
    st = both.launch(dtype, hold, 0, s);
    if (st == GETT_SUCCESS && ex.bytes && gather) {
        const int64_t runs = (width + 7) / 8;
        const CombineJob c = {ws + partsAt, nullptr, nullptr, dX, place, width, 0, stride_dx,
                              (int)tokens, k, (int)width, (int)runs, recip(runs)};
        st = combine_launch(dtype, GETT_FLOAT32, GETT_FLOAT32, c, s);
    }
    return st;
}

gett_status_t gett_combine(gett_dtype_t dtype, int64_t tokens, int k, int64_t cols, const void *H,
                           int64_t stride_h, gett_dtype_t dtype_w, const void *weights,
                           const int32_t *place, const void *residual, int64_t stride_r, void *Y,
                           int64_t stride_y, void *stream)
{
    using namespace gett;
    gett_status_t st = sizes_ok(dtype, tokens, k, 1);
    if (st != GETT_SUCCESS) return st;
    if (dtype_w != GETT_FLOAT32 && dtype_w != dtype) return GETT_ERROR_INVALID_VALUE;
    Extent h, w = {}, p = {}, r = {}, y;
    st = layer_matrix(dtype, tokens * k, cols, H, stride_h, h);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, tokens, cols, Y, stride_y, y);
    if (st == GETT_SUCCESS && residual) st = layer_matrix(dtype, tokens, cols, residual, stride_r, r);
    if (st == GETT_SUCCESS && y.bytes) st = layer_list(tokens * k, type_size(dtype_w), weights, w);
    if (st == GETT_SUCCESS && y.bytes) st = layer_list(tokens * k, 4, place, p);
    if (st != GETT_SUCCESS || !y.bytes) return st;
    const bool inPlace = residual == Y && (tokens == 1 || stride_r == stride_y);
    if (!apart(y, h) || !apart(y, w) || !apart(y, p) || !(inPlace || apart(y, r)))
        return GETT_ERROR_INVALID_VALUE;
    const int64_t runs = (cols + 7) / 8;
    const CombineJob j = {H, weights, residual, Y, place, stride_h, stride_r, stride_y, (int)tokens, k,
                          (int)cols, (int)runs, recip(runs)};
    return combine_launch(dtype, dtype, dtype_w, j, static_cast<hipStream_t>(stream));
}

gett_status_t gett_combine_grad(gett_dtype_t dtype, int64_t tokens, int k, int64_t cols,
                                const void *dY, int64_t stride_dy, const void *H, int64_t stride_h,
                                gett_dtype_t dtype_w, const void *weights, const int32_t *place,
                                int experts, const int32_t *offsets, void *dH, int64_t stride_dh,
                                void *dweights, void *stream)
{
    using namespace gett;
    gett_status_t st = sizes_ok(dtype, tokens, k, experts);
    if (st != GETT_SUCCESS) return st;
    if (dtype_w != GETT_FLOAT32 && dtype_w != dtype) return GETT_ERROR_INVALID_VALUE;
    const int64_t rows = tokens * k;
    Extent y, h = {}, w = {}, p = {}, f = {}, eh = {}, ew = {};
    st = layer_matrix(dtype, tokens, cols, dY, stride_dy, y);
    if (st == GETT_SUCCESS && dweights) st = layer_matrix(dtype, rows, cols, H, stride_h, h);
    if (st == GETT_SUCCESS && dH) st = layer_matrix(dtype, rows, cols, dH, stride_dh, eh);
    if (st == GETT_SUCCESS && eh.bytes) st = layer_list(rows, type_size(dtype_w), weights, w);
    if (st == GETT_SUCCESS && dweights) st = layer_list(rows, type_size(dtype_w), dweights, ew);
    const bool wanted = eh.bytes || ew.bytes;
    if (st == GETT_SUCCESS && wanted) st = layer_list(rows, 4, place, p);
    if (st == GETT_SUCCESS && eh.bytes) st = layer_list(experts + 1, 4, offsets, f);
    if (st != GETT_SUCCESS || !wanted) return st;
    const Extent in[5] = {y, h, w, p, f};
    for (const Extent &e : in)
        if (!apart(eh, e) || !apart(ew, e)) return GETT_ERROR_INVALID_VALUE;
    if (!apart(eh, ew)) return GETT_ERROR_INVALID_VALUE;
    const CombineGradJob j = {dY, H, weights, eh.bytes ? dH : nullptr, dweights, place, offsets, stride_dy,
                              stride_h, stride_dh, (int)tokens, k, (int)cols, experts};
    return combine_grad_launch(dtype, dtype_w, j, static_cast<hipStream_t>(stream));
}

}  // extern "C"
