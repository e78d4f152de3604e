// layers.hip -- dropout and the linear layer of gett_layers.h.
#include "layer_util.hpp"

namespace gett {

namespace {

// Eight columns of a row a lane: one block of random bits, one vector each way.  Bound by
// memory: 16384 x 8192 in bf16 takes 85 to 92 us (537 MB: 5.8 to 6.3 TB/s, more than a
// copy of this size reaches here; a share of it stays in the last-level cache).
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T *X, int64_t ldx, T *Y, int64_t ldy,
                                                      int64_t total, int cols, int runs, Recip runsInv,
                                                      Drop d)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= total) return;
    const int64_t row = id < INT32_MAX ? quotient((uint32_t)id, runs, runsInv) : id / runs;
    const int col = (int)(id - row * runs) * 8, left = cols - col;
    float v[8];
    load8(X + row * ldx + col, left, v);
    if (d.cut) drop8(v, d, d.key(), (uint32_t)row, (uint32_t)col);
    store8(Y + row * ldy + col, left, v);
}

}  // namespace

}  // namespace gett

extern "C" {

gett_status_t gett_dropout(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                           int64_t stride_x, const gett_dropout_t *drop, void *Y, int64_t stride_y,
                           void *stream)
{
    using namespace gett;
    if (!float_type(dtype) || !drop || !drop_ok(drop)) return GETT_ERROR_INVALID_VALUE;
    Extent x, y;
    gett_status_t st = layer_matrix(dtype, rows, cols, X, stride_x, x);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, rows, cols, Y, stride_y, y);
    if (st != GETT_SUCCESS || !x.bytes) return st;
    if (!(X == Y && (rows == 1 || stride_x == stride_y)) && !apart(x, y)) return GETT_ERROR_INVALID_VALUE;
    const int64_t runs = (cols + 7) / 8, total = rows * runs, blocks = (total + 255) / 256;
    if (!fits_launch(blocks, 256)) return GETT_ERROR_NOT_SUPPORTED;
    const Drop d = drop_of(drop);
    return with_type(dtype, [&](auto v) {
        typedef decltype(v) T;
        hipLaunchKernelGGL(dropout_kernel<T>, dim3((unsigned)blocks), dim3(256), 0,
                           static_cast<hipStream_t>(stream), static_cast<const T *>(X), stride_x,
                           static_cast<T *>(Y), stride_y, total, (int)cols, (int)runs, recip(runs), d);
        return launched(hipGetLastError());
    });
}

gett_status_t gett_linear(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k, const void *X,
                          int64_t stride_x, const void *W, int64_t stride_w, const void *bias,
                          int activation, const gett_dropout_t *drop, const void *residual,
                          int64_t stride_r, void *Z, int64_t stride_z, void *Y, int64_t stride_y,
                          void *stream)
{
    using namespace gett;
    if (!float_type(dtype) || !activation_ok(activation) || !drop_ok(drop)) return GETT_ERROR_INVALID_VALUE;
    Extent x, w, b = {}, r = {}, z = {}, y;
    gett_status_t st = layer_matrix(dtype, m, k, X, stride_x, x);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, n, k, W, stride_w, w);
    if (st == GETT_SUCCESS) st = layer_matrix(dtype, m, n, Y, stride_y, y);
    if (st == GETT_SUCCESS && bias) st = layer_list(n, type_size(dtype), bias, b);
    if (st == GETT_SUCCESS && residual) st = layer_matrix(dtype, m, n, residual, stride_r, r);
    if (st == GETT_SUCCESS && Z) st = layer_matrix(dtype, m, n, Z, stride_z, z);
    if (st != GETT_SUCCESS || !y.bytes) return st;
    const bool inPlace = residual == Y && (m == 1 || stride_r == stride_y);
    if (!apart(y, x) || !apart(y, w) || !apart(y, b) || !apart(y, z) || !(inPlace || apart(y, r)) ||
        !apart(z, x) || !apart(z, w) || !apart(z, b) || !apart(z, r))
        return GETT_ERROR_INVALID_VALUE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    Arena arena;
    // (few rows are taken at any address)
    const bool direct = on_grid(dtype, n, k, W, stride_w), few = product_is_few(dtype, kWhole, m, n, 0, direct);
    const bool gridX = few || on_grid(dtype, m, k, X, stride_x), gridW = few || direct;
    Operand ox = operand_of(dtype, m, k, X, stride_x, gridX, arena, m);
    Operand ow = operand_of(dtype, n, k, W, stride_w, gridW, arena, n);
    ProductPlan plan = {};
    if (few) plan.shape = kFewRows;
    else plan = product_plan(dtype, kRowsRows, kWhole, m, n, k, 0);
    const int64_t slots = arena.take(plan.slotBytes);
    Partials hold;
    if (arena.bytes) {
        st = stream_workspace(s, (uint64_t)plan.counters, arena.bytes, hold);
        if (st != GETT_SUCCESS) return st;
        st = place_copy(dtype, ox, hold, m, k, X, stride_x, s);
        if (st == GETT_SUCCESS) st = place_copy(dtype, ow, hold, n, k, W, stride_w, s);
        if (st != GETT_SUCCESS) return st;
    }
    ProductArgs g = product_args(ox, ow, m, n, k);
    g.kM = ox.width;
    g.kN = ow.width;
    g.out = {static_cast<const char *>(bias), static_cast<const char *>(residual),
             static_cast<char *>(Z), static_cast<char *>(Y), stride_r, stride_z, stride_y, activation, 0,
             drop_of(drop)};
    return product_launch_of(dtype, kRowsRows, kWhole, g, plan, hold, slots, s);
}

gett_status_t gett_linear_grad(gett_dtype_t dtype, int64_t m, int64_t n, int64_t k, const void *dY,
                               int64_t stride_dy, const void *Z, int64_t stride_z, const void *X,
                               int64_t stride_x, const void *W, int64_t stride_w, int activation,
                               const gett_dropout_t *drop, void *dX, int64_t stride_dx, void *dW,
                               int64_t stride_dw, void *dbias, void *stream)
{
    using namespace gett;
    if (!float_type(dtype) || !activation_ok(activation) || !drop_ok(drop)) return GETT_ERROR_INVALID_VALUE;
    const bool active = activation != GETT_ACTIVATION_NONE;
    Extent y, z = {}, x = {}, w = {}, ex = {}, ew = {}, eb = {};
    gett_status_t st = layer_matrix(dtype, m, n, dY, stride_dy, y);
    if (st == GETT_SUCCESS && active) st = layer_matrix(dtype, m, n, Z, stride_z, z);
    if (st == GETT_SUCCESS && (k < 0 || k >= kLayerCols))
        st = k < 0 ? GETT_ERROR_INVALID_VALUE : GETT_ERROR_NOT_SUPPORTED;
    if (st == GETT_SUCCESS && dW) st = layer_matrix(dtype, m, k, X, stride_x, x);
    if (st == GETT_SUCCESS && dX) st = layer_matrix(dtype, n, k, W, stride_w, w);
    if (st == GETT_SUCCESS && dX) st = layer_matrix(dtype, m, k, dX, stride_dx, ex);
    if (st == GETT_SUCCESS && dW) st = layer_matrix(dtype, n, k, dW, stride_dw, ew);
    if (st == GETT_SUCCESS && dbias) st = layer_list(n, type_size(dtype), dbias, eb);
    if (st != GETT_SUCCESS) return st;
    const Extent in[4] = {y, z, x, w}, out[3] = {ex, ew, eb};
    for (int i = 0; i < 3; ++i) {
        for (const Extent &e : in)
            if (!apart(out[i], e)) return GETT_ERROR_INVALID_VALUE;
        for (int j = i + 1; j < 3; ++j)
            if (!apart(out[i], out[j])) return GETT_ERROR_INVALID_VALUE;
    }
    if (!ex.bytes && !ew.bytes && !eb.bytes) return GETT_SUCCESS;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Drop d = drop_of(drop);
    const bool products = ex.bytes || ew.bytes, sum = eb.bytes;
    const bool direct = !active && !d.cut && on_grid(dtype, m, n, dY, stride_dy);
    Arena arena;
    Operand oz = operand_of(dtype, m, n, dY, stride_dy, direct || !products, arena, m);
    Operand ox = {nullptr, 16, 0, -1}, ow = ox;
    if (ew.bytes) ox = operand_of(dtype, m, k, X, stride_x, on_grid(dtype, m, k, X, stride_x), arena, m);
    if (ex.bytes) ow = operand_of(dtype, n, k, W, stride_w, on_grid(dtype, n, k, W, stride_w), arena, n);
    const int64_t sumsAt = sum ? arena.take(slope_slots(m, n, 0) * n * 4) : -1;
    BackwardProducts both;
    both.wantX = ex.bytes;
    both.wantW = ew.bytes;
    both.plan(dtype, m, n, k, 0);
    const int64_t slots = arena.take(both.slotBytes());
    Partials hold;
    if (arena.bytes) {
        st = stream_workspace(s, both.counters(), arena.bytes, hold);
        if (st != GETT_SUCCESS) return st;
    }
    char *ws = static_cast<char *>(hold.tiles);
    SlopeJob j = {dY, Z, nullptr, sum ? reinterpret_cast<float *>(ws + sumsAt) : nullptr, stride_dy,
                  stride_z, 0, (int)m, (int)n, activation, d, nullptr, 0, 0, 0, {}};
    if (oz.copyAt >= 0) {
        oz.p = ws + oz.copyAt;
        j.dZ = ws + oz.copyAt;
        j.ldd = oz.width;
    }
    if (j.dZ || j.sums) st = slope_launch(dtype, j, s);
    if (st == GETT_SUCCESS && sum) st = sums_launch(dtype, j, dbias, s);
    if (st == GETT_SUCCESS) st = place_copy(dtype, ox, hold, m, k, X, stride_x, s);
    if (st == GETT_SUCCESS) st = place_copy(dtype, ow, hold, n, k, W, stride_w, s);
    if (st != GETT_SUCCESS) return st;
    ProductArgs &gx = both.x, &gw = both.w;
    gx = product_args(oz, ow, m, k, n);
    gx.kM = oz.width;
    gx.fullN = ow.width;
    gx.out.Y = static_cast<char *>(dX);
    gx.out.ldy = stride_dx;
    gw = product_args(oz, ox, n, k, m);
    gw.fullM = oz.width;
    gw.fullN = ox.width;
    gw.out.Y = static_cast<char *>(dW);
    gw.out.ldy = stride_dw;
    return both.launch(dtype, hold, slots, s);
}

}  // extern "C"
