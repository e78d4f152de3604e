// layer_util.hip -- the passes around the products of product.hpp, all bound by
// the bytes that they move: copies onto the 16-byte grid, the gradient of an
// epilogue, sums of columns, sums of the experts' rows.
#include "layer_util.hpp"

namespace gett {

namespace {

// --------------------------------------------------------------------- copy ---

// Piece after piece of 16 bytes of a copy with rows of `ld` numbers, zeros behind a
// row's last column.  A row of the copy is row order[.] / choices of the source where
// there is an order (rows of no expert stay unwritten; nothing reads them).
template <typename T>
__global__ __launch_bounds__(256) void layer_copy_kernel(CopyJob j)
{
    constexpr int EP = 16 / sizeof(T);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)j.rows * j.pieces) return;
    const int64_t row = id < INT32_MAX ? quotient((uint32_t)id, j.pieces, j.piecesInv) : id / j.pieces;
    const int col = (int)(id - row * j.pieces) * EP;
    int64_t from = row;
    if (j.order) {
        const int32_t r = j.order[row];
        if (r < 0) return;
        from = quotient(min((uint32_t)r, (uint32_t)j.rows - 1), j.choices, j.choicesInv);
    }
    int64_t at = from * j.ld;
    if (j.perMatrix) {
        const int64_t z = quotient((uint32_t)row, j.perMatrix, j.perMatrixInv);
        at = z * j.step + (row - z * j.perMatrix) * j.ld;
    }
    const T *src = reinterpret_cast<const T *>(j.src) + at + col;
    Run<T, EP> v;
    if (col + EP <= j.cols) {
        v = __builtin_bit_cast(Run<T, EP>, load16(src));
    } else {
#pragma unroll
        for (int i = 0; i < EP; ++i) v.v[i] = col + i < j.cols ? src[i] : from_float<T>(0.0f);
    }
    *reinterpret_cast<i4 *>(reinterpret_cast<T *>(j.dst) + row * j.pieces * EP + col) =
        __builtin_bit_cast(i4, v);
}

// ------------------------------------------------------- epilogue's gradient ---

constexpr int kSlopeCols = 256;  // columns of a workgroup: 32 lanes of eight

// Rows of a workgroup: as many as leave four workgroups a CU, between 8 and 64 (1023 x
// 515 in 32 bits, of 64 rows each 25 us, of 8 rows 5.5).
int slope_log2(int64_t m, int64_t n)
{
    const int64_t across = (n + kSlopeCols - 1) / kSlopeCols;
    int l = 3;
    while (l < 6 && (m >> (l + 1)) * across >= 1024) ++l;
    return l;
}

// The slots (runs of 1 << shift rows) of expert e begin with offsets[e] >> shift, plus e.
__device__ __forceinline__ void slope_slots_of(const SlopeJob &j, int e, int &first, int &count)
{
    int b = 0, f = j.m;
    if (j.offsets) {
        b = expert_offset(j.offsets, e, j.m);
        f = expert_offset(j.offsets, e + 1, j.m);
    }
    first = (b >> j.shift) + e;
    count = f > b ? (f - b + (1 << j.shift) - 1) >> j.shift : 0;
}

// dz = dropout(dy) act'(z), written with zeros behind the last column, and the sums
// of each column over the workgroup's rows: eight rows at a time, two loads each on
// their way, the eight partial sums of a column added in the same order each time.
// Bound by memory: 8192 x 8192 in bf16 with GELU and dropout 87 us (403 MB: 4.6 TB/s).
// z comes, and dz goes, in the operands' type: the matrix unit takes no other, and dz in
// two parts would be twice the products' time (900 us for 8192 x 8192 x 4096).  This is
// one rounding more than dx and dw have from their own: in bf16 they are 0.0024 off
// (norms) where one rounding alone is 0.0017, in fp16 0.0003 and 0.0002.  The sums are of
// dz before it is rounded.
template <typename T>
__global__ __launch_bounds__(256) void layer_slope_kernel(SlopeJob j)
{
    __shared__ float sums[8][kSlopeCols];
    const int lane = (int)threadIdx.x & 31, strip = (int)threadIdx.x >> 5;
    const int slot = (int)quotient(blockIdx.x, j.across, j.acrossInv);
    const int size = 1 << j.shift;
    int begin = slot << j.shift, end = j.m;
    if (j.offsets) {
        const int e = expert_of_slot(j.offsets, j.experts, j.m, slot, j.shift);
        const int b = expert_offset(j.offsets, e, j.m);
        begin = b + (slot - ((b >> j.shift) + e)) * size;
        end = e == j.experts ? 0 : expert_offset(j.offsets, e + 1, j.m);   // (none behind the last)
    }
    if (begin + size < end) end = begin + size;
    const int col0 = ((int)blockIdx.x - slot * j.across) * kSlopeCols, col = col0 + lane * 8;
    const int left = j.n - col;
    PhiloxColumn random = {};
    if (j.drop.cut) random = philox_column((uint32_t)col >> 3, j.drop.offset, j.drop.key());
    const bool active = j.activation != GETT_ACTIVATION_NONE;
    float total[8] = {};
    if (left > 0) {
        for (int row0 = begin + strip; row0 < end; row0 += 16) {
            float v[2][8], z[2][8];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                if (row0 + 8 * x < end) {
                    load8(reinterpret_cast<const T *>(j.dY) + (row0 + 8 * x) * j.ldy + col, left, v[x]);
                    if (active)
                        load8(reinterpret_cast<const T *>(j.Z) + (row0 + 8 * x) * j.ldz + col, left, z[x]);
                }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int row = row0 + 8 * x;
                if (row >= end) break;
                if (active) slope8(j.activation, v[x], z[x]);   // (zeros behind the last column)
                // (last: what is dropped is zero, whatever it was)
                if (j.drop.cut) {
                    uint32_t w[4];
                    philox_row(random, (uint32_t)row, w);
                    drop8(v[x], j.drop, w);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) total[i] += v[x][i];
                if (j.dZ)
                    store8(reinterpret_cast<T *>(j.dZ) + row * j.ldd + col,
                           j.ldd - col < 8 ? (int)(j.ldd - col) : 8, v[x]);
            }
        }
    }
    if (!j.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[strip][lane * 8 + i] = total[i];
    __syncthreads();
    const int c = col0 + (int)threadIdx.x;
    if (c >= j.n) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
    j.sums[(int64_t)slot * j.n + c] = t;
}

// A column's sum over the slots of each expert: 32 columns a workgroup, eight strips of
// every eighth slot, added in a fixed order.
template <typename T>
__global__ __launch_bounds__(256) void layer_sums_kernel(SlopeJob j, T *out)
{
    __shared__ float sums[8][32];
    const int lane = (int)threadIdx.x & 31, strip = (int)threadIdx.x >> 5;
    const int e = (int)quotient(blockIdx.x, j.across, j.acrossInv);
    const int c = ((int)blockIdx.x - e * j.across) * 32 + lane;
    int first, count;
    slope_slots_of(j, e, first, count);
    float t[2] = {};
    if (c < j.n) {
        const float *p = j.sums + (int64_t)first * j.n + c;
        int i = strip;
        for (; i + 8 < count; i += 16) {
            t[0] += p[(int64_t)i * j.n];
            t[1] += p[(int64_t)(i + 8) * j.n];
        }
        if (i < count) t[0] += p[(int64_t)i * j.n];
    }
    sums[strip][lane] = t[0] + t[1];
    __syncthreads();
    if (strip || c >= j.n) return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += sums[i][lane];
    out[(int64_t)e * j.n + c] = from_float<T>(v);
}

// ------------------------------------------------------------------ combine ---

// Y[t] = residual[t] + sum_j weights[t, j] H[place[t, j]], eight columns a lane, in
// rising j.  H in T or, for sums of gradients, in 32 bits.  Bound by memory: 8192 x 4
// rows of 2048 in bf16 32 us (168 MB: 5.2 TB/s), in 32 bits 65 (302 MB: 4.7 TB/s).
template <typename T, typename H, typename W>
__global__ __launch_bounds__(256) void combine_kernel(CombineJob j)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)j.tokens * j.runs) return;
    const int64_t t = id < INT32_MAX ? quotient((uint32_t)id, j.runs, j.runsInv) : id / j.runs;
    const int col = (int)(id - t * j.runs) * 8, left = j.cols - col;
    const uint32_t rows = (uint32_t)j.tokens * j.k;
    float v[8] = {};
    if (j.residual) load8(reinterpret_cast<const T *>(j.residual) + t * j.ldr + col, left, v);
    // four rows on their way (one after the other, eight take 5 us of latencies)
    for (int i0 = 0; i0 < j.k; i0 += 4) {
        uint32_t p[4];
        float w[4], x[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = i0 + i < j.k;
            p[i] = there ? (uint32_t)j.place[t * j.k + i0 + i] : rows;
            w[i] = there && j.weights ? to_float(reinterpret_cast<const W *>(j.weights)[t * j.k + i0 + i])
                                      : 1.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p[i] < rows)
                load8(reinterpret_cast<const H *>(j.H) + (int64_t)p[i] * j.ldh + col, left, x[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p[i] < rows)
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] += w[i] * x[i][c];
    }
    store8(reinterpret_cast<T *>(j.Y) + t * j.ldy + col, left, v);
}

// A workgroup for a token t: dH[place] = w dY[t] and dw = dY[t] . H[place] for its
// choices, four rows on their way (8192 x 4 rows of 2048 in bf16: 65 us, 302 MB at
// 4.6 TB/s; with a wavefront for each row, dY[t] read by each, 92 where this had 84).  The rows of dH with the token's own
// numbers are set to zero where they are no expert's.
template <typename T, typename W>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradJob j)
{
    __shared__ float part[4][4];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = (int)blockDim.x >> 6;
    const uint32_t rows = (uint32_t)j.tokens * j.k, row0 = blockIdx.x * j.k;
    const int stride = (int)blockDim.x * 8;
    T *dH = reinterpret_cast<T *>(j.dH);
    const T *dY = reinterpret_cast<const T *>(j.dY) + (int64_t)blockIdx.x * j.ldy;
    for (int i0 = 0; i0 < j.k; i0 += 4) {
        uint32_t p[4];
        float w[4], sum[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = i0 + i < j.k;
            p[i] = there ? (uint32_t)j.place[row0 + i0 + i] : rows;
            w[i] = there && dH ? to_float(reinterpret_cast<const W *>(j.weights)[row0 + i0 + i]) : 0.0f;
        }
        for (int c = tid * 8; c < j.cols; c += stride) {
            const int left = j.cols - c;
            float g[8], x[4][8];
            load8(dY + c, left, g);
            if (j.dweights) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (p[i] < rows) load8(reinterpret_cast<const T *>(j.H) + p[i] * j.ldh + c, left, x[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (p[i] >= rows) continue;
                if (dH) {
                    float v[8];
#pragma unroll
                    for (int y = 0; y < 8; ++y) v[y] = w[i] * g[y];
                    store8(dH + p[i] * j.ldd + c, left, v);
                }
                if (j.dweights) {
#pragma unroll
                    for (int y = 0; y < 8; ++y) sum[i] += g[y] * x[i][y];
                }
            }
        }
        if (!j.dweights) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int d = 32; d; d >>= 1) sum[i] += __shfl_xor(sum[i], d);
            if (lane == 0) part[wave][i] = sum[i];
        }
        __syncthreads();
        if (tid < 4 && i0 + tid < j.k) {
            float v = 0.0f;
            for (int y = 0; y < waves; ++y) v += part[y][tid];
            reinterpret_cast<W *>(j.dweights)[row0 + i0 + tid] = from_float<W>(v);
        }
        __syncthreads();
    }
    if (dH) {
        const int live = expert_offset(j.offsets, j.experts, (int)rows);
        const float zero[8] = {};
        for (int i = 0; i < j.k; ++i)
            if ((int64_t)row0 + i >= live)
                for (int c = tid * 8; c < j.cols; c += stride)
                    store8(dH + (int64_t)(row0 + i) * j.ldd + c, j.cols - c, zero);
    }
}

}  // namespace

// ---------------------------------------------------------------- launchers ---

gett_status_t copy_launch(gett_dtype_t t, const CopyJob &j, hipStream_t s)
{
    const int64_t n = (int64_t)j.rows * j.pieces;
    if (n == 0) return GETT_SUCCESS;
    if (!fits_launch((n + 255) / 256, 256)) return GETT_ERROR_NOT_SUPPORTED;
    return with_type(t, [&](auto v) {
        hipLaunchKernelGGL(layer_copy_kernel<decltype(v)>, dim3((unsigned)((n + 255) / 256)), dim3(256),
                           0, s, j);
        return launched(hipGetLastError());
    });
}

int64_t slope_slots(int64_t m, int64_t n, int experts)
{
    const int l = slope_log2(m, n);
    return experts ? (m >> l) + experts + 1 : (m + (1 << l) - 1) >> l;
}
gett_status_t slope_launch(gett_dtype_t t, SlopeJob j, hipStream_t s)
{
    const int64_t slots = slope_slots(j.m, j.n, j.offsets ? j.experts : 0);
    const int64_t across = (j.n + kSlopeCols - 1) / kSlopeCols;
    if (slots == 0 || across == 0) return GETT_SUCCESS;
    if (!fits_launch(slots * across, 256)) return GETT_ERROR_NOT_SUPPORTED;
    j.shift = slope_log2(j.m, j.n);
    j.across = (int)across;
    j.acrossInv = recip(across);
    return with_type(t, [&](auto v) {
        hipLaunchKernelGGL(layer_slope_kernel<decltype(v)>, dim3((unsigned)(slots * across)),
                           dim3(256), 0, s, j);
        return launched(hipGetLastError());
    });
}
gett_status_t sums_launch(gett_dtype_t t, SlopeJob j, void *out, hipStream_t s)
{
    const int64_t across = (j.n + 31) / 32, blocks = across * (j.offsets ? j.experts : 1);
    if (blocks == 0) return GETT_SUCCESS;
    if (!fits_launch(blocks, 256)) return GETT_ERROR_NOT_SUPPORTED;
    j.shift = slope_log2(j.m, j.n);
    j.across = (int)across;
    j.acrossInv = recip(across);
    return with_type(t, [&](auto v) {
        typedef decltype(v) T;
        hipLaunchKernelGGL(layer_sums_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, j,
                           static_cast<T *>(out));
        return launched(hipGetLastError());
    });
}

gett_status_t combine_launch(gett_dtype_t t, gett_dtype_t tH, gett_dtype_t tw, const CombineJob &j,
                             hipStream_t s)
{
    const int64_t n = (int64_t)j.tokens * j.runs;
    if (n == 0) return GETT_SUCCESS;
    if (!fits_launch((n + 255) / 256, 256)) return GETT_ERROR_NOT_SUPPORTED;
    return with_type(t, [&](auto v) {
        typedef decltype(v) T;
        auto launch = [&](auto h, auto w) {
            hipLaunchKernelGGL((combine_kernel<T, decltype(h), decltype(w)>),
                               dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, j);
            return launched(hipGetLastError());
        };
        if (tH != t) return launch(float(), float());
        return tw == t ? launch(T(), T()) : launch(T(), float());
    });
}
gett_status_t combine_grad_launch(gett_dtype_t t, gett_dtype_t tw, const CombineGradJob &j, hipStream_t s)
{
    if (j.tokens == 0) return GETT_SUCCESS;
    const int threads = j.cols <= 512 ? 64 : j.cols <= 1024 ? 128 : 256;
    if (!fits_launch(j.tokens, threads)) return GETT_ERROR_NOT_SUPPORTED;
    return with_type(t, [&](auto v) {
        typedef decltype(v) T;
        auto launch = [&](auto w) {
            hipLaunchKernelGGL((combine_grad_kernel<T, decltype(w)>), dim3((unsigned)j.tokens),
                               dim3(threads), 0, s, j);
            return launched(hipGetLastError());
        };
        return tw == t ? launch(T()) : launch(float());
    });
}

}  // namespace gett
