// mx_pack.hip -- microscaled 4-bit packing and its inverse.
//
// A block of 32 values x_i becomes s = 2^(floor(log2 max|x|) - 2) and the
// codes of x_i / s (gett_matrix.h has the format).  The maximum is taken on
// the magnitudes' bits as integers, which order as the floats do and put
// infinities and NaNs above everything; the exponent is a field of those
// bits, so the scale is exact.  The division by a power of two, the rounding
// (to nearest, ties to the even code) and the saturation at 6 are one
// conversion instruction for two values.
//
// Bound: memory.  X is read once, also where both orientations are packed: a
// workgroup takes a tile (128 x 128; 32 x 512 where only rows are packed);
// each lane loads eight neighbours of a row, four lanes hold a block, and the
// maximum crosses them in two exchanges.  For the transposed packing the tile
// passes through LDS (unrounded, in X's own type) and a lane takes 32 rows of
// one column; four lanes take one column's four blocks, so 64 bytes of a row
// of codes_t leave together.  Scales are gathered in LDS and leave in whole
// runs.  A bf16 matrix of 16384 x 8192: both orientations in 72-76 us (268 MB
// read, 143 MB written: 5.4-5.7 TB/s, where a copy reaches 5.1), one in 58-60,
// the way back in 58-64; 1 x 4096 in 3.4 and 2.5 us, the launch's own time.
#include "kernel.hpp"
#include "matrix.hpp"
#include "mx.hpp"

namespace gett {
namespace {

constexpr int kT = 128;         // edge of a square tile
constexpr int kThreads = 256;
constexpr int kChunk = 8;       // neighbours of a row one lane takes

// Tiles: 128 x 128 where columns are packed (four blocks of each column); 32 x
// 512 where only rows are read or written, so that a wavefront's access is one
// row's 512 neighbours.
template <bool COLS> struct Tile {
    static constexpr int R = COLS ? kT : 32, C = COLS ? kT : 512;
    static constexpr int LANES = C / kChunk;             // lanes of a row
    static constexpr int ROWS = kThreads / LANES;        // rows of a pass
    static constexpr int PASSES = R / ROWS;
};

__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    // the other lane of the pair, then the other pair of the four
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// the byte of column c of row r among the codes
__device__ __forceinline__ int64_t code_offset(int rows, int r, int c)
{
    return ((int64_t)(c / kTileK) * rows + r) * kTileBytes + (c % kTileK) / 2;
}

// The tile of workgroup `block` of `blocks`: ids of one XCD (workgroups go round
// the eight) are neighbours, in pairs of rows where there are such, so that the
// two tiles that share a line of 128 bytes of codes meet in one L2.
__device__ __forceinline__ void tile_of(int block, int blocks, int tilesC, Recip tilesInv, int &tr,
                                        int &tc)
{
    const int per = blocks >> 3;
    const int id = block < per * 8 ? (block & 7) * per + (block >> 3) : block;
    const int pair = (int)quotient((uint32_t)(id >> 1), tilesC, tilesInv);
    const int inPair = id - 2 * pair * tilesC, left = blocks - 2 * pair * tilesC;
    if (left >= 2 * tilesC) {
        tr = 2 * pair + (inPair & 1);
        tc = inPair >> 1;
    } else {   // a last single row
        tr = 2 * pair;
        tc = inPair;
    }
}

// LDS address (elements) of tile element (r, c): rows follow one another,
// with 32 bytes of skew after every 32 rows, so that the lanes that read four
// blocks of one column fall on different banks.
template <typename T> __device__ __forceinline__ int tile_at(int r, int c)
{
    return r * kT + (r >> 5) * (32 / (int)sizeof(T)) + c;
}

// 16 bytes at an address that is a multiple of 4 or 2
typedef i4 Piece4 __attribute__((aligned(4)));
typedef i4 Piece2 __attribute__((aligned(2)));

// Eight neighbours of a row, as they lie in memory (at any element's address).
template <typename T> struct Chunk {
    static constexpr int N = (int)sizeof(T) / 2;   // 16-byte pieces
    typedef typename std::conditional<sizeof(T) == 4, Piece4, Piece2>::type Piece;
    i4 v[N];
    __device__ __forceinline__ void load(const T *p)
    {
        // read once: past the caches' least recently used lines (51 us where
        // ordinary loads took 58 for 268 MB beside a quarter of that in stores)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = __builtin_nontemporal_load(reinterpret_cast<const Piece *>(p) + i);
    }
    __device__ __forceinline__ void set(const T *p) { __builtin_memcpy(v, p, sizeof(v)); }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void store(T *lds) const   // 16-byte aligned
    {
#pragma unroll
        for (int i = 0; i < N; ++i) reinterpret_cast<i4 *>(lds)[i] = v[i];
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) {
            return __int_as_float(v[i >> 2][i & 3]);
        } else {
            const uint32_t w = (uint32_t)v[0][i >> 1];
            if constexpr (std::is_same<T, bf16>::value)
                return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
            else
                return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w & 0xffffu));
        }
    }
};

// One matrix to pack; tiles of columns and their reciprocal.  `wide`: columns
// are neighbours in memory (stride_col 1).
template <typename T> struct Job {
    const T *X;
    int64_t sr, sc;
    int rows, cols, tilesC, blocks;
    Recip tilesInv;
    bool wide;
    uint8_t *codes, *scales, *codesT, *scalesT;
};

// Workgroups of the first matrix, then those of the second (if there is one).
template <typename T, bool ROWS, bool COLS>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(Job<T> first, Job<T> second)
{
    const bool is2 = (int)blockIdx.x >= first.blocks;
    const T *const X = is2 ? second.X : first.X;
    const int64_t sr = is2 ? second.sr : first.sr, sc = is2 ? second.sc : first.sc;
    const int rows = is2 ? second.rows : first.rows, cols = is2 ? second.cols : first.cols;
    const int tilesC = is2 ? second.tilesC : first.tilesC;
    const bool wide = is2 ? second.wide : first.wide;
    uint8_t *const codes = is2 ? second.codes : first.codes;
    uint8_t *const scales = is2 ? second.scales : first.scales;
    uint8_t *const codesT = is2 ? second.codesT : first.codesT;
    uint8_t *const scalesT = is2 ? second.scalesT : first.scalesT;
    const int block = (int)blockIdx.x - (is2 ? first.blocks : 0);
    __shared__ __attribute__((aligned(16))) T tile[COLS ? kT * kT + 3 * (32 / sizeof(T)) : 1];
    typedef Tile<COLS> Q;
    // [128 columns][row][block], and [column][block]
    __shared__ __attribute__((aligned(16))) uint8_t sRow[ROWS ? Q::C / 128 : 1][ROWS ? Q::R : 1][4];
    __shared__ __attribute__((aligned(16))) uint8_t sCol[COLS ? kT : 1][4];

    const int tid = (int)threadIdx.x;
    int tr, tc;
    tile_of(block, is2 ? second.blocks : first.blocks, tilesC,
            is2 ? second.tilesInv : first.tilesInv, tr, tc);
    const int row0 = tr * Q::R, col0 = tc * Q::C;
    const int tilesK = (int)mx_tiles(cols), tilesKT = (int)mx_tiles(rows);
    // this tile's columns (rows) lie inside the padded row of codes (codes_t)
    const int c8 = (tid % Q::LANES) * kChunk, r0 = tid / Q::LANES;
    const bool inRow = ROWS && col0 + c8 < tilesK * kTileK, inCol = COLS && row0 < tilesKT * kTileK;

    // All passes' loads, with nothing between them.  Rows past the last read it
    // again (their codes are not stored; for the columns they become zeros), and
    // so do chunks past the last column or across it, which are replaced.
    const int left = cols - (col0 + c8);   // columns of this lane's chunk inside X
    Chunk<T> x[Q::PASSES];
    if (wide && cols >= kChunk) {
        const int c = left >= kChunk ? col0 + c8 : cols - kChunk;
#pragma unroll
        for (int p = 0; p < Q::PASSES; ++p) {
            const int r = row0 + r0 + p * Q::ROWS;
            x[p].load(X + (int64_t)(r < rows ? r : rows - 1) * sr + c);
        }
    }
    if (!wide || left < kChunk) {
#pragma unroll
        for (int p = 0; p < Q::PASSES; ++p) {
            const int r = row0 + r0 + p * Q::ROWS;
            const T *src = X + (int64_t)(r < rows ? r : rows - 1) * sr + (int64_t)(col0 + c8) * sc;
            T v[kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = i < left ? src[i * sc] : from_float<T>(0.0f);
            x[p].set(v);
        }
    }
#pragma unroll
    for (int p = 0; p < Q::PASSES; ++p) {
        const int lr = r0 + p * Q::ROWS;
        if constexpr (COLS) {
            if (row0 + lr >= rows) x[p].clear();
            x[p].store(tile + tile_at<T>(lr, c8));
        }
        if constexpr (ROWS) {
            float f[kChunk];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                f[i] = x[p].at(i);
                top = max(top, magnitude(f[i]));
            }
            const uint32_t sb = scale_byte(quad_max(top));
            const uint32_t q = codes8(f, scale_value(sb));
            if (inRow && row0 + lr < rows)
                *reinterpret_cast<uint32_t *>(codes + code_offset(rows, row0 + lr, col0 + c8)) = q;
            if ((tid & 3) == 0) sRow[c8 >> 7][lr][(c8 >> 5) & 3] = (uint8_t)sb;
        }
    }
    __syncthreads();
    if constexpr (COLS) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = j * (kT / 2) + (tid >> 2), b = tid & 3;   // column, block of 32 rows
            float f[32];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                f[i] = to_float(tile[tile_at<T>(b * 32 + i, c)]);
                top = max(top, magnitude(f[i]));
            }
            const uint32_t sb = scale_byte(top);
            const float s = scale_value(sb);
            i4 q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = (int)codes8(f + 8 * i, s);
            if (inCol && col0 + c < cols)
                *reinterpret_cast<i4 *>(codesT + code_offset(cols, col0 + c, row0 + b * 32)) = q;
            sCol[c][b] = (uint8_t)sb;
        }
        __syncthreads();
    }
    // scales: 512 bytes, one 16-byte piece (four rows) a thread
    if constexpr (ROWS) {
        const int r = tid * 4 % Q::R, part = tid * 4 / Q::R, R = (int)mx_scale_rows(rows);
        if (tid < 32 && col0 + part * kT < tilesK * kTileK && row0 + r < R)
            *reinterpret_cast<i4 *>(scales + ((int64_t)(col0 / kT + part) * R + row0 + r) * 4) =
                *reinterpret_cast<const i4 *>(&sRow[part][r][0]);
    }
    if constexpr (COLS) {
        const int c = (tid - 64) * 4, R = (int)mx_scale_rows(cols);   // another wavefront
        if (c >= 0 && c < kT && inCol && col0 + c < R)
            *reinterpret_cast<i4 *>(scalesT + ((int64_t)(row0 / kT) * R + col0 + c) * 4) =
                *reinterpret_cast<const i4 *>(&sCol[c][0]);
    }
}

// A workgroup writes a 32 x 512 tile of values; `wide` as above.
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(
    const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int rows, int cols,
    int tilesC, Recip tilesInv, bool wide, T *__restrict__ X, int64_t sr, int64_t sc)
{
    typedef Tile<false> Q;
    __shared__ __attribute__((aligned(16))) uint8_t sRow[Q::C / 128][Q::R][4];
    const int tid = (int)threadIdx.x;
    int tr, tc;
    tile_of((int)blockIdx.x, (int)gridDim.x, tilesC, tilesInv, tr, tc);
    const int row0 = tr * Q::R, col0 = tc * Q::C;
    const int R = (int)mx_scale_rows(rows);
    const int c8 = (tid % Q::LANES) * kChunk, r0 = tid / Q::LANES;
    const int left = cols - (col0 + c8);
    uint32_t q[Q::PASSES];
#pragma unroll
    for (int p = 0; p < Q::PASSES; ++p) {
        const int r = row0 + r0 + p * Q::ROWS;
        q[p] = 0;
        if (r < rows && left > 0)
            q[p] = *reinterpret_cast<const uint32_t *>(codes + code_offset(rows, r, col0 + c8));
    }
    {
        const int r = tid * 4 % Q::R, part = tid * 4 / Q::R;
        if (tid < 32 && col0 + part * kT < cols && row0 + r < R)
            *reinterpret_cast<i4 *>(&sRow[part][r][0]) = *reinterpret_cast<const i4 *>(
                scales + ((int64_t)(col0 / kT + part) * R + row0 + r) * 4);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < Q::PASSES; ++p) {
        const int lr = r0 + p * Q::ROWS, r = row0 + lr;
        if (r >= rows || left <= 0) continue;
        const uint32_t sb = sRow[c8 >> 7][lr][(c8 >> 5) & 3];
        const float s = scale_value(sb);
        float f[kChunk];
        const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[p], s, 0);
        const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[p], s, 1);
        const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[p], s, 2);
        const f2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[p], s, 3);
        f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1];
        f[4] = c[0], f[5] = c[1], f[6] = d[0], f[7] = d[1];
        T v[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            v[i] = from_float<T>(sb == 255 ? __uint_as_float(0x7fc00000u) : f[i]);
        T *dst = X + (int64_t)r * sr + (int64_t)(col0 + c8) * sc;
        if (wide && left >= kChunk) {
            Chunk<T> c;
            c.set(v);
#pragma unroll
            for (int i = 0; i < Chunk<T>::N; ++i)
                reinterpret_cast<typename Chunk<T>::Piece *>(dst)[i] = c.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < kChunk; ++i)
                if (i < left) dst[i * sc] = v[i];
        }
    }
}

// A job in kernel terms: rows are the direction of the larger stride.
template <typename T> Job<T> job_of(QuantizeJob q)
{
    if (q.sr == 1 && q.sc != 1) {   // the transpose is read along its rows
        std::swap(q.rows, q.cols);
        std::swap(q.sr, q.sc);
        std::swap(q.codes, q.codesT);
        std::swap(q.scales, q.scalesT);
    }
    // enough tiles for X and for the padding of the packed rows
    const int64_t R = q.codesT ? Tile<true>::R : Tile<false>::R;
    const int64_t C = q.codesT ? Tile<true>::C : Tile<false>::C;
    const int64_t tilesR = ((q.codesT ? mx_tiles(q.rows) * kTileK : q.rows) + R - 1) / R;
    const int64_t tilesC = ((q.codes ? mx_tiles(q.cols) * kTileK : q.cols) + C - 1) / C;
    const int64_t blocks = fits_launch(tilesR * tilesC, kThreads) ? tilesR * tilesC : 0;
    return {static_cast<const T *>(q.X), q.sr, q.sc, (int)q.rows, (int)q.cols, (int)tilesC,
            (int)blocks, recip(tilesC), q.sc == 1, static_cast<uint8_t *>(q.codes),
            static_cast<uint8_t *>(q.scales), static_cast<uint8_t *>(q.codesT),
            static_cast<uint8_t *>(q.scalesT)};
}

template <typename T>
gett_status_t quantize_typed(const QuantizeJob *q, int n, hipStream_t stream)
{
    const Job<T> a = job_of<T>(q[0]);
    Job<T> b = {};
    if (n == 2) b = job_of<T>(q[1]);
    if (a.blocks == 0 || (n == 2 && b.blocks == 0)) return GETT_ERROR_NOT_SUPPORTED;
    if (n == 2 && (!a.codes != !b.codes || !a.codesT != !b.codesT ||
                   !fits_launch((int64_t)a.blocks + b.blocks, kThreads))) {   // one launch each
        const gett_status_t st = quantize_typed<T>(q, 1, stream);
        return st == GETT_SUCCESS ? quantize_typed<T>(q + 1, 1, stream) : st;
    }
    const dim3 grid((unsigned)(a.blocks + b.blocks)), block(kThreads);
    if (a.codes && a.codesT)
        hipLaunchKernelGGL((mx_quantize_kernel<T, true, true>), grid, block, 0, stream, a, b);
    else if (a.codes)
        hipLaunchKernelGGL((mx_quantize_kernel<T, true, false>), grid, block, 0, stream, a, b);
    else
        hipLaunchKernelGGL((mx_quantize_kernel<T, false, true>), grid, block, 0, stream, a, b);
    return hipGetLastError() == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
}

template <typename T>
hipError_t dequantize_typed(int64_t rows, int64_t cols, const void *codes, const void *scales,
                            void *X, int64_t sr, int64_t sc, unsigned blocks, int tilesC,
                            hipStream_t stream)
{
    hipLaunchKernelGGL((mx_dequantize_kernel<T>), dim3(blocks), dim3(kThreads), 0, stream,
                       static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales),
                       (int)rows, (int)cols, tilesC, recip(tilesC), sc == 1, static_cast<T *>(X), sr,
                       sc);
    return hipGetLastError();
}

}  // namespace

gett_status_t quantize_launch(gett_dtype_t dtype, const QuantizeJob *q, int n, hipStream_t stream)
{
    QuantizeJob some[2];
    int m = 0;
    for (int i = 0; i < n; ++i)
        if (q[i].rows > 0 && q[i].cols > 0) some[m++] = q[i];
    if (m == 0) return GETT_SUCCESS;
    if (dtype == GETT_FLOAT32) return quantize_typed<float>(some, m, stream);
    if (dtype == GETT_BFLOAT16) return quantize_typed<bf16>(some, m, stream);
    return quantize_typed<_Float16>(some, m, stream);
}

}  // namespace gett

extern "C" {

gett_status_t gett_mx_size(int64_t rows, int64_t cols, uint64_t *code_bytes, uint64_t *scale_bytes)
{
    if (!code_bytes || !scale_bytes || rows < 0 || cols < 0) return GETT_ERROR_INVALID_VALUE;
    if (rows >= gett::kMaxRows || cols >= gett::kMaxCols) return GETT_ERROR_NOT_SUPPORTED;
    *code_bytes = (uint64_t)gett::mx_code_bytes(rows, cols);
    *scale_bytes = (uint64_t)gett::mx_scale_bytes(rows, cols);
    return GETT_SUCCESS;
}

gett_status_t gett_mx_quantize(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                               int64_t stride_row, int64_t stride_col, void *codes, void *scales,
                               void *codes_t, void *scales_t, void *stream)
{
    using namespace gett;
    const gett_status_t st = matrix_ok(dtype, rows, cols, X, stride_row, stride_col);
    if (st != GETT_SUCCESS) return st;
    const bool along = codes || scales, across = codes_t || scales_t;
    if (rows >= kMaxRows || cols >= kMaxRows || (along && cols >= kMaxCols) ||
        (across && rows >= kMaxCols))
        return GETT_ERROR_NOT_SUPPORTED;
    if (rows == 0 || cols == 0) return GETT_SUCCESS;
    if ((!along && !across) || (along && !packed_ok(codes, scales)) ||
        (across && !packed_ok(codes_t, scales_t)))
        return GETT_ERROR_INVALID_VALUE;
    const int64_t span = span_bytes(rows, cols, stride_row, stride_col, type_size(dtype));
    if (span < 0) return GETT_ERROR_NOT_SUPPORTED;
    const void *p[5] = {X, codes, scales, codes_t, scales_t};
    const int64_t n[5] = {span, mx_code_bytes(rows, cols), mx_scale_bytes(rows, cols),
                          mx_code_bytes(cols, rows), mx_scale_bytes(cols, rows)};
    for (int i = 0; i < 5; ++i)
        for (int j = i + 1; j < 5; ++j)
            if (p[i] && p[j] && overlaps(p[i], n[i], p[j], n[j])) return GETT_ERROR_INVALID_VALUE;
    const QuantizeJob q = {rows, cols, X, stride_row, stride_col, codes, scales, codes_t, scales_t};
    return quantize_launch(dtype, &q, 1, static_cast<hipStream_t>(stream));
}

gett_status_t gett_mx_dequantize(gett_dtype_t dtype, int64_t rows, int64_t cols,
                                 const void *codes, const void *scales, void *X,
                                 int64_t stride_row, int64_t stride_col, void *stream)
{
    using namespace gett;
    const gett_status_t st = matrix_ok(dtype, rows, cols, X, stride_row, stride_col);
    if (st != GETT_SUCCESS) return st;
    if (rows >= kMaxRows || cols >= kMaxCols) return GETT_ERROR_NOT_SUPPORTED;
    if (rows == 0 || cols == 0) return GETT_SUCCESS;
    if (!packed_ok(codes, scales)) return GETT_ERROR_INVALID_VALUE;
    const int64_t span = span_bytes(rows, cols, stride_row, stride_col, type_size(dtype));
    if (span < 0 || !matrix_injective(rows, cols, stride_row, stride_col))
        return GETT_ERROR_NOT_SUPPORTED;
    if (overlaps(X, span, codes, mx_code_bytes(rows, cols)) ||
        overlaps(X, span, scales, mx_scale_bytes(rows, cols)))
        return GETT_ERROR_INVALID_VALUE;
    const int64_t tilesC = (cols + Tile<false>::C - 1) / Tile<false>::C;
    const int64_t tiles = (rows + Tile<false>::R - 1) / Tile<false>::R * tilesC;
    if (!fits_launch(tiles, kThreads)) return GETT_ERROR_NOT_SUPPORTED;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (dtype == GETT_FLOAT32)
        e = dequantize_typed<float>(rows, cols, codes, scales, X, stride_row, stride_col,
                                    (unsigned)tiles, (int)tilesC, s);
    else if (dtype == GETT_BFLOAT16)
        e = dequantize_typed<bf16>(rows, cols, codes, scales, X, stride_row, stride_col,
                                   (unsigned)tiles, (int)tilesC, s);
    else
        e = dequantize_typed<_Float16>(rows, cols, codes, scales, X, stride_row, stride_col,
                                       (unsigned)tiles, (int)tilesC, s);
    return e == hipSuccess ? GETT_SUCCESS : GETT_ERROR_HIP;
}

}  // extern "C"
