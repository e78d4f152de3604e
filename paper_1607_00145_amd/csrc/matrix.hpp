// matrix.hpp -- what the matrix operators of gett_matrix.h share: element
// types, argument checks, the packed format's geometry and the conversions
// between floats and 4-bit codes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gett_matrix.h"
#include "plan.hpp"

namespace gett {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------- host checks ---

inline bool float_type(gett_dtype_t t)
{
    return t == GETT_FLOAT32 || t == GETT_BFLOAT16 || t == GETT_FLOAT16;
}
inline int64_t type_size(gett_dtype_t t) { return t == GETT_FLOAT32 ? 4 : 2; }

constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxCols = (int64_t)1 << 24;

// Bytes from a strided matrix's first element to behind its last; -1 where
// that passes 2^62.
inline int64_t span_bytes(int64_t rows, int64_t cols, int64_t sr, int64_t sc, int64_t item)
{
    const __int128 n = ((__int128)(rows - 1) * sr + (__int128)(cols - 1) * sc + 1) * item;
    return n < ((__int128)1 << 62) ? (int64_t)n : -1;
}
// No two elements of a rows x cols matrix share an address, seen from the
// strides alone: the larger stride passes over all of the other direction.
inline bool matrix_injective(int64_t rows, int64_t cols, int64_t sr, int64_t sc)
{
    if (rows <= 1 || cols <= 1) return true;
    const bool byRow = sr >= sc;
    const int64_t inner = byRow ? sc : sr, extent = byRow ? cols : rows, outer = byRow ? sr : sc;
    return (__int128)inner * (extent - 1) < outer;
}

// A launch has fewer than 2^32 threads.
inline bool fits_launch(int64_t blocks, int64_t threads)
{
    return blocks < ((int64_t)1 << 32) / threads;
}

// ------------------------------------------------------------ packed format ---

constexpr int kTileK = 256;    // columns of one tile: 128 bytes of codes, 8 scales a row
constexpr int kTileBytes = 128;
constexpr int kTileBlocks = 8;

__host__ __device__ inline int64_t mx_tiles(int64_t cols) { return (cols + kTileK - 1) / kTileK; }
__host__ __device__ inline int64_t mx_scale_rows(int64_t rows) { return (rows + 15) / 16 * 16; }
inline int64_t mx_code_bytes(int64_t rows, int64_t cols) { return rows * mx_tiles(cols) * kTileBytes; }
inline int64_t mx_scale_bytes(int64_t rows, int64_t cols)
{
    return mx_tiles(cols) * kTileBlocks * mx_scale_rows(rows);
}

// ------------------------------------------------------------- conversions ---

struct bf16 {
    uint16_t v;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_float(bf16 x) { return __uint_as_float((uint32_t)x.v << 16); }

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ _Float16 from_float<_Float16>(float x) { return (_Float16)x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x)
{
    // round to nearest, ties to even; a NaN stays one
    const __bf16 b = (__bf16)x;
    return bf16{__builtin_bit_cast(uint16_t, b)};
}

// N elements at any element address
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T v[N];
};

// The scale byte of a block whose largest magnitude has these bits (without
// the sign): the exponent less two, at least 0; 255 for infinities and NaNs,
// whose magnitudes compare above all others as integers.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}
// 2^(byte - 127); any finite number for the NaN scale
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x3f800000u : byte << 23);
}

// eight floats over `scale` -> eight codes, the first in the low bits
__device__ __forceinline__ uint32_t codes8(const float *x, float scale)
{
    uint32_t o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[0], x[1], scale, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[2], x[3], scale, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[4], x[5], scale, 2);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[6], x[7], scale, 3);
    return o;
}

}  // namespace gett

// Which kernels a call takes, from sizes alone (no HIP call): for tests, which
// assert that they run the variant that they mean to.  Exported, but not part of
// gett_matrix.h.
extern "C" {
// of a product of packed matrices into a row-major C (few rows: edge 0)
struct gett_tiles {
    int64_t edge, slices, shared, workgroups;   // slices of each shared tile
};
void gett_mx_tiles(int64_t m, int64_t n, int64_t k, struct gett_tiles *out);
// of S, b S + c S^2 and the update; edge 32: blocks whose wavefronts share K;
// edge 0: the whole matrix in one workgroup
void gett_orthogonalize_tiles(int64_t batch, int64_t rows, int64_t cols, struct gett_tiles out[3]);
}
