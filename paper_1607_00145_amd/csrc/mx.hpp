// mx.hpp -- what the 4-bit operators' sources share on the host side.
#pragma once
#include "matrix.hpp"

namespace gett {

// status of a matrix argument: element type, extents, strides, pointer
inline gett_status_t matrix_ok(gett_dtype_t dtype, int64_t rows, int64_t cols, const void *X,
                               int64_t sr, int64_t sc)
{
    if (!float_type(dtype) || rows < 0 || cols < 0 || sr < 1 || sc < 1)
        return GETT_ERROR_INVALID_VALUE;
    if (rows > 0 && cols > 0 && (!X || (uintptr_t)X % type_size(dtype)))
        return GETT_ERROR_INVALID_VALUE;
    return GETT_SUCCESS;
}

inline bool packed_ok(const void *codes, const void *scales)
{
    return codes && scales && (uintptr_t)codes % 16 == 0 && (uintptr_t)scales % 16 == 0;
}

// A matrix to pack: along its columns (codes, scales), along its rows (codesT,
// scalesT) or both; null where not wanted.
struct QuantizeJob {
    int64_t rows, cols;
    const void *X;
    int64_t sr, sc;
    void *codes, *scales, *codesT, *scalesT;
};

// Packs one or two matrices of a type, in one launch where they want the same
// packings (mx_pack.hip).  Arguments have been checked.
gett_status_t quantize_launch(gett_dtype_t dtype, const QuantizeJob *jobs, int n,
                              hipStream_t stream);

}  // namespace gett
