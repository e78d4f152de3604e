"""Which of the library's kernels a matrix operator takes (csrc/matrix.hpp,
gett_tiles; no GPU needed): tests assert that they run what they mean to."""
import ctypes

import paper_1607_00145_amd as g


class Tiles(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("edge", "slices", "shared", "workgroups")]


def mx_tiles(m, n, k):
    t = Tiles()
    f = g.load_library().gett_mx_tiles
    f.argtypes, f.restype = [ctypes.c_int64] * 3 + [ctypes.c_void_p], None
    f(m, n, k, ctypes.byref(t))
    return t


def orth_tiles(batch, rows, cols):
    """Of S, b S + c S^2 and the update."""
    t = (Tiles * 3)()
    f = g.load_library().gett_orthogonalize_tiles
    f.argtypes, f.restype = [ctypes.c_int64] * 3 + [ctypes.c_void_p], None
    f(batch, rows, cols, ctypes.byref(t))
    return list(t)
