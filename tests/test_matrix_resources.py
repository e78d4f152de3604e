"""Registers of the matrix operators' kernels, from the built library's code
objects (no GPU): none spills to scratch memory, and the tiles of 256 x 256
keep two wavefronts per SIMD (256 registers)."""
import os
import re
import subprocess

import pytest

import paper_1607_00145_amd as g
from test_kernel_resources import LLVM, code_objects

KERNELS = ["mx_quantize_kernel", "mx_dequantize_kernel", "mx_tile_kernel", "mx_few_kernel",
           "orth_norm_kernel", "orth_start_kernel", "orth_copy_kernel", "orth_product_kernel",
           "orth_short_kernel", "orth_small_kernel"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """mangled name -> (scratch bytes per lane, VGPRs, AGPRs)"""
    if not os.path.exists(f"{LLVM}/llvm-readelf"):
        pytest.skip("llvm-readelf not found")
    tmp, found = tmp_path_factory.mktemp("co"), {}
    for k, co in enumerate(code_objects(g.LIB_PATH)):
        path = tmp / f"{k}.co"
        path.write_bytes(co)
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", str(path)], check=True,
                               capture_output=True, text=True).stdout
        for blk in notes.split("\n  - ")[1:]:
            name = re.search(r"\.name:\s+(\S+)", blk)
            if name and any(x in name.group(1) for x in KERNELS):
                field = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", blk).group(1))
                found[name.group(1)] = (field("private_segment_fixed_size"), field("vgpr_count"),
                                        field("agpr_count"))
    return found


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_kernel_spills(kernels, kernel):
    mine = {n: v for n, v in kernels.items() if kernel in n}
    assert mine, kernel
    assert not {n: v for n, v in mine.items() if v[0] > 0}


@pytest.mark.parametrize("kernel", ["mx_tile_kernel", "orth_product_kernel"])
def test_large_tiles_keep_two_wavefronts(kernels, kernel):
    large = {n: v for n, v in kernels.items()
             if kernel in n and "PanelShapeILi2ELi4ELi4ELi2E" in n}
    assert large
    assert all(v[1] <= 256 for v in large.values()), large
