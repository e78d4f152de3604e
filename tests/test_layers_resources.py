"""Registers of the layers' kernels, from the built library's code objects (no GPU):
none spills to scratch memory, and the large tiles keep two wavefronts per SIMD (256
registers)."""
import os
import re
import subprocess

import pytest

import paper_1607_00145_amd as g
from test_kernel_resources import LLVM, code_objects

KERNELS = ["dropout_kernel", "product_kernel", "product_pair_kernel", "product_slabs_kernel",
           "product_slabs_pair_kernel", "product_few_kernel", "product_row_kernel",
           "layer_copy_kernel", "layer_slope_kernel", "layer_sums_kernel", "combine_kernel",
           "combine_grad_kernel", "route_choose_kernel", "route_small_kernel", "route_scan_kernel",
           "route_place_kernel", "route_grad_kernel"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """mangled name -> (scratch bytes per lane, VGPRs and AGPRs)"""
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
                found[name.group(1)] = (field("private_segment_fixed_size"), field("vgpr_count"))
    return found


@pytest.mark.parametrize("kernel", KERNELS)
def test_no_kernel_spills(kernels, kernel):
    mine = {n: v for n, v in kernels.items() if kernel in n}
    assert mine, kernel
    assert not {n: v for n, v in mine.items() if v[0] > 0}


def test_large_tiles_keep_two_wavefronts(kernels):
    large = {n: v for n, v in kernels.items() if "ProductShapeILi4ELi2ELi2ELi4E" in n}
    assert large
    assert all(v[1] <= 256 for v in large.values()), large
