"""Numbers that a wavefront's lanes hand one another through LDS without a barrier: the
compiler has to be told of it, or it may take a lane's own earlier value for what
another has stored since.  The instructions do not show that it was told (there are
none for it), the compiler's own form of the built sources does."""
import functools
import os
import re
import subprocess

import pytest

from paper_1607_00145_amd import build

HIPCC = "/opt/rocm/bin/hipcc"


@functools.lru_cache(maxsize=None)
def kernels(source, folder):
    """Mangled name -> text of each kernel of a source, after the compiler's first passes."""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    out = folder / f"{source}.ll"
    flags = [f for f in build.COMMON if not f.startswith("-O")] + build.DEVICE
    subprocess.run([HIPCC, "-O1", *flags, "-x", "hip", "--cuda-device-only", "-S", "-emit-llvm", "-o", str(out),
                    os.path.join(build.CSRC, source)], check=True, capture_output=True)
    text = out.read_text()
    return {m.group(1): m.group(2) for m in
            re.finditer(r"^define [^\n]*amdgpu_kernel[^\n]*@(\w+)\([^\n]*\{\n(.*?)^\}", text, re.M | re.S)}


def exchanges(body):
    """How often what lanes stored is made known to the others."""
    return len(re.findall(r'fence syncscope\("wavefront"\) release\n\s*(?:tail )?call void @llvm\.amdgcn\.wave\.barrier\(\)'
                          r'[^\n]*\n\s*fence syncscope\("wavefront"\) acquire', body))


@pytest.fixture(scope="module")
def folder(tmp_path_factory):
    return tmp_path_factory.mktemp("ir")


@pytest.mark.parametrize("source,name", [
    ("route.hip", "route_grad_kernel"), ("route.hip", "route_choose_kernel"), ("route.hip", "route_small_kernel"),
    ("product_f32.hip", "14product_kernel"), ("product_f32.hip", "product_pair_kernel")])
def test_lanes_exchange_through_lds(folder, source, name):
    """Before others read what a lane has stored, and before it stores again."""
    mine = {n: exchanges(b) for n, b in kernels(source, folder).items() if name in n and "Slabs" not in n}
    assert mine
    assert all(v >= 2 for v in mine.values()), mine
