"""What becomes of the per-stream workspace that a captured graph points at
when a later call needs more, and its errors (csrc/workspace.cpp, built here
with g++ against a record of its HIP calls; no GPU)."""
import os
import subprocess

import pytest

from conftest import ROOT


@pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"),
                    reason="HIP headers not found")
def test_growth_leaves_graphs_their_buffers(tmp_path):
    exe = str(tmp_path / "probe")
    csrc = os.path.join(ROOT, "paper_1607_00145_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                    os.path.join(ROOT, "tests", "native", "workspace_probe.cpp"),
                    os.path.join(csrc, "workspace.cpp"), "-pthread", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
