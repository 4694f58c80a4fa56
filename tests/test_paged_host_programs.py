"""Programs that run the paged cache's host code against a stand-in for the HIP runtime, under the address and undefined-behaviour sanitizers."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "hip_stub")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("name,says", [("paged_device_check", "paged device checks passed"), ("paged_grid_check", "paged grid checks passed")])
def test_host_program(tmp_path, name, says):
    exe, csrc = str(tmp_path / name), os.path.join(ROOT, "paper_2601_01204_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-I", STUB, "-I", csrc,
           "-include", os.path.join(STUB, "paged_host_types.h"), "-x", "c++", os.path.join(csrc, "paged_api.hip"), os.path.join(STUB, name + ".cpp"), "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert says in r.stdout
