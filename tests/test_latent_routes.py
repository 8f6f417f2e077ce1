"""The plans of the batches that stand for each way through the absorbed latent attention."""
import os
import shutil
import subprocess

import pytest

from latent_shapes import ROUTES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_21889_amd", "csrc")


def test_batches_take_the_routes_that_they_stand_for(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path / "print_latent_plan")
    res = subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                          "-I", CSRC, os.path.join(ROOT, "tests", "native", "print_latent_plan.cpp"), os.path.join(CSRC, "latent_plan.cpp"),
                          os.path.join(CSRC, "planner.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    text = "".join("256 %d %d %s\n" % (heads, len(new), " ".join("%d %d" % cn for cn in zip(cached, new)))
                   for heads, cached, new, *_ in ROUTES.values())
    lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.split("\n")
    for (name, (_, _, _, row_tile, by_tile, least)), line in zip(ROUTES.items(), lines):
        got = [int(x) for x in line.split()]
        assert got[0] == row_tile and got[1] == by_tile and got[2] >= least, (name, got)
        assert got[3] > got[4] or name in ("rows128_even", "rows128_even_long"), (name, "several workgroups to a tile", got)
        if name == "rows32":  # four waves, as far as that goes (fewer than six units to a workgroup)
            assert got[2] < 6, got
