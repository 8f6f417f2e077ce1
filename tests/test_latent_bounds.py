"""Bounds of the latent attention's counts, compiled from the headers that the kernels use."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_21889_amd", "csrc")


def test_counts_of_the_longest_request_fit_their_types(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path / "latent_bounds")
    res = subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                          "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                          os.path.join(ROOT, "tests", "native", "latent_bounds.cpp"), os.path.join(CSRC, "latent_plan.cpp"),
                          os.path.join(CSRC, "planner.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=60)
    assert run.returncode == 0 and "latent bounds ok" in run.stdout, (run.stdout + run.stderr)[-4000:]
