"""The launches that batches over a 4-bit cache are cut into, on the host: those of the device's tests, and the largest ones allowed."""
import os
import shutil
import subprocess

import pytest

import mx4_batches as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_21889_amd", "csrc")
UNITS = 256  # compute units of the device


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path_factory.mktemp("native") / "mx4_plan_launches")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "native", "mx4_plan_launches.cpp"), os.path.join(CSRC, "mx4_plan.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)

    def run(cached, new, heads):
        text = "%d %d %d %d\n" % (*heads, UNITS, len(cached)) + "\n".join("%d %d" % x for x in zip(cached, new))
        done = subprocess.run([exe], input=text, capture_output=True, text=True, env=env, timeout=60)
        assert done.returncode == 0 and done.stdout.endswith("end\n"), (done.stdout + done.stderr)[-4000:]
        return [(line.split()[0], *map(int, line.split()[1:])) for line in done.stdout.splitlines()[:-1]]

    return run


@pytest.mark.parametrize("name", B.FEW)
def test_every_launch_of_few_rows_has_parts(launches, name):
    cached, new, heads, _ = B.few(name)
    got = launches(cached, new, heads)
    assert [x[0] for x in got] == ["few"] * 3 and [x[2] for x in got] == [120, 120, 10]
    assert all(x[1] == int(name.split()[0]) and x[4] > 0 for x in got)


def test_every_launch_of_many_rows_has_parts(launches):
    got = launches(*B.many())
    many, few = [x for x in got if x[0] == "many"], [x for x in got if x[0] == "few"]
    assert [x[1] for x in many] == [96, 44] and len(few) == 1 and few[0][4] > 0
    # shares of a whole number of units; in the first launch of 64 keys, which end inside tiles, in the second larger ones
    assert [x[2] for x in many] == [0, 0] and many[0][3] == 6 and many[1][3] > 6 and all(x[5] == 1 for x in many)


# (keys of a request are at most 2^30, query rows in all as many)
@pytest.mark.parametrize("cached,new,heads", [(1 << 20, 1 << 20, (32, 8)), (1 << 24, 1 << 20, (32, 8)), ((1 << 30) - 70, 70, (8, 1)),
                                              ((1 << 30) - (1 << 16), 1 << 16, (32, 8)), ((1 << 30) - (1 << 18), 1 << 18, (64, 1)),
                                              ((1 << 30) - (1 << 22), 1 << 22, (64, 1)), (0, 1 << 24, (64, 1)), (0, 1 << 30, (1, 1))])
def test_the_longest_requests(launches, cached, new, heads):
    got = launches([cached], [new], heads)
    assert len(got) == 1 and got[0][0] == "many" and got[0][5] == 1
    assert got[0][2] == 1 or 1 <= got[0][4] <= 2 * UNITS


def test_the_longest_requests_of_few_rows(launches):
    got = launches([(1 << 30) - 1, 5], [1, 1], (8, 1))
    assert [x[0] for x in got] == ["few"] and 2 <= got[0][3] <= 2 * UNITS
