"""How the rotation into the cache is shared out, on the host (plan.hpp and plan.cpp built with g++)."""

import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18502_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers are not available")
    out = str(tmp_path_factory.mktemp("plan") / "libplan.so")
    srcs = [os.path.join(CSRC, "plan.cpp"), os.path.join(ROOT, "tests", "hostsan", "layer_plan_abi.cpp")]
    res = subprocess.run(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                          f"-I{os.path.join(ROOT, 'include')}", *srcs, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    h = ctypes.CDLL(out)
    h.test_rope_log_parts.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int]
    h.test_rope_step.restype = ctypes.c_int64
    return h


@pytest.mark.parametrize("T", [1, 100, 2048, 2049, 8191, 1 << 24, 1 << 30, (1 << 31) - (1 << 23), (1 << 31) - (1 << 23) + 1, (1 << 31) - 1])
def test_the_rotations_items_are_counted_within_32_bits(plan, T):
    """A wave's next item, one step past its last, is still behind all items: it ends."""
    for Hq, H in ((0, 1), (4, 1), (32, 8), (0, 192), (128, 8), (65535, 65535)):
        for g in (1, 2, 4, 8, 16, 32, 64):
            items = T << plan.test_rope_log_parts(T, Hq, H, g)
            assert items - 1 + plan.test_rope_step() < 1 << 32, (Hq, H, g)


def test_the_rotations_parts(plan):
    """Both borders of the rule for 32 + 2 x 8 heads of 128 (8 lanes a row): 6 passes, two parts up to 2048 tokens and
    again from 6667."""
    parts = lambda T: 1 << plan.test_rope_log_parts(T, 32, 8, 8)
    assert [parts(T) for T in (1, 1024, 1025, 2048, 2049, 6666, 6667, 8191)] == [4, 4, 2, 2, 1, 1, 2, 2]
