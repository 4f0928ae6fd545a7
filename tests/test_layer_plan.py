"""How the rotation into the cache is shared out and which kernel a 4-bit linear takes, on the host (plan.hpp and plan.cpp built
with g++): the cases of tests/fp4_cases.py reach every kernel, and each beyond the scales that it holds at a time."""

import ctypes
import os
import shutil
import subprocess

import pytest

from tests import fp4_cases

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
    h.test_plan_fp4.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_void_p]
    h.test_plan_fp4.restype = None
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


def fp4(plan, M, N, K):
    out = (ctypes.c_int * 6)()
    plan.test_plan_fp4(M, N, K, out)
    return tuple(out[:5]), out[5]


def test_the_4_bit_cases_reach_every_variant_beyond_a_panel_of_scales(plan):
    beyond = set()
    for want, M, N, K in fp4_cases.beyond_panels():
        v, panel = fp4(plan, M, N, K)
        assert v == want and panel == fp4_cases.panel(v), (M, N, K, v)
        steps = K // 128
        assert steps > panel and (v[2] == 1 or steps % panel % v[2] != 0), (M, N, K)    # (waves with different numbers of steps)
        assert K % 128 != 0
        beyond.add(v)
    assert len(beyond) == plan.test_fp4_variants() == len(fp4_cases.VARIANTS)


def test_the_4_bit_linears_have_no_other_variants(plan):
    seen = {fp4(plan, M, N, K)[0] for M in (*range(1, 140), 1000, (1 << 20) - 16) for N in (*range(8, 40000, 347), 128256, (1 << 28) - 1)
            for K in (32, 4096, 8192, 8224, 1 << 30)}
    assert seen == set(fp4_cases.VARIANTS)


def test_each_group_of_rows_takes_the_variant_it_names(plan):
    for N, K, want, rows in fp4_cases.ROWS:
        assert {fp4(plan, M, N, K)[0] for M in range(rows[0], rows[-1] + 1)} == {want}, (N, K, rows)
    assert {v for _, _, v, _ in fp4_cases.ROWS} == set(fp4_cases.VARIANTS)
