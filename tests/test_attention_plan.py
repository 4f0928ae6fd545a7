"""Which kernel of the paged attention a call runs, on the host (plan.cpp built with g++): the cases of
tests/attention_variants.py reach every variant and both ways of sharing out the work, and their reference."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import attention as oa
from tests.attention_cases import paged_reference
from tests.attention_variants import CASES, inputs, reference, replay, case

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18502_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers are not available")
    out = str(tmp_path_factory.mktemp("plan") / "libplan.so")
    srcs = [os.path.join(CSRC, "plan.cpp"), os.path.join(ROOT, "tests", "hostsan", "attention_plan_abi.cpp")]
    res = subprocess.run(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                          f"-I{os.path.join(ROOT, 'include')}", *srcs, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    h = ctypes.CDLL(out)
    h.test_plan_paged.argtypes = [ctypes.c_int64] * 6 + [ctypes.c_void_p]
    h.test_plan_paged.restype = None

    def f(*shape):
        got = (ctypes.c_int64 * 6)()
        h.test_plan_paged(*shape, got)
        return tuple(got)
    return f


@pytest.mark.parametrize("at", range(len(CASES)))
def test_each_case_reaches_the_variant_it_names(plan, at):
    c, want = CASES[at]
    got = replay(plan, c)
    for key in ("dp", "tiles", "line", "split", "rounds"):
        assert got[key] == want[key] or (key == "rounds" and not want[key]), (c["name"], key, got)
    if not want["tiles"]:
        assert (got["nq"], got["hg"], got["idle"]) == (want["nq"], want["hg"], want["idle"]), (c["name"], got)


def test_the_cases_reach_every_variant(plan):
    stream, tiles = set(), set()
    for c, w in CASES:
        (tiles if w["tiles"] else stream).add((w["dp"], c["per_tensor"], w["line"]) if w["tiles"] else (w["dp"], w["nq"], w["hg"], w["line"]))
    assert stream >= {(dp, nq, hg, line) for dp in (64, 128, 256) for nq, hg in ((1, 1), (1, 2), (1, 4), (2, 1), (2, 2))
                      for line in (False, True)}
    assert tiles == {(dp, pt, line) for dp in (64, 128, 256) for pt in (False, True) for line in (False, True)}
    # and there are no others
    for T, B, Hq, H, D, L in ((t, b, h * g, h, d, m) for t in (1, 5, 40, 700, 5000) for b in (1, 7, 64) for h in (1, 2, 3, 8)
                              for g in (1, 4, 16) for d in (16, 64, 80, 128, 192, 256) for m in (16, 4096, 100000)):
        dp, nq, hg, til, _, _ = plan(T, B, Hq, H, D, L)
        assert til or (nq, hg) in ((1, 1), (1, 2), (1, 4), (2, 1), (2, 2))


def test_a_workspace_holds_the_parts_of_every_table_width(plan):
    """Asked for without the tables' width: the widest call's."""
    for T, B, Hq, H, D in ((5, 1, 8, 2, 128), (64, 64, 32, 8, 128), (320, 64, 32, 8, 128), (26, 1, 4, 1, 64), (700, 3, 32, 8, 256)):
        most = plan(T, B, Hq, H, D, 2 ** 31 - 1)[5]
        for L in (0, 16, 1000, 30000, 10 ** 6):
            dp, nq, hg, tiles, groups, bytes_ = plan(T, B, Hq, H, D, L)
            rows = (256 if dp == 128 else 128) if tiles else 16 * nq * hg
            assert 16384 + groups * 2 * rows * (dp + 4) * 4 <= bytes_ <= most
            assert 3 * groups * 4 <= 16384


@pytest.mark.parametrize("c", [case("chain", 1, [3, 0, 2], [20, 5, 0], 2, 2, 32), case("tree", 2, [5, 5], [9, 0], 1, 3, 16, nodes=4),
                               case("one scale", 3, [2, 2], [7, 30], 2, 1, 24, per_tensor=True)])
def test_the_reference_is_the_oracle_s(c):
    d = inputs(c)
    want, tol = paged_reference(d)
    out, spread, mag = reference(d)
    assert d["tables"].shape[1] * d["block"] >= d["lens"].max()
    np.testing.assert_allclose(out, want, rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(oa.bound(out, spread, mag, c["D"], int(d["lens"].max())), tol, rtol=1e-10)
