"""Sizes and values at the ends of what the attentions' entry points take, refused on the host before any HIP call."""

import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2606_18502_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18502_amd", "csrc")
OK, UNSUP, HIP, VALUE = 0, 3, 7, 8
A16 = 0x10000            # fake, 16-byte aligned device address: never dereferenced here


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    """The host side without device code: a call that passes every check reports SPEC_ERR_HIP."""
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers are not available")
    out = str(tmp_path_factory.mktemp("host") / "libhost.so")
    srcs = [os.path.join(CSRC, f) for f in ("api.cpp", "validate.cpp", "plan.cpp")]
    srcs.append(os.path.join(ROOT, "tests", "hostsan", "launch_stubs.cpp"))
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                          f"-I{os.path.join(ROOT, 'include')}", *srcs, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return _lib.declare(ctypes.CDLL(out))


def paged(lib, T=20, B=4, Hq=1, H=1, D=16, scale=0.1):
    wsb = lib.spec_fp8_paged_attention_workspace_bytes(max(T, 1), max(B, 1), Hq, H, D)
    return lib.spec_fp8_paged_attention(A16, Hq * D, A16, A16, A16, A16, 0, A16, 1, 1, A16, A16, None, 0, T, B, Hq, H, D, 16, 100,
                                        scale, A16, Hq * D, A16, wsb, None)


def prompt(lib, scale=0.1):
    return lib.spec_prompt_attention_bf16(A16, 16, A16, 16, A16, 16, A16, 20, 4, 1, 1, 16, scale, A16, 16, None)


def test_sequences_leave_room_for_the_kernels_arithmetic(lib):
    """Positions a few sequences further, as the kernels reckon them in 32 bits, still fit."""
    top = 2 ** 31 - 65536
    assert paged(lib, B=top) == HIP
    for B in (top + 1, 2 ** 31 - 255, 2 ** 31 - 1):
        assert paged(lib, B=B) == UNSUP, B


def test_a_softmax_scale_whose_powers_of_two_overflow_is_refused(lib):
    """Scores are taken to base 2: scale * log2(e) has to be finite in fp32, or a score of 0 would be 0 * inf."""
    for f in (lambda s: paged(lib, scale=s), lambda s: prompt(lib, scale=s)):
        assert f(2.0 ** 126) == HIP
        assert f(2.0 ** -149) == HIP
        assert f(2.0 ** 127) == HIP                      # 2^127 log2(e) = 1.4427 * 2^127 < 2^128
        assert f(1.5 * 2.0 ** 127) == VALUE              # 2.16 * 2^127
        assert f(3.4e38) == VALUE
