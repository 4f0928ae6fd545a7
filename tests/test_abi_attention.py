"""What the entry points of the cache read and of the attentions refuse, on the host before any HIP call (these calls
never reach a kernel, so they run without a GPU), and the same cases against the host side built with sanitizers."""

import ctypes
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18502_amd", "csrc")

OK, NULL, SHAPE, UNSUP, ENUM, ALIGN, WS, HIP, VALUE, SCRATCH = range(10)
A16 = 0x10000            # fake, 16-byte aligned device address: never dereferenced here
I31 = 1 << 31


@pytest.fixture(scope="module")
def lib():
    import paper_2606_18502_amd as p
    san = os.environ.get("SPECFP8_ABI_LIB")
    if san:
        from paper_2606_18502_amd import _lib
        return _lib.declare(ctypes.CDLL(san))
    if not os.path.exists(p.LIB_PATH):
        from paper_2606_18502_amd import build
        build.build()
    return p.load_library()


def read(lib, kc=A16, vc=A16, ks=A16, vs=A16, mode=0, slots=A16, T=4, H=8, D=128, num=64, k=A16, ld_k=1024, v=A16,
         ld_v=1024):
    return lib.spec_fp8_kv_cache_read(kc, vc, ks, vs, mode, slots, T, H, D, num, k, ld_k, v, ld_v, None)


def test_kv_cache_read(lib):
    assert read(lib, mode=2) == ENUM
    assert read(lib, T=-1) == SHAPE
    assert read(lib, H=0) == SHAPE
    assert read(lib, num=-1) == SHAPE
    assert read(lib, ld_k=1016) == SHAPE
    assert read(lib, ld_v=1016) == SHAPE
    assert read(lib, D=100, ld_k=800, ld_v=800) == UNSUP
    assert read(lib, D=520, ld_k=4160, ld_v=4160) == UNSUP
    assert read(lib, T=I31) == UNSUP
    assert read(lib, H=1 << 25, ld_k=1 << 32, ld_v=1 << 32) == UNSUP        # H*D
    for name in ("kc", "vc", "ks", "vs", "slots", "k", "v"):
        assert read(lib, **{name: None}) == NULL, name
    for name in ("kc", "vc", "k", "v"):
        assert read(lib, **{name: A16 + 8}) == ALIGN, name
    assert read(lib, slots=A16 + 4) == ALIGN
    assert read(lib, ks=A16 + 2) == ALIGN
    assert read(lib, ld_k=1028) == ALIGN
    assert read(lib, T=0, kc=None, vc=None, ks=None, vs=None, slots=None, k=None, v=None) == OK
    # an empty cache reads as zeros: its pointers are not looked at, the others are
    assert read(lib, num=0, kc=None, vc=None, ks=None, vs=None, k=None) == NULL
    assert read(lib, num=0, kc=None, vc=None, ks=None, vs=None, slots=None) == NULL


def paged(lib, q=A16, ld_q=4096, kc=A16, vc=A16, ks=A16, vs=A16, mode=0, tables=A16, ld_t=16, P=16, lens=A16, cu=None,
          tree=None, N=0, T=20, B=4, Hq=32, H=8, D=128, bs=16, nb=100, scale=0.1, out=A16, ld_out=4096, ws=A16, wsb=None):
    if wsb is None:
        wsb = lib.spec_fp8_paged_attention_workspace_bytes(max(T, 1), max(B, 1), Hq, H, D)
    return lib.spec_fp8_paged_attention(q, ld_q, kc, vc, ks, vs, mode, tables, ld_t, P, lens, cu, tree, N, T, B, Hq, H, D, bs,
                                        nb, scale, out, ld_out, ws, wsb, None)


def test_paged_attention(lib):
    assert paged(lib, mode=2) == ENUM
    assert paged(lib, mode=9) == ENUM
    for bad in (dict(T=-1), dict(B=-1), dict(Hq=0), dict(H=0), dict(D=0), dict(Hq=30), dict(bs=0), dict(nb=-1), dict(P=-1),
                dict(ld_t=15), dict(ld_q=4088), dict(ld_out=4088), dict(T=21), dict(tree=A16), dict(N=4),
                dict(tree=A16, N=4, T=19), dict(tree=A16, N=4, cu=A16), dict(tree=A16, N=-1)):
        assert paged(lib, **bad) == SHAPE, bad
    for bad in (dict(D=100, ld_q=3200, ld_out=3200), dict(D=264, ld_q=8448, ld_out=8448), dict(nb=I31), dict(B=I31, T=0),
                dict(T=1 << 26), dict(Hq=65536, H=65536, ld_q=1 << 23, ld_out=1 << 23), dict(bs=I31), dict(P=1 << 28, ld_t=1 << 28),
                dict(tree=A16, N=65, T=4 * 66), dict(nb=I31 - 1, bs=I31 - 1, P=1), dict(ld_t=1 << 60)):
        assert paged(lib, **bad) == UNSUP, bad
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert paged(lib, scale=bad) == VALUE, bad
    for name in ("q", "out", "kc", "vc", "ks", "vs", "tables", "lens"):
        assert paged(lib, **{name: None}) == NULL, name
    for name in ("q", "out", "kc", "vc"):
        assert paged(lib, **{name: A16 + 8}) == ALIGN, name
    for name in ("ks", "vs", "tables", "lens", "cu"):
        assert paged(lib, **{name: A16 + 2}) == ALIGN, name
    assert paged(lib, tree=A16 + 4, N=4) == ALIGN
    assert paged(lib, ld_q=4100) == ALIGN
    assert paged(lib, ld_out=4100) == ALIGN
    assert paged(lib, ws=None) == WS
    assert paged(lib, wsb=lib.spec_fp8_paged_attention_workspace_bytes(20, 4, 32, 8, 128) - 1) == WS
    assert paged(lib, ws=A16 + 8) == ALIGN
    # nothing to do: nothing is looked at
    nothing = dict(q=None, out=None, kc=None, vc=None, ks=None, vs=None, tables=None, lens=None, ws=None, wsb=0)
    assert paged(lib, T=0, **nothing) == OK
    assert paged(lib, B=0, T=0, **nothing) == OK
    assert paged(lib, T=0, tree=A16, N=0, **nothing) == SHAPE


def test_paged_attention_workspace(lib):
    f = lib.spec_fp8_paged_attention_workspace_bytes
    assert f(20, 4, 32, 8, 128) >= 16384
    for bad in ((0, 4, 32, 8, 128), (20, 0, 32, 8, 128), (20, 4, 0, 8, 128), (20, 4, 32, 0, 128), (20, 4, 30, 8, 128),
                (20, 4, 32, 8, 0), (20, 4, 32, 8, 264), (I31, 4, 32, 8, 128)):
        assert f(*bad) == 0, bad
    for T, B, Hq, H, D in ((1, 1, 1, 1, 8), (1 << 20, 1, 64, 1, 256), (1 << 20, 1 << 20, 32, 8, 128), (65, 1, 4, 4, 256)):
        assert 16384 <= f(T, B, Hq, H, D) < 1 << 30


def prompt(lib, q=A16, ld_q=4096, k=A16, ld_k=1024, v=A16, ld_v=1024, cu=A16, T=20, B=4, Hq=32, H=8, D=128, scale=0.1,
           out=A16, ld_out=4096):
    return lib.spec_prompt_attention_bf16(q, ld_q, k, ld_k, v, ld_v, cu, T, B, Hq, H, D, scale, out, ld_out, None)


def test_prompt_attention(lib):
    for bad in (dict(T=-1), dict(B=-1), dict(Hq=0), dict(H=0), dict(D=0), dict(H=5), dict(ld_q=4088), dict(ld_k=1016),
                dict(ld_v=1016), dict(ld_out=4088)):
        assert prompt(lib, **bad) == SHAPE, bad
    for bad in (dict(D=100), dict(D=264), dict(T=1 << 26), dict(B=I31), dict(B=1 << 21)):
        assert prompt(lib, **bad) == UNSUP, bad
    assert prompt(lib, scale=-0.5) == VALUE
    for name in ("q", "k", "v", "cu", "out"):
        assert prompt(lib, **{name: None}) == NULL, name
        assert prompt(lib, **{name: A16 + 2}) == ALIGN, name
    for name in ("ld_q", "ld_k", "ld_v", "ld_out"):
        assert prompt(lib, **{name: 4100}) == ALIGN, name
    assert prompt(lib, T=0, q=None, k=None, v=None, cu=None, out=None) == OK
    assert prompt(lib, B=0, q=None, k=None, v=None, cu=None, out=None) == OK


def test_the_binding_refuses_what_is_no_device_tensor():
    import torch

    import paper_2606_18502_amd as p
    z = torch.zeros
    q, c, s = z((4, 4, 16), dtype=torch.bfloat16), z((16, 2, 16), dtype=torch.uint8), z((16, 2))
    i = z((2, 1), dtype=torch.int32)
    with pytest.raises(ValueError, match="k_cache must be a CUDA"):
        p.kv_cache_read(c, c, z(4, dtype=torch.int64), s, s)
    with pytest.raises(ValueError, match="q must be a CUDA"):
        p.paged_attention(q, c, c, s, s, i, i[:, 0], 16)
    with pytest.raises(ValueError, match="q must be a CUDA"):
        p.prompt_attention(q, q, q, i[0])


def _runtime(name):
    out = subprocess.run(["g++", f"-print-file-name={name}"], capture_output=True, text=True).stdout.strip()
    return out if os.path.isabs(out) and os.path.exists(out) else None


@pytest.mark.skipif("SPECFP8_ABI_LIB" in os.environ, reason="runs the others")
def test_the_refusals_under_sanitizers(tmp_path):
    """api.cpp, validate.cpp and plan.cpp with AddressSanitizer and UndefinedBehaviorSanitizer, no device code."""
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include") or _runtime("libasan.so") is None:
        pytest.skip("no g++, HIP headers or AddressSanitizer")
    so = str(tmp_path / "libspecfp8_hostsan.so")
    srcs = [os.path.join(CSRC, f) for f in ("api.cpp", "validate.cpp", "plan.cpp")]
    srcs.append(os.path.join(ROOT, "tests", "hostsan", "launch_stubs.cpp"))
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
           "-I/opt/rocm/include", f"-I{os.path.join(ROOT, 'include')}", *srcs, "-o", so]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    env = dict(os.environ, LD_PRELOAD=_runtime("libasan.so"), SPECFP8_ABI_LIB=so,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-s", "-p", "no:cacheprovider", os.path.abspath(__file__),
                          "-k", "not binding"], capture_output=True, text=True, env=env, cwd=ROOT, timeout=300)
    log = res.stdout + res.stderr
    assert res.returncode == 0, log[-4000:]
    assert "ERROR: AddressSanitizer" not in log and "runtime error:" not in log, log[-4000:]
