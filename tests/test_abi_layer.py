"""What the norm, the rotation into the cache and the 4-bit linears refuse, on the host before any HIP call (these calls
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


def norm(lib, x=A16, ld_x=512, res=A16, ld_r=512, w=A16, eps=1e-5, rows=4, cols=512, mode=0, scales=A16, q=A16, ld_q=512,
         sum=A16, ld_s=512, y=A16, ld_y=512):
    return lib.spec_fp8_rms_norm(x, ld_x, res, ld_r, w, eps, rows, cols, mode, scales, q, ld_q, sum, ld_s, y, ld_y, None)


def test_rms_norm(lib):
    assert norm(lib, mode=2) == ENUM
    assert norm(lib, mode=-1) == ENUM
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=-8), dict(ld_x=504), dict(ld_r=504), dict(ld_q=504), dict(ld_s=504),
                dict(ld_y=504)):
        assert norm(lib, **bad) == SHAPE, bad
    wide = dict(ld_x=1 << 21, ld_r=1 << 21, ld_q=1 << 21, ld_s=1 << 21, ld_y=1 << 21)
    for bad in (dict(cols=500), dict(cols=(1 << 20) + 8, **wide), dict(rows=I31)):
        assert norm(lib, **bad) == UNSUP, bad
    for bad in (0.0, -1e-5, 1e-30, float("inf"), float("nan")):
        assert norm(lib, eps=bad) == VALUE, bad
    assert norm(lib, x=None) == NULL
    assert norm(lib, w=None) == NULL
    assert norm(lib, scales=None) == NULL
    assert norm(lib, q=None, y=None) == NULL
    for name in ("x", "res", "w", "q", "sum", "y"):
        assert norm(lib, **{name: A16 + 8}) == ALIGN, name
    for name in ("ld_x", "ld_r", "ld_q", "ld_s", "ld_y"):
        assert norm(lib, **{name: 516}) == ALIGN, name
    assert norm(lib, scales=A16 + 2) == ALIGN
    # what is not there is not looked at
    assert norm(lib, res=None, ld_r=0, sum=None, ld_s=0, q=None, ld_q=0, scales=None, y=A16 + 8) == ALIGN
    assert norm(lib, rows=0, x=None, w=None, q=None, y=None, sum=None, res=None, scales=None) == OK


def rope(lib, q=A16, ld_q=4096, k=A16, ld_k=1024, v=A16, ld_v=1024, pos=A16, freq=A16, R=128, pairs=0, slots=A16, T=4, Hq=32,
         H=8, D=128, num=64, mode=0, ks=A16, vs=A16, kc=A16, vc=A16, qo=A16, ld_qo=4096, ko=A16, ld_ko=1024):
    return lib.spec_fp8_rope_kv_cache_write(q, ld_q, k, ld_k, v, ld_v, pos, freq, R, pairs, slots, T, Hq, H, D, num, mode, ks,
                                            vs, kc, vc, qo, ld_qo, ko, ld_ko, None)


def test_rope_kv_cache_write(lib):
    assert rope(lib, pairs=2) == ENUM
    assert rope(lib, mode=2) == ENUM
    for bad in (dict(T=-1), dict(Hq=-1), dict(H=0), dict(D=0, R=0), dict(num=-1), dict(R=0), dict(R=-8), dict(R=136),
                dict(ld_q=4088), dict(ld_k=1016), dict(ld_v=1016), dict(ld_qo=4088), dict(ld_ko=1016)):
        assert rope(lib, **bad) == SHAPE, bad
    for bad in (dict(R=60), dict(D=100, R=96), dict(D=520, ld_q=1 << 15, ld_k=1 << 15, ld_v=1 << 15, ld_qo=1 << 15, ld_ko=1 << 15),
                dict(T=I31), dict(Hq=65536, ld_q=1 << 24, ld_qo=1 << 24),
                dict(H=65536, ld_k=1 << 24, ld_v=1 << 24, ld_ko=1 << 24),
                *(dict([(name, 1 << 35)]) for name in ("ld_q", "ld_k", "ld_v", "ld_qo", "ld_ko"))):
        assert rope(lib, **bad) == UNSUP, bad
    for name in ("q", "k", "v", "pos", "freq", "slots", "ks", "vs", "kc", "vc", "qo"):
        assert rope(lib, **{name: None}) == NULL, name
    for name in ("q", "k", "v", "kc", "vc", "qo", "ko"):
        assert rope(lib, **{name: A16 + 8}) == ALIGN, name
    for name in ("ks", "vs", "pos"):
        assert rope(lib, **{name: A16 + 2}) == ALIGN, name
    for name in ("freq", "slots"):
        assert rope(lib, **{name: A16 + 4}) == ALIGN, name
    for name in ("ld_q", "ld_k", "ld_v", "ld_qo", "ld_ko"):
        assert rope(lib, **{name: 4100}) == ALIGN, name
    # what is not there is not looked at: no queries, no rotated keys, no cache
    assert rope(lib, Hq=0, q=None, ld_q=0, qo=None, ld_qo=0, ko=None, ld_ko=0, pos=None) == NULL
    assert rope(lib, num=0, ks=None, vs=None, kc=None, vc=None, slots=None) == NULL
    assert rope(lib, T=0, q=None, k=None, v=None, pos=None, freq=None, slots=None, ks=None, vs=None, kc=None, vc=None,
                qo=None) == OK


def quant4(lib, x=A16, rows=4, cols=512, ld_x=512, q=A16, ld_q=256, s=A16, ld_s=16):
    return lib.spec_fp4_quantize(x, rows, cols, ld_x, q, ld_q, s, ld_s, None)


def test_fp4_quantize(lib):
    for bad in (dict(rows=-1), dict(cols=0), dict(ld_x=504), dict(ld_q=240), dict(ld_s=15)):
        assert quant4(lib, **bad) == SHAPE, bad
    assert quant4(lib, cols=496) == UNSUP
    assert quant4(lib, cols=I31, ld_x=I31, ld_q=I31, ld_s=I31) == UNSUP
    for name in ("x", "q", "s"):
        assert quant4(lib, **{name: None}) == NULL, name
    for bad in (dict(x=A16 + 8), dict(q=A16 + 8), dict(ld_x=516), dict(ld_q=264)):
        assert quant4(lib, **bad) == ALIGN, bad
    assert quant4(lib, rows=0, x=None, q=None, s=None) == OK


def gemm4(lib, a=A16, lda=512, sa=A16, mode=0, w=A16, ldw=256, ws=A16, ld_ws=16, M=4, N=64, K=512, y=A16, ldy=64, out=0):
    return lib.spec_fp8_gemm_fp4(a, lda, sa, mode, w, ldw, ws, ld_ws, M, N, K, y, ldy, out, None)


def test_gemm_fp4(lib):
    assert gemm4(lib, mode=2) == ENUM
    assert gemm4(lib, out=2) == ENUM
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(lda=496), dict(ldw=240), dict(ld_ws=15), dict(ldy=56)):
        assert gemm4(lib, **bad) == SHAPE, bad
    for bad in (dict(K=496), dict(K=(1 << 30) + 32, lda=I31, ldw=I31, ld_ws=I31), dict(N=1 << 28, ldy=1 << 28), dict(M=1 << 20)):
        assert gemm4(lib, **bad) == UNSUP, bad
    for name in ("a", "sa", "w", "ws", "y"):
        assert gemm4(lib, **{name: None}) == NULL, name
    for bad in (dict(a=A16 + 8), dict(w=A16 + 8), dict(y=A16 + 8), dict(sa=A16 + 2), dict(lda=520), dict(ldw=264), dict(ldy=68)):
        assert gemm4(lib, **bad) == ALIGN, bad
    assert gemm4(lib, M=0, a=None, sa=None, w=None, ws=None, y=None) == OK


def test_the_binding_refuses_what_is_no_device_tensor():
    import torch

    import paper_2606_18502_amd as p
    z = torch.zeros
    x, c = z((4, 64), dtype=torch.bfloat16), z((4, 64), dtype=torch.uint8)
    h = z((4, 2, 16), dtype=torch.bfloat16)
    for call, name in ((lambda: p.rms_norm(x, x[0]), "x"), (lambda: p.rms_norm_quantize(x, x[0]), "x"),
                       (lambda: p.rope_kv_cache_write(h, h, h, *[c] * 7), "q"), (lambda: p.quantize_fp4(x), "x"),
                       (lambda: p.gemm_fp4(c, x, c, c), "a")):
        with pytest.raises(ValueError, match=f"{name} must be a CUDA"):
            call()


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


def test_sizes_whose_products_exceed_64_bits(lib):
    """Refused by the heads' size alone, before any stride is compared with a product (the sanitized run sees an overflow)."""
    for D in (1 << 60, 1 << 62, (1 << 63) - 8):
        for far in ({}, dict.fromkeys(("ld_q", "ld_k", "ld_v", "ld_qo", "ld_ko"), (1 << 63) - 8)):
            assert rope(lib, D=D, **far) == UNSUP, (D, far)
            assert rope(lib, D=D, R=D, Hq=1, H=1, **far) == UNSUP, (D, far)
