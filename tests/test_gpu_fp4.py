"""GPU parity of spec_fp4_quantize and spec_fp8_gemm_fp4 against oracle/fp4.py.

Codes and scales are bit-exact.  The product is within the matrix cores' accumulation bound of the exact sum (oracle/fp4.py
error_bound) and two fp32 roundings, and within 2e-3 of its row's largest output; the bf16 output is the rounding of the
fp32 one, bit for bit."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import e4m3, fp4, gemm as og, quantize as oq
from tests import fp4_cases
from tests.gpu_util import dev_bf16, dev_f32, dev_u8, host, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (17, 4096), (5, 14336), (70000, 32), (2, 2080)])
def test_quantize_is_exact(rows, cols):
    p = need_gpu()
    x = wl.linear_weights(rows, cols, rows + cols)
    codes, scales = p.quantize_fp4(dev_bf16(x))
    want = fp4.quantize(x)
    np.testing.assert_array_equal(host(codes), want[0])
    np.testing.assert_array_equal(host(scales), want[1])


def test_quantize_of_every_bf16_magnitude():
    """Each finite bf16 value as a group's largest, with smaller ones, ties and zeros of both signs beside it."""
    p = need_gpu()
    top = np.arange(0, 0x7F80, dtype=np.uint16)
    rng = np.random.default_rng(0)
    x = np.zeros((len(top), 32), np.uint16)
    share = rng.integers(0, 33, (len(top), 30)) / 32.0                     # of the largest: ties among them
    x[:, 0] = top
    x[:, 1:31] = wl.bf16_bits_from_f32((wl.f32_from_bf16_bits(top)[:, None] * share).astype(np.float32))
    x[:, 31] = 0x8000
    x ^= (rng.integers(0, 2, x.shape).astype(np.uint16) << 15)
    codes, scales = p.quantize_fp4(dev_bf16(x))
    want = fp4.quantize(x)
    np.testing.assert_array_equal(host(scales), want[1])
    np.testing.assert_array_equal(host(codes), want[0])


def test_quantize_into_views():
    p = need_gpu()
    x = wl.linear_weights(9, 128, 1)
    wide = torch.zeros((9, 160), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:136] = dev_bf16(x)
    q, s = (torch.full((9, n), 0xAB, dtype=torch.uint8, device="cuda") for n in (96, 7))
    got = p.quantize_fp4(wide[:, 8:136], out=q[:, 16:80], scales=s[:, 1:5])
    want = fp4.quantize(x)
    np.testing.assert_array_equal(host(got[0]), want[0])
    np.testing.assert_array_equal(host(got[1]), want[1])
    assert (q[:, :16] == 0xAB).all() and (q[:, 80:] == 0xAB).all() and (s[:, :1] == 0xAB).all() and (s[:, 5:] == 0xAB).all()


def operands(M, N, K, seed):
    a, sa = oq.quantize_rows(wl.linear_activations(M, K, seed, 0.01, 20.0))
    return a, sa, *fp4.quantize(wl.linear_weights(N, K, seed + 1))


def check(y32, y16, a, sa, codes, scales):
    w = fp4.decode(codes, scales)
    ref = fp4.gemm(a, sa, w)
    y = host(y32).astype(np.float64)
    bound = fp4.error_bound(a, sa, w) + 2.0 ** -23 * np.abs(ref)
    assert (np.abs(y - ref) <= bound).all(), (np.abs(y - ref) / np.maximum(bound, 1e-300)).max()
    assert og.rel_error(y, ref) <= 2e-3
    np.testing.assert_array_equal(host_bf16_bits(y16), wl.bf16_bits_from_f32(host(y32)))


@pytest.mark.parametrize("M,N,K", [
    (1, 1, 32), (1, 64, 4096), (2, 33, 64), (3, 100, 96), (5, 200, 160), (7, 65, 480), (8, 256, 512), (9, 250, 544), (15, 31, 1024),
    (16, 48, 2080), (17, 130, 2048), (31, 96, 1056), (33, 96, 4096), (48, 40, 992), (63, 72, 1536), (64, 128, 4096), (65, 40, 576),
    (130, 24, 672), (1, 512, 14336), (4, 96, 14336), (12, 1000, 736), (130, 1000, 96), (200, 4500, 288), (150, 12000, 96),
])
def test_parity(M, N, K):
    p = need_gpu()
    say(f"gemm_fp4 M={M} N={N} K={K}")
    a, sa, w, sw = operands(M, N, K, M + N + K)
    d = dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw)
    y32, y16 = p.gemm_fp4(*d, out_dtype=torch.float32), p.gemm_fp4(*d)
    check(y32, y16, a, sa, w, sw)
    one = dev_f32([0.03125])                                 # one scale for all rows
    if M > 1:
        y = p.gemm_fp4(d[0], one, d[2], d[3], out_dtype=torch.float32)
        check(y, p.gemm_fp4(d[0], one, d[2], d[3]), a, np.float32(0.03125), w, sw)


@pytest.mark.parametrize("M", [3, 11, 27, 50])
@pytest.mark.parametrize("N,K", [(70, 33056), (1300, 33056), (2500, 33056), (5000, 2080), (9000, 1184), (14000, 2080), (17000, 1312), (20000, 352), (33011, 4384), (4500, 16544),
                                 (9000, 8320), (33011, 160)])
def test_every_variant(M, N, K):
    """Numbers of columns on all sides of the variants' borders, K beyond the scales that a workgroup holds at a time; sampled
    columns, the first and last among them."""
    p = need_gpu()
    say(f"gemm_fp4 variants M={M} N={N} K={K}")
    rng = np.random.default_rng(N + K)
    a, sa = oq.quantize_rows(wl.linear_activations(M, K, 1, 0.01, 20.0))
    w = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sw = rng.integers(120, 128, (N, K // 32), dtype=np.uint8)
    d = dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw)
    cols = np.unique(np.concatenate((rng.choice(N, 40), np.arange(17), np.arange(N - 17, N))))
    y32, y16 = p.gemm_fp4(*d, out_dtype=torch.float32), p.gemm_fp4(*d)
    check(y32[:, cols].contiguous(), y16[:, cols].contiguous(), a, sa, w[cols], sw[cols])
    # scales of any address: the same sums
    odd = torch.zeros((N, K // 32 + 5), dtype=torch.uint8, device="cuda")
    odd[:, 3:3 + K // 32] = d[3]
    assert torch.equal(p.gemm_fp4(*d[:3], odd[:, 3:3 + K // 32], out_dtype=torch.float32), y32)


def test_strides_and_what_lies_beside():
    p = need_gpu()
    M, N, K = 6, 90, 288
    a, sa, w, sw = operands(M, N, K, 2)
    da = torch.full((M, K + 64), 0x7F, dtype=torch.uint8, device="cuda")            # NaN codes beside every operand
    dw = torch.full((N, K // 2 + 32), 0x77, dtype=torch.uint8, device="cuda")
    ds = torch.full((N, K // 32 + 4), 255, dtype=torch.uint8, device="cuda")
    da[:, 16:16 + K], dw[:, 16:16 + K // 2], ds[:, 1:1 + K // 32] = dev_u8(a), dev_u8(w), dev_u8(sw)
    out = {}
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.full((M, 128), 7.0, dtype=dtype, device="cuda")
        got = p.gemm_fp4(da[:, 16:16 + K], dev_f32(sa), dw[:, 16:16 + K // 2], ds[:, 1:1 + K // 32], out=y[:, 8:8 + N])
        assert (y[:, :8] == 7.0).all() and (y[:, 8 + N:] == 7.0).all()
        out[dtype] = got.contiguous()
    check(out[torch.float32], out[torch.bfloat16], a, sa, w, sw)


@pytest.mark.parametrize("M,N,K", [(3, 40, 1056), (20, 40, 2112), (50, 40, 608)])
def test_nan_codes_scales_and_extreme_scales(M, N, K):
    """A NaN code reaches its row alone and a scale of 255 its column alone; scales at both ends of E8M0 are what they stand
    for (2^-127 and 2^127), as far as fp32 holds the products."""
    p = need_gpu()
    a, sa, w, sw = operands(M, N, K, 7)
    a[1, 5], a[2, K - 1] = 0x7F, 0xFF
    sw[3, K // 32 - 1], sw[4, 0] = 255, 255
    sw[7, :] = 127 + 100
    sw[8, :] = 127 - 100
    sw[9, ::2] = 0
    y = host(p.gemm_fp4(dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw), out_dtype=torch.float32)).astype(np.float64)
    bad = np.zeros((M, N), bool)
    bad[1:3] = True
    bad[:, 3:5] = True
    np.testing.assert_array_equal(np.isnan(y), bad)
    clean = a.copy()
    clean[1, 5] = clean[2, K - 1] = 0
    sw[3:5] = 127
    wd = fp4.decode(w, sw)
    ref, bound = fp4.gemm(clean, sa, wd), fp4.error_bound(clean, sa, wd)
    bound += 2.0 ** -23 * np.abs(ref) + 2.0 ** -120                     # (2^-127 is below the normal numbers)
    assert (np.abs(y - ref) <= bound)[~bad].all()


def test_a_row_does_not_depend_on_the_others_and_runs_agree():
    """The same row among up to 16, 32 and 64 (and more): within one way of splitting rows the bits are the same."""
    p = need_gpu()
    a, sa, w, sw = operands(80, 300, 4128, 11)
    d = dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw)
    for counts in ((1, 7, 16), (17, 32), (33, 64, 80)):
        rows = [p.gemm_fp4(d[0][:m], d[1][:m], d[2], d[3], out_dtype=torch.float32) for m in counts for _ in range(2)]
        for y in rows[1:]:
            n = min(len(y), len(rows[0]))
            assert torch.equal(y[:n], rows[0][:n])


def test_many_columns_and_far_rows():
    """Offsets beyond 32 bits: weights of a far stride."""
    p = need_gpu()
    N, K, M = 40, 256, 3
    a, sa, w, sw = operands(M, N, K, 13)
    far = 1 << 27
    box = torch.zeros(N * far, dtype=torch.uint8, device="cuda")
    dw, ds = (box.as_strided((N, n), (far, 1), at) for n, at in ((K // 2, 0), (K // 32, 4096 + 1)))
    dw.copy_(dev_u8(w))
    ds.copy_(dev_u8(sw))
    y32 = p.gemm_fp4(dev_u8(a), dev_f32(sa), dw, ds, out_dtype=torch.float32)
    check(y32, p.gemm_fp4(dev_u8(a), dev_f32(sa), dw, ds), a, sa, w, sw)


def test_refused_arguments():
    p = need_gpu()
    d = dict(device="cuda")
    a, sa = torch.zeros((4, 64), dtype=torch.uint8, **d), torch.ones(4, **d)
    w, sw = torch.zeros((8, 32), dtype=torch.uint8, **d), torch.zeros((8, 2), dtype=torch.uint8, **d)
    for call, message in ((lambda: p.gemm_fp4(a, sa, w[:, :16], sw), "activations' K"), (lambda: p.gemm_fp4(a, sa, w, sw[:, :1]), "sw must be"),
                          (lambda: p.gemm_fp4(a, sa, w, sw[:4]), "sw must be"), (lambda: p.gemm_fp4(a, sa[:3], w, sw), "sa must hold"),
                          (lambda: p.gemm_fp4(a, sa, w, sw.float()), "sw must have dtype"),
                          (lambda: p.gemm_fp4(a, sa, w, sw, out_dtype=torch.float16), "out must be bf16 or fp32"),
                          (lambda: p.gemm_fp4(a, sa, w, sw, out=torch.empty((4, 16), **d)), "out must be"),
                          (lambda: p.quantize_fp4(torch.zeros((4, 64), **d)), "x must have dtype"),
                          (lambda: p.quantize_fp4(torch.zeros((4, 64), dtype=torch.bfloat16, **d), out=w), "out must be")):
        with pytest.raises(ValueError, match=message):
            call()
    with pytest.raises(p.SpecError) as e:
        p.quantize_fp4(torch.zeros((4, 48), dtype=torch.bfloat16, **d))
    assert e.value.status == 3
    with pytest.raises(p.SpecError) as e:
        p.gemm_fp4(a[:, :48], sa, w[:, :24], sw[:, :1])
    assert e.value.status == 3
    assert p.gemm_fp4(a[:0], sa[:0], w, sw).shape == (0, 8)
    torch.cuda.synchronize()


@pytest.mark.parametrize("v,M,N,K", fp4_cases.beyond_panels())
def test_every_variant_beyond_a_panel_of_scales(v, M, N, K):
    """Scales, ring and pointers go on in a second and third panel; some waves have no step there, and K ends inside one."""
    p = need_gpu()
    say(f"gemm_fp4 panels variant={v} M={M} N={N} K={K}")
    rng = np.random.default_rng(N + K)
    a, sa = oq.quantize_rows(wl.linear_activations(M, K, 1, 0.01, 20.0))
    w = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sw = rng.integers(120, 128, (N, K // 32), dtype=np.uint8)
    d = dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw)
    cols = np.unique(np.concatenate((rng.choice(N, 24), np.arange(17), np.arange(N - 17, N))))
    y32, y16 = p.gemm_fp4(*d, out_dtype=torch.float32), p.gemm_fp4(*d)
    check(y32[:, cols].contiguous(), y16[:, cols].contiguous(), a, sa, w[cols], sw[cols])


@pytest.mark.parametrize("N,K,v,counts", fp4_cases.ROWS)
def test_a_row_has_the_same_bits_among_all_counts_of_a_variant(N, K, v, counts):
    """First and last rows alone among fewer: a variant's rows do not see each other."""
    p = need_gpu()
    say(f"gemm_fp4 rows variant={v} N={N} K={K}")
    most = counts[-1]
    rng = np.random.default_rng(N + most)
    a, sa = oq.quantize_rows(wl.linear_activations(most, K, 3, 0.01, 20.0))
    w = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sw = rng.integers(120, 128, (N, K // 32), dtype=np.uint8)
    d = dev_u8(a), dev_f32(sa), dev_u8(w), dev_u8(sw)
    whole = p.gemm_fp4(*d, out_dtype=torch.float32)
    for m in counts:
        for rows in (slice(0, m), slice(most - m, most)):
            assert torch.equal(p.gemm_fp4(d[0][rows], d[1][rows], d[2], d[3], out_dtype=torch.float32), whole[rows]), (m, rows)
