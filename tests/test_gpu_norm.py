"""GPU parity of spec_fp8_rms_norm (the residual's addition, the norm, its E4M3 codes) against oracle/norm.py.

The sum is exact: fp32 of two bf16 values, rounded to bf16.  The kernel's y in fp32 is off by at most TOL of itself: the
sum of squares takes at most 64 fused additions in a thread (for rows of up to 65536; cols / 1024 for wider ones), 6 across a
wave and 16 across waves, half of whose relative error (and of h's own rounding, twice) reaches 1/sqrt, and mean, eps,
square root, quotient and the two products round once each: (64 + 6 + 16 + 2) / 2 + 8 = 52 roundings of 2^-24, taken as 64.  bf16 adds half a step, 2^-8.  A code has
to be the one of some value within TOL of y over the kernel's own scale."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import e4m3, norm as on, quantize as oq
from tests.gpu_util import dev_bf16, host, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu

TOL = 64 * 2.0 ** -24
EPS = 1e-5


def tolerance(cols):
    return TOL if cols <= 65536 else (cols / 1024 / 2 + 20) * 2.0 ** -24


def values(t):
    return oq.bf16_to_f32(host_bf16_bits(t)).astype(np.float64)


def inputs(rows, cols, seed, residual=True):
    x = wl.linear_activations(rows, cols, seed, 0.01, 20.0)
    r = wl.linear_activations(rows, cols, seed + 1, 0.01, 50.0) if residual else None
    w = wl.bf16_bits_from_f32((1 + 0.2 * np.random.default_rng(seed).standard_normal(cols)).astype(np.float32))
    return x, r, w


def check_codes(codes, scale, y, tol=TOL):
    """codes [rows, cols] of y (fp64) under the kernel's scale [rows, 1] (fp32 values)."""
    inv = (1.0 / scale.astype(np.float64)).astype(np.float32).astype(np.float64)
    with np.errstate(over="ignore"):
        lo, hi = y * inv * (1 - tol - 2.0 ** -23), y * inv * (1 + tol + 2.0 ** -23)
    a, b, c = (e4m3.decode(e4m3.encode(np.clip(v, -1e30, 1e30).astype(np.float32))) for v in (lo, hi, y * inv))
    got = e4m3.decode(codes)
    assert ((np.minimum(a, b) <= got) & (got <= np.maximum(a, b))).all(), np.abs(got - c).max()


def check(y, out_q, out_s, out_y, static=None):
    tol = tolerance(y.shape[1])
    if out_y is not None:
        err = np.abs(values(out_y) - y)
        assert (err <= np.abs(y) * (2.0 ** -8 + tol) + 2.0 ** -133).all(), (err / np.maximum(np.abs(y), 1e-30)).max()
    if out_q is None:
        return
    if static is None:
        s = host(out_s)
        ref = on.row_scale(y)
        assert (np.abs(s - ref) <= ref * (tol + 2.0 ** -23)).all()
    else:
        s = np.full(len(y), static, np.float32)
    check_codes(host(out_q), s[:, None], y, tol)


@pytest.mark.parametrize("rows,cols,residual,static,normed", [
    (1, 8, True, False, True), (3, 64, True, False, True), (5, 520, False, False, True), (2, 2200, True, True, False),
    (1, 4096, True, False, False), (37, 4096, True, False, True), (320, 4096, True, False, False), (9, 4104, False, True, True),
    (7, 7176, True, False, True), (300, 1000, True, True, True), (3, 16384, True, False, True), (2, 16392, False, False, True),
    (2, 32768, True, False, True), (3, 40008, True, False, True), (1, 65536, True, False, True),
    (2, 32776, True, False, True), (2, 98312, True, True, True), (1, 1 << 20, True, False, True),
])
def test_parity(rows, cols, residual, static, normed):
    p = need_gpu()
    say(f"norm rows={rows} cols={cols} residual={residual} static={static} normed={normed}")
    x, r, w = inputs(rows, cols, rows + cols, residual)
    h = on.residual_sum(x, r)
    y = on.rms_norm(h, w, EPS)
    dx, dr, dw = dev_bf16(x), None if r is None else dev_bf16(r), dev_bf16(w)
    given = torch.full((1,), 0.02, device="cuda") if static else None       # (some values are beyond 448 * 0.02)
    ny = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda") if normed else None
    q, s, total = p.rms_norm_quantize(dx, dw, EPS, residual=dr, per_tensor_scale=given, normed=ny)
    check(y, q, s, ny, np.float32(0.02) if static else None)
    if residual:
        np.testing.assert_array_equal(host_bf16_bits(total), wl.bf16_bits_from_f32(h.astype(np.float32)))
    else:
        assert total is None
    # the bf16 norm alone gives the same values, and a row alone the same bits as among others
    y2, total2 = p.rms_norm(dx, dw, EPS, residual=dr)
    if normed:
        assert torch.equal(y2.view(torch.int16), ny.view(torch.int16))
    if residual:
        assert torch.equal(total2.view(torch.int16), total.view(torch.int16))
    last = p.rms_norm_quantize(dx[-1:], dw, EPS, residual=None if dr is None else dr[-1:], per_tensor_scale=given)
    assert torch.equal(last[0], q[-1:]) and (static or torch.equal(last[1], s[-1:]))


@pytest.mark.parametrize("where,cols", [("residual", 1352), ("x", 1352), ("residual", 33000), ("x", 33000)])
def test_in_place_and_strides(where, cols):
    """Column blocks of wider tensors; the sum over the residual (or x), y over the other; what is beside them stays."""
    p = need_gpu()
    rows, wide = 33, cols + 56
    x, r, w = inputs(rows, cols, 5)
    box = torch.full((2, rows, wide), 7.0, dtype=torch.bfloat16, device="cuda")
    dx, dr = box[0][:, 16:16 + cols], box[1][:, 16:16 + cols]
    dx.copy_(dev_bf16(x))
    dr.copy_(dev_bf16(r))
    h = on.residual_sum(x, r)
    y = on.rms_norm(h, w, EPS)
    codes = torch.full((rows, wide), 0xAB, dtype=torch.uint8, device="cuda")
    ny, ns = (dx, dr) if where == "residual" else (dr, dx)
    q, s, total = p.rms_norm_quantize(dx, dev_bf16(w), EPS, residual=dr, residual_out=ns, normed=ny, out=codes[:, 16:16 + cols])
    assert total is ns
    check(y, q.contiguous(), s, ny.contiguous())
    np.testing.assert_array_equal(host_bf16_bits(ns.contiguous()), wl.bf16_bits_from_f32(h.astype(np.float32)))
    for t, v in ((box[0], 7.0), (box[1], 7.0), (codes, 0xAB)):
        assert (t[:, :16] == v).all() and (t[:, 16 + cols:] == v).all()


@pytest.mark.parametrize("cols", [4096, 40000])
def test_rows_that_are_not_finite_and_rows_beyond_fp32_squares(cols):
    p = need_gpu()
    rows = 12
    x, r, w = inputs(rows, cols, 9)
    xf = wl.f32_from_bf16_bits(x).copy()
    rf = wl.f32_from_bf16_bits(r).copy()
    xf[1, 77] = np.inf
    xf[3, 4095] = np.nan
    rf[5, 0] = -np.inf
    xf[6], rf[6] = 0.0, 0.0                               # zeros: y and codes 0, the least scale
    xf[7] *= 1e25                                          # squares overflow
    rf[8] *= 3e35
    xf[9], rf[9] = xf[9] * 1e-30, rf[9] * 1e-30             # eps alone is left of the norm
    xf[10, 5] = rf[10, 5] = 3e38                            # the sum itself overflows: an infinity
    xf[11] = 0.0
    rf[11] = 0.0
    xf[11, 9] = 3e38                                       # one channel is the whole row
    x, r = wl.bf16_bits_from_f32(xf), wl.bf16_bits_from_f32(rf)
    y = on.rms_norm(on.residual_sum(x, r), w, EPS)
    wild = [1, 3, 5, 10]
    assert np.isnan(y[wild]).all() and np.isfinite(np.delete(y, wild, 0)).all()
    ny = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    q, s, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), EPS, residual=dev_bf16(r), normed=ny)
    fine = [i for i in range(rows) if i not in wild]
    check(y[fine], q[fine], s[fine], ny[fine])
    assert (host(s)[wild + [6]] == 2.0 ** -100).all()
    assert (host(q)[wild] == 0x7F).all() and np.isnan(values(ny)[wild]).all()
    assert not host(q)[6].any() and not values(ny)[6].any()
    # under a given scale, too
    q, _, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), EPS, residual=dev_bf16(r), per_tensor_scale=torch.ones(1, device="cuda"))
    assert (host(q)[wild] == 0x7F).all()
    check_codes(host(q)[fine], np.ones((1, 1), np.float32), y[fine])


def test_large_weights():
    """Products of a value and a weight beyond fp32, although y is within it."""
    p = need_gpu()
    x, _, _ = inputs(4, 512, 3, False)
    x = wl.bf16_bits_from_f32(wl.f32_from_bf16_bits(x) * np.float32(1e10))
    w = wl.bf16_bits_from_f32(np.full(512, 2.0 ** 100, np.float32))
    y = on.rms_norm(on.residual_sum(x), w, EPS)
    ny = torch.empty((4, 512), dtype=torch.bfloat16, device="cuda")
    q, s, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), EPS, normed=ny)
    check(y, q, s, ny)


def test_more_rows_than_one_launch_takes():
    p = need_gpu()
    rows, cols = (1 << 21) + 3, 8
    x = torch.randn((rows, cols), device="cuda").to(torch.bfloat16)
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    r = torch.randn((rows, cols), device="cuda").to(torch.bfloat16)
    q, s, total = p.rms_norm_quantize(x, w, EPS, residual=r)
    for part in (slice(0, 5), slice((1 << 21) - 2, rows)):
        h = on.residual_sum(host_bf16_bits(x[part]), host_bf16_bits(r[part]))
        check(on.rms_norm(h, host_bf16_bits(w), EPS), q[part], s[part], None)
        np.testing.assert_array_equal(host_bf16_bits(total[part]), wl.bf16_bits_from_f32(h.astype(np.float32)))


def test_rows_beyond_32_bits():
    """Row strides that put the second row past 2^31 elements, on every side."""
    p = need_gpu()
    cols, far = 264, 1 << 31
    x, r, w = inputs(2, cols, 31)
    box = torch.zeros(far + 4 * cols, dtype=torch.bfloat16, device="cuda")
    dx, dr, ns, ny = (box.as_strided((2, cols), (far, 1), i * cols) for i in range(4))
    codes = torch.zeros(far + cols, dtype=torch.uint8, device="cuda").as_strided((2, cols), (far, 1))
    dx.copy_(dev_bf16(x))
    dr.copy_(dev_bf16(r))
    q, s, total = p.rms_norm_quantize(dx, dev_bf16(w), EPS, residual=dr, residual_out=ns, normed=ny, out=codes)
    h = on.residual_sum(x, r)
    check(on.rms_norm(h, w, EPS), q.contiguous(), s, ny.contiguous())
    np.testing.assert_array_equal(host_bf16_bits(total.contiguous()), wl.bf16_bits_from_f32(h.astype(np.float32)))


def test_refused_arguments_and_no_rows():
    p = need_gpu()
    d = dict(device="cuda")
    x, w = torch.ones((4, 64), dtype=torch.bfloat16, **d), torch.ones(64, dtype=torch.bfloat16, **d)
    bad = [
        (lambda: p.rms_norm(x.float(), w), "x must have dtype"),
        (lambda: p.rms_norm(x, w[:56]), "weight must be"),
        (lambda: p.rms_norm(x, w.float()), "weight must have dtype"),
        (lambda: p.rms_norm(x, w, residual=x[:3]), "residual must be"),
        (lambda: p.rms_norm(x, w, residual=x, residual_out=x[:, :56]), "residual_out must be"),
        (lambda: p.rms_norm(x, w, out=x[:2]), "out must be"),
        (lambda: p.rms_norm(x, w, residual=x, residual_out=x, out=x), "must differ"),
        (lambda: p.rms_norm_quantize(x, w, residual=x, residual_out=x, normed=x), "must differ"),
        (lambda: p.rms_norm_quantize(x, w, out=torch.empty((4, 56), dtype=torch.uint8, **d)), "out must be"),
        (lambda: p.rms_norm_quantize(x, w, scales=torch.empty(3, **d)), "scales must be"),
        (lambda: p.rms_norm_quantize(x, w, per_tensor_scale=torch.empty(4, **d)), "per_tensor_scale must hold"),
        (lambda: p.rms_norm_quantize(x, w, normed=torch.empty((4, 8), dtype=torch.bfloat16, **d)), "normed must be"),
    ]
    for call, message in bad:
        with pytest.raises(ValueError, match=message):
            call()
    for call, status in ((lambda: p.rms_norm(x, w, eps=0.0), 8), (lambda: p.rms_norm(x[:, :60], w[:60]), 3)):
        with pytest.raises(p.SpecError) as e:
            call()
        assert e.value.status == status
    q, s, total = p.rms_norm_quantize(x[:0], w, residual=x[:0])
    assert q.shape == (0, 64) and s.shape == (0,) and total.shape == (0, 64)
    # no residual, but a place for the sum: x itself
    y, total = p.rms_norm(x, w, residual_out=torch.empty_like(x))
    assert torch.equal(total, x)
    torch.cuda.synchronize()


@pytest.mark.parametrize("cols", [4096, 40000])
def test_an_eps_of_the_size_of_the_squares(cols):
    """Rows on both sides of 2^126, what their squares sum to, under an eps as large as their mean: it counts on either side."""
    p = need_gpu()
    rows = 6
    x = wl.f32_from_bf16_bits(inputs(rows, cols, 13, False)[0]).copy()
    x /= np.sqrt(np.mean(x.astype(np.float64) ** 2, axis=1, keepdims=True)).astype(np.float32)
    mean = 2.0 ** 126 / cols * np.array([0.25, 0.9, 1.1, 4.0, 16.0, 4096.0])
    x = wl.bf16_bits_from_f32(x * np.sqrt(mean)[:, None].astype(np.float32))
    w = inputs(1, cols, 14)[2]
    for eps in (2.0 ** 126 / cols, 2.0 ** 126):
        y = on.rms_norm(on.residual_sum(x), w, eps)
        ny = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
        q, s, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), eps, normed=ny)
        check(y, q, s, ny)


def test_an_eps_near_the_largest_number():
    """The mean of the squares and eps together exceed fp32, although neither does."""
    p = need_gpu()
    eps = float(np.finfo(np.float32).max)
    x = wl.bf16_bits_from_f32(np.outer([3e18, 1.0, 1e30], [1, -1, 0.5, 0.25, -1, 1, 0.75, 1]).astype(np.float32))
    w = inputs(1, 8, 16)[2]
    y = on.rms_norm(on.residual_sum(x), w, eps)
    assert (np.abs(y[0]) > 0.01).all()
    ny = torch.empty((3, 8), dtype=torch.bfloat16, device="cuda")
    q, s, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), eps, normed=ny)
    check(y, q, s, ny)


@pytest.mark.parametrize("cols", [512, 40000])
def test_small_channels_beside_large_ones(cols):
    """A channel whose square exceeds fp32, and channels down to 2^-66 with weights of 2^-3 to 2^40 beside it: y keeps its bits down
    to the least normal number."""
    p = need_gpu()
    rows = 4
    x = wl.f32_from_bf16_bits(inputs(rows, cols, 17, False)[0]).astype(np.float64)
    x = np.copysign(1 + np.abs(x) % 1, x) * 2.0 ** -np.linspace(30, 66, cols)
    x[:, 5], x[1, 7] = 2.0 ** 66, 2.0 ** 70
    x = wl.bf16_bits_from_f32(x.astype(np.float32))
    w = wl.bf16_bits_from_f32((2.0 ** (np.arange(cols) % 44 - 3)).astype(np.float32))
    y = on.rms_norm(on.residual_sum(x), w, EPS)
    normal = np.abs(y) >= 2.0 ** -126
    assert (normal & (np.abs(y) < 2.0 ** -110)).sum() > rows * 20
    ny = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    q, s, _ = p.rms_norm_quantize(dev_bf16(x), dev_bf16(w), EPS, normed=ny)
    check(y, q, s, ny)
