"""GPU parity of spec_fp8_rope_kv_cache_write against oracle/rope.py and oracle/kvcache.py.

The kernel's sine and cosine are off by at most 4 * 2^-24: the fraction of a turn is rounded to fp32 (2^-26 turns, 1.6 * 2^-24
in angle) and sincospi by two units of 2^-24; the 64-bit angle adds |angle| 2^-51.  The rotation rounds twice more, so a rotated
channel is within TOL = 8 * 2^-24 of |x| + |y| of its pair.  A row's largest rotated magnitude is at least half of any
pair's |x| + |y|, so its scale is within 2 TOL and a rounding.  Values' codes and scales are the plain cache write's, bit
for bit; slots that no token names keep what they held."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import e4m3, kvcache as ok, quantize as oq, rope
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, host, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu

TOL = 8 * 2.0 ** -24
SENT_CODE, SENT_SCALE = 0xAB, -1.0


def values(t):
    return oq.bf16_to_f32(host_bf16_bits(t.contiguous())).astype(np.float64)


def make(T, Hq, H, D, R, num_slots, seed, far=131072):
    rng = np.random.default_rng(seed)
    qkv = wl.linear_activations(max(T, 1), (Hq + 2 * H) * D, seed, 0.01, 20.0)[:T]
    pos = rng.integers(0, far, T).astype(np.int32)
    slots = rng.choice(num_slots, T, replace=False).astype(np.int64)
    if T >= 3:
        slots[1] = -1                     # padding
        slots[T - 1] = num_slots + 5      # beyond the cache
        pos[0], pos[2] = 0, far - 1
    return qkv, pos, 500000.0 ** (-np.arange(R // 2) * 2.0 / R), slots


def run(p, qkv, pos, freq, slots, Hq, H, D, num_slots, neighbours=False, static=None, keys=False, in_place=False):
    T = len(pos)
    d = dev_bf16(qkv)
    q, k, v = (d[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
    kc = torch.full((num_slots, H, D), SENT_CODE, dtype=torch.uint8, device="cuda")
    vc = torch.full_like(kc, SENT_CODE)
    if static is None:
        ks = torch.full((num_slots, H), SENT_SCALE, device="cuda")
        vs = torch.full_like(ks, SENT_SCALE)
    else:
        ks, vs = dev_f32([static[0]]), dev_f32([static[1]])
    qo = q if in_place else None
    ko = (k if in_place else torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")) if keys else None
    qo = p.rope_kv_cache_write(q, k, v, dev_i32(pos), torch.from_numpy(freq).cuda(), torch.from_numpy(slots).cuda(), kc, vc, ks,
                               vs, per_tensor=static is not None, interleaved=neighbours, q_out=qo, k_out=ko)
    return qo, ko, kc, vc, ks, vs, d


def check(qkv, pos, freq, slots, Hq, H, D, num_slots, neighbours, static, got, extra=0.0):
    qo, ko, kc, vc, ks, vs, _ = got
    T, R = len(pos), 2 * len(freq)
    x = oq.bf16_to_f32(qkv).astype(np.float64)
    q, k = x[:, :Hq * D].reshape(T, Hq, D), x[:, Hq * D:(Hq + H) * D].reshape(T, H, D)
    tol = TOL + extra
    refs = []
    for a, out in ((q, qo), (k, ko)):
        ref = rope.rotate(a, pos, freq, neighbours)
        near = tol * rope.pair_sums(a, R, neighbours)
        refs.append((ref, near))
        if out is not None and a.size:
            err = np.abs(values(out) - ref)
            assert (err <= np.abs(ref) * 2.0 ** -8 + near * (1 + 2.0 ** -8) + 2.0 ** -133).all()
    # values: the plain write
    rv = np.full((num_slots, H, D), SENT_CODE, np.uint8)
    rvs = np.full((num_slots, H), SENT_SCALE, np.float32)
    ok.kv_cache_write(qkv[:, (Hq + H) * D:], slots, H, D, rv, rvs, None if static is None else static[1])
    np.testing.assert_array_equal(host(vc), rv)
    if static is None:
        np.testing.assert_array_equal(host(vs), rvs)
    # keys
    ref, near = refs[1]
    codes, scales = host(kc), host(ks)
    seen = np.zeros(num_slots, bool)
    for t, s in enumerate(slots):
        if s < 0 or s >= num_slots:
            continue
        seen[s] = True
        if static is None:
            want = np.maximum(np.abs(ref[t]).max(-1) / 448, 2.0 ** -100)
            assert (np.abs(scales[s] - want) <= want * (2 * tol + 2.0 ** -23)).all()
            sc = scales[s].astype(np.float64)[:, None]
        else:
            sc = np.float64(np.float32(static[0]))
        inv = (1.0 / sc).astype(np.float32).astype(np.float64) if static is None else np.float64(np.float32(1.0 / sc))
        lo, hi = ((ref[t] + sign * near[t]) * inv for sign in (-1, 1))
        lo, hi = lo - np.abs(lo) * 2.0 ** -24, hi + np.abs(hi) * 2.0 ** -24
        a, b = (e4m3.decode(e4m3.encode(v.astype(np.float32))) for v in (lo, hi))
        c = e4m3.decode(codes[s])
        assert ((np.minimum(a, b) <= c) & (c <= np.maximum(a, b))).all(), t
    assert (codes[~seen] == SENT_CODE).all()
    if static is None:
        assert (scales[~seen] == SENT_SCALE).all()


@pytest.mark.parametrize("T,Hq,H,D,R,neighbours,static", [
    (1, 32, 8, 128, 128, False, False), (5, 32, 8, 128, 128, True, False), (37, 8, 2, 64, 64, False, True),
    (13, 4, 1, 80, 32, True, True), (13, 3, 3, 80, 40, False, False), (9, 2, 2, 256, 128, False, False), (4, 1, 1, 8, 8, False, False),
    (4, 5, 1, 8, 8, True, False), (6, 2, 1, 24, 16, False, False), (7, 1, 1, 16, 16, False, False), (7, 7, 1, 32, 32, True, False),
    (3, 2, 1, 512, 512, False, False), (3, 1, 1, 504, 8, True, False), (3, 4, 2, 264, 264, False, True), (321, 6, 2, 128, 64, False, False),
    (2500, 4, 2, 64, 64, False, False), (3, 0, 2, 128, 128, False, False), (700, 16, 1, 128, 128, False, False),
])
def test_parity(T, Hq, H, D, R, neighbours, static):
    p = need_gpu()
    say(f"rope T={T} Hq={Hq} H={H} D={D} R={R} neighbours={neighbours} static={static}")
    num_slots = T + 40
    given = (0.03, 0.01) if static else None            # (some values saturate)
    args = make(T, Hq, H, D, R, num_slots, T + D + R)
    got = run(p, *args, Hq, H, D, num_slots, neighbours, given, keys=True)
    check(*args, Hq, H, D, num_slots, neighbours, given, got)
    # without the rotated keys, and over the inputs themselves: the same bits
    again = run(p, *args, Hq, H, D, num_slots, neighbours, given, keys=False)
    over = run(p, *args, Hq, H, D, num_slots, neighbours, given, keys=True, in_place=True)
    for a in (again, over):
        for x, y in zip((got[0], *got[2:6]), (a[0], *a[2:6])):
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    assert torch.equal(over[1].contiguous().view(torch.int16), got[1].view(torch.int16))
    assert torch.equal(over[6][:, (Hq + H) * D:], dev_bf16(args[0])[:, (Hq + H) * D:])       # values stay


def test_positions_of_31_bits_and_negative_ones():
    p = need_gpu()
    T, Hq, H, D = 6, 4, 2, 64
    qkv, _, freq, slots = make(T, Hq, H, D, D, 50, 3)
    pos = np.array([2 ** 31 - 1, -2 ** 31, -1, 123456789, -77777, 2 ** 30], np.int32)
    freq = np.concatenate(([1.0], freq[1:]))
    got = run(p, qkv, pos, freq, slots, Hq, H, D, 50, keys=True)
    check(qkv, pos, freq, slots, Hq, H, D, 50, False, None, got, extra=2.0 ** 31 * 2.0 ** -51)


def test_wide_rows_and_columns_behind_the_heads():
    """Strides beyond the heads on every side; what lies behind them stays."""
    p = need_gpu()
    T, Hq, H, D, wide = 19, 4, 2, 64, 264
    qkv, pos, freq, slots = make(T, Hq, H, D, D, 40, 8)
    d = dev_bf16(qkv)
    boxes = [torch.full((T, wide + 16 * i), 7.0, dtype=torch.bfloat16, device="cuda") for i in range(5)]
    q, k, v, qo, ko = (b[:, 8:8 + h * D].unflatten(1, (h, D)) for b, h in zip(boxes, (Hq, H, H, Hq, H)))
    for t, a, b in ((q, 0, Hq), (k, Hq, Hq + H), (v, Hq + H, Hq + 2 * H)):
        t.copy_(d[:, a * D:b * D].unflatten(1, (b - a, D)))
    kc, vc = (torch.full((40, H, D), SENT_CODE, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((40, H), SENT_SCALE, device="cuda") for _ in range(2))
    out = p.rope_kv_cache_write(q, k, v, dev_i32(pos), torch.from_numpy(freq).cuda(), torch.from_numpy(slots).cuda(), kc, vc, ks, vs,
                                q_out=qo, k_out=ko)
    assert out is qo
    check(qkv, pos, freq, slots, Hq, H, D, 40, False, None, (qo, ko, kc, vc, ks, vs, None))
    for b, h in zip(boxes, (Hq, H, H, Hq, H)):
        assert (b[:, :8] == 7.0).all() and (b[:, 8 + h * D:] == 7.0).all()


def test_an_empty_cache_and_no_tokens():
    p = need_gpu()
    T, Hq, H, D = 5, 4, 2, 64
    qkv, pos, freq, _ = make(T, Hq, H, D, D, 50, 4)
    slots = np.arange(T)
    got = run(p, qkv, pos, freq, slots, Hq, H, D, 0, keys=True)
    check(qkv, pos, freq, slots, Hq, H, D, 0, False, None, got)
    got = run(p, qkv[:0], pos[:0], freq, slots[:0], Hq, H, D, 50)
    assert got[0].shape == (0, Hq, D) and (got[2] == SENT_CODE).all()


def test_a_cache_beyond_32_bits():
    """Slots whose codes lie past 4 GiB: what is written there is what a small cache gets."""
    p = need_gpu()
    T, Hq, H, D = 4, 2, 2, 64
    qkv, pos, freq, _ = make(T, Hq, H, D, D, 50, 17)
    small = run(p, qkv, pos, freq, np.arange(T), Hq, H, D, T)
    n = 2 ** 32 // (H * D) + 8
    kc, vc = (torch.empty((n, H, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty((n, H), device="cuda") for _ in range(2))
    slots = torch.tensor([n - 1, 2 ** 32 // (H * D), 2 ** 31 // (H * D), 0], device="cuda")
    q, k, v = (dev_bf16(qkv)[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
    p.rope_kv_cache_write(q, k, v, dev_i32(pos), torch.from_numpy(freq).cuda(), slots, kc, vc, ks, vs)
    for a, b in zip(small[2:6], (kc, vc, ks, vs)):
        assert torch.equal(a, b[slots])


def test_more_tokens_than_one_grid_covers():
    p = need_gpu()
    T, D, last = 2 ** 24 + 5, 8, 9
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, D), device="cuda", generator=g).to(torch.bfloat16)[:, None]
    pos = (torch.arange(T, device="cuda", dtype=torch.int64) % 5000).to(torch.int32)
    freq = torch.tensor([1.0, 0.3, 0.07, 0.001], dtype=torch.float64, device="cuda")
    slots = torch.full((T,), -1, device="cuda")
    slots[-last:] = torch.arange(last, device="cuda")

    def call(first):
        kc = torch.full((last, 1, D), SENT_CODE, dtype=torch.uint8, device="cuda")
        ks = torch.full((last, 1), SENT_SCALE, device="cuda")
        vc, vs, t = kc.clone(), ks.clone(), x[first:]
        return p.rope_kv_cache_write(t, t, t, pos[first:], freq, slots[first:], kc, vc, ks, vs)[-last:], kc, vc, ks, vs

    for a, b in zip(call(0), call(T - last)):
        assert torch.equal(a, b)


def test_a_row_of_zeros_and_the_plain_writes_scales():
    """A key of zeros has code 0 and the least scale; at position 0 nothing turns: keys are the plain write's, bit for bit."""
    p = need_gpu()
    T, Hq, H, D = 9, 2, 2, 128
    qkv, pos, freq, slots = make(T, Hq, H, D, D, 60, 21)
    qkv[4] = 0
    got = run(p, qkv, 0 * pos, freq, slots, Hq, H, D, 60, keys=True)
    d = dev_bf16(qkv)
    k, v = (d[:, a * D:(a + H) * D].unflatten(1, (H, D)) for a in (Hq, Hq + H))
    kc = torch.full((60, H, D), SENT_CODE, dtype=torch.uint8, device="cuda")
    vc, ks = kc.clone(), torch.full((60, H), SENT_SCALE, device="cuda")
    vs = ks.clone()
    p.kv_cache_write(k, v, torch.from_numpy(slots).cuda(), kc, vc, ks, vs)
    for a, b in zip(got[2:6], (kc, vc, ks, vs)):
        assert torch.equal(a, b)
    assert torch.equal(got[0].contiguous(), d[:, :Hq * D].unflatten(1, (Hq, D)))
    assert torch.equal(got[1], k)
    assert (host(got[4])[slots[4]] == 2.0 ** -100).all() and not host(got[2])[slots[4]].any()


def test_refused_arguments():
    p = need_gpu()
    d = dict(device="cuda")
    T, Hq, H, D = 4, 4, 2, 64
    q, k = torch.ones((T, Hq, D), dtype=torch.bfloat16, **d), torch.ones((T, H, D), dtype=torch.bfloat16, **d)
    kc, ks = torch.zeros((8, H, D), dtype=torch.uint8, **d), torch.zeros((8, H), **d)
    pos, freq, slots = torch.zeros(T, dtype=torch.int32, **d), torch.ones(D // 2, dtype=torch.float64, **d), torch.arange(T, **d)

    def call(**kw):
        a = dict(q=q, k=k, v=k, positions=pos, inv_freq=freq, slot_mapping=slots, k_cache=kc, v_cache=kc.clone(), k_scale=ks,
                 v_scale=ks.clone()) | kw
        return p.rope_kv_cache_write(**a)

    call()
    for kw, message in ((dict(q=q[:3]), "one T and D"), (dict(v=k[:, :1]), "one T and D"), (dict(q=q[..., :32]), "packed side by side"),
                        (dict(positions=pos.long()), "positions must have dtype"), (dict(positions=pos[:3]), "positions must be"),
                        (dict(inv_freq=freq.float()), "inv_freq must have dtype"), (dict(slot_mapping=slots[:2]), "slot_mapping must be"),
                        (dict(k_cache=kc[:, :1].contiguous()), "k_cache and v_cache"), (dict(per_tensor=True), "per-tensor scales"),
                        (dict(q_out=k), "q_out must be"), (dict(k_out=q), "k_out must be"), (dict(k_out=k.float()), "k_out must have dtype")):
        with pytest.raises(ValueError, match=message):
            call(**kw)
    for kw, status in ((dict(inv_freq=freq.repeat(2)), 2), (dict(inv_freq=freq[:3]), 3), (dict(inv_freq=freq[:0]), 2)):
        with pytest.raises(p.SpecError) as e:
            call(**kw)
        assert e.value.status == status
    torch.cuda.synchronize()


def test_far_positions_are_as_accurate_as_near_ones():
    """Pairs whose first channel all but cancels, so that its bf16 holds the angle's absolute error: at positions of 30 and 31
    bits as at near ones, in units of 2^-24: 1.6 |(x, y)| for the fraction of a turn in fp32, 2 (|x| + |y|) for sine and
    cosine, |y| for the first product, and half a step of the result in fp32 and in bf16."""
    p = need_gpu()
    T, Hq, R = 600, 2, 64
    rng = np.random.default_rng(41)
    pos = np.concatenate((rng.integers(0, 1000, T // 3), rng.integers(2 ** 30, 2 ** 31, T // 3), -rng.integers(2 ** 30, 2 ** 31, T // 3)))
    freq = rng.uniform(0.5, 1.0, R // 2)
    angle = pos.astype(np.longdouble)[:, None] * freq.astype(np.longdouble)
    angle = (angle - np.rint(angle / rope.TWO_PI) * rope.TWO_PI).astype(np.float64)
    c, s = np.cos(angle)[:, None, :, None], np.sin(angle)[:, None, :, None]
    # of 128 values x each the one whose nearest y leaves least
    x = (1 + (np.arange(128) + rng.integers(0, 2)) / 128.0)[None, None, None]
    y = oq.bf16_to_f32(wl.bf16_bits_from_f32((x * c / s).astype(np.float32))).astype(np.float64)
    best = np.abs(x * c - y * s).argmin(-1)[..., None]
    x, y = (np.take_along_axis(np.broadcast_to(v, y.shape), best, -1)[..., 0] for v in (x, y))
    q = np.concatenate((x, y), -1).repeat(Hq, 1)
    bits = wl.bf16_bits_from_f32(q.astype(np.float32).reshape(T, Hq * R))
    k = torch.zeros((T, 1, R), dtype=torch.bfloat16, device="cuda")
    cache, scale = torch.zeros((0, 1, R), dtype=torch.uint8, device="cuda"), torch.zeros((0, 1), device="cuda")
    got = p.rope_kv_cache_write(dev_bf16(bits).unflatten(1, (Hq, R)), k, k, dev_i32(pos.astype(np.int32)), torch.from_numpy(freq).cuda(),
                                torch.zeros(T, dtype=torch.int64, device="cuda"), cache, cache, scale, scale)
    ref = rope.rotate(q, pos.astype(np.int32), freq, False)[..., :R // 2]
    x, y = np.abs(q[..., :R // 2]), np.abs(q[..., R // 2:])
    tol = 2.0 ** -24 * (1.6 * np.hypot(x, y) + 2 * (x + y) + y) + np.abs(ref) * (2.0 ** -8 + 2.0 ** -24)
    err = np.abs(values(got)[..., :R // 2] - ref)
    usual = y < 8                                           # (far larger ones stand beside a sine near 0)
    assert usual.mean() > 0.8 and np.median(np.abs(ref)[usual] / (x + y)[usual]) < 2.0 ** -14
    assert (err <= tol).all(), (err / tol).max()
