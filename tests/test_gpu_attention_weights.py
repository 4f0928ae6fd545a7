"""How many bits the attentions keep of a weight: 16 for rows of few keys in tiles and prompts, 8 for the others there, 15 in
the stream of few rows; what a row's result moves by when a call goes from the one to the other."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa, e4m3
from tests.attention_cases import paged_case, within
from tests.attention_variants import reference
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, dev_u8, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu
FEW = 64                                                 # keys of a row whose weights keep 16 bits


def values(t):
    return wl.f32_from_bf16_bits(host_bf16_bits(t)).astype(np.float64)


def prompt_inputs(seed, n, H, G, D):
    rng = np.random.default_rng(seed)
    bits = [wl.bf16_bits_from_f32(rng.standard_normal((n, h, D)).astype(np.float32)) for h in (H * G, H, H)]
    return bits, [wl.f32_from_bf16_bits(b).astype(np.float64) for b in bits]


@pytest.mark.parametrize("lens,H,G,D", [([64], 2, 4, 128), ([1, 2, 33, 63, 0, 64], 1, 4, 128), ([150, 70], 2, 4, 128), ([64, 90], 2, 1, 64),
                                        ([64], 1, 8, 256), ([40, 64], 1, 3, 96), ([70], 1, 128, 64)])
def test_prompt_rows_of_few_keys_keep_16_bits(lens, H, G, D):
    p = need_gpu()
    say(f"weights of prompts {lens} H={H} G={G} D={D}")
    bits, (q, k, v) = prompt_inputs(sum(lens) + D, sum(lens), H, G, D)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    got = values(p.prompt_attention(*[dev_bf16(b) for b in bits], dev_i32(cu)))
    out, spread, mag = oa.prompt_attention(q, k, v, cu, D ** -0.5)
    keys = np.concatenate([np.arange(1, n + 1) for n in lens])
    few = keys <= FEW
    tol = oa.bound(out, spread, mag, D, max(lens), weight=2.0 ** -8)
    fine = oa.bound(out, spread, mag, D, FEW, weight=2.0 ** -16)
    assert within(got[few], out[few], fine[few]) <= 1.0
    assert within(got, out, tol) <= 1.0


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("n,G,D", [(66, 128, 64), (66, 128, 128), (60, 4, 128), (40, 2, 256)])
def test_an_infinite_value_and_rows_of_few_keys(n, G, D, value):
    """What a weight leaves after its rounding may be 0, and 0 * inf is NaN.  (128 heads on one: rows that see all of a tile.)"""
    p = need_gpu()
    bits, _ = prompt_inputs(5, n, 1, G, D)
    q, k, v = (dev_bf16(b) for b in bits)
    cu = dev_i32([0, n])
    clean = values(p.prompt_attention(q, k, v, cu))
    v[2, 0, 5] = float(value)
    out = values(p.prompt_attention(q, k, v, cu))
    np.testing.assert_array_equal(np.delete(out, 5, axis=2), np.delete(clean, 5, axis=2))
    np.testing.assert_array_equal(out[:2], clean[:2])
    np.testing.assert_array_equal(out[2:, :, 5], np.full((n - 2, G), value))


def paged(p, c):
    tree = None if c["tree"] is None else torch.from_numpy(c["tree"].view(np.int64).copy()).cuda()
    return values(p.paged_attention(dev_bf16(c["q_bits"]), dev_u8(c["kc"]), dev_u8(c["vc"]), dev_f32(c["ks"]), dev_f32(c["vs"]),
                                    dev_i32(c["tables"]), dev_i32(c["lens"]), c["block"],
                                    cu_q=None if c["uniform"] else dev_i32(c["cu"]), tree_mask=tree, per_tensor=c["per_tensor"]))


@pytest.mark.parametrize("per_tensor", [False, True])
@pytest.mark.parametrize("new,ctx,H,G,D", [([65, 65], [0, 1], 32, 8, 128), ([40, 40], [3, 20], 32, 4, 64), ([65, 65], [0, 30], 16, 8, 256)])
def test_tile_rows_of_few_keys_keep_16_bits(new, ctx, H, G, D, per_tensor):
    p = need_gpu()
    say(f"weights of tiles new={new} ctx={ctx} H={H} G={G} D={D} per_tensor={per_tensor}")
    c = paged_case(71, new, ctx, H, G, D, per_tensor=per_tensor)
    out, spread, mag = reference(c)
    keys = np.concatenate([x + 1 + np.arange(n) for n, x in zip(new, ctx)])
    few = keys <= FEW
    assert few.sum() >= 64
    got = paged(p, c)
    assert within(got[few], out[few], oa.bound(out, spread, mag, D, FEW, weight=2.0 ** -16)[few]) <= 1.0
    assert within(got, out, oa.bound(out, spread, mag, D, int(c["lens"].max()))) <= 1.0


@pytest.mark.parametrize("D,n,B,H", [(128, 48, 16, 8), (64, 20, 16, 8), (256, 65, 8, 8)])
def test_the_same_rows_by_the_stream_and_by_tiles(D, n, B, H):
    """One row of a sequence more or less changes the kernel (n * 4 rows of a KV head: the switch of plan.cpp).  The rows
    common to both calls differ by their weights' bits (2^-8 and 2^-15 of each term) and the outputs' rounding."""
    p = need_gpu()
    G = 4
    say(f"at the switch D={D} n={n}")
    c = paged_case(72, [n] * B, (100 + 37 * np.arange(B)).tolist(), H, G, D)
    out, spread, mag = reference(c)
    L = int(c["lens"].max())
    tiles = paged(p, c)
    assert within(tiles, out, oa.bound(out, spread, mag, D, L)) <= 1.0
    keep = np.arange(n * B) % n != 0                     # without each sequence's first row
    less = dict(c, q_bits=c["q_bits"][keep])
    stream = paged(p, less)
    fine = oa.bound(out, spread, mag, D, L, weight=2.0 ** -15)
    assert within(stream, out[keep], fine[keep]) <= 1.0
    assert within(tiles[keep], stream, (oa.bound(out, spread, mag, D, L) + fine)[keep]) <= 1.0
    rel = lambda x, y: float(np.sqrt(np.sum((x - y) ** 2) / np.sum(y ** 2)))
    say(f"  error of tiles {rel(tiles[keep], out[keep]):.5f}, of the stream {rel(stream, out[keep]):.5f}, apart {rel(tiles[keep], stream):.5f}")
    assert not np.array_equal(tiles[keep], stream)       # (both kernels have run)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("new,ctx,H,G,D", [([65, 65], 63, 32, 8, 128), ([40, 40], 63, 32, 4, 64), ([65, 65], 63, 16, 8, 256), ([65, 65], 20, 32, 8, 128)])
def test_an_infinite_value_scale_in_tiles_of_few_keys(new, ctx, H, G, D, sign):
    """Seen by every row of the first tiles (64 keys: all of a tile), whose weights enter as two bf16: inf - inf is NaN."""
    p = need_gpu()
    c = paged_case(73, new, [ctx] * 2, H, G, D)
    slot = c["tables"][0, 0] * 16 + 3
    c["vc"][slot, 1, 6] = 0x80
    before = paged(p, c)
    c["vs"][slot, 1] = sign * np.inf
    out = paged(p, c)
    hit = np.zeros(out.shape, bool)
    hit[:new[0], G:2 * G] = True
    np.testing.assert_array_equal(out[~hit], before[~hit])
    code = e4m3.decode(c["vc"][slot, 1])
    got = out[:new[0], G:2 * G]
    np.testing.assert_array_equal(got, np.broadcast_to(np.where(code == 0, np.nan, np.copysign(np.inf, code * sign)), got.shape))
