"""Infinite, NaN and zero values and scales in the attentions: every path has to give what the formula gives in IEEE
arithmetic, wherever the key lies, and zeros for a row that sees nothing."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa, e4m3, tree as ot
from tests.attention_cases import paged_case, paged_reference, within
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, dev_u8, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu


def values(t):
    return wl.f32_from_bf16_bits(host_bf16_bits(t)).astype(np.float64)


def run(p, c):
    tree = None if c["tree"] is None else torch.from_numpy(c["tree"].view(np.int64).copy()).cuda()
    return values(p.paged_attention(dev_bf16(c["q_bits"]), dev_u8(c["kc"]), dev_u8(c["vc"]), dev_f32(c["ks"]), dev_f32(c["vs"]),
                                    dev_i32(c["tables"]), dev_i32(c["lens"]), c["block"],
                                    cu_q=None if c["uniform"] else dev_i32(c["cu"]), tree_mask=tree,
                                    per_tensor=c["per_tensor"]))


STREAM, MORE, TILES = ([4], 2, 4), ([40], 2, 4), ([65, 65], 32, 8)


# ------------------------------------------------- infinite scales of values

@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("place", ["seen by all", "seen by some"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("shape,D", [(STREAM, 128), (MORE, 128), (STREAM, 64), (STREAM, 256), (STREAM, 24), (TILES, 128),
                                     (([40, 40], 32, 4), 64), (([65, 65], 16, 8), 256)])
def test_an_infinite_value_scale_gives_signed_infinities(shape, D, tree, place, sign):
    """sum p v sv with sv infinite: the code's sign decides, a code of 0 gives NaN; other rows and heads are untouched."""
    p = need_gpu()
    new, H, G = shape
    n = new[0]
    say(f"infinite value scale new={new} H={H} G={G} D={D} tree={tree} {place} {sign}")
    masks = None
    if tree:
        parents = np.array([[-1, -1] + [m % 2 for m in range(n - 3)]] * len(new), np.int32)
        masks = ot.tree_attention_masks(parents)[0]
    c = paged_case(61, new, [140] * len(new), H, G, D, tree=masks)
    L = int(c["lens"][0])
    j = 3 if place == "seen by all" else L - n + 2
    slot = c["tables"][0, j // 16] * 16 + j % 16
    c["vc"][slot, 1, 5] = 0x00                           # +0 and -0 among the key's codes
    c["vc"][slot, 1, 6] = 0x80
    before = run(p, c)
    c["vs"][slot, 1] = sign * np.inf
    out = run(p, c)
    seen = np.zeros(out.shape[0], bool)
    seen[:n] = (oa.tree_seen([int(m) for m in masks[0]], L) if tree else oa.chain_seen(n, L))[:, j]
    assert seen.any() and seen[:n].all() == (place == "seen by all")
    hit = np.zeros(out.shape, bool)
    hit[seen, G:2 * G] = True
    np.testing.assert_array_equal(out[~hit], before[~hit])
    code = e4m3.decode(c["vc"][slot, 1])
    want = np.where(code == 0, np.nan, np.copysign(np.inf, code * sign))
    got = out[seen][:, G:2 * G]
    np.testing.assert_array_equal(got, np.broadcast_to(want, got.shape))


# ------------------------------------------------------- scales of a tensor

@pytest.mark.parametrize("shape,D", [(STREAM, 128), (TILES, 128), (([40, 40], 32, 4), 64), (([65, 65], 16, 8), 256), (STREAM, 24)])
def test_a_key_scale_of_zero_gives_equal_weights(shape, D):
    """All scores are 0; keys that a row does not see still have no weight."""
    p = need_gpu()
    new, H, G = shape
    say(f"key scale 0 new={new} H={H} G={G} D={D}")
    c = paged_case(62, new, [70] * len(new), H, G, D, per_tensor=True)
    c["ks"][:] = 0.0
    ref, tol = paged_reference(c)
    assert within(run(p, c), ref, tol) <= 1.0


@pytest.mark.parametrize("which", ["ks", "vs"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("new,lens,H,G,D", [([4, 4], [2, 40], 2, 4, 128), ([90, 90], [61, 300], 32, 8, 128), ([1100], [1002], 4, 8, 128),
                                            ([1100], [1002], 4, 8, 64), ([1100], [1002], 4, 8, 256), ([5, 5], [2, 9], 2, 2, 24)])
def test_rows_that_see_nothing_are_zeros_whatever_the_scales(which, value, new, lens, H, G, D):
    """More rows than tokens: the first rows see none.  One scale of the tensor that is NaN or infinite reaches the others."""
    p = need_gpu()
    say(f"{which} {value} new={new} lens={lens} H={H} G={G} D={D}")
    c = paged_case(63, new, [max(x - n, 0) for x, n in zip(lens, new)], H, G, D, per_tensor=True)
    c["lens"] = np.array(lens, np.int32)
    c[which][:] = value
    out = run(p, c)
    first = 0
    for n, L in zip(new, lens):
        none = max(n - L, 0)
        assert (out[first:first + none] == 0).all()
        if which == "vs" or value != value:              # (infinite scores of both signs: some rows see -inf alone)
            assert not np.isfinite(out[first + none:first + n]).any()
        first += n


# ---------------------------------------------------- scores of -inf, prompts

def prompt(p, q, k, v, lens):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    d = [dev_bf16(wl.bf16_bits_from_f32(x.astype(np.float32))) for x in (q, k, v)]
    return values(p.prompt_attention(*d, dev_i32(cu)))


@pytest.mark.parametrize("D", [128, 96, 80, 72, 64, 40, 8, 256, 200, 136])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n,j", [(150, 3), (150, 100), (20, 0), (20, 7)])
def test_an_infinite_key_element_decides_by_the_query_sign(D, sign, n, j):
    """A score of -inf has no weight (a row with no other is zeros), one of +inf gives NaN: the same for heads that fill
    their tile's columns and for heads that do not."""
    p = need_gpu()
    H, G = 2, 2
    say(f"infinite key element D={D} sign={sign} n={n} j={j}")
    rng = np.random.default_rng(64 + D)
    r = lambda h: wl.f32_from_bf16_bits(wl.bf16_bits_from_f32(rng.standard_normal((n, h, D)).astype(np.float32))).astype(np.float64)
    q, k, v = r(H * G), r(H), r(H)
    ch = 3 % D
    q[:, :, ch] = np.where(np.abs(q[:, :, ch]) < 0.25, 0.25, q[:, :, ch])         # (no 0 * inf)
    plain = oa.attention(q, k, v, oa.chain_seen(n, n), D ** -0.5)
    hidden = oa.chain_seen(n, n)
    hidden[:, j] = False
    without, spread, mag = oa.attention(q, k, v, hidden, D ** -0.5)
    k[j, 1, ch] = sign * np.inf
    out = prompt(p, q, k, v, [n])
    tol = oa.bound(*plain, D, n)
    assert within(out[:, :G], plain[0][:, :G], tol[:, :G]) <= 1.0                # the other KV head
    assert within(out[:j, G:], plain[0][:j, G:], tol[:j, G:]) <= 1.0             # earlier rows
    up = (np.sign(q[j:, G:, ch]) * sign) > 0
    assert np.isnan(out[j:, G:][up]).all()
    tol = oa.bound(without, spread, mag, D, n)
    got, ref, t = out[j:, G:][~up], without[j:, G:][~up], tol[j:, G:][~up]
    assert within(got, ref, t) <= 1.0
    if j == 0:
        assert (out[0, G:][~up[0]] == 0).all()


@pytest.mark.parametrize("value", [np.inf, np.nan])
@pytest.mark.parametrize("D", [128, 64, 256, 96])
@pytest.mark.parametrize("n", [20, 200])
def test_rows_of_scores_of_minus_infinity_alone_are_zeros_whatever_the_values(D, value, n):
    """The first two tokens' keys give -inf to every query; the first one's value is infinite or NaN."""
    p = need_gpu()
    rng = np.random.default_rng(65)
    q = np.abs(rng.standard_normal((n, 2, D))) + 0.25
    k, v = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
    k[:2, 0, 1] = -np.inf
    v[0, 0, 5] = value
    out = prompt(p, q, k, v, [n])
    assert (out[:2] == 0).all()
    assert np.isfinite(np.delete(out, 5, axis=2)).all()


@pytest.mark.parametrize("shape,D", [(STREAM, 128), (MORE, 128), (STREAM, 64), (STREAM, 256), (STREAM, 24), (TILES, 128),
                                     (([40, 40], 32, 4), 64), (([65, 65], 16, 8), 256)])
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_paged_rows_of_scores_of_minus_infinity_alone_are_zeros(shape, D, value):
    """The first two tokens have an infinite key scale and keys below 0, queries above; the first one's value scale is
    infinite or NaN."""
    p = need_gpu()
    new, H, G = shape
    c = paged_case(66, new, [0] * len(new), H, G, D)
    q = np.abs(c["q"]) + 0.25
    c["q_bits"] = wl.bf16_bits_from_f32(q.astype(np.float32))
    for j in range(2):
        slot = c["tables"][0, 0] * 16 + j
        c["kc"][slot, 1] = 0xB8                          # -1
        c["ks"][slot, 1] = np.inf
    c["vs"][c["tables"][0, 0] * 16, 1] = value
    out = run(p, c)
    assert (out[:2, G:2 * G] == 0).all()
    assert np.isfinite(out[:, :G]).all() and np.isfinite(out[new[0]:]).all()
