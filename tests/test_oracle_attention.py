"""Pins of oracle/attention.py, the inputs' shape in tests/attention_cases.py, and that its check rejects mistakes."""

import numpy as np
import pytest
import torch

from oracle import attention as oa, e4m3, kvcache as ok, tree as ot
from tests.attention_cases import CODE_NAN, paged_case, paged_reference, within
import workloads as wl


def test_equals_torch_in_64_bits():
    rng = np.random.default_rng(0)
    n, L, Hq, H, D = 5, 9, 6, 2, 16
    q, k, v = rng.standard_normal((n, Hq, D)), rng.standard_normal((L, H, D)), rng.standard_normal((L, H, D))
    seen = oa.chain_seen(n, L)
    out, spread, mag = oa.attention(q, k, v, seen, 0.3)
    tq = torch.from_numpy(q).permute(1, 0, 2)
    tk = torch.from_numpy(k).permute(1, 0, 2).repeat_interleave(Hq // H, 0)
    tv = torch.from_numpy(v).permute(1, 0, 2).repeat_interleave(Hq // H, 0)
    w = torch.softmax((0.3 * tq @ tk.transpose(1, 2)).masked_fill(~torch.from_numpy(seen), -torch.inf), -1)
    np.testing.assert_allclose(out, (w @ tv).permute(1, 0, 2).numpy(), rtol=1e-12, atol=1e-13)
    assert (spread >= np.abs(out) - 1e-12).all() and (mag > 0).all()


def test_closed_forms():
    D, L = 8, 7
    v = np.arange(L * D, dtype=np.float64).reshape(L, 1, D)
    q = np.ones((1, 1, D))
    same = np.zeros((L, 1, D))
    seen = np.ones((1, L), bool)
    np.testing.assert_allclose(oa.attention(q, same, v, seen, 1.0)[0][0, 0], v.mean(0)[0])      # equal scores: the mean
    one = same.copy()
    one[3] = 100.0
    np.testing.assert_allclose(oa.attention(q, one, v, seen, 1.0)[0][0, 0], v[3, 0])            # one large: that row
    # two scores a, b: weights 1/(1+e^(b-a))
    two = np.array([[0, 1]] * 1, bool)
    k2 = np.zeros((2, 1, D))
    k2[1] = np.log(3.0) / D
    o = oa.attention(q, k2, v[:2], np.ones((1, 2), bool), 1.0)[0][0, 0]
    np.testing.assert_allclose(o, (v[0, 0] + 3 * v[1, 0]) / 4)
    assert (oa.attention(q, k2, v[:2], np.zeros((1, 2), bool), 1.0)[0] == 0).all()               # none seen


def test_hidden_keys_do_not_matter():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((4, 2, 8)), rng.standard_normal((6, 1, 8)), rng.standard_normal((6, 1, 8))
    seen = oa.chain_seen(4, 6)
    ref = oa.attention(q, k, v, seen, 0.5)[0]
    k[5], v[5] = np.nan, np.inf                        # the last token: only the last row sees it
    got = oa.attention(q, k, v, seen, 0.5)[0]
    np.testing.assert_array_equal(got[:3], ref[:3])
    assert not np.isfinite(got[3]).any()


def test_visibility_rules():
    assert oa.chain_seen(3, 5).sum(1).tolist() == [3, 4, 5]
    assert oa.chain_seen(4, 2).sum(1).tolist() == [0, 0, 1, 2]       # more rows than tokens: the first see none
    assert oa.chain_seen(1, 0).shape == (1, 0)
    # a chain-shaped tree is the chain; siblings do not see each other
    masks, depth = ot.tree_attention_masks(np.array([[-1, 0, 1]], np.int32))
    np.testing.assert_array_equal(oa.tree_seen(masks[0], 9), oa.chain_seen(4, 9))
    masks, _ = ot.tree_attention_masks(np.array([[-1, -1, 0]], np.int32))
    np.testing.assert_array_equal(oa.tree_seen(masks[0], 5)[:, 2:], [[0, 0, 0], [1, 0, 0], [0, 1, 0], [1, 0, 1]])
    assert oa.tree_seen(masks[0], 5)[:, :2].all()


def test_gather_and_read_decode_what_the_write_stored():
    rng = np.random.default_rng(2)
    T, H, D, block = 11, 2, 16, 4
    bits = wl.linear_activations(T, H * D, 3)
    table = np.array([2, 0, 5])
    slots = np.array([table[j // block] * block + j % block for j in range(T)], np.int64)
    codes, scales = ok.kv_cache_write(bits, slots, H, D, np.full((24, H, D), CODE_NAN, np.uint8), np.ones((24, H), np.float32))
    x = wl.f32_from_bf16_bits(bits).reshape(T, H, D).astype(np.float64)
    got, there = oa.gather(codes, scales, table, block, T)
    assert there.all()
    assert (np.abs(got - x) <= 2.0 ** -4 * np.abs(x) + scales[slots][..., None] * 2.0 ** -10).all()   # half an E4M3 step
    np.testing.assert_array_equal(oa.kv_cache_read(codes, scales, slots), got)
    back = oa.kv_cache_read(codes, scales, np.array([3, -1, 24, 8], np.int64))
    assert (back[1:3] == 0).all() and (back[3] == got[0]).all()
    _, there = oa.gather(codes, scales, np.array([2, -1, 6]), block, T)      # pages outside the cache
    assert there.tolist() == [True] * 4 + [False] * 7
    # a static scale
    np.testing.assert_array_equal(oa.kv_cache_read(codes, np.array([0.5], np.float32), slots),
                                  0.5 * e4m3.decode(codes[slots]).astype(np.float64))


def test_paged_equals_prompt_on_the_same_values():
    c = paged_case(4, [5, 3], [0, 0], 2, 2, 16, block=4)
    out, tol = paged_reference(c)
    k = np.concatenate([oa.gather(c["kc"], c["ks"], c["tables"][b], 4, c["lens"][b])[0] for b in range(2)])
    v = np.concatenate([oa.gather(c["vc"], c["vs"], c["tables"][b], 4, c["lens"][b])[0] for b in range(2)])
    np.testing.assert_allclose(oa.prompt_attention(c["q"], k, v, c["cu"], c["scale"])[0], out)
    assert (tol > 0).all()


@pytest.mark.parametrize("mistake", ["scale", "one more key", "one key less", "wrong head", "value scale left out"])
def test_the_check_rejects_mistakes(mistake):
    """Planted in the reference's inputs: each moves some output beyond its bound."""
    c = paged_case(5, [3, 3], [20, 7], 2, 2, 32)
    ref, tol = paged_reference(c)
    assert within(ref, ref, tol) == 0.0
    d = dict(c)
    if mistake == "scale":
        d["scale"] = c["scale"] * 1.05
    elif mistake == "one more key":
        d["lens"], d["tables"] = c["lens"] - 1, c["tables"]
        assert within(paged_reference(d)[0], ref, tol) > 1.0
        return
    elif mistake == "one key less":
        t = c["tables"].copy()
        t[0, 0] = -1
        d["tables"] = t
    elif mistake == "wrong head":
        d["kc"] = c["kc"][:, ::-1].copy()
    else:
        d["vs"] = np.ones_like(c["vs"])
    assert within(paged_reference(d)[0], ref, tol) > 1.0
