"""GPU parity of the cache read and of the attentions against oracle/attention.py, within its derived bounds: sizes
around every tile edge, ragged and empty sequences, masks, pages that end inside a tile, strides, values that a row
does not see, long contexts, far offsets, graphs and streams."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa, e4m3, tree as ot
from tests.attention_cases import CODE_NAN, bf16_values, cache, paged_case, paged_reference, within
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, dev_u8, host, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu


def values(t):
    return wl.f32_from_bf16_bits(host_bf16_bits(t)).astype(np.float64)


def on_device(c):
    d = dict(q=dev_bf16(c["q_bits"]), kc=dev_u8(c["kc"]), vc=dev_u8(c["vc"]), ks=dev_f32(c["ks"]), vs=dev_f32(c["vs"]),
             tables=dev_i32(c["tables"]), lens=dev_i32(c["lens"]), cu=None if c["uniform"] else dev_i32(c["cu"]))
    d["tree"] = None if c["tree"] is None else torch.from_numpy(c["tree"].view(np.int64).copy()).cuda()
    return d


def call(p, c, d, **more):
    return p.paged_attention(d["q"], d["kc"], d["vc"], d["ks"], d["vs"], d["tables"], d["lens"], c["block"], cu_q=d["cu"],
                             tree_mask=d["tree"], per_tensor=c["per_tensor"], **more)


def check_paged(c, what):
    p = need_gpu()
    say(what)
    ref, tol = paged_reference(c)
    out = call(p, c, on_device(c))
    worst = within(values(out), ref, tol)
    say(f"  worst {worst:.3f} of the bound")
    assert worst <= 1.0
    return out


# ------------------------------------------------------------------ the read

@pytest.mark.parametrize("T,H,D,per_tensor", [(1, 1, 8, False), (5, 8, 128, False), (37, 3, 80, True), (13, 2, 24, False),
                                              (9, 1, 512, True), (300, 4, 64, False), (11, 5, 512, False), (2100, 1, 40, False),
                                              (7, 300, 8, False)])
def test_kv_cache_read_is_exact(T, H, D, per_tensor):
    p = need_gpu()
    rng = np.random.default_rng(T)
    S = T + 7
    kc, ks = cache(rng, S, H, D, per_tensor)
    vc, vs = cache(rng, S, H, D, per_tensor, spread=30.0)
    kc.reshape(-1)[: min(256, kc.size)] = np.arange(min(256, kc.size), dtype=np.uint8)          # every code, NaN too
    slots = rng.integers(0, S, T)                      # some twice
    if T > 2:
        slots[0], slots[1], slots[2] = -1, S, 2 ** 40
    want = []
    for c, s in ((kc, ks), (vc, vs)):
        x = np.zeros((T, H, D), np.float32)
        for t, sl in enumerate(slots):
            if 0 <= sl < S:
                x[t] = e4m3.decode(c[sl]).astype(np.float32) * (s[sl][:, None] if s.ndim == 2 else s[0])
        want.append(x)
    args = (dev_u8(kc), dev_u8(vc), torch.from_numpy(slots.astype(np.int64)).cuda(), dev_f32(ks), dev_f32(vs))
    k, v = p.kv_cache_read(*args, per_tensor=per_tensor)
    # into column blocks of a wider matrix, whose other columns stay
    wide = torch.full((T, 2 * H * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    k2, v2 = wide[:, :H * D].view(T, H, D), wide[:, H * D:2 * H * D].view(T, H, D)
    r = p.kv_cache_read(*args, per_tensor=per_tensor, k=k2, v=v2)
    assert r[0] is k2 and r[1] is v2
    for got, got2, x in ((k, k2, want[0]), (v, v2, want[1])):
        nan = np.isnan(x)
        g = values(got)
        assert np.isnan(g[nan]).all()
        np.testing.assert_array_equal(host_bf16_bits(got)[~nan], wl.bf16_bits_from_f32(np.where(nan, 0, x))[~nan])
        assert torch.equal(got.contiguous().view(torch.int16), got2.contiguous().view(torch.int16))
    assert (wide[:, 2 * H * D:] == 7.0).all()


def test_kv_cache_read_of_nothing():
    p = need_gpu()
    z = dict(device="cuda")
    c, s = torch.zeros((4, 2, 16), dtype=torch.uint8, **z), torch.ones((4, 2), **z)
    k, v = p.kv_cache_read(c, c, torch.zeros(0, dtype=torch.int64, **z), s, s)
    assert k.shape == v.shape == (0, 2, 16)
    k, v = p.kv_cache_read(c[:0], c[:0], torch.zeros(3, dtype=torch.int64, **z), s[:0], s[:0])
    assert (k == 0).all() and (v == 0).all()


# ------------------------------------------------------- over the paged cache

@pytest.mark.parametrize("new,ctx,H,G,D,block,per_tensor", [
    ([1], [0], 1, 1, 64, 16, False),                 # one token alone
    ([1], [63], 1, 1, 8, 16, False),                 # the smallest head
    ([1], [31], 2, 4, 128, 16, True),
    ([1, 1, 1], [32, 33, 700], 8, 4, 128, 16, False),     # single tokens
    ([5] * 4, [120, 1, 0, 251], 8, 4, 128, 16, False),    # verify rows
    ([8] * 3, [61, 64, 300], 1, 4, 128, 24, True),
    ([3, 0, 1, 7], [5, 9, 0, 130], 2, 3, 96, 16, False),  # ragged rows, none, odd groups
    ([5] * 2, [77, 20], 5, 1, 80, 1, False),              # five heads, pages of one token
    ([4] * 2, [100, 3], 3, 2, 40, 7, False),              # pages that no tile divides, 8-byte rows
    ([2] * 2, [90, 257], 2, 8, 256, 32, False),
    ([1] * 2, [50, 400], 1, 32, 192, 16, True),           # many heads on one
    ([1], [200], 1, 71, 64, 16, False),
    ([17, 33], [40, 300], 2, 4, 128, 16, False),          # chunks
    ([64], [0], 1, 4, 64, 16, False),                     # a prompt through the cache
    ([129, 1], [130, 700], 1, 4, 128, 16, False),
    ([140], [60], 2, 1, 72, 48, True),
    ([70], [33], 1, 2, 256, 16, False),
])
def test_paged_chain(new, ctx, H, G, D, block, per_tensor):
    check_paged(paged_case(len(new) + D, new, ctx, H, G, D, block, per_tensor),
                f"paged new={new} ctx={ctx} H={H} G={G} D={D} block={block} per_tensor={per_tensor}")


@pytest.mark.parametrize("new,ctx,H,G,D,block,per_tensor", [
    ([65, 65], [0, 1], 32, 8, 128, 16, False),       # many rows: tiles of 256, nothing before them
    ([300, 1, 37, 0, 90], [100, 600, 63, 40, 1], 16, 8, 128, 24, False),
    ([70, 66], [640, 5], 32, 8, 128, 16, True),
    ([80, 90], [129, 64], 32, 8, 112, 16, False),    # a head that ends inside its 128 columns
    ([40] * 2, [63, 200], 32, 4, 64, 16, False),     # tiles of 128
    ([129, 1, 70], [1000, 3, 64], 16, 5, 48, 8, True),
    ([65, 70, 65], [30, 300, 2], 16, 8, 256, 16, False),
    ([65, 70, 65], [30, 300, 2], 16, 8, 192, 100, True),
])
def test_paged_tiles_of_many_rows(new, ctx, H, G, D, block, per_tensor):
    check_paged(paged_case(len(new) + D, new, ctx, H, G, D, block, per_tensor),
                f"paged tiles new={new} ctx={ctx} H={H} G={G} D={D} block={block} per_tensor={per_tensor}")


@pytest.mark.parametrize("per_tensor", [False, True])
def test_paged_tiles_of_which_a_few_are_long(per_tensor):
    """One row group of 30000 tokens among short ones: its tile is cut into more parts than one workgroup joins."""
    check_paged(paged_case(25, [1, 130, 130], [30000, 20, 7], 4, 32, 128, per_tensor=per_tensor), "one long tile")


def test_paged_no_tokens_fewer_tokens_than_rows_and_lengths_outside():
    p = need_gpu()
    c = paged_case(3, [3, 3, 3, 3, 3], [10, 4, 6, 13, 0], 2, 2, 64)
    c["lens"] = np.array([0, 2, -5, 10 ** 6, 3], np.int32)      # none; fewer than rows; below 0; beyond the table
    ref, tol = paged_reference(c)
    out = values(call(p, c, on_device(c)))
    assert (out[0:3] == 0).all() and (out[3] == 0).all() and (out[6:9] == 0).all()
    assert within(out, ref, tol) <= 1.0


def test_paged_tables_that_point_outside():
    p = need_gpu()
    c = paged_case(4, [4, 4, 4], [60, 90, 40], 2, 4, 128)
    c["tables"][0, 1] = -1
    c["tables"][1, 3] = 10 ** 9
    c["tables"][2, :] = -2 ** 31                        # no page at all
    ref, tol = paged_reference(c)
    out = values(call(p, c, on_device(c)))
    assert (out[8:] == 0).all() and within(out, ref, tol) <= 1.0
    c["tables"] = c["tables"][:, :0]                     # no table
    out = values(call(p, c, on_device(c)))
    assert (out == 0).all()


@pytest.mark.parametrize("per_tensor", [False, True])
@pytest.mark.parametrize("new,H,G,D", [([4, 4], 2, 4, 128), ([65, 65], 32, 8, 128), ([40, 40], 32, 4, 64), ([3, 3], 2, 2, 24)])
def test_paged_pages_outside_and_no_cache(new, H, G, D, per_tensor):
    """The same for few rows, for tiles and for the smallest heads; then a cache without a page, whose scales are NaN."""
    p = need_gpu()
    c = paged_case(29, new, [120, 40], H, G, D, per_tensor=per_tensor)
    c["tables"][0, 1] = 10 ** 9
    c["tables"][0, 4] = -1
    c["tables"][1, :] = -5
    ref, tol = paged_reference(c)
    d = on_device(c)
    out = values(call(p, c, d))
    assert (out[new[0]:] == 0).all() and within(out, ref, tol) <= 1.0
    c["ks"][:] = np.nan
    c["vs"][:] = np.nan
    c["kc"], c["vc"] = c["kc"][:0], c["vc"][:0]
    if not per_tensor:
        c["ks"], c["vs"] = c["ks"][:0], c["vs"][:0]
    assert (values(call(p, c, on_device(c))) == 0).all()


@pytest.mark.parametrize("N,ctx,H,G,D,per_tensor", [(1, [0, 40], 1, 1, 64, False), (4, [1, 33], 2, 4, 128, False),
                                                    (25, [700, 64], 2, 4, 128, False), (63, [5], 1, 4, 128, True),
                                                    (64, [0, 100], 1, 2, 96, False), (33, [31], 3, 1, 256, False),
                                                    (64, [3, 90], 32, 8, 128, False), (64, [3, 90], 32, 4, 64, True)])
def test_paged_tree(N, ctx, H, G, D, per_tensor):
    p = need_gpu()
    rng = np.random.default_rng(N)
    B = len(ctx)
    parents = np.array([[int(rng.integers(-1, n)) for n in range(N)] for _ in range(B)], np.int32)
    if N > 3:
        parents[0, 3] = 7                                # unreachable: its mask is empty, it sees the prefix and the root
    mask, _ = p.tree_attention_mask(dev_i32(parents))
    masks = host(mask).view(np.uint64)
    np.testing.assert_array_equal(masks, ot.tree_attention_masks(parents)[0])
    c = paged_case(N, [N + 1] * B, ctx, H, G, D, per_tensor=per_tensor, tree=masks)
    check_paged(c, f"tree N={N} ctx={ctx} H={H} G={G} D={D}")


def test_a_chain_shaped_tree_is_the_chain():
    p = need_gpu()
    c = paged_case(7, [6] * 3, [50, 3, 200], 2, 4, 128)
    d = on_device(c)
    chain = call(p, c, d)
    d["tree"] = p.tree_attention_mask(dev_i32(np.tile(np.arange(-1, 4, dtype=np.int32), (3, 1))))[0]
    assert torch.equal(call(p, c, d), chain)


def a_nan_reaches(where, new, tree, H, G, D):
    """Of the first sequence's second KV head."""
    p = need_gpu()
    n = new[0]
    masks = None
    if tree:
        parents = np.array([[-1, -1] + [m % 2 for m in range(n - 3)]] * len(new), np.int32)
        masks = ot.tree_attention_masks(parents)[0]
    c = paged_case(11, new, [70] * len(new), H, G, D, tree=masks)
    L = int(c["lens"][0])
    j = L - n + 2                                        # the second node, or the third token of the chain
    slot = c["tables"][0, j // 16] * 16 + j % 16
    before = values(call(p, c, on_device(c)))
    if where == "K code":
        c["kc"][slot, 1, 5] = CODE_NAN
    elif where == "V code":
        c["vc"][slot, 1, 5] = 0xFF
    elif where == "K scale":
        c["ks"][slot, 1] = np.nan
    else:
        c["vs"][slot, 1] = np.inf
    out = values(call(p, c, on_device(c)))
    seen = np.zeros(out.shape[0], bool)
    seen[:n] = (oa.tree_seen([int(m) for m in masks[0]], L) if tree else oa.chain_seen(n, L))[:, j]
    assert seen.any() and not seen[:n].all()
    hit = np.zeros(out.shape, bool)
    hit[seen, G:2 * G] = True                            # the second KV head's query heads
    np.testing.assert_array_equal(out[~hit], before[~hit])
    if where == "V code":                                # its channel alone
        assert np.isnan(out[seen][:, G:2 * G, 5]).all()
        others = np.delete(np.arange(D), 5)
        assert np.isfinite(out[:, :, others]).all()
    else:
        assert not np.isfinite(out[seen][:, G:2 * G]).any()


@pytest.mark.parametrize("where", ["K code", "V code", "K scale", "V scale"])
@pytest.mark.parametrize("new", [[4], [40]])
@pytest.mark.parametrize("tree", [False, True])
def test_a_nan_reaches_the_rows_that_see_it_and_no_others(where, new, tree):
    a_nan_reaches(where, new, tree, 2, 4, 128)


@pytest.mark.parametrize("where", ["K code", "V code", "K scale", "V scale"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("new,H,G,D", [([65, 65], 32, 8, 128), ([40, 40], 32, 4, 64), ([65, 65], 16, 8, 256)])
def test_a_nan_and_tiles_of_rows(where, tree, new, H, G, D):
    a_nan_reaches(where, new, tree, H, G, D)


def test_paged_strides_and_rows_of_no_sequence():
    p = need_gpu()
    c = paged_case(9, [3, 1, 5], [40, 100, 7], 2, 4, 64, gaps=2)
    ref, tol = paged_reference(c)
    d = on_device(c)
    T, Hq, D = c["q"].shape
    wide = torch.zeros((T, Hq * D + 72), dtype=torch.bfloat16, device="cuda")
    wide[:, 16:16 + Hq * D] = d["q"].view(T, -1)
    d["q"] = wide[:, 16:16 + Hq * D].view(T, Hq, D)
    t = torch.full((3, d["tables"].shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    t[:, 2:2 + d["tables"].shape[1]] = d["tables"]
    d["tables"] = t[:, 2:2 + d["tables"].shape[1]]
    back = torch.full((T, Hq * D + 40), 5.0, dtype=torch.bfloat16, device="cuda")
    out = back[:, 8:8 + Hq * D].view(T, Hq, D)
    assert call(p, c, d, out=out) is out
    assert within(values(out), ref, tol) <= 1.0
    assert (out[:2] == 5).all() and (out[-2:] == 5).all()
    assert (back[:, :8] == 5).all() and (back[:, 8 + Hq * D:] == 5).all()


@pytest.mark.parametrize("new,ctx,H,G,D", [([1, 1, 1], [0, 1, 700], 4, 4, 128), ([5, 5], [2, 300], 2, 4, 64),
                                            ([26], [90], 2, 4, 128), ([2, 3], [40, 0], 1, 2, 256)])
def test_weights_of_few_rows_are_kept_to_15_bits(new, ctx, H, G, D):
    p = need_gpu()
    c = paged_case(17, new, ctx, H, G, D)
    say(f"weights new={new} ctx={ctx} H={H} G={G} D={D}")
    rows = [(int(a), int(e - a)) for a, e in zip(c["cu"][:-1], c["cu"][1:])]
    out, spread, mag = oa.paged_attention(c["q"], c["kc"], c["vc"], c["ks"], c["vs"], c["tables"], c["lens"], c["block"],
                                          c["scale"], rows, None)
    tol = oa.bound(out, spread, mag, D, int(c["lens"].max()), weight=2.0 ** -15)
    assert within(values(call(p, c, on_device(c))), out, tol) <= 1.0


@pytest.mark.parametrize("scale", [1e-3, 40.0])
def test_paged_flat_and_steep_scores(scale):
    """Nearly equal weights, and scores of thousands, where one key takes nearly all."""
    check_paged(paged_case(12, [5, 5], [300, 90], 2, 4, 128, q_scale=scale), f"paged scores of {scale}")


def test_paged_scale_argument():
    p = need_gpu()
    c = paged_case(13, [2, 2], [50, 10], 1, 2, 64)
    c["scale"] = 0.37
    ref, tol = paged_reference(c)
    assert within(values(call(p, c, on_device(c), scale=0.37)), ref, tol) <= 1.0


def test_many_short_sequences():
    rng = np.random.default_rng(5)
    B = 700
    new = rng.integers(0, 4, B).tolist()
    ctx = rng.integers(0, 40, B).tolist()
    check_paged(paged_case(14, new, ctx, 1, 2, 64), "700 short sequences")


@pytest.mark.parametrize("new,ctx,D", [([1, 5, 2], [20000, 30, 5000], 128), ([1], [30011], 64), ([40], [9000], 128)])
def test_long_contexts(new, ctx, D):
    check_paged(paged_case(15, new, ctx, 1, 4, D), f"long contexts {ctx}")


def test_offsets_past_32_bits():
    """Pages at both ends of caches of more than 4 GiB, and scales past 2^30 entries' bytes."""
    p = need_gpu()
    H, D, block = 8, 128, 16
    small = paged_case(16, [3, 3], [60, 29], H, 2, D, block)
    slots = small["kc"].shape[0]
    total = (2 ** 32 // (H * D) // block + 64) * block
    d = on_device(small)
    big = {}
    for name in ("kc", "vc"):
        big[name] = torch.full((total, H, D), CODE_NAN, dtype=torch.uint8, device="cuda")
        big[name][total - slots:] = d[name]
    for name in ("ks", "vs"):
        big[name] = torch.full((total, H), float("nan"), device="cuda")
        big[name][total - slots:] = d[name]
    want = call(p, small, d)
    d.update(big)
    d["tables"] = d["tables"] + (total - slots) // block
    assert torch.equal(call(p, small, d), want)
    ref, tol = paged_reference(small)
    assert within(values(want), ref, tol) <= 1.0
    at = torch.arange(total - 5, total, device="cuda")
    k, v = p.kv_cache_read(big["kc"], big["vc"], at, big["ks"], big["vs"])
    k2, v2 = p.kv_cache_read(big["kc"][-5:].contiguous(), big["vc"][-5:].contiguous(), at - (total - 5), big["ks"][-5:].contiguous(),
                             big["vs"][-5:].contiguous())
    assert torch.equal(k.view(torch.int16), k2.view(torch.int16)) and torch.equal(v.view(torch.int16), v2.view(torch.int16))


def test_one_workspace_for_calls_of_different_shapes_and_the_same_results_twice():
    p = need_gpu()
    cases = [paged_case(20, [1], [5000], 1, 4, 128), paged_case(21, [5] * 6, [900, 30, 0, 2000, 77, 400], 2, 4, 128),
             paged_case(22, [100, 1], [300, 1500], 2, 2, 64), paged_case(23, [1] * 3, [10, 20, 30], 4, 1, 256),
             paged_case(24, [26] * 2, [600, 1200], 1, 4, 128), paged_case(26, [65] * 2, [600, 1200], 32, 8, 128),
             paged_case(27, [40] * 4, [900, 1100, 0, 5], 8, 4, 64), paged_case(28, [3] * 2, [90, 20], 2, 2, 24)]
    need = [p.paged_attention_workspace_bytes(c["T"], len(c["lens"]), c["H"] * c["G"], c["H"], c["D"]) for c in cases]
    ws = torch.zeros(max(need), dtype=torch.uint8, device="cuda")
    ws[16384:] = 0xFF                                    # only the tickets have to be zero
    devs = [on_device(c) for c in cases]
    first = [call(p, c, d).clone() for c, d in zip(cases, devs)]
    for _ in range(2):
        for c, d, want in zip(cases, devs, first):
            assert torch.equal(call(p, c, d, workspace=ws), want)
            assert int(ws[:16384].sum()) == 0
    for c, d, want in zip(cases, devs, first):
        ref, tol = paged_reference(c)
        assert within(values(want), ref, tol) <= 1.0


# -------------------------------------------------------------- over prompts

def prompt_case(seed, lens, H, G, D, gaps=0, q_scale=1.0):
    rng = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32) + gaps
    T = int(cu[-1]) + gaps
    Hq = H * G
    qkv = wl.bf16_bits_from_f32(rng.standard_normal((T, (Hq + 2 * H) * D)).astype(np.float32))
    if q_scale != 1.0:
        f = wl.f32_from_bf16_bits(qkv)
        f[:, :Hq * D] *= q_scale
        qkv = wl.bf16_bits_from_f32(f)
    return dict(qkv=qkv, cu=cu, T=T, H=H, G=G, D=D, scale=D ** -0.5)


def split(c, x):
    T, H, Hq, D = c["T"], c["H"], c["H"] * c["G"], c["D"]
    return (x[:, :Hq * D].reshape(T, Hq, D) if isinstance(x, np.ndarray) else x[:, :Hq * D].view(T, Hq, D),
            x[:, Hq * D:(Hq + H) * D].reshape(T, H, D) if isinstance(x, np.ndarray) else x[:, Hq * D:(Hq + H) * D].view(T, H, D),
            x[:, (Hq + H) * D:].reshape(T, H, D) if isinstance(x, np.ndarray) else x[:, (Hq + H) * D:].view(T, H, D))


def prompt_reference(c):
    q, k, v = split(c, wl.f32_from_bf16_bits(c["qkv"]).astype(np.float64))
    out, spread, mag = oa.prompt_attention(q, k, v, c["cu"], c["scale"])
    return out, oa.bound(out, spread, mag, c["D"], int(max(np.diff(c["cu"]).max(), 1)))


@pytest.mark.parametrize("lens,H,G,D", [
    ([1], 1, 1, 64), ([1, 1, 1], 2, 4, 128), ([2, 31, 32, 33], 1, 4, 128), ([63, 64, 65], 2, 2, 64), ([0, 5, 0, 0, 17, 0], 1, 3, 128),
    ([127, 129], 1, 1, 128), ([257], 1, 4, 128), ([300, 3], 1, 8, 64), ([150], 1, 2, 256), ([90, 40], 3, 1, 80), ([33, 70], 2, 5, 8),
    ([100], 1, 4, 200), ([64, 64], 1, 4, 32), ([520], 1, 1, 128), ([48], 1, 71, 64), ([100], 1, 2, 104),
])
def test_prompt(lens, H, G, D):
    p = need_gpu()
    c = prompt_case(sum(lens) + D, lens, H, G, D)
    say(f"prompt lens={lens} H={H} G={G} D={D}")
    ref, tol = prompt_reference(c)
    q, k, v = split(c, dev_bf16(c["qkv"]))
    out = p.prompt_attention(q, k, v, dev_i32(c["cu"]))
    worst = within(values(out), ref, tol)
    say(f"  worst {worst:.3f} of the bound")
    assert worst <= 1.0
    assert torch.equal(out, p.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), dev_i32(c["cu"])))


def reference_on_device(q, k, v, scale, first=0):
    """One prompt's attention in 64 bits on the device, head by head: (out, spread, mag) as the oracle's."""
    n, Hq, D = q.shape
    outs = [torch.empty((n, Hq, D), dtype=torch.float64, device="cuda") for _ in range(2)]
    mag = torch.empty((n, Hq), dtype=torch.float64, device="cuda")
    hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    for h in range(Hq):
        kk, vv = (x[:, h // (Hq // x.shape[1])].double().contiguous() for x in (k, v))
        kt = kk.t().contiguous()
        qq = q[:, h].double().contiguous()
        w = torch.softmax((torch.mm(qq, kt) * scale).masked_fill(hidden, -torch.inf), -1)
        outs[0][:, h], outs[1][:, h] = torch.mm(w, vv), torch.mm(w, vv.abs())
        mag[:, h] = (torch.mm(qq.abs(), kt.abs()) * scale).masked_fill(hidden, 0).amax(-1)
    return outs[0].cpu().numpy(), outs[1].cpu().numpy(), mag.cpu().numpy()


@pytest.mark.parametrize("n,H,G,D", [(2047, 2, 4, 128), (4100, 1, 2, 64), (1537, 1, 4, 128)])
def test_long_prompt(n, H, G, D):
    p = need_gpu()
    say(f"prompt of {n}, H={H} G={G} D={D}")
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn((n, h, D), device="cuda", generator=g).to(torch.bfloat16) for h in (H * G, H, H))
    out = p.prompt_attention(q, k, v, dev_i32([0, n]))
    o, spread, mag = reference_on_device(q, k, v, D ** -0.5)
    assert within(values(out), o, oa.bound(o, spread, mag, D, n)) <= 1.0


@pytest.mark.parametrize("scale", [1e-3, 40.0])
def test_prompt_flat_and_steep_scores(scale):
    p = need_gpu()
    c = prompt_case(31, [200, 65], 1, 4, 128, q_scale=scale)
    ref, tol = prompt_reference(c)
    q, k, v = split(c, dev_bf16(c["qkv"]))
    assert within(values(p.prompt_attention(q, k, v, dev_i32(c["cu"]))), ref, tol) <= 1.0


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", [1, 2])
@pytest.mark.parametrize("n", [60, 300])
def test_a_later_row_does_not_reach_earlier_ones(which, value, n):
    p = need_gpu()
    c = prompt_case(33, [n, 20], 2, 2, 128)
    parts = [x.contiguous() for x in split(c, dev_bf16(c["qkv"]))]
    cu = dev_i32(c["cu"])
    clean = values(p.prompt_attention(*parts, cu))
    j = n - 13
    parts[which][j, 1, 3] = value
    out = values(p.prompt_attention(*parts, cu))
    hit = np.zeros(out.shape, bool)
    hit[j:n, 2:] = True
    np.testing.assert_array_equal(out[~hit], clean[~hit])
    if which == 2:
        assert not np.isfinite(out[j:n, 2:, 3]).any()
        others = np.delete(np.arange(128), 3)
        np.testing.assert_array_equal(out[:, :, others], clean[:, :, others])
    elif value != value:
        assert np.isnan(out[j:n, 2:]).all()


def test_prompt_rows_of_no_prompt_and_strides():
    p = need_gpu()
    c = prompt_case(34, [20, 37], 2, 2, 64, gaps=3)
    ref, tol = prompt_reference(c)
    x = dev_bf16(c["qkv"])
    x[:3] = float("nan")
    x[-3:] = float("nan")
    q, k, v = split(c, x)
    T, Hq, D = q.shape
    back = torch.full((T, Hq * D + 40), 5.0, dtype=torch.bfloat16, device="cuda")
    out = back[:, 8:8 + Hq * D].view(T, Hq, D)
    assert p.prompt_attention(q, k, v, dev_i32(c["cu"]), out=out) is out
    assert within(values(out), ref, tol) <= 1.0
    assert (out[:3] == 5).all() and (out[-3:] == 5).all() and (back[:, :8] == 5).all() and (back[:, 8 + Hq * D:] == 5).all()
    assert p.prompt_attention(q[:0], k[:0], v[:0], dev_i32([0, 0])).shape == (0, Hq, D)


def test_prompts_many_and_empty():
    p = need_gpu()
    rng = np.random.default_rng(35)
    lens = rng.integers(0, 12, 600).tolist()
    c = prompt_case(35, lens, 1, 2, 64)
    ref, tol = prompt_reference(c)
    q, k, v = split(c, dev_bf16(c["qkv"]))
    assert within(values(p.prompt_attention(q, k, v, dev_i32(c["cu"]))), ref, tol) <= 1.0


# ------------------------------------------------- refusals, graphs, streams

def test_refused_arguments():
    p = need_gpu()
    c = paged_case(40, [2, 2], [20, 9], 2, 2, 64)
    d = on_device(c)
    z = dict(device="cuda")
    bad = [
        (lambda: call(p, c, dict(d, q=d["q"].float())), "q must have dtype"),
        (lambda: call(p, c, dict(d, q=d["q"][:, :, ::2])), "unit stride"),
        (lambda: call(p, c, dict(d, q=d["q"][:, :, :32])), "packed side by side"),
        (lambda: call(p, c, dict(d, q=d["q"][:, :, :32].contiguous())), "same head size"),
        (lambda: call(p, c, dict(d, kc=d["kc"][:-1])), "contiguous \\[num_slots, H, D\\]"),
        (lambda: call(p, c, dict(d, ks=d["ks"][:, :1])), "per-row scales"),
        (lambda: call(p, dict(c, per_tensor=True), d), "per-tensor scales"),
        (lambda: call(p, c, dict(d, lens=d["lens"][:1])), "kv_lens"),
        (lambda: call(p, c, dict(d, lens=d["lens"].long())), "kv_lens must have dtype"),
        (lambda: call(p, c, dict(d, tables=d["tables"].t().contiguous().t())), "block_tables"),
        (lambda: call(p, c, dict(d, cu=dev_i32([0, 2]))), "cu_q"),
        (lambda: call(p, dict(c, block=0), d), "block_size"),
        (lambda: call(p, c, dict(d, tree=torch.zeros((2, 4), dtype=torch.int64, **z))), "B \\* \\(N \\+ 1\\)"),
        (lambda: call(p, c, dict(d, tree=torch.zeros((2, 1), dtype=torch.int64, **z), cu=dev_i32([0, 2, 4]))), "cu_q must be None"),
        (lambda: call(p, c, d, out=torch.empty((4, 4, 32), dtype=torch.bfloat16, **z)), "out must be"),
        (lambda: call(p, c, d, scale="steep"), "could not convert"),
        (lambda: call(p, c, d, workspace=torch.zeros(1 << 24, dtype=torch.uint8)), "workspace must be"),
        (lambda: call(p, c, d, workspace=torch.zeros((1 << 12, 1 << 12), dtype=torch.uint8, **z).t()), "workspace must be contiguous"),
        (lambda: p.prompt_attention(d["q"], d["q"][:, :2], d["q"][:3, :2], dev_i32([0, 4])), "k and v must be"),
        (lambda: p.prompt_attention(d["q"], d["q"], d["q"], dev_i32([[0, 4]])), "cu_seqlens"),
        (lambda: p.kv_cache_read(d["kc"], d["vc"], dev_i32([0]), d["ks"], d["vs"]), "slot_mapping must have dtype"),
        (lambda: p.kv_cache_read(d["kc"], d["vc"], torch.zeros(2, dtype=torch.int64, **z), d["ks"], d["vs"],
                                 k=torch.empty((3, 2, 64), dtype=torch.bfloat16, **z)), "k and v must be"),
    ]
    for i, (f, message) in enumerate(bad):
        with pytest.raises(ValueError, match=message):
            f()
    for f, status in ((lambda: call(p, c, d, scale=0.0), 8), (lambda: call(p, c, d, scale=float("nan")), 8),
                      (lambda: p.prompt_attention(d["q"][:, :3], d["q"][:, :2], d["q"][:, :2], dev_i32([0, 4])), 2),
                      (lambda: call(p, c, dict(d, q=d["q"][:3])), 2),
                      (lambda: p.prompt_attention(*(torch.zeros((2, 1, 264), dtype=torch.bfloat16, **z),) * 3, dev_i32([0, 2])), 3)):
        with pytest.raises(p.SpecError) as e:
            f()
        assert e.value.status == status
    torch.cuda.synchronize()


def test_replays_equal_eager_calls():
    """Prompt, cache write, verify over the cache (split contexts), tree and read in one graph, replayed on new
    inputs with the program's own work between."""
    p = need_gpu()
    H, G, D, block = 2, 4, 128, 16
    Hq = H * G
    n, B, k1, N = 70, 3, 5, 6
    pages = 40
    z = dict(device="cuda")
    x = torch.empty((n, (Hq + 2 * H) * D), dtype=torch.bfloat16, **z)
    q, k, v = x[:, :Hq * D].view(n, Hq, D), x[:, Hq * D:(Hq + H) * D].view(n, H, D), x[:, (Hq + H) * D:].view(n, H, D)
    qv = torch.empty((B * k1, Hq, D), dtype=torch.bfloat16, **z)
    qt = torch.empty((B * (N + 1), Hq, D), dtype=torch.bfloat16, **z)
    slots = torch.empty(n, dtype=torch.int64, **z)
    kc, vc = (torch.empty((3 * pages * block, H, D), dtype=torch.uint8, **z) for _ in range(2))
    ks, vs = (torch.empty((3 * pages * block, H), **z) for _ in range(2))
    cu = dev_i32([0, 30, 30, n])
    tables = torch.empty((B, pages), dtype=torch.int32, **z)
    lens = torch.empty(B, dtype=torch.int32, **z)
    parents = torch.empty((B, N), dtype=torch.int32, **z)
    ws = torch.zeros(max(p.paged_attention_workspace_bytes(t, B, Hq, H, D) for t in (B * k1, B * (N + 1))), dtype=torch.uint8, **z)
    outs = [torch.empty((n, Hq, D), dtype=torch.bfloat16, **z), torch.empty_like(qv), torch.empty_like(qt),
            torch.empty((n, H, D), dtype=torch.bfloat16, **z), torch.empty((n, H, D), dtype=torch.bfloat16, **z)]

    def load(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, qv, qt):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g).to(torch.bfloat16))
        for c in (kc, vc):
            c.copy_(torch.randint(0, 0x7F, c.shape, device="cuda", generator=g, dtype=torch.int32).to(torch.uint8))
        for s in (ks, vs):
            s.copy_(torch.rand(s.shape, device="cuda", generator=g) * 0.01)
        perm = torch.randperm(3 * pages, device="cuda", generator=g)
        tables.copy_(perm.view(B, pages).to(torch.int32))
        lens.copy_(torch.randint(20, pages * block, (B,), device="cuda", generator=g).to(torch.int32))
        slots.copy_(torch.randperm(3 * pages * block, device="cuda", generator=g)[:n])
        rng = np.random.default_rng(seed)
        parents.copy_(dev_i32([[int(rng.integers(-1, m)) if m else -1 for m in range(N)] for _ in range(B)]))

    def step():
        p.prompt_attention(q, k, v, cu, out=outs[0])
        p.kv_cache_write(k, v, slots, kc, vc, ks, vs)
        p.paged_attention(qv, kc, vc, ks, vs, tables, lens, block, out=outs[1], workspace=ws)
        mask, _ = p.tree_attention_mask(parents)
        p.paged_attention(qt, kc, vc, ks, vs, tables, lens, block, tree_mask=mask, out=outs[2], workspace=ws)
        p.kv_cache_read(kc, vc, slots, ks, vs, k=outs[3], v=outs[4])

    load(1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3, 3, 4):
        load(seed)
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        load(seed)
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs, want)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), (seed, i)
        p.prompt_attention(q, k, v, cu)                  # the program's own work


def test_a_side_stream_is_followed():
    p = need_gpu()
    c = paged_case(41, [5] * 4, [400, 30, 900, 8], 2, 4, 128)
    d = on_device(c)
    want = call(p, c, d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.empty_like(want)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):       # a launch on any other stream would not be captured
            call(p, c, d, out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_nothing_is_allocated_with_output_and_workspace_given():
    p = need_gpu()
    c = paged_case(42, [5] * 4, [400, 30, 900, 8], 2, 4, 128)
    d = on_device(c)
    out = call(p, c, d)
    ws = torch.zeros(p.paged_attention_workspace_bytes(c["T"], 4, 8, 2, 128), dtype=torch.uint8, device="cuda")
    made = lambda: torch.cuda.memory_stats()["allocation.all.allocated"]
    before = made()
    call(p, c, d, out=out, workspace=ws)
    assert made() == before


# ------------------------------------------------------------------ together

def test_prompts_then_verify_steps_then_the_read():
    """As a serving program runs them: two prompts' attention, their keys and values into the cache, a drafted chain
    and then a drafted tree over it, each written first; the read gives back what the attentions saw."""
    p = need_gpu()
    H, G, D, block = 2, 4, 128, 16
    Hq, lens, k1, N = H * G, [50, 21], 5, 7
    rng = np.random.default_rng(50)
    n, B = sum(lens), len(lens)
    z = dict(device="cuda")
    pages = 8
    S = B * pages * block
    tables = rng.permutation(B * pages).reshape(B, pages).astype(np.int32)
    kc, vc = (torch.full((S, H, D), CODE_NAN, dtype=torch.uint8, **z) for _ in range(2))
    ks, vs = (torch.full((S, H), float("nan"), **z) for _ in range(2))
    have = [0] * B

    def place(count):
        out = []
        for b, c in enumerate(count):
            j = have[b] + np.arange(c)
            out.append(tables[b, j // block].astype(np.int64) * block + j % block)
            have[b] += c
        return np.concatenate(out)

    def new_rows(T):
        x = wl.bf16_bits_from_f32(rng.standard_normal((T, (Hq + 2 * H) * D)).astype(np.float32))
        d = dev_bf16(x)
        return x, d[:, :Hq * D].view(T, Hq, D), d[:, Hq * D:(Hq + H) * D].view(T, H, D), d[:, (Hq + H) * D:].view(T, H, D)

    def reference(x, count, masks=None):
        c = dict(q=wl.f32_from_bf16_bits(x[:, :Hq * D]).astype(np.float64).reshape(-1, Hq, D), kc=host(kc), vc=host(vc), ks=host(ks),
                 vs=host(vs), tables=tables, lens=np.array(have, np.int32), block=block, scale=D ** -0.5, D=D, tree=masks,
                 cu=np.concatenate([[0], np.cumsum(count)]))
        return paged_reference(c)

    # the prompts
    x, q, k, v = new_rows(n)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    out = p.prompt_attention(q, k, v, dev_i32(cu))
    f = wl.f32_from_bf16_bits(x).astype(np.float64)
    o, spread, mag = oa.prompt_attention(f[:, :Hq * D].reshape(n, Hq, D), f[:, Hq * D:(Hq + H) * D].reshape(n, H, D),
                                         f[:, (Hq + H) * D:].reshape(n, H, D), cu, D ** -0.5)
    assert within(values(out), o, oa.bound(o, spread, mag, D, max(lens))) <= 1.0
    slots = place(lens)
    p.kv_cache_write(k, v, torch.from_numpy(slots).cuda(), kc, vc, ks, vs)
    back, _ = p.kv_cache_read(kc, vc, torch.from_numpy(slots).cuda(), ks, vs)
    step = np.abs(f[:, Hq * D:(Hq + H) * D].reshape(n, H, D))
    # half an E4M3 step (2^-4, or half the smallest one of the row's scale), then half a bf16 step of the result
    half = np.maximum(step * 2.0 ** -4, host(ks)[slots][..., None].astype(np.float64) * 2.0 ** -10)
    assert (np.abs(values(back) - f[:, Hq * D:(Hq + H) * D].reshape(n, H, D)) <= half * (1 + 2.0 ** -7) + (step + half) * 2.0 ** -8).all()
    # the prompt's last rows again, now over the cache, as a chunk
    # a drafted chain
    x, q, k, v = new_rows(B * k1)
    p.kv_cache_write(k, v, torch.from_numpy(place([k1] * B)).cuda(), kc, vc, ks, vs)
    out = p.paged_attention(q, kc, vc, ks, vs, dev_i32(tables), dev_i32(have), block)
    ref, tol = reference(x, [k1] * B)
    assert within(values(out), ref, tol) <= 1.0
    # two drafts accepted, then a tree
    for b in range(B):
        have[b] -= k1 - 3
    parents = np.array([[-1, -1, 0, 0, 1, 2, 5], [-1, 0, 0, 0, 3, 3, 1]], np.int32)
    x, q, k, v = new_rows(B * (N + 1))
    p.kv_cache_write(k, v, torch.from_numpy(place([N + 1] * B)).cuda(), kc, vc, ks, vs)
    mask, _ = p.tree_attention_mask(dev_i32(parents))
    out = p.paged_attention(q, kc, vc, ks, vs, dev_i32(tables), dev_i32(have), block, tree_mask=mask)
    ref, tol = reference(x, [N + 1] * B, host(mask).view(np.uint64))
    assert within(values(out), ref, tol) <= 1.0
