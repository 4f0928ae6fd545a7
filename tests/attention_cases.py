"""Seeded inputs of the attention tests: packed rows, a paged cache, its tables and lengths (numpy)."""

import numpy as np

import workloads as wl
from oracle import attention as oa, e4m3

CODE_NAN = 0x7F


def bf16_values(rng, *shape, scale=1.0):
    """(bf16 bits, their values in float64)."""
    bits = wl.bf16_bits_from_f32((rng.standard_normal(shape) * scale).astype(np.float32))
    return bits, wl.f32_from_bf16_bits(bits).astype(np.float64)


def cache(rng, slots, H, D, per_tensor, spread=1.0):
    """E4M3 codes (no NaN) and scales of values around `spread`."""
    x = rng.standard_normal((slots, H, D)) * spread
    if per_tensor:
        scale = np.array([np.abs(x).max() / 448.0 * 0.9], np.float32)
        codes = e4m3.encode((x / scale[0]).astype(np.float32))
    else:
        scale = (np.abs(x).max(-1) / 448.0).astype(np.float32)
        codes = e4m3.encode((x / scale[..., None]).astype(np.float32))
    return codes.reshape(slots, H, D), scale


def paged_case(seed, new, ctx, H, G, D, block=16, per_tensor=False, tree=None, ragged=None, q_scale=1.0, gaps=0):
    """One call's inputs.  new: rows of each sequence; ctx: tokens before them; gaps: rows of no sequence at both
    ends of q.  Every slot that no token names holds NaN codes and a NaN scale."""
    rng = np.random.default_rng(seed)
    B = len(new)
    L = np.array([c + n for c, n in zip(ctx, new)], np.int32)
    pages = [-(-int(x) // block) for x in L]
    num_blocks = sum(pages) + 3
    P = max(max(pages), 1)
    order = rng.permutation(num_blocks)
    tables = np.full((B, P), -1, np.int32)
    at = 0
    for b, w in enumerate(pages):
        tables[b, :w] = order[at:at + w]
        at += w
    kc, ks = cache(rng, num_blocks * block, H, D, per_tensor)
    vc, vs = cache(rng, num_blocks * block, H, D, per_tensor)
    named = np.zeros(num_blocks * block, bool)
    for b in range(B):
        j = np.arange(L[b])
        named[tables[b, j // block] * block + j % block] = True
    for c in (kc, vc):
        c[~named] = CODE_NAN
    if not per_tensor:
        ks[~named] = np.nan
        vs[~named] = np.nan
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + gaps
    T = int(cu[-1]) + gaps
    qb, q = bf16_values(rng, T, H * G, D, scale=q_scale)
    return dict(q_bits=qb, q=q, kc=kc, vc=vc, ks=ks, vs=vs, tables=tables, lens=L, block=block, cu=cu, T=T, H=H, G=G, D=D,
                per_tensor=per_tensor, tree=tree, uniform=len(set(new)) == 1 and gaps == 0 if ragged is None else not ragged,
                scale=D ** -0.5)


def paged_reference(c):
    rows = [(int(a), int(e - a)) for a, e in zip(c["cu"][:-1], c["cu"][1:])]
    top = c["tables"].shape[1] * c["block"]
    lens = np.clip(c["lens"], 0, top)
    masks = None if c["tree"] is None else [[int(m) for m in row] for row in c["tree"]]
    out, spread, mag = oa.paged_attention(c["q"], c["kc"], c["vc"], c["ks"], c["vs"], c["tables"], lens, c["block"],
                                          c["scale"], rows, masks)
    return out, oa.bound(out, spread, mag, c["D"], int(max(lens.max(), 1)))


def within(got, ref, tol):
    """Every element that has a reference inside its bound; the worst ratio."""
    there = ~np.isnan(ref)
    assert np.isfinite(got[there]).all(), "not finite where it has to be"
    off = np.abs(got - ref)[there] / tol[there]
    return float(off.max()) if off.size else 0.0
