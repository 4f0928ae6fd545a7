"""Attention over packed prompts and over the paged FP8 KV cache, in 64 bits.

Test infrastructure only (see the package docstring): the GPU path never
imports this module.

For one sequence with n rows of queries and L keys, query head g reading KV
head g // (Hq / H):

    out[i] = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - max)

over the keys that row i sees; a row that sees none is zeros.  Keys that a
row does not see are left out of every sum, so their values (NaN included)
do not matter.  A paged cache holds E4M3 codes by slot, with one scale per
(slot, head) or one for all; a token whose page is outside the cache is not
there.

Beside the output each function returns what a bound on a kernel's rounding
needs, per element: spread = sum_j p_ij |v_j| / sum_j p_ij, and per (row, head)
mag = max_j scale sum_d |q_id k_jd| over the keys seen.
"""

from __future__ import annotations

import numpy as np

from . import e4m3


def attention(q, k, v, seen, scale):
    """q [n, Hq, D], k and v [L, H, D] in float64, seen bool [n, L]; returns (out, spread, mag)."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, spread = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    mag = np.zeros((n, Hq))
    for i in range(n):
        js = np.flatnonzero(seen[i])
        if js.size == 0:
            continue
        for g in range(Hq):
            kk, vv = k[js, g // G], v[js, g // G]
            s = scale * (kk @ q[i, g])
            mag[i, g] = scale * np.max(np.abs(kk) @ np.abs(q[i, g]))
            p = np.exp(s - np.max(s))
            out[i, g] = p @ vv / p.sum()
            spread[i, g] = p @ np.abs(vv) / p.sum()
    return out, spread, mag


def chain_seen(n, L):
    """Row i of the last n of L tokens sees token j iff j <= L - n + i."""
    return np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]


def tree_seen(masks, L):
    """Rows of the root and of the N nodes, the last N + 1 of L tokens: the prefix and the root, and node m
    iff bit m of the node's mask is set.  masks: N integers."""
    N = len(masks)
    seen = np.zeros((N + 1, L), bool)
    for i in range(N + 1):
        for j in range(L):
            m = j - (L - N)
            seen[i, j] = m < 0 or (i >= 1 and (int(masks[i - 1]) >> m) & 1 == 1)
    return seen


def gather(codes, scales, table, block_size, L):
    """The first L tokens of a sequence: (values [L, H, D] in float64, which of them there are)."""
    slots_total, H, D = codes.shape
    num_blocks = slots_total // block_size
    x, there = np.zeros((L, H, D)), np.zeros(L, bool)
    for j in range(L):
        page = int(table[j // block_size])
        if 0 <= page < num_blocks:
            slot = page * block_size + j % block_size
            s = scales[slot].astype(np.float64)[:, None] if scales.ndim == 2 else float(scales[0])
            x[j] = e4m3.decode(codes[slot]).astype(np.float64) * s
            there[j] = True
    return x, there


def paged_attention(q, k_cache, v_cache, k_scale, v_scale, tables, kv_lens, block_size, scale, rows, masks=None):
    """q [T, Hq, D] float64; rows: (first, count) of each sequence; masks: integers [B][N] of a tree, or None.
    Rows of no sequence come out as NaN.  Returns (out, spread, mag)."""
    T, Hq, D = q.shape
    out, spread, mag = np.full((T, Hq, D), np.nan), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for b, (first, n) in enumerate(rows):
        L = int(kv_lens[b])
        k, there = gather(k_cache, k_scale, tables[b], block_size, L)
        v, _ = gather(v_cache, v_scale, tables[b], block_size, L)
        seen = (chain_seen(n, L) if masks is None else tree_seen(masks[b], L)) & there[None, :]
        out[first:first + n], spread[first:first + n], mag[first:first + n] = \
            attention(q[first:first + n], k, v, seen, scale)
    return out, spread, mag


def prompt_attention(q, k, v, cu, scale):
    """Packed prompts; rows of no prompt come out as NaN.  Returns (out, spread, mag)."""
    T, Hq, D = q.shape
    out, spread, mag = np.full((T, Hq, D), np.nan), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for a, e in zip(cu[:-1], cu[1:]):
        out[a:e], spread[a:e], mag[a:e] = attention(q[a:e], k[a:e], v[a:e], chain_seen(e - a, e - a), scale)
    return out, spread, mag


def bound(out, spread, mag, D, L, weight=2.0 ** -8):
    """How far a kernel's bf16 output may be from `out`, element by element.

    Half a bf16 step of the result (2^-8 |out|); every p_ij (times its value
    scale) rounded to bf16 once, `weight` = 2^-8 of its term at most: 2^-8 spread
    (as the sum of two, 8 bits and the rest of at most 2^-7 rounded: 2^-15); a score
    is a sum of D exact products in fp32 with the scales and log2(e) as further
    factors and the reference subtracted: (D + 8) 2^-23 of mag (its absolute terms,
    an addition taken to cut its result; the reference is within 8 of the largest:
    8 more), relative in p_ij, once in the sum of p v and once in that of p; the
    sums over L keys in fp32 in any order, with 2^-21 for the exponential:
    (L + 4) 2^-23 each, twice."""
    score = (D + 8) * 2.0 ** -23 * (mag + 8.0)[..., None]
    sums = (L + 4) * 2.0 ** -23
    rel = np.expm1(2 * score) + 2 * sums + weight
    return 2.0 ** -8 * np.abs(out) * (1 + rel) + spread * rel + 2.0 ** -126


def kv_cache_read(codes, scales, slots):
    """bf16-exact inputs of the read: float64 [T, H, D] values dec(code) * scale, zeros outside the cache."""
    out = np.zeros((len(slots),) + codes.shape[1:])
    for t, s in enumerate(slots):
        if 0 <= s < codes.shape[0]:
            sc = scales[s].astype(np.float64)[:, None] if scales.ndim == 2 else float(scales[0])
            out[t] = e4m3.decode(codes[s]).astype(np.float64) * sc
    return out
