"""Calls that reach every variant of the paged attention's kernels and both ways of sharing out their work, and a replay
of the sharing on the host that tells which ones a call reaches."""

import numpy as np

from oracle import attention as oa, e4m3, tree as ot
from tests.attention_cases import paged_case


def case(name, seed, new, ctx, H, G, D, width=0, per_tensor=False, nodes=0, block=16):
    """new, ctx: a number or (least, most) for `count` sequences, or lists.  width: tokens that a table row can name."""
    return dict(name=name, seed=seed, new=new, ctx=ctx, H=H, G=G, D=D, width=width, per_tensor=per_tensor, nodes=nodes, block=block)


def some(seed, count, least, most, more=()):
    return np.random.default_rng(seed).integers(least, most + 1, count).tolist() + list(more)


# dp: D padded; nq: 16s of rows; hg: KV heads a workgroup; tiles: matrix tiles of many rows; line: equal ranges of one line
# (otherwise cells); split: a unit of several steps lies in several ranges or cells; rounds: joined in two rounds; idle: a
# workgroup's last head is past the last KV head.
def wants(dp, nq, hg, tiles=False, line=False, split=True, rounds=False, idle=False):
    return dict(dp=dp, nq=nq, hg=hg, tiles=tiles, line=line, split=split, rounds=rounds, idle=idle)


WIDE = 40000
CASES = []


def add(c, **w):
    CASES.append((c, wants(**w)))


# ---- few rows, few sequences: cells; the wide tables keep several heads in a workgroup
for _dp, _D, _H in ((64, 64, 5), (128, 128, 6), (256, 256, 3)):
    add(case("four heads", _dp, [4, 4, 4], [700, 33, 0], _H, 4, _D, WIDE), dp=_dp, nq=1, hg=4, idle=True)
    add(case("two heads", _dp + 1, [1, 1, 1], [900, 64, 31], 2, 8, _D, WIDE), dp=_dp, nq=1, hg=2)
    add(case("two heads of 32 rows", _dp + 2, [5, 5, 5], [1000, 3, 250], 3, 4, _D, WIDE), dp=_dp, nq=2, hg=2, idle=True)
    add(case("one head", _dp + 3, [2, 2], [1500, 40], 1, 5, _D), dp=_dp, nq=1, hg=1)
    add(case("one head of 32 rows", _dp + 4, [6, 6], [1500, 40], 1, 4, _D), dp=_dp, nq=2, hg=1)
add(case("four heads, one scale", 20, [3, 3, 3, 3], [500, 1, 90, 1], 7, 5, 112, WIDE, per_tensor=True), dp=128, nq=1, hg=4, idle=True)
add(case("two heads of 32 rows, one scale", 21, [8, 8, 8], [500, 1, 90], 4, 4, 48, WIDE, per_tensor=True), dp=64, nq=2, hg=2)
add(case("four heads, a tree", 22, [4, 4, 4], [400, 60, 5], 6, 4, 128, WIDE, nodes=3), dp=128, nq=1, hg=4, idle=True)
add(case("two heads, a tree", 23, [8, 8], [30, 400], 2, 4, 128, WIDE, nodes=7), dp=128, nq=2, hg=2)
add(case("four heads, pages of 24", 24, [1, 1, 1], [777, 24, 47], 4, 8, 192, WIDE - WIDE % 24, block=24), dp=256, nq=1, hg=4)

# ---- few rows, many sequences: one line, with one long context among short ones
for _dp, _D, _H in ((64, 64, 6), (128, 128, 5), (256, 192, 3)):
    add(case("four heads, a line", _dp + 5, [2] * 70, some(1, 69, 0, 500, [9000]), _H, 4, _D, WIDE),
        dp=_dp, nq=1, hg=4, line=True, rounds=True, idle=True)
    add(case("two heads, a line", _dp + 6, [1] * 90, some(2, 89, 0, 1200, [15000]), 2, 8, _D, WIDE),
        dp=_dp, nq=1, hg=2, line=True, rounds=True)
    add(case("two heads of 32 rows, a line", _dp + 7, [5] * 70, some(3, 69, 0, 900, [15000]), 3, 4, _D, WIDE),
        dp=_dp, nq=2, hg=2, line=True, rounds=True, idle=True)
    add(case("one head, a line", _dp + 8, [1] * 280, some(4, 279, 0, 300, [30000]), 1, 3, _D), dp=_dp, nq=1, hg=1, line=True, rounds=True)
    add(case("one head of 32 rows, a line", _dp + 9, [5] * 280, some(5, 279, 0, 300, [30000]), 1, 4, _D),
        dp=_dp, nq=2, hg=1, line=True, rounds=True)
add(case("ragged rows, none among them, a line", 30, some(6, 70, 0, 6), some(7, 69, 0, 600, [5000]), 8, 4, 128, WIDE),
    dp=128, nq=1, hg=4, line=True)
add(case("one scale, a line", 31, some(8, 70, 1, 8), some(9, 70, 0, 900), 4, 4, 128, WIDE, per_tensor=True),
    dp=128, nq=2, hg=2, line=True)
add(case("a tree, a line", 32, [4] * 64, some(10, 64, 0, 700), 8, 4, 128, WIDE, nodes=3), dp=128, nq=1, hg=4, line=True)
add(case("a tree of 32 rows, a line", 33, [8] * 64, some(11, 64, 0, 900), 4, 4, 128, WIDE, nodes=7), dp=128, nq=2, hg=2, line=True)
add(case("rows of several 32s, a line", 34, [26] * 20, some(12, 20, 100, 900), 8, 4, 128), dp=128, nq=2, hg=1, line=True)

# ---- many rows: tiles
for _dp, _D, _n, _H, _ctx in ((64, 64, 30, 32, [60, 1100, 500, 0]), (128, 128, 50, 32, [60, 1100, 500, 0]), (256, 224, 70, 16, [60, 1100, 0])):
    for _pt in (False, True):
        add(case("tiles, cells", _dp + 10 + _pt, [_n] * len(_ctx), _ctx, _H, 4, _D, per_tensor=_pt), dp=_dp, nq=1, hg=1, tiles=True)
        add(case("tiles, a line", _dp + 12 + _pt, [_n] * 9, some(13, 8, 900, 1600, [6000]), 16, 4, _D, per_tensor=_pt),
            dp=_dp, nq=1, hg=1, tiles=True, line=True)
add(case("tiles of ragged rows, a line", 40, some(14, 10, 0, 120), some(15, 10, 0, 2500), 16, 4, 128), dp=128, nq=1, hg=1, tiles=True, line=True)
add(case("tiles of a tree, a line", 41, [50] * 8, some(16, 8, 800, 1500), 16, 4, 96, nodes=49), dp=128, nq=1, hg=1, tiles=True, line=True)


def inputs(c):
    """The call's inputs (attention_cases.paged_case), with tables that name pages of others past a sequence's end."""
    B = len(c["new"])
    masks = None
    rng = np.random.default_rng(c["seed"])
    if c["nodes"]:
        parents = np.array([[int(rng.integers(-1, n)) for n in range(c["nodes"])] for _ in range(B)], np.int32)
        masks = ot.tree_attention_masks(parents)[0]
    d = paged_case(c["seed"], c["new"], c["ctx"], c["H"], c["G"], c["D"], c["block"], c["per_tensor"], tree=masks)
    P = max(d["tables"].shape[1], c["width"] // c["block"])
    t = rng.integers(0, d["kc"].shape[0] // c["block"], (B, P)).astype(np.int32)
    t[:, :d["tables"].shape[1]] = np.where(d["tables"] < 0, t[:, :d["tables"].shape[1]], d["tables"])
    d["tables"] = t
    return d


_DECODED = e4m3.decode_table()


def reference(c):
    """attention_cases.paged_reference's results for tables without holes, by matrix products: (out, spread, mag)."""
    T, Hq, D = c["q"].shape
    G = c["G"]
    out, spread, mag = np.full((T, Hq, D), np.nan), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for b, (first, end) in enumerate(zip(c["cu"][:-1], c["cu"][1:])):
        n, L = int(end - first), int(c["lens"][b])
        if n == 0:
            continue
        j = np.arange(L)
        slots = c["tables"][b, j // c["block"]].astype(np.int64) * c["block"] + j % c["block"]
        seen = oa.chain_seen(n, L) if c["tree"] is None else oa.tree_seen([int(m) for m in c["tree"][b]], L)
        sees = np.repeat(seen, G, 0)                         # rows (token, head of the group)
        for h in range(c["H"]):
            k, v = (_DECODED[x[slots, h]] * (s[slots, h].astype(np.float64)[:, None] if s.ndim == 2 else float(s[0]))
                    for x, s in ((c["kc"], c["ks"]), (c["vc"], c["vs"])))
            q = c["q"][first:end, h * G:(h + 1) * G].reshape(n * G, D)
            s = np.where(sees, c["scale"] * (q @ k.T), -np.inf)
            top = s.max(1, keepdims=True)
            none = np.isneginf(top[:, 0])
            w = np.exp(s - np.where(np.isneginf(top), 0.0, top))
            w /= np.where(none, 1.0, w.sum(1))[:, None]
            out[first:end, h * G:(h + 1) * G] = (w @ v).reshape(n, G, D)
            spread[first:end, h * G:(h + 1) * G] = (w @ np.abs(v)).reshape(n, G, D)
            m = np.where(sees, c["scale"] * (np.abs(q) @ np.abs(k).T), 0.0).max(1)
            mag[first:end, h * G:(h + 1) * G] = m.reshape(n, G)
    return out, spread, mag


# ------------------------------------------------------------------ the replay

def replay(plan, c):
    """What the call's kernel does: plan(T, B, Hq, H, D, max_len) -> (dp, nq, hg, tiles, groups, bytes).  The kernels cut
    units (sequence, rows of a KV head's group, heads) of key steps into cells, or all of them on one line into equal
    ranges."""
    H, G, B, T = c["H"], c["G"], len(c["new"]), sum(c["new"])
    lens = [x + n for x, n in zip(c["ctx"], c["new"])]
    max_len = max(-(-max(lens) // c["block"]), 1, c["width"] // c["block"]) * c["block"]
    dp, nq, hg, tiles, groups, _ = plan(T, B, H * G, H, c["D"], max_len)
    if tiles:
        waves = 8 if dp == 128 else 4
        rows, step, cell, extra, heads = 32 * waves, 64, 8, 3, 1
    else:
        kw = 4 // hg
        rows, step, cell, extra, heads = 16 * nq, 32 * kw, 3, 5 if kw == 1 else 3, hg
    nhg = -(-H // heads)
    bound = (T * G // rows + B) * nhg
    grid = min(min(bound, groups) * max(((max_len + step - 1) // step + 1) // cell, 1), groups)
    units = []
    for n, L in zip(c["new"], lens):
        units += [max(-(-int(L) // step), 1)] * (-(-n * G // rows) * nhg)
    cells = [max((s + 1) // cell, 1) for s in units]
    line = sum(cells) > grid
    split = rounds = False
    if not line:
        split, rounds = max(cells) > 1, max(cells) > 24
    else:
        total = sum(s + extra for s in units)
        place = 0
        for s in units:
            at = place + extra
            parts = ((at + s) * grid - 1) // total - ((at + 1) * grid - 1) // total + 1
            split |= parts > 1
            rounds |= parts > 24
            place += s + extra
    return dict(dp=dp, nq=nq, hg=hg, tiles=bool(tiles), line=line, split=split, rounds=rounds, idle=H % heads != 0)
