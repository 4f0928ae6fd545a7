"""GPU parity of every variant of the paged attention's kernels, in cells and on one line, against the definition in 64
bits (tests/attention_variants.py; tests/test_attention_plan.py pins which call reaches what)."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa
from tests.attention_cases import within
from tests.attention_variants import CASES, inputs, reference
from tests.gpu_util import dev_bf16, dev_f32, dev_i32, dev_u8, host_bf16_bits, need_gpu, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("at", range(len(CASES)))
def test_variant(at):
    """Few rows within the bound of weights kept to 15 bits, tiles within that of 8; the same results in a workspace
    that other calls have used."""
    p = need_gpu()
    c, w = CASES[at]
    say(f"{c['name']}: B={len(c['new'])} H={c['H']} G={c['G']} D={c['D']} {w}")
    d = inputs(c)
    tree = None if d["tree"] is None else torch.from_numpy(d["tree"].view(np.int64).copy()).cuda()
    args = (dev_bf16(d["q_bits"]), dev_u8(d["kc"]), dev_u8(d["vc"]), dev_f32(d["ks"]), dev_f32(d["vs"]), dev_i32(d["tables"]),
            dev_i32(d["lens"]), d["block"])
    more = dict(cu_q=None if d["uniform"] else dev_i32(d["cu"]), tree_mask=tree, per_tensor=d["per_tensor"])
    out = p.paged_attention(*args, **more)
    ref, spread, mag = reference(d)
    tol = oa.bound(ref, spread, mag, c["D"], int(max(d["lens"].max(), 1)), weight=2.0 ** -8 if w["tiles"] else 2.0 ** -15)
    got = wl.f32_from_bf16_bits(host_bf16_bits(out)).astype(np.float64)
    worst = within(got, ref, tol)
    say(f"  worst {worst:.3f} of the bound")
    assert worst <= 1.0
    ws = torch.zeros(p.paged_attention_workspace_bytes(d["T"], len(c["new"]), c["H"] * c["G"], c["H"], c["D"]), dtype=torch.uint8,
                     device="cuda")
    for _ in range(2):
        again = p.paged_attention(*args, **more, workspace=ws)
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))
        assert int(ws[:16384].sum()) == 0


def call(p, d):
    tree = None if d["tree"] is None else torch.from_numpy(d["tree"].view(np.int64).copy()).cuda()
    out = p.paged_attention(dev_bf16(d["q_bits"]), dev_u8(d["kc"]), dev_u8(d["vc"]), dev_f32(d["ks"]), dev_f32(d["vs"]),
                            dev_i32(d["tables"]), dev_i32(d["lens"]), d["block"], tree_mask=tree, per_tensor=d["per_tensor"])
    return wl.f32_from_bf16_bits(host_bf16_bits(out)).astype(np.float64)


@pytest.mark.parametrize("where", ["K code", "V code", "K scale", "V scale"])
@pytest.mark.parametrize("at", [i for i, (c, w) in enumerate(CASES)
                                if not w["tiles"] and not w["line"] and w["hg"] > 1 and len(set(c["new"])) == 1 and not c["per_tensor"]])
def test_a_nan_stays_with_its_head_and_the_rows_that_see_it(at, where):
    """Several heads in a workgroup: of the first sequence's last KV head, in the last token."""
    p = need_gpu()
    c, w = CASES[at]
    say(f"{c['name']} D={c['D']} {where}")
    d = inputs(c)
    h, G, n, L = c["H"] - 1, c["G"], c["new"][0], int(d["lens"][0])
    slot = d["tables"][0, (L - 1) // d["block"]] * d["block"] + (L - 1) % d["block"]
    before = call(p, d)
    dict(zip(("K code", "V code", "K scale", "V scale"), (d["kc"], d["vc"], d["ks"], d["vs"])))[where][(slot, h, 5)[:2 + ("code" in where)]] = \
        0x7F if "code" in where else np.nan
    out = call(p, d)
    seen = oa.chain_seen(n, L)[:, -1] if d["tree"] is None else oa.tree_seen([int(m) for m in d["tree"][0]], L)[:, -1]
    hit = np.zeros(out.shape, bool)
    hit[np.flatnonzero(seen), h * G:(h + 1) * G] = True
    if where == "V code":
        hit[:, :, np.arange(c["D"]) != 5] = False
    np.testing.assert_array_equal(out[~hit], before[~hit])
    assert hit.any() and np.isnan(out[hit]).all()
