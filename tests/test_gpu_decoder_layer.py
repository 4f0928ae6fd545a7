"""A drafter's decoder layer from the framework's calls alone, as a serving program runs it: norm into codes, QKV linear,
rotation into the paged cache, attention over it, output linear, norm with the residual, gated FFN -- prompts first, then a
step of a few new rows, eagerly and as a captured graph.

Each stage is checked against its oracle on what the stage before it left on the device, so that a stage's tolerance
is its own; the captured step is compared with the eager one bit for bit."""

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import e4m3, fp4, norm as on, quantize as oq, rope
from tests.gpu_util import dev_bf16, dev_i32, host, host_bf16_bits, need_gpu

pytestmark = pytest.mark.gpu

C, HQ, H, D, I, PAGE, EPS = 256, 4, 2, 64, 512, 16, 1e-5
QKV = (HQ + 2 * H) * D


class Layer:
    """Weights (the QKV linear in E4M3, the others in 4 bits), the cache, and one pass over new rows."""

    def __init__(self, p, blocks, seed=0):
        self.p = p
        rng = np.random.default_rng(seed)
        w = lambda n, k, s: dev_bf16(wl.linear_weights(n, k, seed + s, 0.08))
        self.qkv = p.quantize(w(QKV, C, 1))
        self.o, self.gate_up, self.down = (p.quantize_fp4(w(n, k, s)) for n, k, s in ((C, HQ * D, 2), (2 * I, C, 3), (C, I, 4)))
        self.n1, self.n2 = (dev_bf16(wl.bf16_bits_from_f32((1 + 0.2 * rng.standard_normal(C)).astype(np.float32))) for _ in range(2))
        self.freq = torch.from_numpy(10000.0 ** (-np.arange(D // 2) * 2.0 / D)).cuda()
        self.kc, self.vc = (torch.zeros((blocks * PAGE, H, D), dtype=torch.uint8, device="cuda") for _ in range(2))
        self.ks, self.vs = (torch.zeros((blocks * PAGE, H), device="cuda") for _ in range(2))

    def run(self, x, residual, positions, slots, attend, keys=None):
        """attend(q, k, v) -> attention's output; returns every intermediate."""
        p, r = self.p, {}
        r["codes"], r["scales"], r["sum"] = p.rms_norm_quantize(x, self.n1, EPS, residual=residual)
        r["qkv"] = p.gemm(r["codes"], r["scales"], *self.qkv)
        q, k, v = (r["qkv"][:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, HQ), (HQ, HQ + H), (HQ + H, HQ + 2 * H)))
        r["q"] = p.rope_kv_cache_write(q, k, v, positions, self.freq, slots, self.kc, self.vc, self.ks, self.vs, k_out=keys)
        r["att"] = attend(r["q"], keys, v)
        r["att_codes"], r["att_scales"] = p.quantize(r["att"].flatten(1))
        r["o"] = p.gemm_fp4(r["att_codes"], r["att_scales"], *self.o)
        r["codes2"], r["scales2"], r["sum2"] = p.rms_norm_quantize(r["o"], self.n2, EPS, residual=r["sum"])
        r["gate_up"] = p.gemm_fp4(r["codes2"], r["scales2"], *self.gate_up)
        r["h_codes"], r["h_scales"] = p.quantize(r["gate_up"], silu_mul=True)
        r["y"] = p.gemm_fp4(r["h_codes"], r["h_scales"], *self.down)
        return r


def values(t):
    return oq.bf16_to_f32(host_bf16_bits(t)).astype(np.float64)


def check_norm(x, residual, weight, codes, scales, total):
    """As in the norm's own tests: y within 64 * 2^-24, then half an E4M3 step (2^-4, and 2^-10 of the subnormal step)."""
    h = on.residual_sum(host_bf16_bits(x), host_bf16_bits(residual))
    np.testing.assert_array_equal(host_bf16_bits(total), wl.bf16_bits_from_f32(h.astype(np.float32)))
    y = on.rms_norm(h, host_bf16_bits(weight), EPS)
    s = host(scales).astype(np.float64)[:, None]
    err = np.abs(e4m3.decode(host(codes)) * s - y)
    assert (err <= np.abs(y) * (2.0 ** -4 + 2.0 ** -17) + s * 2.0 ** -10).all()


def check_linear4(codes, scales, w, y):
    a, sa, wd = host(codes), host(scales), fp4.decode(host(w[0]), host(w[1]))
    ref = fp4.gemm(a, sa, wd)
    assert (np.abs(values(y) - ref) <= fp4.error_bound(a, sa, wd) * (1 + 2.0 ** -8) + np.abs(ref) * 2.0 ** -8 + 1e-30).all()


def check_stages(layer, x, residual, positions, slots, r):
    check_norm(x, residual, layer.n1, r["codes"], r["scales"], r["sum"])
    q = values(r["qkv"][:, :HQ * D]).reshape(-1, HQ, D)
    k = values(r["qkv"][:, HQ * D:(HQ + H) * D]).reshape(-1, H, D)
    freq, pos = host(layer.freq), host(positions)
    for a, got, half in ((q, values(r["q"]), 2.0 ** -8), (k, None, 2.0 ** -4)):
        ref = rope.rotate(a, pos, freq, False)
        near = 8 * 2.0 ** -24 * rope.pair_sums(a, D, False)
        s = 0.0
        if got is None:
            at = host(slots)
            s = host(layer.ks)[at].astype(np.float64)[..., None]
            got = e4m3.decode(host(layer.kc)[at]) * s
        assert (np.abs(got - ref) <= np.abs(ref) * half + 2 * near + s * 2.0 ** -10).all()
    check_linear4(r["att_codes"], r["att_scales"], layer.o, r["o"])
    check_norm(r["o"], r["sum"], layer.n2, r["codes2"], r["scales2"], r["sum2"])
    check_linear4(r["codes2"], r["scales2"], layer.gate_up, r["gate_up"])
    check_linear4(r["h_codes"], r["h_scales"], layer.down, r["y"])


def rows(T, seed):
    return dev_bf16(wl.linear_activations(T, C, seed, 0.02, 8.0))


def test_prompts_then_a_step_eager_and_captured():
    p = need_gpu()
    lens, new = [37, 1, 80], 3
    B, width = len(lens), 8
    layer = Layer(p, B * width)
    order = np.random.default_rng(5).permutation(B * width).astype(np.int32)
    tables = order.reshape(B, width)
    slot = lambda b, j: int(tables[b, j // PAGE]) * PAGE + j % PAGE

    # ---- the prompts: rotated keys in bf16 for their attention, codes into the cache
    T = sum(lens)
    pos = dev_i32(np.concatenate([np.arange(n) for n in lens]))
    slots = torch.tensor([slot(b, j) for b, n in enumerate(lens) for j in range(n)], device="cuda")
    cu = dev_i32(np.concatenate(([0], np.cumsum(lens))))
    x, res = rows(T, 1), rows(T, 2)
    keys = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
    r = layer.run(x, res, pos, slots, lambda q, k, v: p.prompt_attention(q, k, v, cu), keys)
    check_stages(layer, x, res, pos, slots, r)

    # ---- a step: `new` rows of each sequence over the cache
    T = B * new
    x, res = rows(T, 3), rows(T, 4)
    pos = dev_i32(np.concatenate([n + np.arange(new) for n in lens]))
    slots = torch.tensor([slot(b, n + j) for b, n in enumerate(lens) for j in range(new)], device="cuda")
    tab, kv_lens = dev_i32(tables), dev_i32([n + new for n in lens])
    ws = torch.zeros(p.paged_attention_workspace_bytes(T, B, HQ, H, D), dtype=torch.uint8, device="cuda")
    attend = lambda q, k, v: p.paged_attention(q, layer.kc, layer.vc, layer.ks, layer.vs, tab, kv_lens, PAGE, workspace=ws)
    eager = layer.run(x, res, pos, slots, attend)
    check_stages(layer, x, res, pos, slots, eager)
    # the attention read what was appended: its output against the definition over the cache
    kd = e4m3.decode(host(layer.kc)) * host(layer.ks).astype(np.float64)[..., None]
    vd = e4m3.decode(host(layer.vc)) * host(layer.vs).astype(np.float64)[..., None]
    q = values(eager["q"])
    for b, n in enumerate(lens):
        at = np.array([slot(b, j) for j in range(n + new)])
        for i in range(new):
            t, L = b * new + i, n + i + 1
            for g in range(HQ):
                s = (kd[at[:L], g // (HQ // H)] @ q[t, g]) / np.sqrt(D)
                w = np.exp(s - s.max())
                want = w @ vd[at[:L], g // (HQ // H)] / w.sum()
                # bf16 of the output, and the weights' 2^-15 of the terms' magnitudes with their fp32 sums
                near = (w @ np.abs(vd[at[:L], g // (HQ // H)]) / w.sum()) * 2.0 ** -13
                assert (np.abs(values(eager["att"])[t, g] - want) <= np.abs(want) * 2.0 ** -8 + near).all()

    # ---- the same step captured; other inputs copied in, replayed between eager work
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(x, res, pos, slots, attend)                  # (warm on this stream)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer.run(x, res, pos, slots, attend)
    for seed in (11, 12, 13, 14):
        x.copy_(rows(T, seed))
        res.copy_(rows(T, seed + 50))
        layer.kc.view(-1, H, D)[slots] = 0                     # what the step appends is its own work
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in captured.items()}
        cache = layer.kc.clone(), layer.ks.clone()
        layer.kc.view(-1, H, D)[slots] = 0
        again = layer.run(x, res, pos, slots, attend)
        for n in got:
            assert torch.equal(got[n].view(torch.uint8), again[n].view(torch.uint8)), n
        assert torch.equal(cache[0], layer.kc) and torch.equal(cache[1], layer.ks)
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Calls on two streams share nothing: each gives what it gives alone."""
    p = need_gpu()
    w = dev_bf16(wl.linear_weights(1000, 4096, 3))
    wq = p.quantize_fp4(w)
    weight = torch.ones(4096, dtype=torch.bfloat16, device="cuda")
    xs = [dev_bf16(wl.linear_activations(m, 4096, m, 0.01, 20.0)) for m in (5, 64)]

    def step(x):
        q, s, _ = p.rms_norm_quantize(x, weight)
        return q, p.gemm_fp4(q, s, *wq)

    want = [step(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(5):
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(step(x))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
