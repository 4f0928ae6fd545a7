"""Performance cases of what stands between the linears of a decoder layer and of the 4-bit linears of a drafter: the
residual's addition with the root-mean-square norm and its E4M3 output, the position rotation of queries and keys on
their way into the paged FP8 cache, and products of few rows with weights held in 4 bits.

A serving program calls them once per layer and step: the norm hands E4M3 codes and scales to the QKV and gate|up
linears, the QKV output is rotated and appended to the cache that the attention reads, and a drafter that runs over a
few rows keeps its weights as OCP MXFP4 (E2M1 codes, one E8M0 scale for 32 of them), because it is bound by reading
them.  Sizes are those of workloads/configs.py (hidden 4096, FFN 14336, QKV 6144, vocabulary 128256, 32 query and 8 KV
heads of 128, steps of 320 rows), their tensor-parallel shards, and ragged sizes around them.

listed() are the fixed cases, draw(rng) one more of the same ranges; prepare/run/work/exact describe one case each.
`own` selects the framework's kernels; without it run() computes the same in elementary torch operations.
"""

from __future__ import annotations

import math

import torch

own = False

HIDDEN, INTER, QKV, VOCAB = 4096, 14336, 6144, 128256
KV_HEADS, GROUP, HEAD_DIM, PAGE = 8, 4, 128, 16
EPS = 1e-5
GROUP4 = 32                                  # 4-bit codes that share a scale


# ---------------------------------------------------------------- the cases

def _norm(name, T, C, residual=True, static=False, normed=False):
    """static: a given scale for all rows; normed: the bf16 values beside the codes."""
    return dict(name=name, kind="norm", T=T, C=C, residual=residual, static=static, normed=normed)


def _rope(name, T, far, H=KV_HEADS, G=GROUP, D=HEAD_DIM, R=HEAD_DIM, interleaved=False, per_tensor=False, keys=False):
    """T tokens at positions below `far`; R of D channels rotated; keys: the rotated keys also as bf16."""
    return dict(name=name, kind="rope", T=T, far=far, H=H, G=G, D=D, R=R, interleaved=interleaved, per_tensor=per_tensor,
                keys=keys)


def _linear4(name, M, N, K, static=False):
    return dict(name=name, kind="linear4", M=M, N=N, K=K, static=static)


def listed():
    return [
        # one token of one sequence: bound by latency
        _norm("norm_t1", 1, HIDDEN),
        # the rows of a serving verify step (B = 64, k = 4), into the QKV or gate|up linear
        _norm("norm_t320", 320, HIDDEN),
        # a prompt chunk of a wider model under a calibrated scale, first layer (nothing to add), values kept too
        _norm("norm_t1005_static", 1005, 7176, residual=False, static=True, normed=True),
        # the rows of a long prompt: a stream over memory
        _norm("norm_t8191", 8191, HIDDEN),
        # one token of one sequence far into its context: bound by latency
        _rope("rope_t1", 1, 131072),
        # the new rows of a serving verify step
        _rope("rope_t320", 320, 4096),
        # one tensor-parallel shard of eight, heads of 80 rotated in part and by neighbours, a calibrated scale
        _rope("rope_t1005_shard", 1005, 32768, H=1, D=80, R=32, interleaved=True, per_tensor=True),
        # a long prompt, whose attention takes the rotated keys in bf16
        _rope("rope_t8191", 8191, 8191, keys=True),
        # a drafter's QKV linear for one sequence: a small weight stream, bound by latency
        _linear4("linear4_m1_qkv", 1, QKV, HIDDEN),
        # its down projection for a few sequences: few output rows, a long sum
        _linear4("linear4_m5_down", 5, HIDDEN, INTER),
        # its gate|up linear at the serving batch
        _linear4("linear4_m64_gate_up", 64, 2 * INTER, HIDDEN, static=True),
        # the output layer of a drafter over the full vocabulary: the largest weight stream of a draft step
        _linear4("linear4_m8_head", 8, VOCAB, HIDDEN),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "rope", "linear4"))
    if kind == "norm":
        C = rng.choice((HIDDEN, HIDDEN, 8 * _log_int(rng, 32, 2048)))
        T = _log_int(rng, 1, min(8191, 8191 * HIDDEN // C))
        c = _norm("", T, C, rng.random() < 0.7, rng.random() < 0.3, rng.random() < 0.3)
    elif kind == "rope":
        H, G, D = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 4, 4, 8)), rng.choice((64, 80, 128, 128, 256))
        R = rng.choice((D, D, D // 2))
        T = _log_int(rng, 1, min(8191, 8191 * 48 * 128 // (H * (G + 2) * D)))
        c = _rope("", T, _log_int(rng, 512, 131072), H, G, D, R, rng.random() < 0.3, rng.random() < 0.3, rng.random() < 0.3)
    else:
        M, tp = _log_int(rng, 1, 64), rng.choice((1, 1, 4, 8))
        N, K = rng.choice(((QKV // tp, HIDDEN), (HIDDEN, HIDDEN // tp), (2 * INTER // tp, HIDDEN), (HIDDEN, INTER // tp),
                           (HIDDEN, 2 * HIDDEN), (VOCAB // tp if M <= 8 else VOCAB // 8, HIDDEN),
                           (_log_int(rng, 100, 16384), GROUP4 * _log_int(rng, 4, 448))))
        c = _linear4("", M, N, K, rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _outliers(g, x, share=0.005, scale=30.0):
    """Some channels of the last axis much larger than the others, as a decoder's activations have them."""
    big = torch.rand(x.shape[-1], device="cuda", generator=g) < share
    return x * torch.where(big, scale, 1.0)


def _to_fp4(w):
    """MXFP4 of fp32 w [N, K]: packed codes [N, K/2] (the even channel in the low half) and scale bytes [N, K/32].

    A group's scale is 2^e with e from its largest magnitude rounded to E2M1's one bit after the point: that value
    lands on 4 or 6, or below."""
    N, K = w.shape
    x = w.view(N, K // GROUP4, GROUP4)
    _, ex = torch.frexp(x.abs().amax(-1) * 8.0 / 7.0)              # (7 and more of 2^e would round to 8)
    e = (ex - 3).clamp(-100, 125)
    v = torch.ldexp(x, -e[..., None])
    m = v.abs().clamp_max_(6.0)
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    m = torch.round(m / step) * step
    code = torch.where(m < 2.0, m * 2.0, torch.where(m < 4.0, m + 2.0, m / 2.0 + 4.0)).to(torch.uint8)
    code |= (v < 0).to(torch.uint8) << 3
    code = code.view(N, K)
    wide = torch.zeros((N, (K // GROUP4 + 3) // 4 * 4), dtype=torch.uint8, device="cuda")
    wide[:, :K // GROUP4] = (e + 127).to(torch.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, wide[:, :K // GROUP4]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "norm":
        T, C = case["T"], case["C"]
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        s["x"] = _outliers(g, _randn(g, T, C)).to(torch.bfloat16)
        s["weight"] = (1.0 + 0.2 * _randn(g, C)).to(torch.bfloat16)
        s["residual"] = _outliers(g, 3.0 * _randn(g, T, C)).to(torch.bfloat16) if case["residual"] else None
        s["sum"] = torch.empty((T, C), **bf16) if case["residual"] else None
        s["normed"] = torch.empty((T, C), **bf16) if case["normed"] else None
        s["codes"] = torch.empty((T, C), dtype=torch.uint8, device="cuda")
        # calibrated on other data: hardly any value is beyond it
        s["scale"] = torch.full((1,), 24.0 / 448.0, device="cuda") if case["static"] else torch.empty(T, device="cuda")
        return s
    if case["kind"] == "rope":
        T, H, D, R = case["T"], case["H"], case["D"], case["R"]
        Hq = H * case["G"]
        # the QKV projection's output, read in place
        qkv = torch.empty((T, (Hq + 2 * H) * D), dtype=torch.bfloat16, device="cuda")
        qkv[:, :(Hq + H) * D] = _outliers(g, _randn(g, T, (Hq + H) * D), 0.01, 20.0).to(torch.bfloat16)
        qkv[:, (Hq + H) * D:] = _randn(g, T, H * D).to(torch.bfloat16)
        s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + H) * D].view(T, H, D)
        s["v"] = qkv[:, (Hq + H) * D:].view(T, H, D)
        s["positions"] = torch.randint(0, case["far"], (T,), device="cuda", generator=g, dtype=torch.int32)
        s["inv_freq"] = 500000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
        slots = (T + T // 4 + PAGE) // PAGE * PAGE
        pages = torch.randperm(slots // PAGE, device="cuda", generator=g)
        slot = (pages[:, None] * PAGE + torch.arange(PAGE, device="cuda")).view(-1)[:T]
        if T > 1:                                                  # padding of the batch
            slot = torch.where(torch.rand(T, device="cuda", generator=g) < 0.02, -1, slot)
        s["slots"] = slot.contiguous()
        for w in ("k", "v"):
            s[w + "_cache"] = torch.zeros((slots, H, D), dtype=torch.uint8, device="cuda")
            s[w + "_scale"] = (torch.full((1,), 0.05, device="cuda") if case["per_tensor"]
                               else torch.ones((slots, H), device="cuda"))
        s["q_out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda") if case["keys"] else None
        return s
    M, N, K = case["M"], case["N"], case["K"]
    x = _outliers(g, _randn(g, M, K))
    s["a_scale"] = x.abs().amax().view(1) / 448.0 if case["static"] else x.abs().amax(-1) / 448.0
    s["a"] = (x / (s["a_scale"] if case["static"] else s["a_scale"][:, None])).clamp(-448, 448).to(torch.float8_e4m3fn)
    s["a"] = s["a"].view(torch.uint8)
    s["w"], s["w_scale"] = _to_fp4(_randn(g, N, K) * 0.02)
    s["y"] = torch.empty((M, (N + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :N]
    return s


# ------------------------------------------------------------- the plain form

def _e4m3(x, scale):
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _row_scale(x):
    return (x.abs().amax(-1) / 448.0).clamp_min(2.0 ** -100)


def _plain_norm(s):
    h = s["x"].float()
    out = {}
    if s["residual"] is not None:
        h = h + s["residual"].float()
        out["sum"] = h.to(torch.bfloat16)
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    if s["normed"] is not None:
        out["normed"] = y.to(torch.bfloat16)
    if s["case"]["static"]:
        out["codes"] = _e4m3(y, s["scale"])
    else:
        out["scale"] = _row_scale(y)
        out["codes"] = _e4m3(y, out["scale"][:, None])
    return out


def _rotated(x, cos, sin, R, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _plain_rope(s):
    case = s["case"]
    angle = s["positions"].double()[:, None, None] * s["inv_freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotated(s["q"], cos, sin, case["R"], case["interleaved"]).to(torch.bfloat16)
    k = _rotated(s["k"], cos, sin, case["R"], case["interleaved"])
    there = s["slots"] >= 0
    at = s["slots"][there]
    out = {"q": q}
    for w, x in (("k", k), ("v", s["v"].float())):
        codes, scale = s[w + "_cache"].view(torch.float8_e4m3fn), s[w + "_scale"]
        if case["per_tensor"]:
            x = _e4m3(x, scale)
        else:
            row = _row_scale(x)
            x = _e4m3(x, row[..., None])
            scale[at] = row[there]
            out[w + "_scale"] = scale
        s[w + "_cache"][at] = x.view(torch.uint8)[there]
        out[w + "_cache"] = codes
    if s["k_out"] is not None:
        out["keys"] = k.to(torch.bfloat16)
    return out


def _plain_linear4(s):
    case = s["case"]
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    grid = torch.cat((grid, -grid))
    w = torch.stack((grid[(s["w"] & 15).int()], grid[(s["w"] >> 4).int()]), -1).view(case["N"], -1, GROUP4)
    w = torch.ldexp(w, s["w_scale"].int()[..., None] - 127).view(case["N"], case["K"])
    y = torch.matmul(s["a"].view(torch.float8_e4m3fn).float(), w.t())
    return (y * s["a_scale"].view(-1, 1)).to(torch.bfloat16)


# --------------------------------------------------------------------- a pass

def run(s):
    case = s["case"]
    if not own:
        return {"norm": _plain_norm, "rope": _plain_rope, "linear4": _plain_linear4}[case["kind"]](s)
    import paper_2606_18502_amd as p
    if case["kind"] == "norm":
        given = s["scale"] if case["static"] else None
        p.rms_norm_quantize(s["x"], s["weight"], EPS, residual=s["residual"], per_tensor_scale=given,
                            residual_out=s["sum"], normed=s["normed"], out=s["codes"],
                            scales=None if case["static"] else s["scale"])
        out = {"codes": s["codes"].view(torch.float8_e4m3fn)}
        if not case["static"]:
            out["scale"] = s["scale"]
        if case["residual"]:
            out["sum"] = s["sum"]
        if case["normed"]:
            out["normed"] = s["normed"]
        return out
    if case["kind"] == "rope":
        p.rope_kv_cache_write(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["slots"], s["k_cache"],
                              s["v_cache"], s["k_scale"], s["v_scale"], per_tensor=case["per_tensor"],
                              interleaved=case["interleaved"], q_out=s["q_out"], k_out=s["k_out"])
        out = {"q": s["q_out"], "k_cache": s["k_cache"].view(torch.float8_e4m3fn),
               "v_cache": s["v_cache"].view(torch.float8_e4m3fn)}
        if not case["per_tensor"]:
            out["k_scale"], out["v_scale"] = s["k_scale"], s["v_scale"]
        if case["keys"]:
            out["keys"] = s["k_out"]
        return out
    return p.gemm_fp4(s["a"], s["a_scale"], s["w"], s["w_scale"], out=s["y"])


def work(case):
    if case["kind"] == "norm":
        T, C = case["T"], case["C"]
        each = 2 + 1 + (4 if case["residual"] else 0) + (2 if case["normed"] else 0)
        return {"bytes": T * C * each + 2 * C + 4 * (1 if case["static"] else T), "flops": 6 * T * C}
    if case["kind"] == "rope":
        T, H, D, R = case["T"], case["H"], case["D"], case["R"]
        Hq = H * case["G"]
        each = 4 * Hq * D + 2 * H * D * (2 + 1) + (2 * H * D if case["keys"] else 0) + 8 + 4
        return {"bytes": T * (each + (0 if case["per_tensor"] else 8 * H)) + 4 * R,
                "flops": T * (3 * (Hq + H) * R + 4 * H * D)}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": N * K // 2 + N * K // GROUP4 + M * K + 4 * (1 if case["static"] else M) + 2 * M * N, "flops": 2 * M * N * K}


# ------------------------------------------- the definition, in 64 bits

def _exact_norm(s, case):
    x, w = s["x"].double(), s["weight"].double()
    out = {}
    if case["residual"]:
        x = out["sum"] = x + s["residual"].double()
    y = w * x / torch.sqrt(torch.sum(x ** 2, 1) / case["C"] + EPS)[:, None]
    if case["normed"]:
        out["normed"] = y
    if case["static"]:
        out["codes"] = torch.clip(y / s["scale"].double(), -448, 448)
    else:
        out["scale"] = torch.max(torch.abs(y), 1).values / 448
        out["codes"] = y / out["scale"][:, None]
    return out


def _exact_rope(s, case):
    R, T, D = case["R"], case["T"], case["D"]
    i = torch.arange(R // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
    phase = torch.polar(torch.ones((T, R // 2), dtype=torch.float64, device="cuda"),
                        torch.outer(s["positions"].double(), s["inv_freq"]))

    def turned(x):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * phase[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    k = turned(s["k"])
    out = {"q": turned(s["q"])}
    if case["keys"]:
        out["keys"] = k
    slots = s["slots"].tolist()
    token = [t for t in range(T) if slots[t] >= 0]
    slot = [slots[t] for t in token]
    for w, x in (("k", k), ("v", s["v"].double())):
        codes = torch.zeros(s[w + "_cache"].shape, dtype=torch.float64, device="cuda")
        if case["per_tensor"]:
            codes[slot] = torch.clip(x[token] / s[w + "_scale"].double(), -448, 448)
        else:
            row = torch.max(torch.abs(x), 2).values / 448
            scale = torch.ones(s[w + "_scale"].shape, dtype=torch.float64, device="cuda")
            scale[slot] = row[token]
            codes[slot] = (x / row[..., None])[token]
            out[w + "_scale"] = scale
        out[w + "_cache"] = codes
    return out


def _exact_linear4(s, case):
    """Halves of a byte as sign, two exponent bits and one of fraction, exponent 0 without the leading one."""
    a = s["a"].view(torch.float8_e4m3fn).double() * s["a_scale"].double().view(-1, 1)
    pieces = []
    for w, e in zip(s["w"].split(8192), s["w_scale"].split(8192)):
        values = []
        for half in (w % 16, w // 16):
            sign = 1.0 - 2.0 * (half // 8).double()
            power, fraction = (half // 2 % 4).double(), (half % 2).double()
            values.append(sign * torch.where(power == 0, fraction / 2, (1 + fraction / 2) * 2 ** (power - 1)))
        x = torch.stack(values, 2).reshape(w.shape[0], case["K"])
        x = x * torch.repeat_interleave(2.0 ** (e.double() - 127), GROUP4, 1)
        pieces.append(torch.mm(a, x.t().contiguous()))
    return torch.cat(pieces, 1)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "linear4": _exact_linear4}[case["kind"]](s, case)
