"""Performance cases of the attention of a verify step: the FP8 KV cache read back, attention of new tokens over the
paged cache, and attention over the prompt that fills it.

A serving program calls them between the QKV projection and the output projection: the prompt's attention reads the
bf16 QKV output in place, its keys and values go to the paged E4M3 cache, and from then on the new rows of every step
(one token, a drafted chain with the last accepted token, a drafted tree, or the next chunk of a long prompt) attend
to the cache.  Head counts and sizes are those of workloads/configs.py (32 query heads, 8 KV heads of 128, pages of 16
tokens, contexts of 512 to 4096 tokens), their tensor-parallel shards, and ragged sizes around them.

listed() are the fixed cases, draw(rng) one more of the same ranges; prepare/run/work/exact describe one case each.
`own` selects the framework's kernels; without it run() computes the same in elementary torch operations.
"""

from __future__ import annotations

import math

import torch

own = False

KV_HEADS, GROUP, HEAD_DIM, PAGE = 8, 4, 128, 16

# A 25-node draft tree in the style of a top-k expansion (depth 6 along the top branch).
TREE25 = "-1 -1 -1 -1 0 0 0 1 1 2 3 4 4 4 5 7 11 11 12 14 16 16 18 20 20"


# ---------------------------------------------------------------- the cases

def _read(name, T, H=KV_HEADS, D=HEAD_DIM, per_tensor=False):
    return dict(name=name, kind="read", T=T, H=H, D=D, per_tensor=per_tensor)


def _paged(name, B, n, ctx, H=KV_HEADS, G=GROUP, D=HEAD_DIM, page=PAGE, per_tensor=False, tree=""):
    """B sequences with n[0]..n[1] new rows and ctx[0]..ctx[1] tokens before them in the cache."""
    return dict(name=name, kind="paged", B=B, n_min=n[0], n_max=n[1], ctx_min=ctx[0], ctx_max=ctx[1], H=H, G=G, D=D,
                page=page, per_tensor=per_tensor, tree=tree)


def _prompt(name, B, n, H=KV_HEADS, G=GROUP, D=HEAD_DIM):
    return dict(name=name, kind="prompt", B=B, n_min=n[0], n_max=n[1], H=H, G=G, D=D)


def listed():
    return [
        # the tokens of one small verify step looked up in the cache: bound by latency
        _read("read_t5", 5),
        # the contexts of a serving batch read back as bf16 (moving sequences to another instance): a stream over memory
        _read("read_t70001", 70001),
        # one sequence generating token by token with a short context: bound by latency
        _paged("decode_b1", 1, (1, 1), (700, 700)),
        # token by token at the serving batch: a stream over the cache
        _paged("decode_b64", 64, (1, 1), (512, 4096)),
        # the flagship verify step (B = 64, k = 4): five rows a sequence over the same cache
        _paged("verify_b64", 64, (5, 5), (512, 4096)),
        # one tensor-parallel shard of eight (one KV head), longer chains, a static scale, pages of 24 tokens
        _paged("verify_b13_shard", 13, (8, 8), (301, 2999), H=1, page=24, per_tensor=True),
        # drafted trees of 25 nodes and the root, each row under its own mask
        _paged("tree_b16", 16, (26, 26), (512, 4096), tree=TREE25),
        # two sequences with very long contexts: few rows, a long axis
        _paged("decode_long_b2", 2, (1, 1), (60001, 131071)),
        # the next chunks of two long prompts beside sequences that generate: products over long rows
        _paged("chunk_b6", 6, (1, 2000), (100, 6000)),
        # short prompts packed together, down to one token
        _prompt("prompt_short_b7", 7, (1, 130)),
        # a prefill batch of ragged prompts (the paper's exceed 1,000 tokens)
        _prompt("prompt_b9", 9, (200, 2100)),
        # one long prompt: bound by the matrix cores
        _prompt("prompt_8191", 1, (8191, 8191)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _random_tree(rng, N):
    return " ".join(str(rng.randint(-1, m - 1)) for m in range(N))


def draw(rng):
    kind = rng.choice(("read", "paged", "paged", "paged", "paged", "prompt", "prompt"))
    H, G, D = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 4, 4, 4, 8)), rng.choice((64, 128, 128, 128, 256))
    per_tensor = rng.random() < 0.3
    if kind == "read":
        c = _read("", _log_int(rng, 1, 70000 * 8 * 128 // (8 * 256)), H, D, per_tensor)
    elif kind == "prompt":
        hi = _log_int(rng, 1, 4096)
        c = _prompt("", _log_int(rng, 1, max(1, min(32, 8191 // hi))), (max(1, hi // rng.choice((1, 4, 50))), hi), H, min(G, 4),
                    min(D, 128))
    else:
        page, rows = rng.choice((16, 16, 32, 24, 1)), rng.choice(("one", "chain", "chain", "tree", "chunk"))
        B = _log_int(rng, 1, 64)
        ctx = _log_int(rng, 16, min(65536, 200000 // B))
        n = {"one": 1, "chain": rng.randint(2, 9), "tree": rng.randint(4, 48), "chunk": 0}[rows]
        tree = _random_tree(rng, n - 1) if rows == "tree" else ""
        if rows == "chunk":
            B, ctx, n = min(B, 5), min(ctx, 6000), _log_int(rng, 16, 2000)
        G = min(G, 4) if rows in ("tree", "chunk") else G
        D = min(D, 128) if ctx * B > 64 * 1024 or rows == "chunk" else D
        c = _paged("", B, (max(1, n // 50) if rows == "chunk" else n, n), (max(1, ctx // rng.choice((1, 8))), ctx), H, G, D,
                   page, per_tensor, tree)
    del c["name"]
    return c


def _spread(lo, hi, B, phase):
    """B lengths from lo to hi, ragged, the same for every seed: lo and hi themselves, then a low-discrepancy sequence."""
    mid = [lo + int((hi - lo) * ((phase + 0.6180339887498949 * b) % 1.0)) for b in range(B)]
    return ([hi] + mid[2:] + [lo])[:B] if B > 1 else [hi]


def _lengths(case):
    """(new rows, cached tokens with the new ones) of each sequence."""
    B = case["B"]
    new = _spread(case["n_min"], case["n_max"], B, 0.37)
    if case["kind"] == "prompt":
        return new, new
    return new, [c + n for c, n in zip(_spread(case["ctx_min"], case["ctx_max"], B, 0.11), new)]


# ------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _outliers(g, x, share=0.01, scale=20.0):
    """Some channels of the last axis much larger than the others, as the projections' outputs have them."""
    big = torch.rand(x.shape[-1], device="cuda", generator=g) < share
    return x * torch.where(big, scale, 1.0)


def _cache(g, slots, H, D, per_tensor, outliers):
    """E4M3 codes [slots, H, D] and their scales, as the cache holds them."""
    x = _randn(g, slots, H, D)
    if outliers:
        x = _outliers(g, x.view(slots, H * D)).view(slots, H, D)
    amax = x.abs().amax(-1) if not per_tensor else x.abs().amax().view(1)
    scale = (amax / 448.0).clamp_min(2.0 ** -100)
    codes = (x / (scale[..., None] if not per_tensor else scale)).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), scale


def _cu(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _tree_masks(parents):
    """The nodes on each node's root path (itself included), as 64 bits."""
    bits = []
    for m, up in enumerate(parents):
        bits.append((1 << m) | (bits[up] if up >= 0 else 0))
    return torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H, D = case["H"], case["D"]
    s = dict(case=case)
    if case["kind"] == "read":
        T = case["T"]
        slots = (T + T // 4 + 16) // 16 * 16
        s["k_cache"], s["k_scale"] = _cache(g, slots, H, D, case["per_tensor"], True)
        s["v_cache"], s["v_scale"] = _cache(g, slots, H, D, case["per_tensor"], False)
        # whole pages in any order, the last one cut
        pages = torch.randperm(slots // PAGE, device="cuda", generator=g)
        s["slots"] = (pages[:, None] * PAGE + torch.arange(PAGE, device="cuda")).view(-1)[:T].contiguous()
        s["k"] = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
        s["v"] = torch.empty_like(s["k"])
        return s
    new, total = _lengths(case)
    Hq, T = H * case["G"], sum(new)
    # the QKV projection's output, read in place
    qkv = torch.empty((T, (Hq + 2 * H) * D), dtype=torch.bfloat16, device="cuda")
    qkv[:, :Hq * D] = _randn(g, T, Hq * D).to(torch.bfloat16)
    qkv[:, Hq * D:(Hq + H) * D] = _outliers(g, _randn(g, T, H * D)).to(torch.bfloat16)
    qkv[:, (Hq + H) * D:] = _randn(g, T, H * D).to(torch.bfloat16)
    s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
    s["out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    s["max_new"], s["max_total"] = max(new), max(total)
    s["cu"] = _cu(new)
    if case["kind"] == "prompt":
        s["k"] = qkv[:, Hq * D:(Hq + H) * D].view(T, H, D)
        s["v"] = qkv[:, (Hq + H) * D:].view(T, H, D)
        return s
    B, page = case["B"], case["page"]
    need = [(t + page - 1) // page for t in total]
    s["k_cache"], s["k_scale"] = _cache(g, sum(need) * page, H, D, case["per_tensor"], True)
    s["v_cache"], s["v_scale"] = _cache(g, sum(need) * page, H, D, case["per_tensor"], False)
    order = torch.randperm(sum(need), device="cuda", generator=g).to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, w in enumerate(need):
        table[b, :w] = order[at:at + w]
        at += w
    s["table"], s["lens"] = table, torch.tensor(total, dtype=torch.int32).cuda()
    s["ragged"] = len(set(new)) > 1
    s["mask"] = None
    if case["tree"]:
        s["mask"] = _tree_masks([int(x) for x in case["tree"].split()]).repeat(B, 1).cuda()
    return s


# ------------------------------------------------------------- the plain form

def _softmax_product(q, k, v, seen, scale):
    """softmax(scale q k^T over the keys seen) v in 32 bits: q [B,Hq,n,D], k and v [B,H,L,D], seen [B,1,n,L]."""
    B, Hq, n, D = q.shape
    H, L = k.shape[1], k.shape[2]
    s = torch.matmul(q.reshape(B, H, Hq // H * n, D), k.transpose(2, 3).contiguous()).view(B, Hq, n, L) * scale
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    s = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, H, Hq // H * n, L), v.contiguous()).view(B, Hq, n, D)
    return o / total.masked_fill(total == 0.0, 1.0)


def _rows(cu, most):
    """Row numbers [B, most] of packed sequences and which of them there are."""
    at = torch.arange(most, device="cuda")
    there = at < (cu[1:] - cu[:-1])[:, None]
    return (cu[:-1, None] + at).masked_fill(~there, 0).long(), there


def _decoded(codes, scale, per_tensor):
    x = codes.view(torch.float8_e4m3fn).to(torch.float32)
    return x * (scale if per_tensor else scale[..., None])


def _plain_paged(s):
    case, cu, lens = s["case"], s["cu"].long(), s["lens"].long()
    page, pt, D = case["page"], case["per_tensor"], case["D"]
    rows, there = _rows(cu, s["max_new"])
    q = s["q"].float()[rows].permute(0, 2, 1, 3)
    pos = torch.arange(s["max_total"], device="cuda")
    slot = s["table"].long()[:, pos // page] * page + pos % page
    k = _decoded(s["k_cache"][slot], s["k_scale"] if pt else s["k_scale"][slot], pt).permute(0, 2, 1, 3)
    v = _decoded(s["v_cache"][slot], s["v_scale"] if pt else s["v_scale"][slot], pt).permute(0, 2, 1, 3)
    new = cu[1:] - cu[:-1]
    i = torch.arange(s["max_new"], device="cuda")
    if s["mask"] is None:
        seen = pos <= ((lens - new)[:, None] + i)[..., None]
    else:
        N = s["mask"].shape[1]
        node = pos - (lens - N)[:, None]
        bits = (s["mask"][:, :, None] >> node.clamp(0, 63)[:, None, :]) & 1
        bits = torch.cat([torch.zeros_like(bits[:, :1]), bits], 1)
        seen = (node[:, None, :] < 0) | (bits == 1)
    seen = (seen & (pos < lens[:, None])[:, None, :])[:, None]
    o = _softmax_product(q, k, v, seen, D ** -0.5).permute(0, 2, 1, 3)
    return o[there].to(torch.bfloat16)


def _plain_prompt(s):
    cu, D = s["cu"].long(), s["case"]["D"]
    rows, there = _rows(cu, s["max_new"])
    q, k, v = (s[x].float()[rows].permute(0, 2, 1, 3) for x in ("q", "k", "v"))
    at = torch.arange(s["max_new"], device="cuda")
    seen = (at <= at[:, None]) & there[:, None, None, :]
    return _softmax_product(q, k, v, seen, D ** -0.5).permute(0, 2, 1, 3)[there].to(torch.bfloat16)


def _plain_read(s):
    pt = s["case"]["per_tensor"]
    return tuple(_decoded(s[c][s["slots"]], s[x] if pt else s[x][s["slots"]], pt).to(torch.bfloat16)
                 for c, x in (("k_cache", "k_scale"), ("v_cache", "v_scale")))


# --------------------------------------------------------------------- a pass

def run(s):
    case = s["case"]
    if not own:
        return {"read": _plain_read, "paged": _plain_paged, "prompt": _plain_prompt}[case["kind"]](s)
    import paper_2606_18502_amd as p
    if case["kind"] == "read":
        return p.kv_cache_read(s["k_cache"], s["v_cache"], s["slots"], s["k_scale"], s["v_scale"],
                               per_tensor=case["per_tensor"], k=s["k"], v=s["v"])
    if case["kind"] == "prompt":
        return p.prompt_attention(s["q"], s["k"], s["v"], s["cu"], out=s["out"])
    if "workspace" not in s:             # a serving program's own, kept for all its calls
        T, Hq, D = s["q"].shape
        n = p.paged_attention_workspace_bytes(T, case["B"], Hq, case["H"], D)
        s["workspace"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
    return p.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lens"],
                             case["page"], cu_q=s["cu"] if s["ragged"] else None, tree_mask=s["mask"],
                             per_tensor=case["per_tensor"], out=s["out"], workspace=s["workspace"])


def work(case):
    H, D = case["H"], case["D"]
    code = 2 * H * D + (0 if case.get("per_tensor") else 8 * H)          # bytes of a cached token
    if case["kind"] == "read":
        return {"bytes": case["T"] * (code + 4 * H * D + 8), "flops": 2 * case["T"] * H * D}
    new, total = _lengths(case)
    Hq, T = H * case["G"], sum(new)
    if case["kind"] == "prompt":
        return {"bytes": T * (2 * Hq + 2 * H) * D * 2, "flops": 2 * D * Hq * sum(n * (n + 1) for n in new)}
    if case["tree"]:
        parents = [int(x) for x in case["tree"].split()]
        depth = [0]
        for up in parents:
            depth.append(depth[up + 1] + 1)
        pairs = sum((t - len(parents)) * n + sum(depth) for n, t in zip(new, total))
    else:
        pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(new, total))
    tables = sum((t + case["page"] - 1) // case["page"] for t in total) * 4
    return {"bytes": sum(total) * code + 4 * T * Hq * D + tables, "flops": 4 * D * Hq * pairs}


# ------------------------------------------- the definition, in 64 bits

def _e4m3_table():
    """The 256 values of OCP E4M3: bias 7, subnormals below 2^-6, NaN at S.1111.111."""
    vals = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        vals.append(-mag if c & 128 else mag)
    return torch.tensor(vals, dtype=torch.float64, device="cuda")


def exact(case, seed):
    s = prepare(case, seed)
    H, D = case["H"], case["D"]
    table = _e4m3_table()

    def cached(which, slots):
        x = table[s[which + "_cache"][slots].long()]
        sc = s[which + "_scale"].double()
        return x * (sc if case["per_tensor"] else sc[slots][..., None])

    if case["kind"] == "read":
        return tuple(torch.cat([cached(w, part) for part in s["slots"].split(8192)]) for w in ("k", "v"))
    new, total = _lengths(case)
    G, outs, first = case["G"], [], 0
    parents = [int(x) for x in case["tree"].split()] if case.get("tree") else []
    for b, (n, L) in enumerate(zip(new, total)):
        q = s["q"][first:first + n].double()
        if case["kind"] == "prompt":
            k, v = s["k"][first:first + n].double(), s["v"][first:first + n].double()
        else:
            j = torch.arange(L, device="cuda")
            slots = s["table"][b].long()[torch.div(j, case["page"], rounding_mode="floor")] * case["page"] + j % case["page"]
            k, v = cached("k", slots), cached("v", slots)
        hidden = torch.ones((n, L), dtype=torch.bool, device="cuda").triu(L - n + 1)
        if parents:
            hidden = torch.zeros((n, L), dtype=torch.bool)
            hidden[:, L - len(parents):] = True
            for m in range(len(parents)):
                up = m
                while up >= 0:
                    hidden[m + 1, L - len(parents) + up] = False
                    up = parents[up]
            hidden = hidden.cuda()
        o = torch.empty((n, H * G, D), dtype=torch.float64, device="cuda")
        for h in range(H * G):
            kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
            for r in range(0, n, 2048):
                w = torch.mm(q[r:r + 2048, h].contiguous(), kh.t().contiguous()) / math.sqrt(D)
                w = torch.softmax(w.masked_fill(hidden[r:r + 2048], -math.inf), -1)
                o[r:r + 2048, h] = torch.mm(w, vh)
        outs.append(o)
        first += n
    return torch.cat(outs)
