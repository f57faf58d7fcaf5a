"""Performance cases of softmax attention over whole sequences and of the layer norm: what a block needs where it does not use agents.

    attend         softmax attention, causal or not, of dense batches, packed sequences of different lengths, or few queries over long caches;
                   groups of heads share a head of keys and values
    attend_bwd     its gradient: of queries, keys and values, from the forward call's results
    layer_norm     y = (x - mean) / sqrt(var + eps) * weight + bias
    layer_norm_bwd its gradient: of x, the weight and the bias

Sizes are those of the package's workloads (14 x 14 tokens in 3 heads, 56 x 56 with 64 channels, 64 x 64 in 8 heads of 40, 128 x 128 in 8 heads of
64), with packed images and prompts beside them.  `run` computes the plain form where `own` is false, else it calls the package.
"""
import math
import random

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def _attend(name, entry, form, batch, queries, keys, heads, kv_heads, head_dim, dtype, causal, lens=0):
    """form: "dense" (all sequences `queries` by `keys` long; from one fused projection where they are equal), "packed" (up to that long, one after
    the other) or "cache" (`queries` each, over room for `keys` that is partly filled).  `lens` picks the lengths."""
    case = {"entry": entry, "form": form, "batch": batch, "queries": queries, "keys": keys, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "causal": causal, "lens": lens}
    return dict(case, name=name) if name else case


def _norm(name, entry, rows, channels, dtype):
    case = {"entry": entry, "rows": rows, "channels": channels, "dtype": dtype}
    return dict(case, name=name) if name else case


def listed():
    return [
        # One image through a small classifier's block in fp32: latency is everything.
        _attend("attend_deit_f32_b1", "attend", "dense", 1, 196, 196, 3, 3, 64, "f32", False),
        # Generation: one new token each for 16 entries of a batch, over caches of different fill.
        _attend("attend_token_bf16_b16", "attend", "cache", 16, 1, 16384, 16, 4, 128, "bf16", True, 1),
        # Images of any aspect ratio, packed: 32 of up to 64 x 64 tokens.
        _attend("attend_packed_bf16", "attend", "packed", 32, 4096, 4096, 8, 8, 64, "bf16", False, 2),
        # The diffusion network's 64 x 64 latents, heads of 40 channels.
        _attend("attend_sd_f16_b2", "attend", "dense", 2, 4096, 4096, 8, 8, 40, "f16", False),
        # Prompts of different lengths, causal, four heads to a head of keys.
        _attend("attend_prompts_bf16", "attend", "packed", 8, 8192, 8192, 16, 4, 128, "bf16", True, 3),
        # The largest: full attention where the high-resolution grid would use agents.
        _attend("attend_hires128_bf16_b2", "attend", "dense", 2, 16384, 16384, 8, 8, 64, "bf16", False),
        # Training of the classifier on 128 images, and on packed prompts.
        _attend("attend_bwd_deit_bf16_b128", "attend_bwd", "dense", 128, 196, 196, 3, 3, 64, "bf16", False),
        _attend("attend_bwd_prompts_bf16", "attend_bwd", "packed", 8, 4096, 4096, 16, 4, 128, "bf16", True, 4),
        # The norms around them: one image in fp32, the high-resolution grid with 512 channels; training at 56 x 56 and in the diffusion network.
        _norm("norm_deit_f32_b1", "layer_norm", 196, 192, "f32"),
        _norm("norm_hires256_bf16_b2", "layer_norm", 131072, 512, "bf16"),
        _norm("norm_bwd_pvt_bf16_b64", "layer_norm_bwd", 200704, 64, "bf16"),
        _norm("norm_bwd_sd_f16_b2", "layer_norm_bwd", 8192, 320, "f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MOST = 4 * 16384 * 16384 * 64 * 16         # operations of the largest listed case


def draw(rng):
    """One more case: sequences of one token to 16384, one to 128 of them, 1 to 32 heads of 32 to 128 channels in groups of 1 to 8; norms of one row to
    200704 with 1 to 4096 channels, odd ones among them."""
    dtype = rng.choice(["bf16"] * 5 + ["f16"] * 3 + ["f32"] * 2)
    if rng.random() < 0.35:
        while True:
            rows, channels = _log_int(rng, 1, 200704), _log_int(rng, 1, 4096)
            if rng.random() < 0.6:
                channels = (channels + 31) // 32 * 32
            if rows * channels <= (131072 * 512 if dtype != "f32" else 65536 * 512):
                return _norm("", rng.choice(["layer_norm", "layer_norm_bwd"]), rows, channels, dtype)
    while True:
        entry, form = rng.choice(["attend"] * 3 + ["attend_bwd"] * 2), rng.choice(["dense", "packed", "packed", "cache"])
        d, group, kv = rng.choice([32, 40, 64, 64, 64, 80, 96, 128, 128]), rng.choice([1, 1, 1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
        batch, queries, causal = _log_int(rng, 1, 128), _log_int(rng, 1, 16384), rng.random() < 0.5
        keys = queries
        if form == "cache":
            entry, queries = "attend", _log_int(rng, 1, 64)
            keys = max(queries, _log_int(rng, 16, 65536))
        elif form == "packed" and rng.random() < 0.3:                   # a cached beginning
            keys = queries + _log_int(rng, 1, 4096)
        if batch * keys * kv * d > 1 << 28 or batch * queries * kv * group * d > 1 << 26 or kv * group > 32:
            continue
        if 4 * batch * queries * keys * kv * group * d * (2.5 if entry == "attend_bwd" else 1) * (8 if dtype == "f32" else 1) > MOST:
            continue
        return _attend("", entry, form, batch, queries, keys, kv * group, kv, d, dtype, causal, rng.randrange(1 << 20))


def _lengths(c):
    """Queries and keys of each sequence."""
    rng, n = random.Random(c["lens"]), c["batch"]
    if c["form"] == "dense":
        return [c["queries"]] * n, [c["keys"]] * n
    if c["form"] == "cache":
        return [c["queries"]] * n, [rng.randint(max(c["queries"], c["keys"] // 2), c["keys"]) for _ in range(n)]
    q = [_log_int(rng, max(1, c["queries"] // 8), c["queries"]) for _ in range(n)]
    return q, [m + rng.randint(0, c["keys"] - c["queries"]) for m in q]


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dt)

    s = {"case": c}
    if c["entry"].startswith("layer_norm"):
        M, C = c["rows"], c["channels"]
        # a residual stream: channels with means of their own
        s["x"] = (torch.randn((M, C), generator=g, device="cuda") * 1.5 + torch.randn((C,), generator=g, device="cuda") * 0.5).to(dt)
        s["w"], s["b"] = normal((C,), 0.1, 1.0), normal((C,), 0.1)
        if c["entry"] == "layer_norm_bwd":
            s["dy"] = normal((M, C))
        if own:
            s["mod"] = _handle(1, 1, 64, 1, dt)
        return s
    B, h, kv, d, (nq, nk) = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], _lengths(c)
    s["nq"], s["nk"] = nq, nk
    if c["form"] == "packed":
        B, N, M = 1, sum(nq), sum(nk)
        s["q_offsets"], s["k_offsets"] = _offsets(nq), _offsets(nk)
    else:
        N, M = c["queries"], c["keys"]
        if c["form"] == "cache":
            s["k_lengths"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
    if N == M:                             # one fused projection
        qkv = normal((B, N, h + 2 * kv, d))
        s["q"], s["k"], s["v"] = (x.permute(0, 2, 1, 3) for x in qkv.split([h, kv, kv], 2))
    else:
        s["q"], s["k"], s["v"] = normal((B, N, h, d)).permute(0, 2, 1, 3), normal((B, kv, M, d)), normal((B, kv, M, d))
    if c["entry"] == "attend_bwd":
        s["do"] = normal((B, h, N, d))
    if own:
        s["mod"] = _handle(B, h, d, max(N, M), dt)
        s["args"] = {"causal": c["causal"], **{n: s[n] for n in ("q_offsets", "k_offsets", "k_lengths") if n in s}}
        if c["entry"] == "attend_bwd":     # what the forward call left
            s["out"], s["lse"] = s["mod"].attend(s["q"], s["k"], s["v"], need_lse=True, **s["args"])
    return s


def _handle(batch, heads, head_dim, tokens, dtype):
    from paper_2312_08874_b200 import AgentAttention
    return AgentAttention(batch, heads, head_dim, tokens, 1, dtype)


def run(state):
    s, c = state, state["case"]
    if c["entry"] == "attend":
        return s["mod"].attend(s["q"], s["k"], s["v"], **s["args"]) if own else _plain_attend(s)
    if c["entry"] == "attend_bwd":
        if own:
            return s["mod"].attend_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["do"], **s["args"])
        return _plain_attend_bwd(s)
    if c["entry"] == "layer_norm":
        return s["mod"].layer_norm(s["x"], s["w"], s["b"], eps=EPS) if own else _plain_norm(s)
    return s["mod"].layer_norm_backward(s["x"], s["dy"], s["w"], s["b"], eps=EPS) if own else _plain_norm_bwd(s)


def _spans(s):
    """(batch entries, rows of queries, rows of keys) of what can be computed together."""
    c = s["case"]
    if c["form"] == "dense":
        return [(slice(None), slice(None), slice(None))]
    if c["form"] == "cache":
        return [(slice(b, b + 1), slice(None), slice(0, n)) for b, n in enumerate(s["nk"])]
    spans, q, k = [], 0, 0
    for n, m in zip(s["nq"], s["nk"]):
        spans.append((slice(0, 1), slice(q, q + n), slice(k, k + m)))
        q, k = q + n, k + m
    return spans


def _pieces(s):
    """The spans in pieces whose scores take a gigabyte at most: (entries, queries, keys, heads of keys, place of the first query in its sequence)."""
    c, group = s["case"], s["case"]["heads"] // s["case"]["kv_heads"]
    for b, q, k in _spans(s):
        B, n, m = (len(range(*x.indices(t))) for x, t in zip((b, q, k), (s["q"].shape[0], s["q"].shape[2], s["k"].shape[2])))
        first, step = q.start or 0, max(1, (1 << 28) // (m * group))       # rows x heads of keys x entries
        heads, rows = max(1, min(c["kv_heads"], step // n)), min(n, step)
        entries = max(1, min(B, step // (n * heads)))
        for e in range(0, B, entries):
            be = slice(b.indices(s["q"].shape[0])[0] + e, b.indices(s["q"].shape[0])[0] + min(B, e + entries))
            for h in range(0, c["kv_heads"], heads):
                for r in range(0, n, rows):
                    yield be, slice(first + r, first + min(n, r + rows)), k, slice(h, min(c["kv_heads"], h + heads)), r + m - n


def _plain_scores(s, b, q, k, heads, at):
    """Probabilities [entries, heads of keys, group, queries, keys], with the queries [.. group, queries, d], keys and values [.. 1, keys, d]."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    x = s["q"][b].unflatten(1, (c["kv_heads"], group))[:, heads, :, q].float()
    y, v = (s[n][b, heads, k].float().unsqueeze(2) for n in ("k", "v"))
    p = x @ y.transpose(-1, -2) * c["head_dim"] ** -0.5
    if c["causal"]:
        i, j = torch.arange(x.shape[-2], device="cuda")[:, None], torch.arange(y.shape[-2], device="cuda")
        p = torch.where(j <= i + at, p, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True), x, y, v


def _plain_attend(s):
    c = s["case"]
    out = torch.empty_like(s["q"], memory_format=torch.contiguous_format).unflatten(1, (c["kv_heads"], -1))
    for b, q, k, heads, at in _pieces(s):
        p, _, _, v = _plain_scores(s, b, q, k, heads, at)
        out[b, heads, :, q] = (p @ v).to(out.dtype)
    return out.flatten(1, 2)


def _plain_attend_bwd(s):
    c, scale = s["case"], s["case"]["head_dim"] ** -0.5
    dq, dk, dv = (torch.zeros(s[n].shape, device="cuda") for n in "qkv")
    dq, do = (t.unflatten(1, (c["kv_heads"], -1)) for t in (dq, s["do"]))
    for b, q, k, heads, at in _pieces(s):
        p, x, y, v = _plain_scores(s, b, q, k, heads, at)
        g = do[b, heads, :, q].float()
        dv[b, heads, k] += (p.transpose(-1, -2) @ g).sum(2)
        dp = g @ v.transpose(-1, -2)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
        dq[b, heads, :, q] = ds @ y
        dk[b, heads, k] += (ds.transpose(-1, -2) @ x).sum(2)
    return {n: t.to(s["q"].dtype) for n, t in (("dq", dq.flatten(1, 2)), ("dk", dk), ("dv", dv))}


def _plain_norm_rows(s):
    x = s["x"].float()
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_norm(s):
    return (_plain_norm_rows(s)[0] * s["w"].float() + s["b"].float()).to(s["x"].dtype)


def _plain_norm_bwd(s):
    xh, r = _plain_norm_rows(s)
    dy = s["dy"].float()
    g = dy * s["w"].float()
    dx = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dw": (dy * xh).sum(0), "db": dy.sum(0)}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["entry"].startswith("layer_norm"):
        x, w, b = (s[n].double().requires_grad_() for n in ("x", "w", "b"))
        with torch.enable_grad():
            y = torch.nn.functional.layer_norm(x, (c["channels"],), w, b, EPS)
        if c["entry"] == "layer_norm":
            return y.detach()
        return dict(zip(("dx", "dw", "db"), torch.autograd.grad(y, (x, w, b), s["dy"].double())))
    group, back = c["heads"] // c["kv_heads"], c["entry"] == "attend_bwd"
    got = {n: torch.zeros(s[n[1:]].shape, dtype=torch.float64, device="cuda") for n in ("dq", "dk", "dv")} if back else None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at_q = at_k = 0
    for i, (n, m) in enumerate(zip(s["nq"], s["nk"])):
        b = 0 if c["form"] == "packed" else i
        rq, rk = slice(at_q, at_q + n), slice(at_k, at_k + m)
        if c["form"] == "packed":
            at_q, at_k = at_q + n, at_k + m
        hidden = torch.ones((n, m), dtype=torch.bool, device="cuda").triu(1 + m - n) if c["causal"] else None
        together = max(1, min(c["heads"], (1 << 28) // (n * m)))            # heads at once
        for h in range(0, c["heads"], together):
            hs = torch.arange(h, min(c["heads"], h + together), device="cuda")
            q = s["q"][b, hs, rq].double().requires_grad_(back)
            k, v = (s[t][b, :, rk].double()[hs // group].requires_grad_(back) for t in "kv")
            with torch.set_grad_enabled(back):
                x = torch.einsum("hid,hjd->hij", q, k) / math.sqrt(c["head_dim"])
                if hidden is not None:
                    x = x.masked_fill(hidden, -math.inf)
                o = torch.einsum("hij,hjd->hid", torch.softmax(x, -1), v)
            del x
            out[b, hs, rq] = o.detach()
            if back:
                a, e, f = torch.autograd.grad(o, (q, k, v), s["do"][b, hs, rq].double())
                got["dq"][b, hs, rq] = a
                for name, t in (("dk", e), ("dv", f)):
                    got[name][b, :, rk] = got[name][b, :, rk].index_add(0, hs // group, t)
    return got if back else out


def work(case):
    c, es = case, 4 if case["dtype"] == "f32" else 2
    if c["entry"].startswith("layer_norm"):
        M, C = c["rows"], c["channels"]
        if c["entry"] == "layer_norm":
            return {"bytes": (2 * M * C + 2 * C) * es, "flops": 8 * M * C}
        return {"bytes": (3 * M * C + C) * es + 8 * C, "flops": 15 * M * C}
    nq, nk = _lengths(c)
    pairs = 0
    for n, m in zip(nq, nk):               # causal: query i has m - n + i + 1 keys (m >= n)
        pairs += n * (m - n) + n * (n + 1) // 2 if c["causal"] else n * m
    queries, keys, d = sum(nq) * c["heads"], sum(nk) * c["kv_heads"], c["head_dim"]
    if c["entry"] == "attend":
        return {"bytes": 2 * (queries + keys) * d * es, "flops": 4 * pairs * c["heads"] * d}
    # reads the inputs, the result, its gradient and the rows' statistics, writes three gradients
    return {"bytes": (4 * queries + 4 * keys) * d * es + 4 * queries, "flops": 10 * pairs * c["heads"] * d}
