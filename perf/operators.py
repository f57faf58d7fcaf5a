"""Performance cases of what stands around the attention in a transformer block: queries and keys with rotary positions (and norms of each
head), and the gated feed-forward product.

    rotate       rotary positions with one to three axes on queries and keys; with "norm", an RMS norm of each head in the same pass
    rotate_bwd   its gradient: fp32 gradients of the prepared queries and keys in, gradients of the projections' outputs (and gains) out
    gated        H = act(X Wg^T + bg) * (X Wu^T + bu)
    gated_bwd    its gradient: X, the weights and the biases

Sizes are those of the package's workloads (14 x 14 tokens in 3 heads, 56 x 56 in 1, 64 x 64 in 8 heads of 40, 128 x 128 and 256 x 256 in 8 heads
of 64) with a video grid and packed images beside them.  `run` computes the plain form where `own` is false, else it calls the package.
"""
import math

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def _rotate(name, entry, batch, heads, head_dim, extent, channels, dtype, pairs, norm, qkv, given=False):
    t, h, w = (1,) * (3 - len(extent)) + tuple(extent)
    a, b, c = (0,) * (3 - len(channels)) + tuple(channels)
    case = {"entry": entry, "batch": batch, "heads": heads, "head_dim": head_dim, "axes": len(extent), "t": t, "h": h, "w": w,
            "ct": a, "ch": b, "cw": c, "dtype": dtype, "pairs": pairs, "norm": norm, "qkv": qkv, "given": given}
    return dict(case, name=name) if name else case


def _gated(name, entry, rows, channels, hidden, dtype, act, bias):
    case = {"entry": entry, "rows": rows, "channels": channels, "hidden": hidden, "dtype": dtype, "act": act, "bias": bias}
    return dict(case, name=name) if name else case


def listed():
    return [
        # One image through a small classifier's block in fp32: latency is everything.
        _rotate("rotate_deit_f32_b1", "rotate", 1, 3, 64, (14, 14), (32, 32), "f32", False, False, False),
        # Two clips of 8 frames on a 45 x 80 grid, time, height and width as axes, read from the fused projection.
        _rotate("rotate_video_bf16_b2", "rotate", 2, 8, 64, (8, 45, 80), (16, 24, 24), "bf16", False, False, True),
        # First stage of a pyramid network: one head, many images; norms and positions in one pass.
        _rotate("norm_pvt_bf16_b64", "rotate", 64, 1, 64, (56, 56), (32, 32), "bf16", False, True, True),
        # Images of any aspect ratio: positions come with the tokens, heads of 40 channels, neighbouring channels as pairs.
        _rotate("norm_packed_f16_b4", "rotate", 4, 8, 40, (75, 117), (20, 20), "f16", True, True, False, True),
        # The largest grid.
        _rotate("norm_hires256_bf16_b2", "rotate", 2, 8, 64, (256, 256), (32, 32), "bf16", False, True, True),
        # Training: the gradients of a batch of images, and of a high-resolution grid.
        _rotate("norm_bwd_deit_bf16_b128", "rotate_bwd", 128, 3, 64, (14, 14), (32, 32), "bf16", False, True, True),
        _rotate("norm_bwd_hires128_bf16_b2", "rotate_bwd", 2, 8, 64, (128, 128), (32, 32), "bf16", False, True, True),
        # The feed-forward part of the classifier's block for one image, in fp32.
        _gated("gated_deit_f32_b1", "gated", 196, 192, 512, "f32", "silu", False),
        # The diffusion network's block: 64 x 64 latents of two images, 320 channels, GELU gate with biases; inference and fine-tuning.
        _gated("gated_sd_f16_b2", "gated", 8192, 320, 1280, "f16", "gelu", True),
        _gated("gated_bwd_sd_f16_b2", "gated_bwd", 8192, 320, 1280, "f16", "gelu", True),
        # High-resolution grid, 512 channels; a hidden size of 8/3 of them that is no multiple of a tile.
        _gated("gated_hires128_bf16_b2", "gated", 32768, 512, 1368, "bf16", "silu", False),
        # Training on a batch of 128 images.
        _gated("gated_bwd_deit_bf16_b128", "gated_bwd", 25088, 192, 512, "bf16", "gelu", True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: one token to a grid of 256 x 256, heads of 32 to 128 channels, one to three axes, both kinds of pairs; one row to 32768,
    32 to 640 channels, hidden sizes of 2 to 4 times that (multiples of 8)."""
    dtype = rng.choice(["bf16"] * 5 + ["f16"] * 3 + ["f32"] * 2)
    if rng.random() < 0.5:
        while True:
            d, axes = rng.choice([32, 40, 64, 64, 64, 80, 128]), rng.choice([1, 2, 2, 2, 3])
            extent = tuple(_log_int(rng, 1, (0, 4096, 256, 48)[axes]) for _ in range(axes))
            heads, batch = rng.choice([1, 2, 3, 4, 8]), _log_int(rng, 1, 128)
            entry, norm = rng.choice(["rotate"] * 3 + ["rotate_bwd"] * 2), rng.random() < 0.6
            total = batch * heads * math.prod(extent) * d
            most = 2 * 8 * 65536 * 64 // (2 if dtype == "f32" else 1) // (4 if entry == "rotate_bwd" else 1)
            if total > most:
                continue
            seg = d // axes // 2 * 2 if rng.random() < 0.7 else max(2, d // axes // 4 * 2)
            return _rotate("", entry, batch, heads, d, extent, (seg,) * axes, dtype, rng.random() < 0.4, norm, rng.random() < 0.6, rng.random() < 0.3)
    while True:
        c = rng.choice([32, 64, 96, 128, 192, 256, 320, 384, 512, 640])
        f = int(c * rng.choice([2, 8 / 3, 3, 4]) + 7) // 8 * 8
        entry, rows = rng.choice(["gated", "gated_bwd"]), _log_int(rng, 1, 32768)
        if f == 3072 or rows * c * f * (3 if entry == "gated_bwd" else 1) > (32768 * 512 * 1368 if dtype != "f32" else 4096 * 320 * 1280):
            continue
        return _gated("", entry, rows, c, f, dtype, rng.choice(["silu", "gelu", "gelu_tanh"]), rng.random() < 0.5)


def _pairs(case):
    """For each rotated pair: its two channels, its axis (of the case's axes) and its rank among the axis's pairs, and how many these are."""
    first, second, axis, rank, count, at = [], [], [], [], [], 0
    for a, seg in enumerate([case["ct"], case["ch"], case["cw"]][3 - case["axes"]:]):
        half = seg // 2
        for j in range(half):
            first.append(at + (2 * j if case["pairs"] else j))
            second.append(at + (2 * j + 1 if case["pairs"] else j + half))
            axis.append(a)
            rank.append(j)
            count.append(half)
        at += seg
    return first, second, axis, rank, count


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(shape, std=1.0, mean=0.0, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dtype)

    s = {"case": c}
    if c["entry"].startswith("gated"):
        M, C, F = c["rows"], c["channels"], c["hidden"]
        # normalised activations, weights that keep their variance
        s["x"], s["wg"], s["wu"] = normal((M, C)), normal((F, C), C ** -0.5), normal((F, C), C ** -0.5)
        s["bg"], s["bu"] = (normal((F,), 0.1), normal((F,), 0.1)) if c["bias"] else (None, None)
        if c["entry"] == "gated_bwd":
            s["dh"] = normal((M, F))
        if own:
            s["mod"] = _handle(1, 1, 64, 1, dt)
        return s
    B, h, d, N = c["batch"], c["heads"], c["head_dim"], c["t"] * c["h"] * c["w"]
    if c["qkv"]:
        qkv = normal((B, N, 3, h, d))
        s["q"], s["k"] = (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(2))
    else:
        s["q"], s["k"] = normal((B, h, N, d)), normal((B, h, N, d))
    first, second, axis, rank, count = _pairs(c)
    s["first"], s["second"], s["axis"] = (torch.tensor(v, device="cuda") for v in (first, second, axis))
    # frequencies of each axis from one radian a step down to a hundredth
    s["freq"] = torch.tensor([100.0 ** (-j / n) for j, n in zip(rank, count)], dtype=torch.float32, device="cuda")
    t = torch.arange(N, device="cuda").expand(B if c["given"] else 1, N)
    w = torch.full((1, 1), c["w"], device="cuda")
    if c["given"]:        # an image's own width in each entry
        w = torch.randint(max(1, c["w"] // 2), c["w"] + 1, (B, 1), generator=g, device="cuda")
    grid = torch.stack([t // (w * c["h"]), t // w % c["h"], t % w], -1)[..., 3 - c["axes"]:].float().contiguous()
    s["grid"], s["positions"] = grid, grid if c["given"] else None
    s["gq"], s["gk"] = (normal((d,), 0.1, 1.0), normal((d,), 0.1, 1.0)) if c["norm"] else (None, None)
    if c["entry"] == "rotate_bwd":
        s["dq"], s["dk"] = (normal((B, h, N, d), dtype=torch.float32) for _ in range(2))
    if own:
        from paper_2312_08874_b200 import Rotary
        s["mod"] = _handle(B, h, d, N, dt)
        s["rotary"] = Rotary(s["freq"], [c["ct"], c["ch"], c["cw"]][3 - c["axes"]:], [c["t"], c["h"], c["w"]][3 - c["axes"]:],
                             positions=s["positions"], pairs=c["pairs"])
    return s


def _handle(batch, heads, head_dim, tokens, dtype):
    from paper_2312_08874_b200 import AgentAttention
    return AgentAttention(batch, heads, head_dim, tokens, 1, dtype)


def run(state):
    s, c = state, state["case"]
    if c["entry"] == "rotate":
        if own:
            q, k = s["mod"].rotate(s["q"], s["k"], s["rotary"], q_gain=s["gq"], k_gain=s["gk"], eps=EPS if c["norm"] else None)
            return {"q": q, "k": k}
        return {"q": _plain_rotate(s, s["q"], s["gq"]), "k": _plain_rotate(s, s["k"], s["gk"])}
    if c["entry"] == "rotate_bwd":
        if own:
            if not c["norm"]:
                return s["mod"].rotate_backward(s["dq"], s["dk"], s["rotary"])
            return s["mod"].rotate_backward(s["dq"], s["dk"], s["rotary"], q=s["q"], k=s["k"], q_gain=s["gq"], k_gain=s["gk"], eps=EPS)
        dq, dgq = _plain_rotate_bwd(s, s["dq"], s["q"], s["gq"])
        dk, dgk = _plain_rotate_bwd(s, s["dk"], s["k"], s["gk"])
        return {"dq": dq, "dk": dk, "dq_gain": dgq, "dk_gain": dgk} if c["norm"] else {"dq": dq, "dk": dk}
    args = {"b_gate": s["bg"], "b_up": s["bu"], "activation": c["act"]}
    if c["entry"] == "gated":
        return s["mod"].gated(s["x"], s["wg"], s["wu"], **args) if own else _plain_gated(s)
    return s["mod"].gated_backward(s["x"], s["wg"], s["wu"], s["dh"], **args) if own else _plain_gated_bwd(s)


def _turned(s, x, sign):
    angle = (s["grid"][:, :, s["axis"]] * s["freq"])[:, None]          # [1 or B, 1, N, pairs]
    cos, sin = torch.cos(angle), torch.sin(angle) * sign
    u, v = x[..., s["first"]], x[..., s["second"]]
    y = x.clone()
    y[..., s["first"]] = u * cos - v * sin
    y[..., s["second"]] = u * sin + v * cos
    return y


def _plain_rotate(s, x, gain):
    y = x.float()
    if gain is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain.float()
    return _turned(s, y, 1.0).to(x.dtype)


def _plain_rotate_bwd(s, g, x, gain):
    g = _turned(s, g, -1.0)
    if gain is None:
        return g, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh, gg = x * r, g * gain.float()
    return r * (gg - xh * (gg * xh).mean(-1, keepdim=True)), (g * xh).sum((0, 1, 2))


def _plain_act(act, g):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _plain_projections(s):
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    if s["bg"] is not None:
        g, u = g + s["bg"].float(), u + s["bu"].float()
    return x, wg, wu, g, u


def _plain_gated(s):
    x, wg, wu, g, u = _plain_projections(s)
    return (_plain_act(s["case"]["act"], g)[0] * u).to(s["x"].dtype)


def _plain_gated_bwd(s):
    x, wg, wu, g, u = _plain_projections(s)
    a, da = _plain_act(s["case"]["act"], g)
    dh = s["dh"].float()
    dg, du = dh * u * da, dh * a
    got = {"dx": dg @ wg + du @ wu, "dw_gate": dg.t() @ x, "dw_up": du.t() @ x}
    if s["bg"] is not None:
        got["db_gate"], got["db_up"] = dg.sum(0), du.sum(0)
    return {k: v.to(s["x"].dtype) for k, v in got.items()}


def exact(case, seed):
    s, c = prepare(case, seed), case
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if c["entry"].startswith("gated"):
        g = torch.nn.functional.linear(wide["x"], wide["wg"], wide.get("bg"))
        u = torch.nn.functional.linear(wide["x"], wide["wu"], wide.get("bu"))
        leaf = g.clone().requires_grad_()
        with torch.enable_grad():
            if c["act"] == "silu":
                a = torch.nn.functional.silu(leaf)
            else:
                a = torch.nn.functional.gelu(leaf, approximate="tanh" if c["act"] == "gelu_tanh" else "none")
        if c["entry"] == "gated":
            return a.detach() * u
        dh = wide["dh"]
        dg, = torch.autograd.grad(a, leaf, dh * u)
        du = dh * a.detach()
        out = {"dx": torch.cat([dg, du], 1) @ torch.cat([wide["wg"], wide["wu"]], 0), "dw_gate": torch.einsum("mf,mc->fc", dg, wide["x"]),
               "dw_up": torch.einsum("mf,mc->fc", du, wide["x"])}
        return dict(out, db_gate=dg.sum(0), db_up=du.sum(0)) if c["bias"] else out
    pos = s["grid"].double()
    phase = torch.stack([pos[..., a] * f for a, f in zip(s["axis"].tolist(), wide["freq"])], -1).unsqueeze(1)
    turn = torch.polar(torch.ones_like(phase), phase)

    def spin(x, turn):
        y = x.clone()
        z = torch.complex(x.index_select(-1, s["first"]).contiguous(), x.index_select(-1, s["second"]).contiguous()) * turn
        return y.index_copy_(-1, s["first"], z.real.contiguous()).index_copy_(-1, s["second"], z.imag.contiguous())

    def norm(x):
        return x / (x.pow(2).sum(-1, keepdim=True) / c["head_dim"] + EPS).sqrt()

    got = {}
    for n in ("q", "k"):
        x, gain = wide[n], wide.get("g" + n)
        if c["entry"] == "rotate":
            got[n] = spin(norm(x) * gain if c["norm"] else x, turn)
            continue
        back = spin(wide["d" + n], turn.conj())
        got["d" + n] = back
        if c["norm"]:
            leaf, lg = x.clone().requires_grad_(), gain.clone().requires_grad_()
            with torch.enable_grad():
                y = norm(leaf) * lg
            got["d" + n], got[f"d{n}_gain"] = torch.autograd.grad(y, (leaf, lg), back)
    return got


def work(case):
    c, es = case, 4 if case["dtype"] == "f32" else 2
    if c["entry"].startswith("gated"):
        M, C, F = c["rows"], c["channels"], c["hidden"]
        weights, bias = 2 * F * C * es, 2 * F * es if c["bias"] else 0
        if c["entry"] == "gated":
            return {"bytes": (M * C + M * F) * es + weights + bias, "flops": 4 * M * C * F}
        # reads X, the weights and dH, writes dX and the weights' gradients; both projections again, dX, dW
        return {"bytes": (2 * M * C + M * F) * es + 2 * weights + 2 * bias, "flops": 12 * M * C * F}
    N, d = c["t"] * c["h"] * c["w"], c["head_dim"]
    count = 2 * c["batch"] * c["heads"] * N * d                        # elements of Q and K
    small = (c["ct"] + c["ch"] + c["cw"]) * 2 + (c["batch"] * N * c["axes"] * 4 if c["given"] else 0) + (2 * d * es if c["norm"] else 0)
    if c["entry"] == "rotate":
        return {"bytes": 2 * count * es + small, "flops": count * (7 if c["norm"] else 3)}
    return {"bytes": count * (8 + (es if c["norm"] else 0)) + small + (8 * d if c["norm"] else 0), "flops": count * (14 if c["norm"] else 3)}
