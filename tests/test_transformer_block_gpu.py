"""The example block: its operators together, inference against training form and both against the formulas in 64 bits.

Tolerances: some ten roundings to bf16 stand between input and result (relative 1.7e-3 each in the 2-norm, added as squares: 5e-3, and what the
residual keeps of them less), the attention's gradients 1e-2 (its own tests); the sum of both in squares, with a factor of two: 1e-2 and 3e-2.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "transformer_block.py")


def load():
    spec = importlib.util.spec_from_file_location("transformer_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(block, x, p):
    B, N, h, d = block.shape
    H, W, n = block.grid_h, block.grid_w, block.agents
    rms = lambda t: t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    q, k, v = (rms(x) @ p["w_qkv"].T).view(B, N, 3, h, d).permute(2, 0, 3, 1, 4)
    t = torch.arange(N, device="cuda")
    half = d // 4 * 2
    freq = block.rotary.freq.double()
    angle = torch.cat([(t // W)[:, None] * freq[:half // 2], (t % W)[:, None] * freq[half // 2:]], 1)

    def turn(y):
        parts = []
        for a in range(2):
            u, w = y[..., a * half:a * half + half // 2], y[..., a * half + half // 2:(a + 1) * half]
            c, s = angle[:, a * half // 2:(a + 1) * half // 2].cos(), angle[:, a * half // 2:(a + 1) * half // 2].sin()
            parts += [u * c - w * s, u * s + w * c]
        return torch.cat(parts + [y[..., 2 * half:]], -1)
    q, k = turn(rms(q) * p["q_gain"]), turn(rms(k) * p["k_gain"])
    pool = int(n ** 0.5)
    agents = torch.nn.functional.adaptive_avg_pool2d(q.reshape(B * h, H, W, d).permute(0, 3, 1, 2), pool).flatten(2).transpose(1, 2).view(B, h, n, d)
    va = torch.softmax(agents @ k.transpose(-1, -2) * d ** -0.5, -1) @ v
    o = torch.softmax(q @ agents.transpose(-1, -2) * d ** -0.5, -1) @ va
    image = v.permute(0, 1, 3, 2).reshape(B, h * d, H, W)
    o = o + torch.nn.functional.conv2d(image, p["dwc"].view(h * d, 1, 3, 3), padding=1, groups=h * d).view(B, h, d, N).transpose(-1, -2)
    x = x + o.transpose(1, 2).reshape(B, N, h * d) @ p["w_out"].T
    y = rms(x)
    g = y @ p["w_gate"].T
    return x + (g * torch.sigmoid(g) * (y @ p["w_up"].T)) @ p["w_down"].T


def test_block_matches_the_formulas():
    m = load()
    block = m.Block(2, 2, 64, 16, 16, 4, hidden=344)
    x = torch.randn((2, 256, 128), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    leaf = x.clone().requires_grad_()
    out = block(leaf)
    inferred = block.infer(x)
    weight = torch.randn(out.shape, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    out.backward(weight)
    wide = {n: t.detach().double().requires_grad_() for n, t in block.named_parameters()}
    xd = x.double().requires_grad_()
    ref = reference(block, xd, wide)
    ref.backward(weight.double())
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(out, ref) <= 1e-2 and rel(inferred, ref) <= 1e-2
    assert rel(leaf.grad, xd.grad) <= 3e-2
    for n, t in block.named_parameters():
        assert rel(t.grad, wide[n].grad) <= 3e-2, n
    assert block.mod.query_status() == 0


def test_example_runs(capsys):
    load().main()
    text = capsys.readouterr().out
    losses = [float(line.split()[-1]) for line in text.splitlines() if line.startswith("step")]
    assert len(losses) == 5 and losses[-1] < losses[0] and "status 0" in text


def test_results_on_another_stream_take_no_memory_in_use():
    """A tensor freed while work of the current stream has yet to read it: a call on another stream does not get its memory for results or workspace."""
    from paper_2312_08874_b200 import AgentAttention, Rotary
    M, C, F, B, h, N, d = 512, 320, 1280, 4, 8, 256, 64
    mod = AgentAttention(B, h, d, N, 1, torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, wg, wu, dh = ((torch.randn(s, generator=gen, device="cuda") * f).bfloat16() for s, f in (((M, C), 1.0), ((F, C), C ** -0.5), ((F, C), C ** -0.5), ((M, F), 1.0)))
    q, k = (torch.randn((B, h, N, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    gq, gk = q.float(), k.float()
    gain = torch.ones(d, device="cuda").bfloat16()
    rotary = Rotary(Rotary.frequencies((32, 32)), (32, 32), (16, 16))
    norm = dict(q_gain=gain, k_gain=gain, eps=1e-6)
    calls = [(lambda s: [mod.gated(x, wg, wu, stream=s)], [(M, F)]),
             (lambda s: list(mod.gated_backward(x, wg, wu, dh, stream=s).values()), [(M, C), (F, C), (F, C)]),
             (lambda s: list(mod.rotate(q, k, rotary, stream=s, **norm)), [(B, h, N, d)] * 2),
             (lambda s: list(mod.rotate_backward(gq, gk, rotary, q=q, k=k, stream=s, **norm).values()), [(B, h, N, 2 * d)] * 2)]
    side = torch.cuda.Stream()
    for call, shapes in calls:
        want = call(None)
        victims = [torch.randn(s, device="cuda").bfloat16() for s in shapes for _ in range(2)] + [torch.randn(1 << n, device="cuda").bfloat16() for n in (16, 20, 23)]
        kept, read = [v.clone() for v in victims], [torch.empty_like(v) for v in victims]
        torch.cuda.synchronize()
        torch.cuda._sleep(30_000_000)                        # 15 ms and more, in which the call below ends
        for r, v in zip(read, victims):
            r.copy_(v)
        del v, victims
        got = call(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(read, kept)) and all(torch.equal(a, b) for a, b in zip(got, want))
