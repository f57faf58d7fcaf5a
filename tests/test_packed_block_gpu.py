"""The example block of packed images: its operators together, inference and training form against the formulas in 64 bits, and each image by itself.

Tolerances: some fourteen roundings to bf16 stand between input and result (relative 1.7e-3 each in the 2-norm, added as squares: 6e-3, and what the residual keeps
of them less), with a factor of two: 1.2e-2; gradients pass twice as many and the rounded slopes of the attention: 3e-2.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_block.py")


def load():
    spec = importlib.util.spec_from_file_location("packed_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(block, packing, x, p):
    h, d, half = block.heads, block.head_dim, block.half
    T = x.shape[0]
    norm = lambda t, w, b: (t - t.mean(-1, keepdim=True)) / (t.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt() * w + b  # noqa: E731
    q, k, v = (norm(x, p["norm1_w"], p["norm1_b"]) @ p["w_qkv"].T).view(T, 3, h, d).permute(1, 2, 0, 3)
    freq, place = block.freq.double(), packing.positions[0].double()
    angle = torch.cat([place[:, :1] * freq[:half // 2], place[:, 1:] * freq[half // 2:]], 1)

    def turn(y):
        parts = []
        for a in range(2):
            u, w = y[..., a * half:a * half + half // 2], y[..., a * half + half // 2:(a + 1) * half]
            c, s = angle[:, a * half // 2:(a + 1) * half // 2].cos(), angle[:, a * half // 2:(a + 1) * half // 2].sin()
            parts += [u * c - w * s, u * s + w * c]
        return torch.cat(parts + [y[..., 2 * half:]], -1)
    q, k = turn(q), turn(k)
    at = packing.offsets.tolist()
    o = torch.cat([torch.softmax(q[:, a:b] @ k[:, a:b].transpose(-1, -2) * d ** -0.5, -1) @ v[:, a:b] for a, b in zip(at, at[1:])], 1)
    x = x + o.transpose(0, 1).reshape(T, h * d) @ p["w_out"].T
    y = norm(x, p["norm2_w"], p["norm2_b"])
    g = y @ p["w_gate"].T
    return x + (g * torch.sigmoid(g) * (y @ p["w_up"].T)) @ p["w_down"].T


def test_block_matches_the_formulas():
    m = load()
    grids = [(9, 14), (1, 1), (16, 16), (3, 50)]
    packing = m.Packing(grids)
    block = m.Block(4, 64, 688, packing.tokens)
    with torch.no_grad():
        for t in (block.norm1_w, block.norm2_w, block.norm1_b, block.norm2_b):
            t += 0.2 * torch.randn(t.shape, generator=torch.Generator().manual_seed(5)).to(t)
    x = torch.randn((packing.tokens, 256), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    leaf = x.clone().requires_grad_()
    out, inferred = block(leaf, packing), block.infer(x, packing)
    weight = torch.randn(out.shape, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    out.backward(weight)
    wide = {n: t.detach().double().requires_grad_() for n, t in block.named_parameters()}
    xd = x.double().requires_grad_()
    ref = reference(block, packing, xd, wide)
    ref.backward(weight.double())
    rel = lambda a, b: float((a.detach().double() - b.detach()).norm() / b.detach().norm())  # noqa: E731
    assert rel(out, ref) <= 1.2e-2 and rel(inferred, ref) <= 1.2e-2
    assert rel(leaf.grad, xd.grad) <= 3e-2
    for n, t in block.named_parameters():
        assert rel(t.grad, wide[n].grad) <= 3e-2, n
    # an image alone is what it is among others
    at = packing.offsets.tolist()
    for i, g in enumerate(grids):
        alone = block.infer(x[at[i]:at[i + 1]].clone(), m.Packing([g]))
        assert rel(alone, inferred[at[i]:at[i + 1]].double()) <= 5e-3
    assert block.mod.query_status() == 0


def test_example_runs(capsys):
    load().main()
    text = capsys.readouterr().out
    assert text.count("step") == 3 and "nan" not in text and "status 0" in text
