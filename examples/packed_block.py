"""A transformer block on images of any sizes, one after the other in one sequence of tokens: layer norms, rotary positions, softmax attention inside
each image, the gated feed-forward product, all of this package.  The projections and residuals are plain torch.

    python examples/packed_block.py            # training steps and inference on 12 images of up to 48 x 48 tokens

`Block.infer` uses the package's calls directly; `Block.forward` is the same block for training, `torch.autograd.Function`s around the forward and backward calls.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2312_08874_b200 import AgentAttention, Rotary  # noqa: E402


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, mod, x, weight, bias):
        ctx.mod = mod
        ctx.save_for_backward(x, weight, bias)
        return mod.layer_norm(x, weight, bias)

    @staticmethod
    def backward(ctx, d_out):
        x, weight, bias = ctx.saved_tensors
        g = ctx.mod.layer_norm_backward(x, d_out.contiguous(), weight, bias)
        return None, g["dx"], g["dw"].to(weight.dtype), g["db"].to(bias.dtype)


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, mod, rotary, q, k):
        ctx.mod, ctx.rotary, ctx.dtype = mod, rotary, q.dtype
        return mod.rotate(q, k, rotary)

    @staticmethod
    def backward(ctx, dq, dk):
        g = ctx.mod.rotate_backward(dq.float().contiguous(), dk.float().contiguous(), ctx.rotary)
        return None, None, g["dq"].to(ctx.dtype), g["dk"].to(ctx.dtype)


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, mod, offsets, q, k, v):
        out, lse = mod.attend(q, k, v, q_offsets=offsets, need_lse=True)
        ctx.mod, ctx.offsets = mod, offsets
        ctx.save_for_backward(q, k, v, out, lse)
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, out, lse = ctx.saved_tensors
        g = ctx.mod.attend_backward(q, k, v, out, lse, d_out.contiguous(), q_offsets=ctx.offsets)
        return None, None, g["dq"], g["dk"], g["dv"]


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, mod, x, w_gate, w_up):
        ctx.mod = mod
        ctx.save_for_backward(x, w_gate, w_up)
        return mod.gated(x, w_gate, w_up)

    @staticmethod
    def backward(ctx, d_out):
        x, w_gate, w_up = ctx.saved_tensors
        g = ctx.mod.gated_backward(x, w_gate, w_up, d_out.contiguous())
        return None, g["dx"], g["dw_gate"], g["dw_up"]


class Packing:
    """Where the tokens of images of the given grids lie: offsets of the images, positions of the tokens."""

    def __init__(self, grids):
        at, places = [0], []
        for h, w in grids:
            at.append(at[-1] + h * w)
            t = torch.arange(h * w)
            places.append(torch.stack([t // w, t % w], 1))
        self.tokens = at[-1]
        self.offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
        self.positions = torch.cat(places)[None].float().cuda()


class Block(torch.nn.Module):
    def __init__(self, heads, head_dim, hidden, max_tokens, dtype=torch.bfloat16, seed=0):
        super().__init__()
        C = heads * head_dim
        self.heads, self.head_dim = heads, head_dim
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return torch.nn.Parameter((torch.randn((rows, cols), generator=g) * cols ** -0.5).to(dtype).cuda())
        self.w_qkv, self.w_out = weight(3 * C, C), weight(C, C)
        self.w_gate, self.w_up, self.w_down = weight(hidden, C), weight(hidden, C), weight(C, hidden)
        self.norm1_w, self.norm2_w = (torch.nn.Parameter(torch.ones(C, dtype=dtype, device="cuda")) for _ in range(2))
        self.norm1_b, self.norm2_b = (torch.nn.Parameter(torch.zeros(C, dtype=dtype, device="cuda")) for _ in range(2))
        self.half = head_dim // 4 * 2                                    # channels of the rows, and of the columns
        self.freq = Rotary.frequencies((self.half, self.half))
        self.mod = AgentAttention(1, heads, head_dim, max_tokens, 1, dtype)

    def rotary(self, packing):
        return Rotary(self.freq, (self.half, self.half), positions=packing.positions)

    def _views(self, x):
        qkv = torch.nn.functional.linear(x, self.w_qkv).view(1, x.shape[0], 3, self.heads, self.head_dim)
        return (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3))

    @torch.no_grad()
    def infer(self, x, packing):
        """x: [tokens, channels]."""
        mod, (q, k, v) = self.mod, self._views(self.mod.layer_norm(x, self.norm1_w, self.norm1_b))
        mod.rotate(q, k, self.rotary(packing), out=(q, k))               # in place, inside the fused projection's output
        a = mod.attend(q, k, v, q_offsets=packing.offsets)
        x = x + torch.nn.functional.linear(a.permute(0, 2, 1, 3).reshape(x.shape), self.w_out)
        return x + torch.nn.functional.linear(mod.gated(mod.layer_norm(x, self.norm2_w, self.norm2_b), self.w_gate, self.w_up), self.w_down)

    def forward(self, x, packing):
        mod, (q, k, v) = self.mod, self._views(_Norm.apply(self.mod, x, self.norm1_w, self.norm1_b))
        q, k = _Rotate.apply(mod, self.rotary(packing), q, k)
        a = _Attend.apply(mod, packing.offsets, q, k, v)
        x = x + torch.nn.functional.linear(a.permute(0, 2, 1, 3).reshape(x.shape), self.w_out)
        return x + torch.nn.functional.linear(_Gated.apply(mod, _Norm.apply(mod, x, self.norm2_w, self.norm2_b), self.w_gate, self.w_up), self.w_down)


def main():
    grids = [(48, 48), (30, 40), (17, 23), (48, 20)] * 3
    packing = Packing(grids)
    block = Block(8, 64, hidden=1368, max_tokens=packing.tokens)
    optimizer = torch.optim.SGD(block.parameters(), lr=1.0)
    x, target = (torch.randn((packing.tokens, 512), device="cuda").bfloat16() for _ in range(2))
    for step in range(3):
        loss = (block(x, packing).float() - target.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        print(f"step {step}: loss {loss.item():.4f}")
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for i in range(25):
        if i == 5:
            start.record()
        block.infer(x, packing)
    end.record()
    end.synchronize()
    print(f"inference: {start.elapsed_time(end) / 20 * 1e3:.1f} us a block of {packing.tokens} tokens, status {block.mod.query_status()}")


if __name__ == "__main__":
    main()
