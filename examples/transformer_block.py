"""A transformer block on a token grid whose operators come from this package: norms of queries and keys with rotary positions, Agent Attention, the
gated feed-forward product.  The projections, residuals and the norms of the channels are plain torch.

    python examples/transformer_block.py            # inference and training steps of a 56 x 56 grid, 8 heads of 64 channels

`Block.infer` prepares queries and keys in place, inside the fused projection's output, from where the attention reads them.  `Block.forward` is the same
block for training: three `torch.autograd.Function`s around the package's forward and backward calls.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2312_08874_b200 import AgentAttention, Rotary  # noqa: E402


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, block, q, k, q_gain, k_gain):
        ctx.block = block
        ctx.save_for_backward(q, k, q_gain, k_gain)
        return block.mod.rotate(q, k, block.rotary, q_gain=q_gain, k_gain=k_gain, eps=block.eps)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, q_gain, k_gain = ctx.saved_tensors
        g = ctx.block.mod.rotate_backward(dq.float(), dk.float(), ctx.block.rotary, q=q, k=k, q_gain=q_gain, k_gain=k_gain, eps=ctx.block.eps)
        return None, g["dq"].to(q.dtype), g["dk"].to(k.dtype), g["dq_gain"].to(q.dtype), g["dk_gain"].to(k.dtype)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, block, q, k, v, dwc):
        ctx.block = block
        ctx.save_for_backward(q, k, v, dwc)
        return block.mod.forward(q, k, v, block.grid_h, block.grid_w, block.agents, dwc_weight=dwc)

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, dwc = ctx.saved_tensors
        b = ctx.block
        g = b.mod.backward(q, k, v, d_out.contiguous(), b.grid_h, b.grid_w, b.agents, dwc_weight=dwc)
        return None, g["dq"].to(q.dtype), g["dk"].to(q.dtype), g["dv"].to(q.dtype), g["dwd"].to(q.dtype)


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, block, x, w_gate, w_up):
        ctx.block = block
        ctx.save_for_backward(x, w_gate, w_up)
        return block.mod.gated(x, w_gate, w_up, activation=block.activation)

    @staticmethod
    def backward(ctx, d_out):
        x, w_gate, w_up = ctx.saved_tensors
        g = ctx.block.mod.gated_backward(x, w_gate, w_up, d_out.contiguous(), activation=ctx.block.activation)
        return None, g["dx"], g["dw_gate"], g["dw_up"]


class Block(torch.nn.Module):
    def __init__(self, batch, heads, head_dim, grid_h, grid_w, pool, hidden, dtype=torch.bfloat16, activation="silu", seed=0):
        super().__init__()
        self.grid_h, self.grid_w, self.agents, self.activation, self.eps = grid_h, grid_w, pool * pool, activation, 1e-6
        self.shape = (batch, grid_h * grid_w, heads, head_dim)
        C = heads * head_dim
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols, std=None):
            return torch.nn.Parameter((torch.randn((rows, cols), generator=g) * (cols ** -0.5 if std is None else std)).to(dtype).cuda())
        self.w_qkv, self.w_out = weight(3 * C, C), weight(C, C)
        self.w_gate, self.w_up, self.w_down = weight(hidden, C), weight(hidden, C), weight(C, hidden)
        self.q_gain, self.k_gain = (torch.nn.Parameter(torch.ones(head_dim, dtype=dtype, device="cuda")) for _ in range(2))
        self.dwc = torch.nn.Parameter(weight(heads * head_dim, 9, 0.1).detach().view(heads, head_dim, 3, 3))
        half = head_dim // 4 * 2                                         # channels of the rows, and of the columns
        self.rotary = Rotary(Rotary.frequencies((half, half)), (half, half), (grid_h, grid_w))
        self.mod = AgentAttention(batch, heads, head_dim, grid_h * grid_w, self.agents, dtype)

    def _norm(self, x):
        return torch.nn.functional.rms_norm(x, x.shape[-1:], eps=self.eps)

    def _views(self, x):
        B, N, h, d = self.shape
        qkv = torch.nn.functional.linear(self._norm(x), self.w_qkv).view(B, N, 3, h, d)
        return (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3))

    @torch.no_grad()
    def infer(self, x):
        B, N, h, d = self.shape
        q, k, v = self._views(x)
        self.mod.rotate(q, k, self.rotary, q_gain=self.q_gain, k_gain=self.k_gain, eps=self.eps, out=(q, k))
        a = self.mod.forward_strided(q, k, v, self.grid_h, self.grid_w, self.agents, dwc_weight=self.dwc)
        x = x + torch.nn.functional.linear(a.permute(0, 2, 1, 3).reshape(B, N, h * d), self.w_out)
        return x + torch.nn.functional.linear(self.mod.gated(self._norm(x), self.w_gate, self.w_up, activation=self.activation), self.w_down)

    def forward(self, x):
        B, N, h, d = self.shape
        q, k, v = self._views(x)
        q, k = _Rotate.apply(self, q, k, self.q_gain, self.k_gain)
        a = _Attention.apply(self, q, k, v.contiguous(), self.dwc)
        x = x + torch.nn.functional.linear(a.permute(0, 2, 1, 3).reshape(B, N, h * d), self.w_out)
        return x + torch.nn.functional.linear(_Gated.apply(self, self._norm(x), self.w_gate, self.w_up), self.w_down)


def main():
    batch, heads, head_dim, side, pool = 2, 8, 64, 56, 7
    block = Block(batch, heads, head_dim, side, side, pool, hidden=1368)
    optimizer = torch.optim.SGD(block.parameters(), lr=20.0)
    x, target = (torch.randn((batch, side * side, heads * head_dim), device="cuda").bfloat16() for _ in range(2))
    for step in range(5):
        loss = (block(x).float() - target.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        print(f"step {step}: loss {loss.item():.4f}")
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for i in range(25):
        if i == 5:
            start.record()
        block.infer(x)
    end.record()
    end.synchronize()
    print(f"inference: {start.elapsed_time(end) / 20 * 1e3:.1f} us a block, status {block.mod.query_status()}")


if __name__ == "__main__":
    main()
