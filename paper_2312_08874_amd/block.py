"""A transformer block of this package's operators, for inference and training, as an example of their use together:

    u = rms(x) w1;  q, k, v = slices of u Wqkv^T + bqkv;  q, k = normed for each head and rotated by their place on the grid
    y = x + (agent attention of q, k, v) Wout^T + bout
    z = y + gated feed-forward block of rms(y) w2

Matrix products and the norms over the whole width are torch's; everything between them is one call of the library, and
torch.autograd.Function ties its backward pass to autograd, once: a second derivative through them is an error.

    python -m paper_2312_08874_amd.block [--dtype bf16] [--batch 8] [--side 32] [--width 512] [--heads 8] [--steps 20]

trains one block on synthetic data (its output is to reproduce a fixed random linear map of its input) and prints the loss.
"""
import argparse
import math
import time

import torch
from torch.autograd.function import once_differentiable

from . import binding


class _Attention(torch.autograd.Function):
    """The fused projection's output [B,T,3,H,d] -> [B,T,H,d]: norm and rotation of q and k, then agent attention."""

    @staticmethod
    def forward(ctx, qkv, w_q, w_k, rope, eps, grids):
        q, k, v = (t.permute(0, 2, 1, 3) for t in qkv.unbind(2))
        turned = torch.empty_like(qkv)      # q, k and v share their strides: v goes along
        turned[:, :, 2] = qkv[:, :, 2]
        tq, tk, tv = (t.permute(0, 2, 1, 3) for t in turned.unbind(2))
        binding.agent_qk_norm_fwd(q, k, rope, weights=(w_q, w_k), eps=eps, out=(tq, tk))
        out = torch.empty_like(qkv[:, :, 0], memory_format=torch.contiguous_format)
        binding.agent_attn_fwd(tq, tk, tv, out=out.permute(0, 2, 1, 3), **grids)
        ctx.save_for_backward(qkv, w_q, w_k, turned)
        ctx.rope, ctx.eps, ctx.grids = rope, eps, grids
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        qkv, w_q, w_k, turned = ctx.saved_tensors
        q, k, _ = (t.permute(0, 2, 1, 3) for t in qkv.unbind(2))
        tq, tk, tv = (t.permute(0, 2, 1, 3) for t in turned.unbind(2))
        g = binding.agent_attn_bwd(tq, tk, tv, d_out.contiguous().permute(0, 2, 1, 3), **ctx.grids)
        d_qkv = torch.empty_like(qkv)
        dq, dk, dv = (t.permute(0, 2, 1, 3) for t in d_qkv.unbind(2))
        dv.copy_(g["dV"])
        w = binding.agent_qk_norm_bwd(q, k, g["dQ"], g["dK"], ctx.rope, weights=(w_q, w_k), eps=ctx.eps, out=(dq, dk))
        return d_qkv, w["dw_q"], w["dw_k"], None, None, None


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, activation):
        y, saved = binding.agent_gated_ffn_fwd(x, w_gate, w_up, w_down, activation=activation, save=True)
        ctx.save_for_backward(x, w_gate, w_up, w_down, saved)
        ctx.activation = activation
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, saved = ctx.saved_tensors
        g = binding.agent_gated_ffn_bwd(x, dy.contiguous(), saved, w_gate, w_up, w_down, activation=ctx.activation)
        return g["dx"], g["dw_gate"], g["dw_up"], g["dw_down"], None


def _rms(x, w, eps):
    v = x.float()
    return (v * (v.square().mean(-1, keepdim=True) + eps).rsqrt() * w).to(x.dtype)


class AgentBlock(torch.nn.Module):
    """x [B, T, width] -> [B, T, width]; T = the cells of `grid`.  hidden: of the feed-forward block (default 8/3 of the width)."""

    def __init__(self, width, heads, grid, agent_grid, *, hidden=None, activation="silu", base=10000.0, eps=1e-6, dtype=torch.bfloat16,
                 device="cuda", seed=0):
        super().__init__()
        d, hidden = width // heads, hidden or width * 8 // 3
        assert width % heads == 0 and d % 4 == 0, "heads of a multiple of four channels"
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=gen, device=device) / math.sqrt(cols)).to(dtype))

        def ones(n):
            return torch.nn.Parameter(torch.ones(n, device=device))
        self.heads, self.d, self.activation, self.eps = heads, d, activation, eps
        self.grids = dict(grid=tuple(grid), agent_grid=tuple(agent_grid))
        self.rope = binding.Rope((d // 4, d // 4), grid=grid, base=base)
        self.w_qkv, self.w_out = weight(3 * width, width), weight(width, width)
        self.b_qkv = torch.nn.Parameter(torch.zeros(3 * width, device=device, dtype=dtype))
        self.b_out = torch.nn.Parameter(torch.zeros(width, device=device, dtype=dtype))
        self.w_gate, self.w_up, self.w_down = weight(hidden, width), weight(hidden, width), weight(width, hidden)
        self.norm1, self.norm2, self.norm_q, self.norm_k = ones(width), ones(width), ones(d), ones(d)

    def forward(self, x):
        B, T, C = x.shape
        training = torch.is_grad_enabled()
        qkv = torch.nn.functional.linear(_rms(x, self.norm1, self.eps), self.w_qkv, self.b_qkv).view(B, T, 3, self.heads, self.d)
        if training:
            o = _Attention.apply(qkv, self.norm_q, self.norm_k, self.rope, self.eps, self.grids)
        else:      # q and k in place, where the projection wrote them
            q, k, v = (t.permute(0, 2, 1, 3) for t in qkv.unbind(2))
            binding.agent_qk_norm_fwd(q, k, self.rope, weights=(self.norm_q, self.norm_k), eps=self.eps, out=(q, k))
            o = torch.empty(B, T, self.heads, self.d, dtype=x.dtype, device=x.device)
            binding.agent_attn_fwd(q, k, v, out=o.permute(0, 2, 1, 3), **self.grids)
        y = x + torch.nn.functional.linear(o.view(B, T, C), self.w_out, self.b_out)
        u = _rms(y, self.norm2, self.eps)
        if training:
            return y + _FeedForward.apply(u, self.w_gate, self.w_up, self.w_down, self.activation)
        return y + binding.agent_gated_ffn_fwd(u, self.w_gate, self.w_up, self.w_down, activation=self.activation)


def main():
    p = argparse.ArgumentParser(description="Trains one transformer block on synthetic data.")
    p.add_argument("--dtype", default="bf16", choices=("bf16", "f16", "f32"))
    for name, value in (("batch", 8), ("side", 32), ("agents", 7), ("width", 512), ("heads", 8), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    dtype = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[a.dtype]
    block = AgentBlock(a.width, a.heads, (a.side, a.side), (a.agents, a.agents), dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.batch, a.side * a.side, a.width, generator=gen, device="cuda").to(dtype)
    target = x.float() @ (torch.randn(a.width, a.width, generator=gen, device="cuda") / math.sqrt(a.width))
    optimizer = torch.optim.AdamW(block.parameters(), lr=1e-3)
    for step in range(a.steps):
        torch.cuda.synchronize()
        start = time.perf_counter()
        loss = (block(x).float() - target).square().mean()
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        torch.cuda.synchronize()
        print("step %3d  loss %.4f  %.2f ms" % (step, loss.item(), 1e3 * (time.perf_counter() - start)), flush=True)
    with torch.no_grad():
        print("inference loss %.4f" % (block(x).float() - target).square().mean().item())


if __name__ == "__main__":
    main()
