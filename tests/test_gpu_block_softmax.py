"""The transformer block with softmax attention and with layer norms against the same block in 64 bits on the host, with autograd's
gradients.  Tolerances: test_gpu_block, whose count of roundings one behind the other these blocks keep below (the attention rounds
its weights and its result, a layer norm its result and its sum)."""
import pytest
import torch

from tests.rotary_reference import rotate
from tests.test_gpu_block import off

pytestmark = pytest.mark.gpu


def reference(block, x, grid, agent_grid):
    w = {n: p.detach().cpu().double().requires_grad_() for n, p in block.named_parameters()}
    B, T, C = x.shape
    H, d, eps = block.heads, block.d, block.eps

    def rms(v, g):
        return v / (v.square().mean(-1, keepdim=True) + eps).sqrt() * g

    def norm(v, name):
        if not block.layer:
            return rms(v, w[name])
        c = v - v.mean(-1, keepdim=True)
        return rms(c, w[name]) + w[name + "_b"]
    qkv = (norm(x, "norm1") @ w["w_qkv"].t() + w["b_qkv"]).view(B, T, 3, H, d).permute(2, 0, 3, 1, 4)
    p = d // 4
    spec = dict(pairs=(p, p), pairing="halves", grid=grid, freqs=[10000.0 ** (-j / p) for j in range(p)] * 2)
    q, k, v = rotate(rms(qkv[0], w["norm_q"]), spec), rotate(rms(qkv[1], w["norm_k"]), spec), qkv[2]
    if agent_grid is None:
        o = torch.softmax(q @ k.transpose(-1, -2) * d ** -0.5, -1) @ v
    else:
        image = q.reshape(B * H, *grid, d).permute(0, 3, 1, 2)
        a = torch.nn.functional.adaptive_avg_pool2d(image, agent_grid).flatten(2).transpose(1, 2).reshape(B, H, -1, d)
        va = torch.softmax(a @ k.transpose(-1, -2) * d ** -0.5, -1) @ v
        o = torch.softmax(q @ a.transpose(-1, -2) * d ** -0.5, -1) @ va
    y = x + o.permute(0, 2, 1, 3).reshape(B, T, C) @ w["w_out"].t() + w["b_out"]
    u = norm(y, "norm2")
    g = u @ w["w_gate"].t()
    return y + (g * torch.sigmoid(g) * (u @ w["w_up"].t())) @ w["w_down"].t(), w


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("attention,norm", [("softmax", "rms"), ("softmax", "layer"), ("agent", "layer")])
def test_block_and_its_gradients(attention, norm, dtype):
    from paper_2312_08874_amd.block import AgentBlock
    grid, agent_grid = (9, 7), (3, 3) if attention == "agent" else None
    block = AgentBlock(96, 3, grid, agent_grid, dtype=dtype, attention=attention, norm=norm)
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(2, 63, 96, generator=gen).to(dtype)
    dz = torch.randn(2, 63, 96, generator=gen).to(dtype)
    with torch.no_grad():
        for name, p in block.named_parameters():
            if name.startswith("norm"):
                p.add_(0.2 * torch.randn(p.shape, generator=gen).cuda())
    x64 = x.double().requires_grad_()
    want, leaves = reference(block, x64, grid, agent_grid)
    want.backward(dz.double())
    xg = x.cuda().requires_grad_()
    got = block(xg)
    got.backward(dz.cuda())
    one = 2 * (torch.finfo(dtype).eps / 2 + (260 * 2.0 ** -24))
    assert off(got, want) <= 12 * one
    assert off(xg.grad, x64.grad) <= 24 * one
    for name, p in block.named_parameters():
        assert off(p.grad, leaves[name].grad) <= 24 * one, name
    with torch.no_grad():
        assert off(block(x.cuda()), want) <= 12 * one


def test_gradients_are_the_loss_differences():
    """A step of t along the gradient and back changes the loss by 2 t times its length, but for a share of (t / the weights' length of 8
    and more)^2 < 1e-5.  The loss adds 6912 values of about 2, each off by up to 2^-18 of it in fp32; at random these come to 83 x 2^-17
    < 7e-4, and t = 2^-6 times lengths of over 5 makes steps of over 0.15."""
    from paper_2312_08874_amd.block import AgentBlock
    block = AgentBlock(64, 2, (6, 6), dtype=torch.float32, attention="softmax", norm="layer", seed=1)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, c = (torch.randn(3, 36, 64, generator=gen, device="cuda") for _ in range(2))

    def loss():
        return (block(x).double() * c).sum()
    loss().backward()
    t = 2.0 ** -6
    for name in ("w_qkv", "norm1", "norm2_b", "w_out", "w_gate"):
        p = dict(block.named_parameters())[name]
        assert p.grad.norm() > 5, name
        way = p.grad / p.grad.norm()
        with torch.no_grad():
            p.add_(way, alpha=t)
            up = loss()
            p.sub_(way, alpha=2 * t)
            down = loss()
            p.add_(way, alpha=t)
        assert abs((up - down).item() / (2 * t) / p.grad.norm().item() - 1) < 1e-2, name


def test_second_derivatives_are_refused():
    from paper_2312_08874_amd.block import AgentBlock, _Attention, _LayerNorm
    block = AgentBlock(32, 2, (4, 4), dtype=torch.float32, attention="softmax", norm="layer")
    gen = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randn(2, 16, 3, 2, 16, generator=gen, device="cuda", requires_grad=True)
    b = torch.randn(2, 16, 32, generator=gen, device="cuda", requires_grad=True)
    for x, call in ((a, lambda: _Attention.apply(a, block.norm_q, block.norm_k, block.rope, block.eps, None)),
                    (b, lambda: _LayerNorm.apply(b, None, block.norm1, block.norm1_b, 1e-5))):
        first, = torch.autograd.grad(call().square().sum(), x)
        again = call()
        graph, = torch.autograd.grad(again.square().sum(), x, create_graph=True)
        assert torch.equal(graph.detach(), first)
        with pytest.raises(RuntimeError, match="differentiate twice"):
            (again.sum() + graph.square().sum()).backward()


def test_arguments():
    from paper_2312_08874_amd.block import AgentBlock
    with pytest.raises(AssertionError):
        AgentBlock(32, 2, (4, 4))
    with pytest.raises(AssertionError):
        AgentBlock(32, 2, (4, 4), (2, 2), attention="linear")
    with pytest.raises(AssertionError):
        AgentBlock(32, 2, (4, 4), (2, 2), norm="batch")
