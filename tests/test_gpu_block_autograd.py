"""What autograd may ask of the transformer block beyond a backward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("part", ["attention", "feed_forward"])
def test_second_derivatives_are_refused(part):
    """The operators have no second derivative, so one that goes through them is an error, not a sum without their part."""
    from paper_2312_08874_amd.block import AgentBlock, _Attention, _FeedForward
    block = AgentBlock(32, 2, (4, 4), (2, 2), dtype=torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(1)
    if part == "attention":
        x = torch.randn(2, 16, 3, 2, 16, generator=gen, device="cuda", requires_grad=True)
        out = _Attention.apply(x, block.norm_q, block.norm_k, block.rope, block.eps, block.grids)
    else:
        x = torch.randn(2, 16, 32, generator=gen, device="cuda", requires_grad=True)
        out = _FeedForward.apply(x, block.w_gate, block.w_up, block.w_down, "silu")
    first, = torch.autograd.grad(out.square().sum(), x)      # once is what they are for
    again = _Attention.apply(x, block.norm_q, block.norm_k, block.rope, block.eps, block.grids) if part == "attention" else \
        _FeedForward.apply(x, block.w_gate, block.w_up, block.w_down, "silu")
    graph, = torch.autograd.grad(again.square().sum(), x, create_graph=True)
    assert torch.equal(graph.detach(), first)
    with pytest.raises(RuntimeError, match="differentiate twice"):      # a loss with a penalty on its gradient
        (again.sum() + graph.square().sum()).backward()
