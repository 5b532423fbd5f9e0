"""Which results of the gated feed-forward block count as apart from its inputs: columns of one buffer."""
import ctypes

import pytest
import torch

from paper_2312_08874_amd import binding
from tests.test_gated_ffn_cpu import A, bwd, desc, fwd


def test_columns_that_meet_are_refused():
    """Rows of 64 elements (bf16), 200 apart, of 12 rows; y starts inside x's columns, x inside y's, before or behind in memory."""
    d = desc(x_stride=200, y_stride=200, dx_stride=200)
    for off in (2, 126, -2, -126, 400 - 126, 400 + 126, -400 + 126, 5 * 400 + 64):
        assert fwd(d, y=A + off) == -6, off
        assert bwd(d, dx=A + off) == -6, off                   # x
        assert bwd(d, dx=9 * A + off) == -6, off               # dy
    d = desc(x_stride=200, y_stride=208)                       # no common period
    assert fwd(d, y=A + 128) == -6
    d = desc(x_stride=200, y_stride=200)
    assert fwd(d, y=2 * A + 128) == -6                         # inside a weight, which is one piece


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 200])
def test_columns_of_one_buffer(rows, dtype):
    """x, y, dy and dx side by side in one buffer: the bits of dense tensors, and nothing else written."""
    from tests.test_gpu_gated_ffn import inputs, run, weights
    s = inputs(dtype, rows, 72, 100, False)
    want = run(binding, s, "silu")
    buffer = torch.full((rows, 5 * 72), 7.0, dtype=s["x"].dtype, device="cuda")
    x, y, gap, dx, dy = buffer.split(72, dim=1)
    x.copy_(s["x"]), dy.copy_(s["dy"])
    _, saved = binding.agent_gated_ffn_fwd(x, **weights(s), save=True, out=y)
    assert torch.equal(y, want["y"])
    d, w = binding._ffn_call(x, s["w_gate"], s["w_up"], s["w_down"], None, None, None, "silu")
    d.y_stride = d.dx_stride = 5 * 72
    workspace = torch.empty(binding.lib().agent_gated_ffn_bwd_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device="cuda")
    status = binding.lib().agent_gated_ffn_bwd(
        ctypes.byref(d), x.data_ptr(), ctypes.byref(w), saved.data_ptr(), dy.data_ptr(), workspace.data_ptr(), workspace.numel(),
        dx.data_ptr(), ctypes.byref(binding.aa_ffn_grads()), torch.cuda.current_stream().cuda_stream)
    assert status == 0
    assert torch.equal(dx, want["dx"]) and torch.equal(x, s["x"]) and torch.equal(dy, s["dy"]) and bool((gap == 7.0).all())
