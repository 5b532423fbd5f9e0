"""Norm and rotation of queries without keys: nothing of the keys' is looked at, in any shape of the launch."""
import ctypes

import pytest
import torch

from paper_2312_08874_amd import binding

pytestmark = pytest.mark.gpu


def _ref(t):
    return ctypes.byref(binding.aa_view(t.data_ptr(), 0, 0, 0))


@pytest.mark.parametrize("heads", [1, 2, 3, 5, 9])
def test_weights_of_keys_that_are_not_there(heads):
    """w_k names the results' own memory (w_k is no input without keys, so no alias), where reading it would be seen: it holds NaN."""
    gen = torch.Generator(device="cuda").manual_seed(heads)
    q, dy = (torch.randn(2, heads, 37, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = 1 + 0.1 * torch.randn(64, generator=gen, device="cuda")
    want, = binding.agent_qk_norm_fwd(q, None, weights=(w, None))[:1]
    grads = binding.agent_qk_norm_bwd(q, None, dy, None, weights=(w, None))
    d = binding.aa_rotary(batch=2, tokens=37, heads_q=heads, heads_k=0, d=64, dtype=binding.AA_BF16)
    L, stream = binding.lib(), torch.cuda.current_stream().cuda_stream
    out = torch.full_like(q, float("nan"))
    norm = binding.aa_qk_norm(w.data_ptr(), out.data_ptr(), 0, 1e-6)
    assert L.agent_qk_norm_fwd(ctypes.byref(d), ctypes.byref(norm), _ref(q), None, _ref(out), None, stream) == 0
    assert torch.equal(out, want)
    dq, dw = torch.full_like(q, float("nan")), torch.empty_like(w)
    norm = binding.aa_qk_norm(w.data_ptr(), dq.data_ptr(), 0, 1e-6)
    need = L.agent_qk_norm_bwd_workspace_bytes(ctypes.byref(d), ctypes.byref(norm))
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert L.agent_qk_norm_bwd(ctypes.byref(d), ctypes.byref(norm), _ref(q), None, _ref(dy), None, workspace.data_ptr(), need, _ref(dq),
                               None, dw.data_ptr(), None, stream) == 0
    assert torch.equal(dq, grads["dq"]) and torch.equal(dw, grads["dw_q"])
