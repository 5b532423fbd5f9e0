"""NaN and infinities in fp32 softmax attention, whose operands are taken apart into bf16 terms where there are many queries: they reach what they
touch, as they do in the kernel of few queries, which takes fp32 as it is, and nothing else."""
import pytest
import torch

import __graft_entry__ as entry
from tests import softmax_reference as ref
from tests.test_gpu_softmax import close
from tests.test_gpu_softmax_edges import inputs, run


def test_terms_are_taken_where_nan_is_honoured():
    assert entry.unit_flags("csrc/softmax.hip") == [] and entry.unit_flags("csrc/softmax_f32.hip") == ["-fno-honor-nans"]


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=["nan", "inf", "-inf"])
@pytest.mark.parametrize("nq,nk,d", [(200, 200, 64), (150, 130, 128), (3, 2500, 64)], ids=["many", "wide", "few"])
def test_what_is_not_finite_reaches_what_it_touches(nq, nk, d, bad):
    q, k, v, g = inputs("f32", 1, 3, 3, nq, nk, d)
    want = ref.attention(q, k, v, False, ref.spans(1, nq, nk), do=g)
    row, key = nq // 2, nk // 3
    q[0, 0, row, 5], v[0, 1, key, 2], g[0, 2, row, 1] = bad, bad, bad
    out, grads = run(q, k, v, g)
    rows, keys, channels = torch.arange(nq) != row, torch.arange(nk) != key, torch.arange(d) != 2
    assert bool(torch.isnan(out[0, 0, row]).all())                  # q . k of either sign
    close(out[0, 0][rows], tuple(t[0, 0][rows] for t in want["out"]), "the other rows")
    assert bool((~torch.isfinite(out[0, 1, :, 2])).all())           # every row weighs the key
    close(out[0, 1][:, channels], tuple(t[0, 1][:, channels] for t in want["out"]), "the other channels")
    close(out[0, 2], tuple(t[0, 2] for t in want["out"]), "the head whose gradient alone is not finite")
    close(grads["dQ"][0, 2][rows], tuple(t[0, 2][rows] for t in want["dQ"]), "dQ of the other rows")
    assert bool((~torch.isfinite(grads["dQ"][0, 2, row])).any()) and bool((~torch.isfinite(grads["dV"][0, 2, :, 1])).all())
    assert bool((~torch.isfinite(grads["dK"][0, 2])).any())
