"""The gated feed-forward block where a value between its products, an input or a gate leaves the element type's range: a result
is within its bound (tests/ffn_reference.py) or no finite number, and never a finite number that is wrong."""
import pytest
import torch

from tests import ffn_reference as ref
from tests.test_gpu_gated_ffn import inputs, run

pytestmark = pytest.mark.gpu
ROWS = [1, 4, 5, 17, 64]      # of the kernels of few tokens; 300 rows of a small block beside them
HALF = {"f16": torch.float16, "bf16": torch.bfloat16}


def right(got, want, what):
    """Within the bound where the result is finite; returns which are."""
    value, bound = want
    got = got.double().reshape(value.shape)
    finite = torch.isfinite(got)
    off = torch.where(finite, (got - value).abs() - bound, torch.full_like(value, -1.0))
    assert bool((off <= 0).all()), "%s: off by %.3g more than allowed, at %d of %d" % (
        what, off.max(), int((off > 0).sum()), off.numel())
    return finite


@pytest.mark.parametrize("rows", ROWS + [300])
def test_gradient_of_down_where_h_is_beyond_the_largest_number(rows):
    """h of channel 5 is some 40000 to 500000, its rounding to fp16 partly infinite: so is the gradient there, and no other."""
    s = inputs("f16", rows, 8, 24, False)
    s["x"], s["dy"] = 0.5 + s["x"].abs().clamp(max=1.0), 0.01 * s["dy"]
    s["w_gate"][5] = s["w_up"][5] = 40.0
    s["w_down"][:, 5] = 0.001
    from paper_2312_08874_amd import binding
    want, got = ref.block(s, "relu"), run(binding, s, "relu")
    h = (s["x"].double() @ s["w_gate"].double().t()).clamp(min=0) * (s["x"].double() @ s["w_up"].double().t())
    beyond = bool((h[:, 5] > 65520).any())
    assert beyond and not bool((h.abs() > 65000)[:, torch.arange(24, device="cuda") != 5].any())
    finite = right(got["dw_down"], want["dw_down"], "dw_down")
    assert not bool(finite[:, 5].any()) and bool(finite[:, :5].all()) and bool(finite[:, 6:].all())
    for name in ("y", "dx", "dw_gate", "dw_up"):
        right(got[name], want[name], name)
