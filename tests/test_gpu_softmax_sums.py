"""What the forward pass of softmax attention sums its weights to: lse of rows that see few keys, in calls that take the keys in ranges.

The bound is softmax_reference's without u: a row all of whose tiles are the first of a wave is summed in fp32 before it is rounded.  That
sum, what rounding took (a difference of two sums) and their total are off by (3 n + 20) e, scores by a, and the logarithm with its
reference by 2 e |lse| and, at 16 powers of two at the most, 32 e."""
import pytest
import torch

from tests import softmax_reference as ref
from tests.test_gpu_softmax import ints
from tests.test_gpu_softmax_edges import inputs

pytestmark = pytest.mark.gpu
E = ref.E


def lse_of(saved, out):
    return saved[:4 * out[..., 0].numel()].view(torch.float32).view(out.shape[:3]).double().cpu()


# B, Hq, Hk, queries, keys, d; lengths of the keys or None (causal)
RANGES = [(1, 4, 4, 2048, 2048, 64, None), (1, 2, 2, 1700, 1700, 32, None), (2, 8, 4, 3, 4000, 64, [200, 2]), (1, 2, 1, 1, 3000, 128, [5])]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", RANGES, ids=lambda c: "x".join(map(str, c[:6])))
def test_lse_of_rows_with_few_keys_in_ranges(case, dtype):
    from paper_2312_08874_amd import binding
    B, Hq, Hk, nq, nk, d, lengths = case
    q, k, v, _ = inputs(dtype, B, Hq, Hk, nq, nk, d)
    kw = dict(causal=True) if lengths is None else dict(lengths=(None, ints(lengths)))
    out, saved = binding.agent_softmax_attn_fwd(q, k, v, save=True, **kw)
    lse = lse_of(saved, out)
    rows = 120 if lengths is None else nq      # of up to as many keys
    for b in range(B):
        for h in range(Hq):
            x, y = q[b, h, :rows].double().cpu(), k[b, h * Hk // Hq].double().cpu()
            n = torch.arange(1, rows + 1) if lengths is None else torch.full((rows,), lengths[b])
            seen = torch.arange(nk)[None] < n[:, None]
            want = torch.logsumexp((x @ y.t() * d ** -0.5).masked_fill(~seen, -float("inf")), -1)
            size = torch.where(seen, x.abs() @ y.abs().t() * d ** -0.5, 0.0).amax(-1)
            bound = (d + 2) * E * size + 4 * E * (2 * size + 6) + (3 * n + 52) * E + 2 * E * want.abs()
            off = (lse[b, h, :rows] - want).abs()
            assert bool((off <= bound).all()), (off / bound).max()
