"""fp16's weights that are far below a row's largest, in the forward pass of softmax attention.

Times 2^6 beside a reference that is one of them, a weight is rounded by u or by half of 2^-24, which is 2^-31 of the reference, and the
weights' sum is at least that: with n of them o is off by 2^-31 (sum of |v| + n |o|) beyond softmax_reference's bound."""
import pytest
import torch

from tests import softmax_reference as ref
from tests.test_gpu_softmax import close

pytestmark = pytest.mark.gpu
E = ref.E


# B, heads, queries, keys, low: the others' scores below the first key's
SMALL = [(1, 2, 1, 65536, 17.55), (8, 8, 1, 65536, 17.55), (1, 1, 40, 60000, 18.0), (8, 8, 512, 16384, 17.55), (2, 16, 1000, 8192, 19.0), (64, 16, 3, 1400, 17.0)]


@pytest.mark.parametrize("case", SMALL, ids=lambda c: "x".join(map(str, c)))
def test_many_small_weights_beside_a_large_one(case):
    """The first key takes most of the weight, and the values of the others, each with next to none, are the result."""
    from paper_2312_08874_amd import binding
    B, H, nq, nk, low = case
    d = 32
    gen = torch.Generator().manual_seed(4)
    q = torch.zeros(B, H, nq, d, dtype=torch.float16, device="cuda")
    k = (0.25 * torch.randn(B, H, nk, d, generator=gen)).half().cuda()
    v = (0.5 + torch.rand(B, H, nk, d, generator=gen)).half().cuda()
    q[..., 0], q[..., 1] = 1.0, 1.0
    k[..., 0] = 0.0
    k[:, :, 0, 0], k[:, :, 0, 1], v[:, :, 0] = low, 0.0, 0.0
    out = binding.agent_softmax_attn_fwd(q, k, v, scale=1.0)
    u = ref.unit(torch.float16)
    for b, h in ((0, 0), (B - 1, H - 1)):
        x, y, z = (t[b, h].double().cpu() for t in (q[:, :, :4], k, v))
        s = x @ y.t()
        p = torch.softmax(s, -1)
        o = p @ z
        a = (d + 2) * E * (x.abs() @ y.abs().t()).amax(-1, keepdim=True) + 4 * E * (low + 16)
        bound = (2 * a + 2 * u + (nk + 8) * E) * o + 2.0 ** -31 * (z.sum(0) + nk * o)
        close(out[b, h, :4], (o, u * (o + bound) + bound + ref.smallest(torch.float16)), "out")
