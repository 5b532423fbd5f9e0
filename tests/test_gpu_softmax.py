"""Softmax attention on the GPU, forward and backward, against its definition in 64 bits; bounds: softmax_reference."""
import pytest
import torch

from tests import softmax_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def tokens(gen, dtype, B, H, N, d, layout, std=1.0):
    """[B,H,N,d] in its layout; "qkv": a slice of a fused projection, "odd": rows 3 elements longer than their channels, off any
    alignment."""
    def rnd(*shape):
        return (std * torch.randn(*shape, generator=gen)).to(dtype).cuda()
    if layout == "dense":
        return rnd(B, H, N, d)
    if layout == "token":
        return rnd(B, N, H, d).permute(0, 2, 1, 3)
    if layout == "odd":
        return rnd(B, H, N, d + 3)[..., 1:d + 1]
    return rnd(B, N, 3, H, d)[:, :, 1].permute(0, 2, 1, 3)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def mixed(mix, B, nq, nk):
    """Keyword arguments of the calls, and the sequences."""
    if mix is None:
        return {}, ref.spans(B, nq, nk)
    if mix[0] == "packed":
        starts = tuple(ints([sum(v[:i]) for i in range(len(v) + 1)]) for v in mix[1:])
        return {"starts": starts}, ref.spans(B, nq, nk, starts=starts)
    lengths = tuple(None if v is None else ints(v) for v in mix[1:])
    return {"lengths": lengths}, ref.spans(B, nq, nk, lengths=lengths)


def close(got, want, what):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape, what
    inf = torch.isinf(value)
    assert bool((got[inf] == value[inf]).all()), what + ": infinities"
    off = ((got - value).abs() - bound)[~inf]
    assert bool(torch.isfinite(got[~inf]).all()), what + ": not finite"
    assert bool((off <= 0).all()), "%s: off by %.3g more than allowed, at %d of %d" % (what, off.max(), int((off > 0).sum()), off.numel())


# dtype, B, Hq, Hk, queries, keys, d, causal, layout, mix
CASES = [
    ("bf16", 2, 3, 3, 196, 196, 64, False, "qkv", None),
    ("f16", 1, 4, 2, 130, 130, 128, True, "token", None),
    ("f32", 2, 2, 2, 77, 77, 48, True, "dense", None),
    ("bf16", 1, 2, 1, 300, 300, 32, True, "dense", None),
    ("f16", 2, 2, 2, 65, 191, 40, False, "token", None),
    ("bf16", 1, 6, 2, 33, 257, 96, True, "token", None),
    ("f32", 1, 2, 1, 129, 65, 128, False, "token", None),
    ("bf16", 1, 2, 2, 90, 40, 64, True, "dense", None),          # the first fifty queries see nothing
    ("f16", 1, 1, 1, 1, 1, 8, True, "dense", None),
    ("bf16", 3, 8, 8, 1, 301, 64, True, "token", None),
    ("f16", 2, 16, 4, 1, 1500, 128, True, "token", None),
    ("f32", 2, 4, 1, 1, 1200, 64, False, "dense", None),
    ("bf16", 2, 8, 1, 3, 700, 80, True, "token", None),
    ("bf16", 2, 3, 3, 50, 70, 20, False, "token", None),         # rows of 40 bytes
    ("f16", 1, 2, 1, 70, 70, 33, True, "odd", None),
    ("f32", 1, 2, 2, 70, 50, 30, True, "odd", None),
    ("bf16", 1, 2, 2, 70, 90, 64, False, "odd", None),
    ("bf16", 1, 2, 1, 70, 150, 256, True, "dense", None),
    ("f16", 1, 1, 1, 100, 100, 200, False, "token", None),
    ("f32", 1, 2, 1, 40, 70, 256, True, "dense", None),
    ("f32", 1, 1, 1, 40, 70, 136, False, "token", None),
    ("bf16", 1, 2, 2, 200, 200, 64, True, "qkv", ("packed", [64, 0, 1, 100, 33], [64, 0, 1, 100, 33])),      # two rows behind
    ("f16", 1, 4, 2, 150, 260, 48, True, "token", ("packed", [0, 40, 9, 0, 90], [7, 130, 0, 3, 80])),
    ("f32", 1, 2, 1, 60, 60, 32, False, "dense", ("packed", [13, 47], [13, 47])),
    ("bf16", 1, 4, 1, 70, 900, 64, True, "token", ("packed", [1] * 70, [0, 1, 63, 64, 65] + [10] * 65)),
    ("bf16", 3, 2, 2, 130, 130, 64, True, "token", ("padded", [130, 1, 64], [130, 1, 64])),
    ("f16", 3, 4, 2, 1, 400, 128, True, "token", ("padded", None, [400, 0, 17])),
    ("f32", 2, 2, 2, 50, 66, 24, False, "dense", ("padded", [0, 50], [66, 3])),
    ("bf16", 2, 2, 2, 70, 90, 64, False, "qkv", ("padded", [70, 33], None)),
    ("f16", 1, 2, 2, 1100, 1100, 64, True, "token", None),
    ("bf16", 1, 1, 1, 17, 5000, 128, False, "dense", None),
    ("f32", 1, 2, 1, 5, 3000, 32, True, "dense", None),
    ("bf16", 16, 16, 4, 140, 140, 16, True, "token", None),      # enough blocks for the kernel of many queries
    ("f16", 32, 8, 8, 130, 200, 64, True, "token", None),
    ("f32", 24, 12, 12, 40, 40, 24, False, "dense", None),
    ("bf16", 12, 12, 12, 257, 70, 128, False, "qkv", None),
]


def _inputs(case, seed=3, std=1.0):
    dtype, B, Hq, Hk, nq, nk, d, causal, layout, mix = case
    gen = torch.Generator().manual_seed(seed)
    q, g = (tokens(gen, DT[dtype], B, Hq, nq, d, layout, std) for _ in range(2))
    k, v = (tokens(gen, DT[dtype], B, Hk, nk, d, layout, std) for _ in range(2))
    kw, where = mixed(mix, B, nq, nk)
    return q, k, v, g, dict(causal=causal, **kw), where


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention_and_its_gradients(case):
    from paper_2312_08874_amd import binding
    q, k, v, g, kw, where = _inputs(case)
    want = ref.attention(q, k, v, case[7], where, do=g)
    out = binding.agent_softmax_attn_fwd(q, k, v, **kw)
    close(out, want["out"], "out")
    again, saved = binding.agent_softmax_attn_fwd(q, k, v, save=True, **kw)
    assert torch.equal(out, again)
    lse = saved[:4 * out[..., 0].numel()].view(torch.float32).view(out.shape[:3])
    used = want["used_q"][:, None, :].expand(lse.shape)
    close(lse.cpu()[used], tuple(t[used] for t in want["lse"]), "lse")
    grads = binding.agent_softmax_attn_bwd(q, k, v, out, saved, g, **kw)
    for name in ("dQ", "dK", "dV"):
        close(grads[name], want[name], name)
    more = binding.agent_softmax_attn_bwd(q, k, v, out, saved, g, **kw)
    assert all(torch.equal(grads[n], more[n]) for n in grads)
