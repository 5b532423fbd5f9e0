"""Softmax attention, backward, where blocks of keys have no queries to go over: the last tiles of causal sequences whose queries are taken in
ranges, and sequences with keys and no queries; heads whose values lie in LDS (65 to 128 channels of 16 bits).  Which sizes lead there is
checked without a GPU in test_softmax_lds_waits; bounds: softmax_reference."""
import pytest
import torch

from tests import softmax_reference as ref
from tests.softmax_plans import CAUSAL
from tests.test_gpu_softmax import close, ints
from tests.test_gpu_softmax_edges import inputs, run

pytestmark = pytest.mark.gpu


def check(dtype, B, Hq, Hk, nq, nk, d, causal, where, **kw):
    q, k, v, g = inputs(dtype, B, Hq, Hk, nq, nk, d)
    want = ref.attention(q, k, v, causal, where, do=g)
    out, grads = run(q, k, v, g, causal=causal, **kw)
    close(out, want["out"], "out")
    for n in grads:
        close(grads[n], want[n], n)
    for _ in range(3):
        _, again = run(q, k, v, g, causal=causal, **kw)
        assert all(torch.equal(again[n], grads[n]) for n in grads)
    return grads


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", CAUSAL, ids=lambda c: "x".join(map(str, c)))
def test_causal_sequences_in_ranges(case, dtype):
    B, Hq, Hk, nq, nk, d, _ = case
    check(dtype, B, Hq, Hk, nq, nk, d, True, ref.spans(B, nq, nk))


def zeros(t):
    return bool((t.contiguous().view(torch.int16) == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [80, 96, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
def test_keys_without_queries(causal, d, dtype):
    lengths = (ints([0, 150, 0]), ints([200, 170, 33]))
    grads = check(dtype, 3, 4, 2, 150, 200, d, causal, ref.spans(3, 150, 200, lengths=lengths), lengths=lengths)
    assert all(zeros(grads[n][b]) for n in ("dK", "dV") for b in (0, 2))
    starts = (ints([0, 0, 70, 70, 150, 150]), ints([0, 64, 100, 133, 190, 200]))
    grads = check(dtype, 1, 4, 2, 150, 200, d, causal, ref.spans(1, 150, 200, starts=starts), starts=starts)
    assert all(zeros(grads[n][:, :, at]) for n in ("dK", "dV") for at in (slice(0, 64), slice(100, 133), slice(190, 200)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_keys_without_queries_in_a_larger_call(dtype):
    """P and dS of one rounding."""
    lengths = (ints([600, 0, 600, 0, 0, 64, 600, 0]), ints([600, 600, 64, 1, 513, 600, 600, 65]))
    grads = check(dtype, 8, 8, 8, 600, 600, 96, True, ref.spans(8, 600, 600, lengths=lengths), lengths=lengths)
    assert all(zeros(grads[n][b]) for n in ("dK", "dV") for b in (1, 3, 4, 7))
