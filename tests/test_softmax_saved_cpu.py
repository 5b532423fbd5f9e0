"""What softmax attention keeps for its backward pass: the rounding of out only where a row may see few keys."""
import ctypes

import pytest

from paper_2312_08874_amd import binding
from tests.test_softmax_cpu import A, desc

LSE, LOW = 2 * 4 * 12 * 4 // 256 * 256 + 256, 2 * 4 * 12 * 32 * 2


def saved(**kw):
    return binding.lib().agent_softmax_attn_saved_bytes(ctypes.byref(desc(**kw)))


@pytest.mark.parametrize("dtype", [binding.AA_BF16, binding.AA_F16])
def test_the_rounding_of_out_is_kept_for_rows_of_few_keys(dtype):
    assert saved(dtype=dtype, tokens_k=512) == LSE + LOW
    assert saved(dtype=dtype, tokens_k=513) == LSE                      # every row sees all of them
    assert saved(dtype=dtype, tokens_k=513, lengths_q=A) == LSE
    for some in (dict(causal=1), dict(lengths_k=A)):
        assert saved(dtype=dtype, tokens_k=513, **some) == LSE + LOW, some
    packed = saved(dtype=dtype, batch=1, tokens_k=513, sequences=3, starts_q=A, starts_k=A)
    assert packed == 256 + LOW // 2
    assert saved(dtype=binding.AA_F32, tokens_k=513) == saved(dtype=binding.AA_F32) == LSE
