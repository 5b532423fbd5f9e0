"""Rotary positions and norms of more tokens than one launch may have blocks for."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "r.cpp").write_text('''#include "%s/paper_2312_08874_amd/csrc/rotary.h"
extern "C" int layers(long long rows, int heads, int lanes, long long* blocks, long long* reach) {
  const aa::RotaryPlan p = aa::rotary_plan({1, lanes, 1}, rows, heads, 0, false, false);
  const int n = aa::rotary_layers(p);
  *blocks = p.blocks;      // reach: the first token behind the last block's, which the kernel counts in 32 bits
  *reach = ((n > 1 ? (long long)n * aa::kRotaryLaunchBlocks : p.blocks) + 0ll) * ((4 / p.across) << (6 - p.shift));
  return n;
}
''' % ROOT)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(at / "r.so"), str(at / "r.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "r.so"))
    lib.layers.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    return lib


def test_launches_stay_below_the_most_threads(rule):
    blocks, reach = ctypes.c_longlong(), ctypes.c_longlong()
    several = 0
    for rows in (1, 1000, 1 << 22, (1 << 25) + 3, 1 << 26, (1 << 30) + 77, (1 << 31) - 1):
        for heads in (1, 3, 16):
            for lanes in (1, 4, 16, 32):
                n = rule.layers(rows, heads, lanes, ctypes.byref(blocks), ctypes.byref(reach))
                assert (n - 1) << 23 < blocks.value <= n << 23 and n < 65536 and rows <= reach.value <= 1 << 32
                several += n > 1
    assert several > 5
    assert rule.layers(1 << 22, 16, 4, ctypes.byref(blocks), ctypes.byref(reach)) == 1


@pytest.mark.gpu
def test_more_tokens_than_one_launch_takes():
    """2^30 tokens and some, three heads of one channel, in place: 2^24 blocks.  The norm of one channel is x / sqrt(x^2 + eps)."""
    from paper_2312_08874_amd import binding
    tokens, heads = (1 << 30) + 77, 3
    q = torch.empty(1, heads, tokens, 1, dtype=torch.bfloat16, device="cuda")
    piece = 1 << 27

    def values(h, lo, n):
        i = torch.arange(lo, lo + n, device="cuda", dtype=torch.int32)
        return ((i % 1021 - 510 + h).float() / 64).bfloat16()
    for h in range(heads):
        for lo in range(0, tokens, piece):
            n = min(piece, tokens - lo)
            q[0, h, lo:lo + n, 0] = values(h, lo, n)
    binding.agent_qk_norm_fwd(q, None, eps=0.25, out=(q, None))
    for h in range(heads):
        for lo in range(0, tokens, piece):
            n = min(piece, tokens - lo)
            x = values(h, lo, n).float()
            want = x / (x * x + 0.25).sqrt()
            off = (q[0, h, lo:lo + n, 0].float() - want).abs()
            assert bool((off <= (2.0 ** -8 + 16 * 2.0 ** -24) * want.abs()).all()), (h, lo)
