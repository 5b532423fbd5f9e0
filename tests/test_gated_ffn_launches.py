"""The gated feed-forward block of more rows than one launch may have blocks for along x, and of tensors beyond 2^31 elements."""
import ctypes
import os
import subprocess

import pytest
import torch

from tests import ffn_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_layers_of_a_launch(tmp_path):
    """Every block of a launch is in one layer, and no layer reaches 2^32 threads along x."""
    (tmp_path / "r.cpp").write_text('''#include "%s/paper_2312_08874_amd/csrc/ffn.h"
extern "C" unsigned layers(long long blocks) { return aa::ffn_layers(blocks); }
extern "C" unsigned most() { return aa::kFfnLaunchBlocks; }
''' % ROOT)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(tmp_path / "r.so"), str(tmp_path / "r.cpp")], check=True)
    lib = ctypes.CDLL(str(tmp_path / "r.so"))
    lib.layers.argtypes = [ctypes.c_longlong]
    most = lib.most()
    assert most * 512 < 1 << 32 and most % 8 == 0
    for blocks in (1, 8, most - 1, most, most + 1, 1 << 24, 1 << 28):
        n = lib.layers(blocks)
        assert (n - 1) * most < blocks <= n * most and n < 65536


def _room(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip("needs %d GB of GPU memory" % gigabytes)


@pytest.mark.gpu
def test_most_rows_of_one_channel():
    """2^30 rows, whose second product has 2^24 tiles: y = relu(x) x."""
    from paper_2312_08874_amd import binding
    _room(200)
    rows, piece = 1 << 30, 1 << 27
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")

    def values(lo):      # of few bits: their squares are exact
        return ((torch.arange(lo, lo + piece, device="cuda", dtype=torch.int32) % 29 - 14) / 4.0).bfloat16()
    for lo in range(0, rows, piece):
        x[lo:lo + piece, 0] = values(lo)
    y = binding.agent_gated_ffn_fwd(x, one, one, one, activation="relu")
    for lo in range(0, rows, piece):
        v = values(lo).float()
        assert torch.equal(y[lo:lo + piece, 0].float(), v.clamp(min=0) * v), lo
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(270001, 8200, 40), (270001, 40, 8200)], ids=["wide rows", "wide hidden rows"])
def test_tensors_beyond_two_thousand_million_elements(shape):
    """x and y, or h and what is kept of it, pass 2^31 elements.  Every row of x is one of 1013; a weight's gradient is that of the 1013
    rows, each counted as often as it is there."""
    from paper_2312_08874_amd import binding
    from tests.test_gpu_gated_ffn import inputs, weights
    _room(120)
    T, C, F = shape
    few = 1013
    s = inputs("bf16", few, C, F, True)
    at = torch.arange(T, device="cuda") % few
    x, dy = s["x"][at], s["dy"][at]
    y, saved = binding.agent_gated_ffn_fwd(x, **weights(s), activation="silu", save=True)
    got = binding.agent_gated_ffn_bwd(x, dy, saved, **weights(s), activation="silu")
    del saved, x, dy
    want = ref.block(s, "silu")
    for name, all_rows in (("y", y), ("dx", got["dx"])):
        value, bound = want[name]
        for lo in range(0, T, few):
            rows = all_rows[lo:lo + few].double()
            assert bool(((rows - value[:len(rows)]).abs() <= bound[:len(rows)]).all()), (name, lo)
    # sums over T rows: T products a value, in any order; rounded once
    counts = torch.bincount(at, minlength=few).double()
    v = {k: t.double() for k, t in s.items()}
    g, u = v["x"] @ v["w_gate"].t() + v["b_gate"], v["x"] @ v["w_up"].t() + v["b_up"]
    a, d = ref.act("silu", g)
    dh = v["dy"] @ v["w_down"]
    for name, left, right in (("dw_gate", dh * u * d, v["x"]), ("dw_up", dh * a, v["x"]), ("dw_down", v["dy"], a * u)):
        value = (left * counts[:, None]).t() @ right
        size = (left.abs() * counts[:, None]).t() @ right.abs()
        # one operand rounded to bf16, sums of C products in it (each off by few 2^-24 of their size, here by some 2^-12 at most)
        bound = (2.0 ** -8 + 2.0 ** -11 + (T + 4) * 2.0 ** -24) * size + 2.0 ** -8 * value.abs()
        assert bool(((got[name].double() - value).abs() <= bound).all()), name
    del y, got
    torch.cuda.empty_cache()
