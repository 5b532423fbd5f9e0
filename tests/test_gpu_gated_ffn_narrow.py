"""Gated feed-forward block in fp32 where its products take 64 x 96 tiles, and the gradients of the biases; bounds as in
tests/ffn_reference.py."""
import ctypes
import os
import subprocess

import pytest
import torch

from tests import ffn_reference as ref
from tests.test_gpu_gated_ffn import check, inputs, run

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# rows, width, hidden: whole columns of tiles, the last one in part, results of any alignment, sums in parts or not
SHAPES = [(1000, 96, 256), (4000, 288, 768), (1000, 130, 300), (1000, 576, 1531), (10664, 96, 100)]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "r.cpp").write_text('''#include "%s/paper_2312_08874_amd/csrc/ffn.h"
extern "C" void tile(long long M, long long N, long long M2, long long N2, long long k, int narrow, int* out) {
  const aa::FfnTile t = aa::ffn_tile(M, N, M2, N2, (k + 31) / 32, 4, true, false, 256, narrow);
  out[0] = t.rows, out[1] = t.cols, out[2] = t.full, out[3] = t.parts, out[4] = t.each;
}
extern "C" int pitch(int hidden) { return aa::ffn_pitch(hidden); }
''' % ROOT)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-o", str(at / "r.so"), str(at / "r.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "r.so"))
    lib.tile.argtypes = [ctypes.c_longlong] * 5 + [ctypes.c_int, ctypes.c_void_p]

    def products(T, C, F, narrow=1):
        P, out = lib.pitch(F), []
        for M, N, M2, N2, k in ((T, C, 0, 0, F), (T, C, 0, 0, 2 * P), (2 * P, C, C, F, T)):
            t = (ctypes.c_int * 5)()
            lib.tile(M, N, M2, N2, k, narrow, t)
            tiles = -(-M // t[0]) * -(-N // t[1]) + -(-M2 // t[0]) * -(-N2 // t[1])
            assert (t[2] == tiles) == (t[3] == 1) and 0 <= t[2] <= tiles
            assert (t[3] - 1) * t[4] < (k + 31) // 32 <= t[3] * t[4]
            out.append(tuple(t))
        return out
    return products


def test_cases_reach_the_tiles(rule):
    reached = {(i, t[3] > 1) for shape in SHAPES for i, t in enumerate(rule(*shape)) if t[1] == 96}
    assert {(0, False), (1, True), (1, False), (2, True), (2, False)} <= reached
    assert all(t[1] != 96 for shape in SHAPES for t in rule(*shape, narrow=0))


def test_most_rows():
    from paper_2312_08874_amd import binding
    for rows, taken in ((1 << 30, True), ((1 << 30) + 1, False), ((1 << 31) - 1, False)):
        for query in (binding.lib().agent_gated_ffn_workspace_bytes, binding.lib().agent_gated_ffn_bwd_workspace_bytes,
                      binding.lib().agent_gated_ffn_saved_bytes):
            assert (query(ctypes.byref(binding.aa_ffn(rows, 1, 1, 0, 0, 0, 0, 0))) > 0) == taken


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_block_and_its_gradients(shape):
    from paper_2312_08874_amd import binding
    s = inputs("f32", *shape, biases=True)
    want, got = ref.block(s, "gelu"), run(binding, s, "gelu")
    assert set(got) == set(want)
    for name in got:
        check(got[name], want[name], name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(1, 5, 3), (255, 63, 65), (257, 72, 130), (513, 130, 64), (20000, 8, 24)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_the_biases(shape, dtype):
    """All of them at once and one alone, dy with rows apart."""
    from paper_2312_08874_amd import binding
    T, C, F = shape
    s = inputs(dtype, T, C, F, biases=True)
    wide = torch.zeros(T, C + 24, dtype=s["dy"].dtype, device="cuda")
    wide[:, :C], s["dy"] = s["dy"], wide[:, :C]
    want, got = ref.block(s, "silu"), run(binding, s, "silu")
    for name in ("db_gate", "db_up", "db_down"):
        check(got[name], want[name], name)
    for alone in ("b_gate", "b_up", "b_down"):
        one = {k: v for k, v in s.items() if not k.startswith("b_") or k == alone}
        want, got = ref.block(one, "silu"), run(binding, one, "silu")
        check(got["d" + alone], want["d" + alone], alone + " alone")
