"""Gated feed-forward block in fp32 where its products take 64 x 96 tiles, the gradients of the biases, and few tokens, whose h, dgate
and dup are two terms; bounds as in tests/ffn_reference.py."""
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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 216, 512), (4, 64, 130), (5, 40, 77), (16, 128, 300), (17, 64, 96), (40, 96, 250), (64, 72, 200), (500, 64, 130)],
                         ids=lambda s: "x".join(map(str, s)))
def test_few_tokens_lose_nothing_between_the_products(shape, dtype):
    """y (up to 64 tokens) and dx: bounds of operands rounded to 2^-15 (two terms of 8 bits or more) instead of the element type."""
    from paper_2312_08874_amd import binding
    s = inputs(dtype, *shape, biases=False)
    got = run(binding, s, "silu")
    v = {k: t.double() for k, t in s.items()}
    g, u = v["x"] @ v["w_gate"].t(), v["x"] @ v["w_up"].t()
    e = torch.sigmoid(g)
    a, d = g * e, e * (1 + g * (1 - e))
    T, C, F = shape
    U, half, fine, low = 2.0 ** -24, torch.finfo(s["x"].dtype).eps / 2, 2.0 ** -15, 2.0 ** -20
    eg = (C + 4) * U * (v["x"].abs() @ v["w_gate"].abs().t()) + 2.0 ** -19 * (1 + g.abs())
    eu = (C + 4) * U * (v["x"].abs() @ v["w_up"].abs().t())
    h, eh = a * u, u.abs() * 1.2 * eg + a.abs() * eu + eg * eu + fine * (a * u).abs() + low
    y = h @ v["w_down"].t()
    bound = half * y.abs() + eh @ v["w_down"].abs().t() + (2 * F + 4) * U * (h.abs() @ v["w_down"].abs().t()) + low
    assert T > 64 or bool(((got["y"].double() - y).abs() <= bound).all())
    dh = v["dy"] @ v["w_down"]
    edh = (C + 4) * U * (v["dy"].abs() @ v["w_down"].abs())
    dg, du = dh * u * d, dh * a
    edg = dh.abs() * (d.abs() * eu + (u.abs() + eu) * 1.1 * eg) + (u * d).abs() * edh + 2 * fine * dg.abs() + low
    edu = dh.abs() * 1.2 * eg + a.abs() * edh + 2 * fine * du.abs() + low
    dx = dg @ v["w_gate"] + du @ v["w_up"]
    size = dg.abs() @ v["w_gate"].abs() + du.abs() @ v["w_up"].abs()
    bound = half * dx.abs() + edg @ v["w_gate"].abs() + edu @ v["w_up"].abs() + (4 * F + 4) * U * size + low
    assert bool(((got["dx"].double() - dx).abs() <= 1.01 * bound).all())      # 1.01: second orders


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 4, 5, 17, 64])
def test_few_tokens_with_h_beyond_the_largest_number(rows):
    """h = 300 * 300 is beyond fp16, its product with 1/2 is not; an infinite h makes an infinite y, and other rows stay as they are."""
    from paper_2312_08874_amd import binding
    x = torch.full((rows, 1), 2.0, dtype=torch.float16, device="cuda")
    x[0] = 300.0
    one = torch.ones(1, 1, dtype=torch.float16, device="cuda")
    y = binding.agent_gated_ffn_fwd(x, one, one, 0.5 * one, activation="relu")
    assert y[0].item() == torch.tensor(45000.0).half().item() and bool((y[1:] == 2.0).all())
    for dtype in (torch.float16, torch.bfloat16):
        z = x.to(dtype)
        z[0] = float("inf")
        y = binding.agent_gated_ffn_fwd(z, one.to(dtype), one.to(dtype), one.to(dtype), activation="relu")
        assert y[0].item() == float("inf") and bool((y[1:] == 4.0).all())
