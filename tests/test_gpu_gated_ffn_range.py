"""The gated feed-forward block where a value between its products, an input or a gate leaves the element type's range: a result
is within its bound (tests/ffn_reference.py) or no finite number, and never a finite number that is wrong."""
import math

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


@pytest.mark.parametrize("rows", ROWS + [300])
@pytest.mark.parametrize("big", ["dgate", "dup"])
def test_gradients_where_dgate_or_dup_is_beyond_the_largest_number(big, rows):
    """One token's dgate or dup of channel 5 is some 70000 to 130000: two terms of fp16 hold it, and its products with x of 1/64 are
    well inside the range, so that every gradient is right."""
    from paper_2312_08874_amd import binding
    s = inputs("f16", rows, 8, 24, False)
    s["x"] = ((1.0 + s["x"].abs().clamp(max=1.0)) / 64).half()
    s["dy"] = 0.01 * s["dy"]
    s["dy"][0] = 25.0
    s["w_down"][:, 5] = 1.0
    large, small = ("w_up", "w_gate") if big == "dgate" else ("w_gate", "w_up")
    s[large][5], s[small][5] = 2500.0, 0.05
    want, got = ref.block(s, "relu"), run(binding, s, "relu")
    dh = s["dy"].double() @ s["w_down"].double()
    factor = (s["x"].double() @ s[large].double().t())[0, 5]
    assert 66000 < float(dh[0, 5] * factor) < 130000
    for name in got:
        assert bool(right(got[name], want[name], name).all()), name


@pytest.mark.parametrize("rows", ROWS + [300])
def test_gradients_with_two_terms_of_dgate_and_dup(rows):
    """dw_gate and dw_up: dgate and dup in two terms are off by 2^-22 (fp16: 2 x 11 bits), not by 2^-11; an odd number of tokens, and
    widths that end inside a tile."""
    from paper_2312_08874_amd import binding
    s = inputs("f16", rows, 72, 90, False)
    got = run(binding, s, "sigmoid")
    v = {k: t.double() for k, t in s.items()}
    g, u = v["x"] @ v["w_gate"].t(), v["x"] @ v["w_up"].t()
    U, T, C = 2.0 ** -24, rows, 72
    eg, eu = ((C + 4) * U * (v["x"].abs() @ v[w].abs().t()) for w in ("w_gate", "w_up"))
    e = torch.sigmoid(g)
    ee = 0.25 * eg + 2.0 ** -19 * (1 + g.abs())      # of act and of its derivative, whose slopes are below 1 / 4
    dh, edh = v["dy"] @ v["w_down"], (C + 4) * U * (v["dy"].abs() @ v["w_down"].abs())
    p, q = u * e * (1 - e), e
    ep, eq = (e * (1 - e)) * eu + (u.abs() + eu) * ee + 2.0 ** -16 * p.abs(), ee + 2.0 ** -16 * q
    for name, f, ef in (("dw_gate", p, ep), ("dw_up", q, eq)):
        d = dh * f
        ed = dh.abs() * ef + (f.abs() + ef) * edh + (2.0 ** -21 + U) * d.abs() + 2.0 ** -25      # the last: a subnormal second term
        want = d.t() @ v["x"]
        bound = ed.t() @ v["x"].abs() + (2 * T + 4) * U * (d.abs().t() @ v["x"].abs()) + 2.0 ** -11 * want.abs() + 2.0 ** -25
        off = (got[name].double() - want).abs() - 1.01 * bound      # 1.01: second orders
        assert bool((off <= 0).all()), "%s: off by %.3g more than allowed" % (name, off.max())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", ROWS + [300])
def test_an_infinite_gradient_of_y_reaches_the_weights_gradients(rows, dtype):
    """dy of one token is infinite in channel 3: its dgate and dup are infinite, and so is what they or dy make of finite, nonzero x
    and h; the other channels of dw_down do not meet it."""
    from paper_2312_08874_amd import binding
    s = inputs(dtype, rows, 24, 40, True)
    s["x"] = torch.where(s["x"] == 0, torch.ones_like(s["x"]), s["x"])
    s["w_down"] = torch.where(s["w_down"] == 0, torch.ones_like(s["w_down"]), s["w_down"])
    clean = run(binding, s, "silu")
    s["dy"][rows // 2, 3] = float("inf")
    got = run(binding, s, "silu")
    for name in ("dw_gate", "dw_up", "db_gate", "db_up"):
        assert not bool(torch.isfinite(got[name]).any()), name
    assert not bool(torch.isfinite(got["dx"][rows // 2]).any())
    assert not bool(torch.isfinite(got["dw_down"][3]).any()) and not bool(torch.isfinite(got["db_down"][3]).any())
    others = [c for c in range(24) if c != 3]
    assert torch.equal(got["dw_down"][others], clean["dw_down"][others])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["relu", "sigmoid"])
@pytest.mark.parametrize("rows", [1, 17, 300, 3000])
def test_gates_of_minus_infinity_switch_their_channels_off(rows, kind, dtype):
    """As a bias of -10000 does, bit for bit: act and its derivative are 0 at both."""
    from paper_2312_08874_amd import binding
    s = inputs(dtype, rows, 40, 200, True)
    s["b_gate"][::3] = -10000.0
    want = run(binding, s, kind)
    s["b_gate"][::3] = float("-inf")
    got = run(binding, s, kind)
    for name in want:
        assert bool(torch.isfinite(want[name]).all()) and torch.equal(got[name], want[name]), name
    assert not bool(got["dw_gate"][::3].any()) and not bool(got["dw_down"][:, ::3].any())
    s["x"][0, 0] = float("nan")      # and no number stays none
    assert bool(run(binding, s, kind)["y"][0].isnan().all())


@pytest.mark.parametrize("dtype,far", [("bf16", 1e4), ("bf16", 1e20), ("f16", 1e4), ("f32", 1e4), ("f32", 1e20)])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows", [1, 17, 300])
def test_far_gates_are_those_of_relu(rows, kind, dtype, far):
    """At +-10000 and at +-1e20, whose square is beyond fp32, the activations and their slopes are relu's to the last bit."""
    from paper_2312_08874_amd import binding
    s = inputs(dtype, rows, 40, 200, True)
    s["b_gate"] = torch.where(s["b_gate"] > 0, far, -far).to(s["x"].dtype)
    s["w_down"] = (s["w_down"].double() / far * 100).to(s["x"].dtype)
    want, got = run(binding, s, "relu"), run(binding, s, kind)
    for name in want:
        assert not bool(want[name].isnan().any()) and torch.equal(got[name], want[name]), name      # dw_down may be beyond fp16


def _tails(kind, g):
    """act(g) / g, act(g) and its slope without a difference of numbers near 1, which 1 + erf and 1 + tanh are far out."""
    if kind == "gelu":
        e = 0.5 * torch.special.erfc(-g * 0.5 ** 0.5)
        return e, g * e, e + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5
    c = 2 * (2 / math.pi) ** 0.5
    z, slope = (g, 1.0) if kind == "silu" else (c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g * g))
    e, rest = torch.sigmoid(z), torch.sigmoid(-z)
    return e, g * e, e + g * e * rest * slope


def one_channel(rows, kind, dtype, lo, hi):
    """One hidden channel, whose gate is x's first channel and whose up is large: (gates, up, act(gates) up, its slopes times up, and
    the type's half rounding and smallest step)."""
    from paper_2312_08874_amd import binding
    up = {"f16": 2.0 ** 14, "bf16": 1.0, "f32": 1.0}[dtype]
    x = torch.ones(rows, 2, device="cuda")
    x[:, 0] = torch.linspace(lo, hi, rows)
    x = x.to(torch.float32 if dtype == "f32" else HALF[dtype])

    def matrix(*v):
        return torch.tensor(v, device="cuda").to(x.dtype)
    s = {"x": x, "w_gate": matrix([1.0, 0.0]), "w_up": matrix([0.0, up]), "w_down": matrix([1.0], [0.0]),
         "dy": matrix([1.0, 0.0]).expand(rows, 2).contiguous()}
    got = run(binding, s, kind)
    info = torch.finfo(x.dtype)
    return x[:, 0].double(), up, got["y"][:, 0].double(), got["dx"][:, 0].double(), info.eps / 2, info.smallest_normal * info.eps


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows", [16, 64, 241, 30001])
def test_tails_of_the_activations(rows, kind, dtype):
    """An error of act shows against act itself.  Bounds, relative: exp of |z| <= 42 with the roundings of its argument and of z,
    4 * 42 * 2^-24; the fit, 1 / x and what follows, 2^-18; h or dgate, and the result, rounded once each; what the forward pass
    keeps, 2^-16.  The slope of a negative gate is a difference: relative to the sum of its parts."""
    g, up, y, dx, half, low = one_channel(rows, kind, dtype, -9, 3)
    parts, a, d = _tails(kind, g)
    rest = (d - parts).abs()
    near = 4 * 42 * 2.0 ** -24 + 2.0 ** -18
    assert bool(((y - a * up).abs() <= (near + 2.01 * half) * (a * up).abs() + low).all())
    bound = (near + 2.0 ** -16) * (parts + rest) * up + 2.01 * half * (d * up).abs() + low
    assert bool(((dx - d * up).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [16, 64, 241, 30001])
def test_slope_of_the_sigmoid_on_both_sides(rows, dtype):
    """Up to 13, where it is 2e-6.  Bounds as above, with exp of |z| <= 13."""
    g, up, y, dx, half, low = one_channel(rows, "sigmoid", dtype, -13, 13)
    e, rest = torch.sigmoid(g), torch.sigmoid(-g)
    near = 4 * 13 * 2.0 ** -24 + 2.0 ** -18
    assert bool(((y - e * up).abs() <= (near + 2.01 * half) * e * up + low).all())
    assert bool(((dx - e * rest * up).abs() <= (near + 2.0 ** -16 + 2.01 * half) * e * rest * up + low).all())
