"""The gated feed-forward block on the GPU against its definition in 64 bits; tests/ffn_reference.py derives the bounds."""
import pytest
import torch

from tests import ffn_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
WEIGHTS = ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down")


def inputs(dtype, T, C, F, biases, seed=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(std, *shape):
        return (std * torch.randn(*shape, generator=gen, device="cuda")).to(DT[dtype])
    s = {"x": rnd(1.0, T, C), "w_gate": rnd(C ** -0.5, F, C), "w_up": rnd(C ** -0.5, F, C), "w_down": rnd(F ** -0.5, C, F),
         "dy": rnd(1.0, T, C)}
    if biases:
        s.update(b_gate=rnd(0.3, F), b_up=rnd(0.3, F), b_down=rnd(0.3, C))
    return s


def weights(s):
    return {k: s[k] for k in WEIGHTS if k in s}


def check(got, want, what):
    value, bound = want
    got = got.double().reshape(value.shape)
    assert bool(torch.isfinite(got).all()), what + ": not finite"
    off = (got - value).abs() - bound
    assert bool((off <= 0).all()), "%s: off by %.3g more than allowed, at %d of %d" % (
        what, off.max(), int((off > 0).sum()), off.numel())


def run(binding, s, kind, **kw):
    y, saved = binding.agent_gated_ffn_fwd(s["x"], **weights(s), activation=kind, save=True, **kw)
    return {"y": y, **binding.agent_gated_ffn_bwd(s["x"], s["dy"], saved, **weights(s), activation=kind, **kw)}


# rows from one to several tiles, widths below, at and behind every step and tile, odd ones, long sums cut into parts
SHAPES = [(1, 1, 1), (1, 8, 16), (1, 64, 171), (2, 40, 24), (3, 33, 65), (5, 129, 31), (16, 64, 128), (17, 72, 200), (31, 96, 256),
          (32, 257, 130), (63, 128, 64), (65, 200, 333), (100, 7, 9), (130, 320, 864), (257, 192, 512), (300, 264, 704),
          (1000, 64, 176), (2049, 48, 40), (777, 512, 1365), (4100, 96, 257), (20000, 32, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_block_and_its_gradients(shape, dtype):
    from paper_2312_08874_amd import binding
    kind = ("silu", "gelu", "gelu_tanh", "relu", "sigmoid")[sum(shape) % 5]
    s = inputs(dtype, *shape, biases=shape[0] % 2 == 1)
    want, got = ref.block(s, kind), run(binding, s, kind)
    assert set(got) == {k for k in want if not k.startswith("db_") or "b_gate" in s}
    for name in got:
        check(got[name], want[name], name)
    y = binding.agent_gated_ffn_fwd(s["x"], **weights(s), activation=kind)      # keeping nothing
    assert torch.equal(y, got["y"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
def test_activations_over_their_whole_range(kind, dtype):
    """One channel a row carries the gate through: far negative, around zero, far positive."""
    from paper_2312_08874_amd import binding
    g = torch.cat([torch.linspace(-30, 30, 241), torch.tensor([-100.0, -1e4, 100.0, 1e4, 0.0, -0.0, 1e-6])])
    s = inputs(dtype, g.numel(), 16, 16, False)
    s["x"][:, 0], s["x"][:, 1:] = g.to(DT[dtype]).cuda(), 1.0
    s["w_gate"].zero_()
    s["w_gate"][:, 0] = 1.0
    want, got = ref.block(s, kind), run(binding, s, kind)
    for name in got:
        check(got[name], want[name], name)


@pytest.mark.parametrize("dtype,shape", [("bf16", (9000, 512, 1365)), ("f16", (4200, 1032, 2750)), ("f32", (3000, 288, 768)),
                                         ("bf16", (40, 1024, 4096)), ("f16", (1, 2048, 5504))])
def test_larger_blocks(dtype, shape):
    from paper_2312_08874_amd import binding
    s = inputs(dtype, *shape, biases=True)
    want, got = ref.block(s, "silu"), run(binding, s, "silu")
    for name in got:
        check(got[name], want[name], name)


def test_gradients_against_differences():
    """<gradient, direction> against central differences of the 64-bit definition, in fp32."""
    from paper_2312_08874_amd import binding
    for kind in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        s = inputs("f32", 37, 40, 56, True)
        got = run(binding, s, kind)
        gen = torch.Generator(device="cuda").manual_seed(4)

        def loss(name, t):
            return float((ref.block({**s, name: t}, kind, backward=False)["y"][0] * s["dy"].double()).sum())
        for name in ("x",) + WEIGHTS:
            v = torch.randn(s[name].shape, generator=gen, device="cuda", dtype=torch.float64)
            h = 1e-5
            diff = (loss(name, s[name].double() + h * v) - loss(name, s[name].double() - h * v)) / (2 * h)
            terms = got["d" + name].double() * v
            assert abs(float(terms.sum()) - diff) <= 1e-5 * float(terms.abs().sum()), (kind, name)


def _apart(t, by):
    """The same values in rows `by` elements further apart."""
    big = torch.full((t.shape[0], t.shape[1] + by), float("nan"), dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by", [8, 3])
@pytest.mark.parametrize("rows", [5, 200])
def test_rows_apart_and_addresses_off_alignment(dtype, by, rows):
    """NaN between the rows reaches nothing; tensors one element off 16 bytes give the bits of aligned ones."""
    from paper_2312_08874_amd import binding
    s = inputs(dtype, rows, 136, 200, True)
    want = run(binding, s, "silu")
    t = dict(s, x=_apart(s["x"], by), dy=_apart(s["dy"], by))
    got = run(binding, t, "silu")
    for name in want:
        assert torch.equal(got[name], want[name]), name
    out = _apart(torch.zeros_like(s["x"]), by)
    binding.agent_gated_ffn_fwd(s["x"], **weights(s), out=out)
    assert torch.equal(out, want["y"])

    def off(t):
        return torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].reshape(t.shape)
    for some in (WEIGHTS[:1], WEIGHTS[1:2], WEIGHTS[2:], WEIGHTS):
        got = run(binding, {k: off(v) if k in some else v for k, v in s.items()}, "silu")
        for name in want:
            assert torch.equal(got[name], want[name]), (name, some)


def test_more_axes_and_wanted_gradients():
    from paper_2312_08874_amd import binding
    s = inputs("bf16", 60, 64, 96, True)
    want = run(binding, s, "gelu")
    x, dy = s["x"].reshape(3, 4, 5, 64), s["dy"].reshape(3, 4, 5, 64)
    y, saved = binding.agent_gated_ffn_fwd(x, **weights(s), activation="gelu", save=True)
    assert y.shape == x.shape and torch.equal(y.reshape(60, 64), want["y"])
    only = binding.agent_gated_ffn_bwd(x, dy, saved, **weights(s), activation="gelu", want_weight_grads=False)
    assert set(only) == {"dx"} and torch.equal(only["dx"].reshape(60, 64), want["dx"])
    rest = binding.agent_gated_ffn_bwd(x, dy, saved, **weights(s), activation="gelu", want_dx=False)
    assert "dx" not in rest and all(torch.equal(rest[k], want[k]) for k in rest)


@pytest.mark.parametrize("rows", [4, 70])
def test_rows_that_are_no_numbers_stay_alone(rows):
    """In y and dx; a weight's gradient sums over the rows, so it is no number either."""
    from paper_2312_08874_amd import binding
    s = inputs("bf16", rows, 72, 100, True)
    clean = run(binding, s, "silu")
    bad = dict(s, x=s["x"].clone(), dy=s["dy"].clone())
    bad["x"][1, 5], bad["dy"][2, 7] = float("nan"), float("inf")
    got = run(binding, bad, "silu")
    others = [r for r in range(rows) if r not in (1, 2)]
    assert torch.equal(got["y"][others], clean["y"][others]) and torch.equal(got["y"][2], clean["y"][2])
    assert bool(got["y"][1].isnan().all())
    assert torch.equal(got["dx"][others], clean["dx"][others])
    assert not bool(torch.isfinite(got["dx"][1]).any()) and not bool(torch.isfinite(got["dx"][2]).any())
    assert bool(got["dw_gate"].isnan().any())


@pytest.mark.parametrize("dtype,shape", [("bf16", (1, 512, 1365)), ("bf16", (640, 256, 688)), ("f32", (50, 96, 256))])
def test_same_bits_stale_workspaces_another_stream_and_a_graph(dtype, shape):
    from paper_2312_08874_amd import binding
    s = inputs(dtype, *shape, biases=True)
    want = run(binding, s, "silu")
    desc, _ = binding._ffn_call(s["x"], *(s[k] for k in WEIGHTS), "silu")
    import ctypes
    sizes = [int(f(ctypes.byref(desc))) for f in (binding.lib().agent_gated_ffn_workspace_bytes,
                                                  binding.lib().agent_gated_ffn_bwd_workspace_bytes)]
    stale = torch.full((max(sizes),), 255, dtype=torch.uint8, device="cuda")      # NaN wherever nothing is written
    again = run(binding, s, "silu", workspace=stale)
    for name in want:
        assert torch.equal(again[name], want[name]), name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pass
    again = run(binding, s, "silu", stream=side)
    side.synchronize()
    for name in want:
        assert torch.equal(again[name], want[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(binding, s, "silu")
    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(3):
        for name in ("x", "dy", "w_up"):
            s[name].copy_(torch.randn(s[name].shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = run(binding, s, "silu")
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(got[name], eager[name]), name


def test_prepared_call():
    from paper_2312_08874_amd import binding
    s = inputs("f16", 3, 320, 856, True)
    out = torch.empty_like(s["x"])
    call = binding.prepare_gated_ffn(s["x"], **weights(s), activation="gelu", out=out)
    for _ in range(2):
        s["x"].mul_(0.5)
        call()
        assert torch.equal(out, binding.agent_gated_ffn_fwd(s["x"], **weights(s), activation="gelu"))
