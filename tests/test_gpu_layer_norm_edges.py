"""Layer norm where it can go wrong: results in place of inputs, large means and rows of one value, rows that are NaN, more elements than
31 bits count, other streams, captured graphs."""
import pytest
import torch

from tests import layer_norm_reference as ref
from tests.test_gpu_layer_norm import DT, close, rows_of

pytestmark = pytest.mark.gpu


def inputs(dtype, rows, width, layout="dense", mean=0.0, seed=6):
    gen = torch.Generator().manual_seed(seed)
    x, r, dy, ds = (rows_of(gen, DT[dtype], rows, width, layout, mean=m) for m in (mean, 0.0, 0.0, 0.0))
    w, b = (m + 0.3 * torch.randn(width, generator=gen).cuda() for m in (1.0, 0.0))
    return x, r, dy, ds, w, b


@pytest.mark.parametrize("dtype,rows,width", [("bf16", 700, 512), ("f32", 300, 1030), ("f16", 5, 9000)])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_results_in_place(dtype, rows, width, layout):
    from paper_2312_08874_amd import binding
    x, r, dy, ds, w, b = inputs(dtype, rows, width, layout)

    def copy(t):
        return t.clone() if layout == "dense" else torch.cat([t, t[:, :3]], 1)[:, :width]
    y, s, saved = binding.agent_layer_norm_fwd(x, w, b, residual=r, save=True)
    for y_at, s_at in ((0, None), (1, None), (0, 1), (1, 0), (None, 1)):
        mine = [copy(x), copy(r)]
        got = binding.agent_layer_norm_fwd(mine[0], w, b, residual=mine[1], out=None if y_at is None else mine[y_at],
                                           sum_out=None if s_at is None else mine[s_at])
        assert torch.equal(got[0], y) and torch.equal(got[1], s), (y_at, s_at)
        assert y_at is None or got[0].data_ptr() == mine[y_at].data_ptr()
    want = binding.agent_layer_norm_bwd(x, dy, saved, w, b, residual=r, dsum=ds)
    for at in range(4):
        mine = [copy(t) for t in (x, r, dy, ds)]
        got = binding.agent_layer_norm_bwd(mine[0], mine[2], saved, w, b, residual=mine[1], dsum=mine[3], out=mine[at])
        assert all(torch.equal(got[n], want[n]) for n in want), at
    alone = binding.agent_layer_norm_bwd(x, dy, saved, w, b, residual=r, dsum=ds, want_weight_grads=False)
    assert set(alone) == {"dx"} and torch.equal(alone["dx"], want["dx"])
    weights = binding.agent_layer_norm_bwd(x, dy, saved, w, b, residual=r, dsum=ds, want_dx=False)
    assert set(weights) == {"dw", "db"} and all(torch.equal(weights[n], want[n]) for n in weights)


@pytest.mark.parametrize("dtype,mean", [("f32", 3000.0), ("bf16", 60.0), ("f16", 500.0)])
def test_large_means_and_rows_of_one_value(dtype, mean):
    from paper_2312_08874_amd import binding
    x, _, dy, _, w, b = inputs(dtype, 40, 520, mean=mean)
    x[3], x[7] = 1.0, 0.0
    y, saved = binding.agent_layer_norm_fwd(x, w, b, eps=1e-3, save=True)
    close(y, ref.forward(x, w, b, 1e-3)["y"], "y")
    assert torch.equal(y[7], b.to(x.dtype))
    grads = binding.agent_layer_norm_bwd(x, dy, saved, w, b)
    want = ref.backward(x, dy, w, b, 1e-3)
    for n in grads:
        close(grads[n], want[n], n)


def test_a_row_that_is_nan_stays_alone():
    from paper_2312_08874_amd import binding
    for width in (96, 5000):
        x, r, dy, ds, w, b = inputs("bf16", 70, width)
        y, s, saved = binding.agent_layer_norm_fwd(x, w, b, residual=r, save=True)
        dx = binding.agent_layer_norm_bwd(x, dy, saved, w, b, residual=r, dsum=ds)["dx"]
        x[5, 17], r[33, 0] = float("nan"), float("inf")
        z, _, stats = binding.agent_layer_norm_fwd(x, w, b, residual=r, save=True)
        dz = binding.agent_layer_norm_bwd(x, dy, stats, w, b, residual=r, dsum=ds)["dx"]
        rest = [i for i in range(70) if i not in (5, 33)]
        assert bool(torch.isnan(z[5]).all()) and bool(torch.isnan(z[33]).any())
        assert torch.equal(z[rest], y[rest]) and torch.equal(dz[rest], dx[rest])


def test_more_elements_than_31_bits_count():
    from paper_2312_08874_amd import binding
    rows, width = (1 << 20) + 3, 2080
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda").normal_()
    dy = torch.empty_like(x).normal_()
    w = torch.rand(width, device="cuda")
    y, saved = binding.agent_layer_norm_fwd(x, w, save=True)
    dx = binding.agent_layer_norm_bwd(x, dy, saved, w)["dx"]
    for at in (0, (1 << 31) // width - 1, rows - 4):
        part = x[at:at + 4].clone()
        z, stats = binding.agent_layer_norm_fwd(part, w, save=True)
        assert torch.equal(y[at:at + 4], z)
        assert torch.equal(dx[at:at + 4], binding.agent_layer_norm_bwd(part, dy[at:at + 4].clone(), stats, w)["dx"])


def both(x, r, dy, ds, w, b, **kw):
    from paper_2312_08874_amd import binding
    y, s, saved = binding.agent_layer_norm_fwd(x, w, b, residual=r, save=True, **kw)
    g = binding.agent_layer_norm_bwd(x, dy, saved, w, b, residual=r, dsum=ds, **kw)
    return [y, s, g["dx"], g["dw"], g["db"]]


def test_on_another_stream():
    t = inputs("f16", 3000, 768)
    want = both(*t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = both(*t, stream=side)
    b = both(*t)
    with torch.cuda.stream(side):
        c = both(*t)
    torch.cuda.synchronize()
    for got in (a, b, c):
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype,rows,width", [("bf16", 900, 512), ("f32", 3, 20000)])
def test_captured_and_replayed(dtype, rows, width):
    graphs = []
    for seed in (1, 2):
        t = inputs(dtype, rows, width, seed=seed)
        both(*t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = both(*t)
        graphs.append((graph, t, result))
    for turn in range(4):
        for graph, t, _ in graphs:
            for x in t:
                x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(turn)).to(x.dtype))
        for graph, *_ in graphs:
            graph.replay()
        for _, t, result in graphs:
            assert all(torch.equal(p, q) for p, q in zip(result, both(*t))), turn


def test_prepared_calls_and_refusals():
    from paper_2312_08874_amd import binding
    x, r, dy, ds, w, b = inputs("bf16", 50, 128)
    y, s = torch.empty_like(x), torch.empty_like(x)
    call = binding.prepare_layer_norm(x, w, b, residual=r, out=y, sum_out=s)
    for _ in range(2):
        call()
        want = binding.agent_layer_norm_fwd(x, w, b, residual=r)
        assert torch.equal(y, want[0]) and torch.equal(s, want[1])
        x.neg_()
    for bad in (dict(weight=w[:64]), dict(weight=w.half()), dict(weight=w, bias=b.bfloat16()), dict(residual=r[:, :64]), dict(residual=r.float()),
                dict(weight=w.cpu()), dict(out=y.t().contiguous().t())):
        with pytest.raises((AssertionError, RuntimeError)):
            binding.agent_layer_norm_fwd(x, **bad)
    with pytest.raises(RuntimeError, match="AA_ERR_ALIAS"):
        binding.agent_layer_norm_fwd(x[1:], out=x[:-1])
    with pytest.raises((AssertionError, RuntimeError)):
        binding.agent_layer_norm_fwd(x[:0])
