"""The gated feed-forward block in 64 bits, and how far a result may be off it.

Bounds go through the formulas from left to right.  U = 2^-24 is a rounding of fp32, half one of the element type, relative to the
value.  A sum of K products in any order is off by at most (K + 4) U times the sum of their magnitudes (K additions, the
products' own rounding, the bias).  The activations and their derivatives have slopes of at most 1.2 and 1.1, and are computed with
an error of `act` (1 + |g|): hardware exp and reciprocal for 16-bit types, expf and erfcf for fp32.  What the backward pass keeps of
the forward pass has 24 bits (16 of them significant), for fp32 all."""
import math

import torch

U = 2.0 ** -24


def act(kind, g):
    if kind == "silu":
        e = torch.sigmoid(g)
        return g * e, e * (1 + g * (1 - e))
    if kind == "gelu":
        e = torch.special.ndtr(g)
        return g * e, e + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    if kind == "sigmoid":
        e = torch.sigmoid(g)
        return e, e * (1 - e)
    on = (g > 0).double()
    return g * on, on


def block(s, kind, backward=True):
    """s: dict of tensors (any type) x, w_*, b_* or absent, dy.  Returns {name: (value, bound)} in float64."""
    dtype = s["x"].dtype
    half, low = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    kept, fn = (0.0, 2.0 ** -21) if dtype == torch.float32 else (2.0 ** -16, 2.0 ** -19)
    v = {k: t.double() for k, t in s.items() if t is not None}
    x, wg, wu, wd = v["x"].reshape(-1, v["x"].shape[-1]), v["w_gate"], v["w_up"], v["w_down"]
    T, C = x.shape
    F = wg.shape[0]
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    bg, bu, bd = (v.get(k, zero) for k in ("b_gate", "b_up", "b_down"))

    def rounded(value, off):
        return value, off + half * value.abs() + low
    g, u = x @ wg.t() + bg, x @ wu.t() + bu
    eg, eu = (C + 4) * U * (x.abs() @ wg.abs().t() + bg.abs()), (C + 4) * U * (x.abs() @ wu.abs().t() + bu.abs())
    a, d = act(kind, g)
    ea = 1.2 * eg + fn * (1 + g.abs())
    h = a * u
    eh = rounded(h, u.abs() * ea + a.abs() * eu + ea * eu)[1]
    y = h @ wd.t() + bd
    out = {"y": rounded(y, eh @ wd.abs().t() + (F + 4) * U * (h.abs() @ wd.abs().t() + bd.abs()))}
    if not backward:
        return out
    dy = v["dy"].reshape(T, C)
    dh, edh = dy @ wd, (C + 4) * U * (dy.abs() @ wd.abs())
    p = u * d
    ep = d.abs() * eu + (u.abs() + eu) * (1.1 * eg + fn * (1 + g.abs())) + kept * p.abs()
    if kind == "relu":      # next to its corner either slope is right
        ep = ep + u.abs() * (g.abs() <= eg).double()
    dg, edg = rounded(dh * p, dh.abs() * ep + (p.abs() + ep) * edh)
    eq = ea + kept * a.abs()
    du, edu = rounded(dh * a, dh.abs() * eq + (a.abs() + eq) * edh)
    out["dx"] = rounded(dg @ wg + du @ wu, edg @ wg.abs() + edu @ wu.abs() + (2 * F + 4) * U * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()))
    for name, e, ee in (("gate", dg, edg), ("up", du, edu)):
        out["dw_" + name] = rounded(e.t() @ x, ee.t() @ x.abs() + (T + 4) * U * (e.abs().t() @ x.abs()))
        out["db_" + name] = rounded(e.sum(0), ee.sum(0) + (T + 4) * U * e.abs().sum(0))
    out["dw_down"] = rounded(dy.t() @ h, dy.abs().t() @ eh + (T + 4) * U * (dy.abs().t() @ h.abs()))
    out["db_down"] = rounded(dy.sum(0), (T + 4) * U * dy.abs().sum(0))
    return out
