"""Layer norm and its gradients in 64 bits on the host, with the error that a pass in fp32 may have.

Bounds, per element, u = half a step of the type of a result, e = 2^-24, C channels, R rows; m(x) = mean |x| of a row.  A sum of n terms is
off by n e of the sum of their magnitudes at the most.  The sum s of x and r: e |s|.  The mean: (C + 2) e m(s); what is left of s
without it: that + 2 e (|s| + |mean|) =: dc; the deviation's square by 2 dc |c| averaged and (C + 4) e of itself, its root's inverse
relative by half that.  h = c r is off by dc r + |h| (relative of r + 2 e)."""
import torch

E = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def rounded(value, bound, dtype):
    return value, half_step(dtype) * (value.abs() + bound) + bound + smallest(dtype)


def forward(x, w, b, eps, residual=None):
    s = x.double().cpu()
    ds = torch.zeros_like(s)
    if residual is not None:
        s = s + residual.double().cpu()
        ds = E * s.abs()
    C = s.shape[-1]
    mean = s.mean(-1, keepdim=True)
    dmean = (C + 2) * E * s.abs().mean(-1, keepdim=True) + ds.mean(-1, keepdim=True)
    c = s - mean
    dc = ds + dmean + 2 * E * (s.abs() + mean.abs())
    var = c.square().mean(-1, keepdim=True)
    dvar = 2 * (dc * c.abs()).mean(-1, keepdim=True) + dc.square().mean(-1, keepdim=True) + (C + 4) * E * var
    r = (var + eps).rsqrt()
    rel = 0.5 * dvar / (var + eps) * 1.5 + 4 * E      # the square root's slope over an error of under a third
    h = c * r
    dh = dc * r * (1 + rel) + h.abs() * (rel + 2 * E)
    W = torch.ones(C, dtype=torch.float64) if w is None else w.double().cpu()
    Bs = torch.zeros(C, dtype=torch.float64) if b is None else b.double().cpu()
    y = h * W + Bs
    dy = dh * W.abs() + 2 * E * ((h * W).abs() + Bs.abs())
    return {"y": rounded(y, dy, x.dtype), "sum": rounded(s, ds, x.dtype), "h": (h, dh), "r": (r, rel), "mean": (mean, dmean)}


def backward(s, dy, w, b, eps, dsum=None, residual=None):
    """From the normed rows s (+ residual) as they are."""
    f = forward(s, None, None, eps, residual)
    (h, dh), (r, rel) = f["h"], f["r"]
    C, R = s.shape[-1], s.numel() // s.shape[-1]
    d = dy.double().cpu()
    W = torch.ones(C, dtype=torch.float64) if w is None else w.double().cpu()
    g = d * W
    mg, mgh = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dmg = (C + 4) * E * g.abs().mean(-1, keepdim=True)
    dmgh = (C + 6) * E * (g * h).abs().mean(-1, keepdim=True) + (g.abs() * dh).mean(-1, keepdim=True)
    t = g - mg - h * mgh
    dt = 3 * E * (g.abs() + mg.abs() + (h * mgh).abs()) + dmg + dh * (mgh.abs() + dmgh) + h.abs() * dmgh
    dx = r * t
    bound = r * (dt * (1 + rel) + t.abs() * (rel + 2 * E))
    if dsum is not None:
        dx = dx + dsum.double().cpu()
        bound = bound + 2 * E * dx.abs()
    flat = lambda v: v.reshape(R, C)      # noqa: E731
    out = {"dx": rounded(dx, bound, s.dtype)}
    if w is not None:
        out["dw"] = rounded(flat(d * h).sum(0), flat(d.abs() * dh).sum(0) + (R + 4) * E * flat((d * h).abs()).sum(0), w.dtype)
    if b is not None:
        out["db"] = rounded(flat(d).sum(0), (R + 4) * E * flat(d.abs()).sum(0), b.dtype)
    return out
