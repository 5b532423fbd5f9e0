"""Rotation by positions and the norm of queries and keys in 64 bits, on the host: the reference of the GPU tests."""
import torch


def pair_channels(pairs, pairing):
    P, out, start = sum(pairs), [], 0
    for p in pairs:
        for j in range(p):
            out.append({"adjacent": (2 * (start + j), 2 * (start + j) + 1), "halves": (start + j, P + start + j),
                        "axis_halves": (2 * start + j, 2 * start + p + j)}[pairing])
        start += p
    return out


def positions_of(rope_spec, B, N):
    """[B, N, axes] float64, from the grid or from the tensor given."""
    if rope_spec.get("positions") is not None:
        p = rope_spec["positions"].double().cpu()
        return p.expand(B, *p.shape[-2:]) if p.dim() == 2 else p
    axes = torch.meshgrid(*(torch.arange(g, dtype=torch.float64) for g in rope_spec["grid"]), indexing="ij")
    return torch.stack([a.reshape(-1) for a in axes], -1).expand(B, N, len(axes))


def rotate(x, rope_spec, back=False):
    """x [B,H,N,d] float64; rope_spec: dict(pairs, pairing, grid or positions, freqs) or None."""
    if rope_spec is None:
        return x.clone()
    pos = positions_of(rope_spec, x.shape[0], x.shape[2])
    out, axis = x.clone(), [a for a, p in enumerate(rope_spec["pairs"]) for _ in range(p)]
    for j, (c0, c1) in enumerate(pair_channels(rope_spec["pairs"], rope_spec["pairing"])):
        phi = pos[:, None, :, axis[j]] * rope_spec["freqs"][j] * (-1.0 if back else 1.0)
        out[..., c0] = x[..., c0] * phi.cos() - x[..., c1] * phi.sin()
        out[..., c1] = x[..., c0] * phi.sin() + x[..., c1] * phi.cos()
    return out


def weight_of(w, H, d):
    if w is None:
        return torch.ones(1, 1, 1, d, dtype=torch.float64)
    w = w.double().cpu()
    return w.reshape(1, 1, 1, d) if w.dim() == 1 else w.reshape(1, H, 1, d)


def norm_fwd(x, w, eps, rope_spec):
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return rotate(x * r * weight_of(w, x.shape[1], x.shape[3]), rope_spec)


def norm_bwd(x, w, eps, rope_spec, dy):
    """dx, dw (dw shaped like the weight), and the magnitudes their rounding errors go by."""
    d = x.shape[3]
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    z = rotate(dy, rope_spec, back=True)
    u = z * weight_of(w, x.shape[1], d)
    dx = r * u - x * r ** 3 * (u * x).mean(-1, keepdim=True)
    scale = r * u.abs().amax(-1, keepdim=True) + x.abs() * r ** 3 * (u * x).abs().mean(-1, keepdim=True)
    terms = z * x * r
    zmax = z.abs().amax(-1, keepdim=True) * (x * r).abs()
    axes = (0, 1, 2) if w is None or w.dim() == 1 else (0, 2)
    return dx, scale, terms.sum(axes), zmax.sum(axes)


def eps_of(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Half the spacing of the subnormal numbers."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
