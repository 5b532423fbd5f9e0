"""Softmax attention and its gradients in 64 bits on the host, with the error that a pass in fp32 with 16-bit operands may have.

Bounds, per element, u = half a step of the element type, e = 2^-24.  A score is off by (d + 2) e of the sum of its terms'
magnitudes, its exponential by that and 4 e of the exponent, which is at most the score's distance from the row's largest plus the
kernel's slack of 8 ln 2; call it a.  A weight is rounded once more, by u, and lse, the sum of rounded weights, is off by a + u at the
most.  So, with A = sum of p |v| and n keys:
  o:   u |o| + (2 a + 2 u + (n + 8) e) A
  lse: a + u + (n + 8) e + 2 e |lse|
Backward, p = exp(score - lse) is off by b = 2 a + u + 2 e |lse| + (n + 8) e relative, t = do . v - D by the error of o in D and by
(d + 2) e of the terms' magnitudes, ds = p t by p (b |t| + its error), and both are rounded, by u; sums over n more terms add (n + 8) e.
fp16 numbers below 2^-14 are rounded to a step of 2^-24, which p (forward: times 1 or less, backward: times 2^12) and ds (times 2^15
over twice the largest |do| |v| at the least a quarter of that) may be.
An exponential under 2^-126 is 0, and so is an operand of a product in bf16 or fp32: p is off by 2^-126 for either, o relative to its row's
weights by no more, ds = p t by |t| times that and by 2^-126 for itself as an operand."""
import torch

E = 2.0 ** -24
ZERO = 2 * 2.0 ** -126


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def spans(B, nq, nk, starts=None, lengths=None):
    """(batch element, first query, queries, first key, keys) of every sequence."""
    if starts is not None:
        sq, sk = (s.tolist() for s in starts)
        return [(0, a, b - a, c, d - c) for a, b, c, d in zip(sq, sq[1:], sk, sk[1:])]
    lq = [nq] * B if lengths is None or lengths[0] is None else lengths[0].tolist()
    lk = [nk] * B if lengths is None or lengths[1] is None else lengths[1].tolist()
    return [(b, 0, q, 0, k) for b, (q, k) in enumerate(zip(lq, lk))]


def attention(q, k, v, causal, where, scale=None, do=None, peak=0.0):
    """{"out", "lse"} and, with do, {"dQ", "dK", "dV"}: each (value, bound), rows of no sequence 0 (lse -inf) with bound 0.
    peak: of the call's rows, where these are some of them, the largest |do| |v|."""
    dtype = q.dtype
    u = 0.0 if dtype == torch.float32 else unit(dtype)
    fine = 2.0 ** -25 if dtype == torch.float16 else 0.0
    round_out = unit(dtype)
    Q, K, V = (t.detach().double().cpu() for t in (q, k, v))
    G = None if do is None else do.detach().double().cpu()
    B, H, N, d = Q.shape
    group = H // K.shape[1]
    c = d ** -0.5 if not scale else scale
    res = {n: [torch.zeros_like(t), torch.zeros_like(t)] for n, t in (("out", Q), ("dQ", Q), ("dK", K), ("dV", V))}
    res["lse"] = [torch.full((B, H, N), -float("inf"), dtype=torch.float64), torch.zeros(B, H, N, dtype=torch.float64)]
    res["used_q"], res["used_k"] = torch.zeros(B, N, dtype=torch.bool), torch.zeros(B, K.shape[2], dtype=torch.bool)
    if G is not None and not peak:
        peak = max((G[b, :, a:a + n].norm(dim=-1).max().item() for b, a, n, _, _ in where if n), default=0.0) * \
            max((V[b, :, a:a + n].norm(dim=-1).max().item() for b, _, _, a, n in where if n), default=0.0)
    for b, q0, nq, k0, nk in where:
        res["used_q"][b, q0:q0 + nq], res["used_k"][b, k0:k0 + nk] = True, True
        if nq == 0 or nk == 0:
            continue
        rows, keys = slice(q0, q0 + nq), slice(k0, k0 + nk)
        seen = torch.ones(nq, nk, dtype=torch.bool)
        if causal:
            seen = seen.tril(nk - nq)
        for h in range(H):
            x, y, z = Q[b, h, rows], K[b, h // group, keys], V[b, h // group, keys]
            s = (x @ y.t() * c).masked_fill(~seen, -float("inf"))
            lse = torch.logsumexp(s, -1, keepdim=True)
            empty = torch.isinf(lse)
            p = torch.where(seen & ~empty, (s - lse.masked_fill(empty, 0.0)).exp(), 0.0)
            size = torch.where(seen, x.abs() @ y.abs().t() * c, 0.0).amax(-1, keepdim=True)
            n = seen.sum(-1, keepdim=True).double()
            a = (d + 2) * E * size + 4 * E * (2 * size + 6)
            A, o = p @ z.abs(), p @ z
            do_o = (2 * a + 2 * u + (n + 8) * E) * A + (fine + ZERO) * (seen.double() @ z.abs())
            res["out"][0][b, h, rows] = o
            res["out"][1][b, h, rows] = round_out * (o.abs() + do_o) + do_o + smallest(dtype)
            level = lse.masked_fill(empty, 0.0)
            res["lse"][0][b, h, rows] = lse[:, 0]
            res["lse"][1][b, h, rows] = (a + u + (n + 8) * E + fine * n + 2 * E * level.abs())[:, 0] + 1e-30
            if G is None:
                continue
            g = G[b, h, rows]
            # D takes o with what rounding took from it, rounded in its turn
            off_o = do_o + (round_out if dtype == torch.float32 else round_out ** 2) * (o.abs() + do_o) + smallest(dtype)
            rel = 2 * a + u + (n + 8) * E + 2 * E * level.abs() + fine * n
            D = (g * o).sum(-1, keepdim=True)
            t = g @ z.t() - D
            dt = (d + 2) * E * (g.abs() @ z.abs().t() + (g * o).abs().sum(-1, keepdim=True)) + \
                (g.abs() * off_o).sum(-1, keepdim=True)
            ds = p * t
            off_p = p * (rel + u) + (fine * 2.0 ** -12 + ZERO) * seen
            off_s = p * (rel * t.abs() + dt) * (1 + u) + u * ds.abs() + (fine * peak * 2.0 ** -12 * seen) + 4 * E * p * (t.abs() + D.abs())
            off_s = off_s + ZERO * (t.abs() + 1) * seen
            sums = (max(nq * group, nk) + 8) * E
            res["dQ"][0][b, h, rows] = c * (ds @ y)
            res["dQ"][1][b, h, rows] = c * (off_s @ y.abs() + sums * (ds.abs() @ y.abs()))
            res["dK"][0][b, h // group, keys] += c * (ds.t() @ x)
            res["dK"][1][b, h // group, keys] += c * (off_s.t() @ x.abs() + sums * (ds.abs().t() @ x.abs()))
            res["dV"][0][b, h // group, keys] += p.t() @ g
            res["dV"][1][b, h // group, keys] += off_p.t() @ g.abs() + sums * (p.t() @ g.abs())
    for n in ("dQ", "dK", "dV"):
        value, bound = res[n]
        res[n][1] = torch.where(res["used_q" if n == "dQ" else "used_k"][:, None, :, None],
                                round_out * (value.abs() + bound) + bound + smallest(dtype), 0.0)
    return res
