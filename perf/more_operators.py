"""Performance cases of softmax attention (whole sequences, causal or not, shared keys, packed and padded sequences, single
tokens over a long cache) and of layer norm with the residual sum before it, both forward and backward.

Where `own` is false, run() computes the plain form: elementary torch operations in 32 bits, rounded once at the end.  Where
it is true, run() calls paper_2312_08874_amd.binding as a program does: forward calls prepared once on fixed buffers, as a
serving loop keeps them, training steps through the ordinary entry points.

A case is a flat dict.  "kind":

  attn, attn_train    o = softmax(q k^T / sqrt(d)) v over the keys that a query sees; _train: and dq, dk, dv
  norm, norm_train    y = layer norm of x (+ residual), and the sum; _train: and all gradients

Attention: batch, heads_q query heads on heads_k key heads, tokens_q, tokens_k, width d, causal (the last query sees the last
key), layout of the token tensors ("dense" [B,H,N,d], "token" [B,N,H,d], "qkv": slices of a fused projection
[B,N,Hq+2Hk,d]), mix: "whole" (every row in use), "padded" (sequences of their own lengths, from the start of each of
the batch), "packed" (`sequences` of their own lengths one behind the other in one run of rows, which they need not fill);
lengths are drawn from mix_seed.
Norm: rows, width, residual, affine ("none", "weight", "both"), weights ("f32" or "x": the type of x).
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


def _attn(name, kind, dtype, batch, heads, tokens, d, causal, layout, mix="whole", sequences=0, mix_seed=0):
    c = {"kind": kind, "dtype": dtype, "batch": batch, "heads_q": heads[0], "heads_k": heads[1], "tokens_q": tokens[0],
         "tokens_k": tokens[1], "d": d, "causal": causal, "layout": layout, "mix": mix, "sequences": sequences,
         "mix_seed": mix_seed}
    return dict(name=name, **c) if name else c


def _norm(name, kind, dtype, rows, width, residual, affine, weights):
    c = {"kind": kind, "dtype": dtype, "rows": rows, "width": width, "residual": residual, "affine": affine,
         "weights": weights}
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one new token for each of four sequences over short caches: nothing but latency
        _attn("attn_one_token", "attn", "bf16", 4, (8, 8), (1, 300), 64, True, "token", "padded", 0, 1),
        # one new token for each of eight sequences of up to 65536, keys shared by four query heads
        _attn("attn_one_token_long", "attn", "f16", 8, (16, 4), (1, 65536), 128, True, "token", "padded", 0, 2),
        # a block of a small vision transformer, inference on a batch of images
        _attn("attn_deit", "attn", "bf16", 64, (3, 3), (196, 196), 64, False, "qkv"),
        # windows of 7 x 7 in the late stage of a hierarchical vision transformer
        _attn("attn_windows", "attn", "f16", 2048, (12, 12), (49, 49), 32, False, "qkv"),
        # a long prompt, keys shared by four query heads, a length that divides by nothing
        _attn("attn_prompt", "attn", "f16", 1, (16, 4), (8191, 8191), 128, True, "token"),
        # training on images of many sizes, packed into one run of tokens
        _attn("attn_packed_train", "attn_train", "bf16", 1, (8, 8), (8192, 8192), 64, False, "qkv", "packed", 37, 3),
        # training a causal model with shared keys
        _attn("attn_causal_train", "attn_train", "bf16", 2, (16, 4), (4096, 4096), 128, True, "token"),
        # training at 128 x 128 tokens, every token seeing every other: the largest
        _attn("attn_highres_train", "attn_train", "bf16", 1, (8, 8), (128 * 128, 128 * 128), 64, False, "qkv"),
        # training in 32 bits on an image whose sides divide by nothing
        _attn("attn_ragged_f32_train", "attn_train", "f32", 8, (6, 6), (31 * 43, 31 * 43), 48, False, "dense"),
        # the norm before a block for four new tokens: nothing but latency
        _norm("norm_few_tokens", "norm", "bf16", 4, 4096, True, "both", "x"),
        # training at 128 x 128 tokens
        _norm("norm_highres_train", "norm_train", "bf16", 128 * 128, 512, True, "both", "f32"),
        # training a large block on 65536 tokens
        _norm("norm_large_train", "norm_train", "f16", 65536, 2048, True, "both", "x"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges that the listed ones span: 1 to 16384 queries on 1 to 65536 keys of 8 to 128 channels, 1
    to 16 heads, 1 to 512 sequences; 1 to 65536 rows of 16 to 8192 channels.  At most the listed cases' work."""
    kind = rng.choice(("attn", "attn", "attn", "attn_train", "attn_train", "norm", "norm_train"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f16", "f32"))
    if kind.startswith("norm"):
        while True:
            rows, width = _log_int(rng, 1, 65536), _log_int(rng, 16, 8192)
            if rng.random() < 0.7:
                width = (width + 7) // 8 * 8
            if rows * width * (2 if dtype == "f32" else 1) <= 65536 * 2048:
                break
        return _norm(None, kind, dtype, rows, width, rng.random() < 0.6, rng.choice(("none", "weight", "both", "both")),
                     rng.choice(("f32", "x")))
    train = kind == "attn_train"
    while True:
        d = rng.choice((8, 16, 20, 32, 40, 48, 64, 64, 64, 80, 96, 128, 128, 128))
        heads_k = rng.choice((1, 2, 3, 4, 5, 6, 8, 8))
        heads_q = heads_k * rng.choice((1, 1, 1, 2, 3, 4, 8))
        batch, mix, sequences = _log_int(rng, 1, 512), rng.choice(("whole", "whole", "padded", "packed")), 0
        form = rng.choice(("one", "chunk", "self", "self", "self", "cross"))
        if form == "one":
            tokens = (1, _log_int(rng, 2, 65536))
        elif form == "chunk":
            n = _log_int(rng, 2, 2048)
            tokens = (n, n + _log_int(rng, 1, 16384))
        elif form == "self":
            tokens = (_log_int(rng, 2, 16384),) * 2
        else:
            tokens = (_log_int(rng, 2, 8192), _log_int(rng, 2, 8192))
        if mix == "packed":
            batch, sequences = 1, _log_int(rng, 1, 512)
            if form == "one":
                sequences = min(sequences, 64)
                tokens = (sequences, tokens[1])
            elif sequences > tokens[0]:
                continue
        pairs = batch * heads_q * tokens[0] * tokens[1]
        rows = batch * (heads_q * tokens[0] + heads_k * tokens[1])
        heavy = (14 if train else 4) * (8 if dtype == "f32" else 1)
        if heads_q <= 16 and pairs <= 8 * 16384 ** 2 and pairs * d * heavy <= 8 * 16384 ** 2 * 64 * 14 and rows * d <= 3e8:
            break
    layout = rng.choice(("dense", "token", "qkv") if form == "self" else ("dense", "token"))
    causal = rng.random() < (0.2 if form == "cross" else 0.5)
    return _attn(None, kind, dtype, batch, (heads_q, heads_k), tokens, d, causal, layout, mix, sequences, rng.randrange(1 << 20))


# --- lengths ---

def _cut(rng, total, parts):
    """`parts` lengths, some of them perhaps 0, that add up to at most `total`."""
    used = total if rng.random() < 0.5 else total - rng.randint(0, total // 16)
    at = sorted(rng.randint(0, used) for _ in range(parts - 1))
    return [b - a for a, b in zip([0] + at, at + [used])]


def _lengths(case):
    """Lengths of every sequence's queries and keys, on the host."""
    rng = random.Random(case["mix_seed"])
    nq, nk, B = case["tokens_q"], case["tokens_k"], case["batch"]
    if case["mix"] == "packed":
        S = case["sequences"]
        if nq == S:      # one token each
            return [1] * S, _cut(rng, nk, S)
        lq = _cut(rng, nq, S)
        return lq, (lq if nq == nk else _cut(rng, nk, S))
    if case["mix"] == "padded":
        lk = [rng.randint(max(1, nk // 8), nk) for _ in range(B)]
        return (lk if nq == nk else [nq] * B), lk
    return [nq] * B, [nk] * B


# --- inputs ---

def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def rnd(*shape, std=1.0, type=dtype):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(std).to(type)

    if case["kind"].startswith("norm"):
        T, C = case["rows"], case["width"]
        # activations of a residual stream: a mean of their own for each channel, every 97th channel large
        spread = torch.where(torch.arange(C, device="cuda") % 97 == 5, 12.0, 1.0)
        offset = rnd(C, std=0.3, type=torch.float32)

        def stream():
            return torch.randn(T, C, generator=gen, device="cuda").mul_(spread).add_(offset).to(dtype)
        s = {"x": stream()}
        if case["residual"]:
            s["r"] = stream()
        wtype = torch.float32 if case["weights"] == "f32" else dtype
        if case["affine"] != "none":
            s["w"] = (1.0 + rnd(C, std=0.2, type=torch.float32)).to(wtype)
        if case["affine"] == "both":
            s["b"] = rnd(C, std=0.2, type=wtype)
        if case["kind"] == "norm_train":
            s["dy"] = rnd(T, C)
            if case["residual"]:
                s["dsum"] = rnd(T, C)
        return s
    B, Hq, Hk, nq, nk, d = (case[k] for k in ("batch", "heads_q", "heads_k", "tokens_q", "tokens_k", "d"))

    def tokens(H, N):
        return rnd(B, N, H, d).permute(0, 2, 1, 3) if case["layout"] != "dense" else rnd(B, H, N, d)

    if case["layout"] == "qkv":
        fused = rnd(B, nq, Hq + 2 * Hk, d).permute(0, 2, 1, 3)
        s = {"q": fused[:, :Hq], "k": fused[:, Hq:Hq + Hk], "v": fused[:, Hq + Hk:]}
    else:
        s = {"q": tokens(Hq, nq), "k": tokens(Hk, nk), "v": tokens(Hk, nk)}
    if case["kind"] == "attn_train":
        s["do"] = tokens(Hq, nq)
    return s


def _mixed(case):
    """What tells the sequences apart, as device tensors: keyword arguments of the attention."""
    lq, lk = _lengths(case)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    if case["mix"] == "packed":
        starts = [[sum(v[:i]) for i in range(len(v) + 1)] for v in (lq, lk)]
        return {"starts": (ints(starts[0]), ints(starts[1]))}
    if case["mix"] == "padded":
        return {"lengths": (ints(lq), ints(lk))}
    return {}


def prepare(case, seed):
    s = _inputs(case, seed)
    state = {"case": case, "in": s}
    if case["kind"].startswith("attn"):
        state["mixed"] = _mixed(case)
    if own:
        from paper_2312_08874_amd import binding
        state["binding"] = binding
        if case["kind"] == "attn":
            # rows that belong to no sequence stay zeros
            q = s["q"]
            state["out"] = torch.zeros(q.shape[0], q.shape[2], q.shape[1], q.shape[3], dtype=q.dtype, device="cuda").permute(0, 2, 1, 3) \
                if case["layout"] != "dense" else torch.zeros_like(q)
            state["call"] = binding.prepare_softmax_attn(q, s["k"], s["v"], causal=case["causal"], out=state["out"], **state["mixed"])
        elif case["kind"] == "norm":
            state["out"] = (torch.empty_like(s["x"]),) + ((torch.empty_like(s["x"]),) if case["residual"] else ())
            state["call"] = binding.prepare_layer_norm(s["x"], s.get("w"), s.get("b"), residual=s.get("r"), eps=EPS, out=state["out"][0],
                                                       sum_out=state["out"][1] if case["residual"] else None)
    return state


# --- one pass ---

def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    case, s = state["case"], state["in"]
    if "call" in state:
        state["call"]()
        return state["out"]
    binding = state["binding"]
    if case["kind"] == "norm_train":
        y, *total, saved = binding.agent_layer_norm_fwd(s["x"], s.get("w"), s.get("b"), residual=s.get("r"), eps=EPS, save=True)
        # from what the sum is of: its rounding would show in the weights' gradients
        g = binding.agent_layer_norm_bwd(s["x"], s["dy"], saved, s.get("w"), s.get("b"), residual=s.get("r"), dsum=s.get("dsum"))
        return {"y": y, **({"sum": total[0]} if total else {}), **g}
    mixed = state["mixed"]
    out, lse = binding.agent_softmax_attn_fwd(s["q"], s["k"], s["v"], causal=case["causal"], save=True, **mixed)
    return {"out": out, **binding.agent_softmax_attn_bwd(s["q"], s["k"], s["v"], out, lse, s["do"], causal=case["causal"], **mixed)}


def _plain(state):
    case, s = state["case"], state["in"]
    return _plain_norm(case, s) if case["kind"].startswith("norm") else _plain_attn(case, s, state["mixed"])


def _seen(case, mixed, device):
    """Which keys a query sees, [1 or B, nq, nk]."""
    nq, nk = case["tokens_q"], case["tokens_k"]
    i, j = torch.arange(nq, device=device)[None, :, None], torch.arange(nk, device=device)[None, None, :]
    if case["mix"] == "packed":
        sq, sk = mixed["starts"]
        # the sequence of a row: how many sequences end at it or before; rows behind the last belong to none
        oq, ok = torch.searchsorted(sq[1:], i.flatten(), right=True), torch.searchsorted(sk[1:], j.flatten(), right=True)
        last = len(sq) - 2
        lag = (sk[1:] - sq[1:])[oq.clamp(max=last)]      # the ends of a sequence's queries and keys lie so far apart
        seen = (oq[:, None] == ok[None, :]) & (oq <= last)[:, None]
        if case["causal"]:
            seen = seen & (j[0] <= i[0] + lag[:, None])
        return seen[None]
    if case["mix"] == "padded":
        lq, lk = (v[:, None, None] for v in mixed["lengths"])
    else:
        lq, lk = nq, nk
    seen = (j < lk) & (i < lq)
    return seen & (j <= i + (lk - lq)) if case["causal"] else seen


def _plain_attn(case, s, mixed):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    B, Hq, nq, d = q.shape
    Hk, nk = k.shape[1:3]
    G, scale = Hq // Hk, d ** -0.5
    seen = _seen(case, mixed, q.device)[:, None, None]
    kt, vt = k.transpose(2, 3).contiguous(), v.transpose(2, 3).contiguous()

    def rows(t):      # the query heads that share keys as rows of one product
        return t.reshape(B, Hk, G * nq, t.shape[-1])

    p = (rows(q) @ kt).mul_(scale).view(B, Hk, G, nq, nk).masked_fill_(~seen, -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m.masked_fill(m == -math.inf, 0.0)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_(min=1e-30)).view(B, Hk, G * nq, nk)
    o = p @ v
    out = o.view(B, Hq, nq, d).to(s["q"].dtype)
    if case["kind"] == "attn":
        return out
    do = rows(s["do"].float())
    dv = p.transpose(2, 3).contiguous() @ do
    ds = (do @ vt).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    ds = torch.where(p > 0, ds, 0.0)
    dq = (ds @ k).view(B, Hq, nq, d)
    dk = ds.transpose(2, 3).contiguous() @ rows(q)
    return {"out": out, "dQ": dq.to(out.dtype), "dK": dk.to(out.dtype), "dV": dv.to(out.dtype)}


def _plain_norm(case, s):
    dtype = s["x"].dtype
    x = s["x"].float() + s["r"].float() if case["residual"] else s["x"].float()
    w = s["w"].float() if "w" in s else 1.0
    c = x - x.mean(-1, keepdim=True)
    rs = (c.square().mean(-1, keepdim=True) + EPS).rsqrt()
    h = c * rs
    y = h * w
    if "b" in s:
        y = y + s["b"].float()
    if case["kind"] == "norm":
        return (y.to(dtype),) + ((x.to(dtype),) if case["residual"] else ())
    dy = s["dy"].float()
    g = dy * w
    dx = (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True)) * rs
    out = {"y": y.to(dtype)}
    if case["residual"]:
        out["sum"] = x.to(dtype)
        dx = dx + s["dsum"].float()
    out["dx"] = dx.to(dtype)
    if "w" in s:
        out["dw"] = (dy * h).sum(0).to(s["w"].dtype)
    if "b" in s:
        out["db"] = dy.sum(0).to(s["b"].dtype)
    return out


# --- what a pass cannot do without ---

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    train = case["kind"].endswith("_train")
    if case["kind"].startswith("norm"):
        elements = case["rows"] * case["width"]
        tensors = (4 + 2 if train else 2 + 2) if case["residual"] else (4 if train else 2)
        weights = {"none": 0, "weight": 1, "both": 2}[case["affine"]] * (2 if train else 1)
        return {"bytes": es * tensors * elements + (4 if case["weights"] == "f32" else es) * weights * case["width"],
                "flops": (22 if train else 8) * elements}
    pairs = rows_q = rows_k = 0
    for lq, lk in zip(*_lengths(case)):
        rows_q, rows_k = rows_q + lq, rows_k + lk
        if not case["causal"]:
            pairs += lq * lk
        elif lq:
            first = max(0, lq - lk)                      # queries before it see nothing
            pairs += sum((lk - lq + 1 + first, lk)) * (lq - first) // 2
    per = 4 if train else 2
    return {"bytes": es * case["d"] * per * (case["heads_q"] * rows_q + case["heads_k"] * rows_k),
            "flops": (14 if train else 4) * case["d"] * case["heads_q"] * pairs}


# --- the operators' definitions in 64 bits ---

def exact(case, seed):
    """From the definitions, sequence by sequence and head by head, gradients by differentiation of the forward pass."""
    s = _inputs(case, seed)
    return _exact_norm(case, s) if case["kind"].startswith("norm") else _exact_attn(case, s)


def _exact_norm(case, s):
    train = case["kind"] == "norm_train"
    v = {k: t.double().requires_grad_(train and k in ("x", "w", "b")) for k, t in s.items()}
    total = v["x"] + v["r"] if case["residual"] else v["x"]
    var, mean = torch.var_mean(total, -1, correction=0, keepdim=True)
    y = (total - mean) / torch.sqrt(var + EPS)
    if "w" in v:
        y = v["w"] * y
    if "b" in v:
        y = v["b"] + y
    if not train:
        return (y,) + ((total,) if case["residual"] else ())
    leaves = [k for k in ("x", "w", "b") if k in v]
    g = dict(zip(leaves, torch.autograd.grad([y] + ([total] if case["residual"] else []), [v[k] for k in leaves],
                                             [v["dy"]] + ([v["dsum"]] if case["residual"] else []))))
    out = {"y": y.detach()}
    if case["residual"]:
        out["sum"] = total.detach()
    out["dx"] = g["x"]
    out.update({"d" + k: g[k] for k in ("w", "b") if k in g})
    return out


def _exact_attn(case, s):
    train = case["kind"] == "attn_train"
    q, k, v = (s[n].double() for n in ("q", "k", "v"))
    group, scale = case["heads_q"] // case["heads_k"], 1.0 / math.sqrt(case["d"])
    lq, lk = _lengths(case)
    packed = case["mix"] == "packed"
    out, dq, dk, dv = (torch.zeros_like(t) for t in (q, q, k, v))
    # whole batches of equal lengths go together, as many as 2 GB of scores hold
    if case["mix"] == "whole":
        each = max(1, int(2 ** 28 / (case["tokens_q"] * case["tokens_k"])))
        parts = [(slice(b, b + each), 0, lq[0], 0, lk[0]) for b in range(0, case["batch"], each)]
    else:
        parts, aq, ak = [], 0, 0
        for b, (n, m) in enumerate(zip(lq, lk)):
            parts.append((slice(0, 1) if packed else slice(b, b + 1), aq, n, ak, m))
            if packed:
                aq, ak = aq + n, ak + m
    if len(parts) * case["heads_q"] > 20000:
        return None
    for at, fq, n, fk, m in parts:
        if n == 0 or m == 0:
            continue
        here = None
        if case["causal"]:
            here = torch.ones(n, m, dtype=torch.bool, device="cuda").tril(m - n)
        heads = range(case["heads_q"]) if n * m > 2 ** 22 else [slice(h * group, (h + 1) * group) for h in range(case["heads_k"])]
        for h in heads:
            hq = h if isinstance(h, slice) else slice(h, h + 1)
            hk = hq.start // group
            x = q[at, hq, fq:fq + n].clone().requires_grad_(train)
            y, z = (t[at, hk:hk + 1, fk:fk + m].clone().requires_grad_(train) for t in (k, v))
            score = torch.matmul(x, y.transpose(-1, -2).contiguous()) * scale
            if here is not None:
                score = score.masked_fill(~here, -math.inf)
                # a query that sees nothing: its weights are all zero
                weight = torch.softmax(score.masked_fill(~here.any(-1, keepdim=True), 0.0), -1) * here
            else:
                weight = torch.softmax(score, -1)
            o = torch.matmul(weight, z)
            out[at, hq, fq:fq + n] = o.detach()
            if train:
                gx, gy, gz = torch.autograd.grad(o, [x, y, z], s["do"][at, hq, fq:fq + n].double())
                dq[at, hq, fq:fq + n] = gx
                dk[at, hk:hk + 1, fk:fk + m] += gy
                dv[at, hk:hk + 1, fk:fk + m] += gz
    return {"out": out, "dQ": dq, "dK": dk, "dV": dv} if train else out
