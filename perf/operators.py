"""Operators of a decoder layer's training step around the attention, for timing: token embedding, normalisation
with the residual stream, and the gated feed-forward block, forward and backward.

A case is one call, or one forward and its backward, on a packed row of tokens.  Token counts and widths are
those of the package's workloads (workloads.py), of its tests, or lie between them.  Activations, their gradients
and the residual stream are N(0, 1); weights have the variance that keeps a projection's output at 1.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One token at a time through a frozen model: the residual is added and normalised.  A launch's latency.
        {"name": "norm-one-token", "op": "norm", "pass": "forward", "tokens": 1, "hidden": 4096, "kind": "rms",
         "residual": True, "x": "bf16", "weight": "bf16"},
        # The residual stream of a layer on the pack of the benchmark with lengths of every size.
        {"name": "norm-llama3-8b", "op": "norm", "pass": "forward", "tokens": 16215, "hidden": 4096, "kind": "rms",
         "residual": True, "x": "bf16", "weight": "bf16"},
        # Gradients on the largest pack, parameters kept in fp32, the residual stream's own gradient added.
        {"name": "norm-multi-turn-backward", "op": "norm", "pass": "backward", "tokens": 31041, "hidden": 4096,
         "kind": "layer", "residual": True, "x": "bf16", "weight": "f32"},
        # The tiny configuration (four heads of 64) in fp32, forward and backward.
        {"name": "norm-tiny-step", "op": "norm", "pass": "step", "tokens": 672, "hidden": 256, "kind": "layer",
         "residual": False, "x": "f32", "weight": "f32"},
        # A width that fills no vector and an odd number of tokens.
        {"name": "norm-ragged-step", "op": "norm", "pass": "step", "tokens": 5465, "hidden": 1237, "kind": "layer",
         "residual": True, "x": "bf16", "weight": "bf16"},
        # The first operation of a step on many short samples.
        {"name": "embed-short-many", "op": "embed", "pass": "forward", "tokens": 7965, "hidden": 4096,
         "vocab": 128256, "x": "bf16", "grad": "bf16"},
        # The table's gradient: most of the vocabulary does not occur, some tokens occur hundreds of times.
        {"name": "embed-llama3-8b-backward", "op": "embed", "pass": "backward", "tokens": 16215, "hidden": 4096,
         "vocab": 128256, "x": "bf16", "grad": "bf16"},
        # A gradient kept in fp32, with a width and a vocabulary that divide by little.
        {"name": "embed-ragged-backward", "op": "embed", "pass": "backward", "tokens": 31041, "hidden": 1002,
         "vocab": 50257, "x": "bf16", "grad": "f32"},
        # One token through the block: the weights are read once, nothing is kept for a backward pass.
        {"name": "ffn-one-token", "op": "ffn", "pass": "forward", "tokens": 1, "hidden": 4096, "ffn": 14336},
        # The tiny configuration's step: launches.
        {"name": "ffn-tiny-step", "op": "ffn", "pass": "step", "tokens": 672, "hidden": 256, "ffn": 696},
        # A small model's step on a small odd pack.
        {"name": "ffn-small-step", "op": "ffn", "pass": "step", "tokens": 1815, "hidden": 2048, "ffn": 5632},
        # A layer of the benchmark's model on its pack, forward and backward.
        {"name": "ffn-llama3-8b-step", "op": "ffn", "pass": "step", "tokens": 16215, "hidden": 4096, "ffn": 14336},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "embed", "ffn", "ffn"))
    if op == "norm":
        x, weight = rng.choice((("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")))
        return {"op": op, "pass": rng.choice(("forward", "backward", "step")), "tokens": _log_uniform(rng, 1, 32768),
                "hidden": _log_uniform(rng, 64, 8192), "kind": rng.choice(("layer", "rms")),
                "residual": rng.random() < 0.6, "x": x, "weight": weight}
    if op == "embed":
        x, grad = rng.choice((("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")))
        return {"op": op, "pass": rng.choice(("forward", "backward")), "tokens": _log_uniform(rng, 1, 32768),
                "hidden": _log_uniform(rng, 16, 4096), "vocab": _log_uniform(rng, 300, 131072), "x": x, "grad": grad}
    case = {"op": op, "pass": rng.choice(("forward", "step", "step")), "tokens": _log_uniform(rng, 1, 16000),
            "hidden": 8 * _log_uniform(rng, 8, 512), "ffn": 8 * _log_uniform(rng, 16, 1792)}
    return case


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=gen, device="cuda")
    return (t.mul_(std) if std != 1.0 else t).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, D = case["tokens"], case["hidden"]
    s = dict(case)
    if case["op"] == "norm":
        dtype, wtype = DTYPES[case["x"]], DTYPES[case["weight"]]
        rms = case["kind"] == "rms"
        s["x"] = _normal(gen, T, D, dtype=dtype)
        s["residual"] = _normal(gen, T, D, std=2.0, dtype=dtype) if case["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(wtype)
        s["bias"] = None if rms else _normal(gen, D, std=0.2, dtype=wtype)
        s["eps"], s["rms"] = 1e-5, rms
        s["d_out"] = _normal(gen, T, D, dtype=dtype)
        s["d_total"] = _normal(gen, T, D, dtype=dtype) if case["residual"] else None
        # what a forward pass would have left for the backward pass: mean and 1 / deviation of each row
        wide = s["x"].double()
        mean = torch.zeros_like(wide[:, 0]) if rms else wide.mean(1)
        s["stats"] = torch.stack([mean, ((wide - mean[:, None]).square().mean(1) + s["eps"]).rsqrt()]).float()
    elif case["op"] == "embed":
        vocab, dtype = case["vocab"], DTYPES[case["x"]]
        # token frequencies fall as 1 / rank, as in text
        u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
        s["ids"] = ((vocab + 1) ** u - 1).long().clamp_(0, vocab - 1).to(torch.int32)
        s["scale"] = D ** 0.5
        if case["pass"] == "forward":
            s["table"] = _normal(gen, vocab, D, std=D ** -0.5, dtype=dtype)
        else:
            s["d_out"] = _normal(gen, T, D, dtype=dtype)
    else:
        F = case["ffn"]
        s["x"] = _normal(gen, T, D)
        s["w"] = [_normal(gen, D, F, std=D ** -0.5), _normal(gen, D, F, std=D ** -0.5), _normal(gen, F, D, std=F ** -0.5)]
        s["d_out"] = _normal(gen, T, D)
    return s


def _plain_norm(s, x):
    """Output, statistics and, where there is a residual, the sum that was normalised (rounded to its type first)."""
    total = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    wide = total.float()
    mean = torch.zeros_like(wide[:, 0]) if s["rms"] else wide.mean(1)
    centred = wide - mean[:, None]
    rstd = (centred.square().mean(1) + s["eps"]).rsqrt()
    out = centred * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        out = out + s["bias"].float()
    return [out.to(x.dtype), torch.stack([mean, rstd])] + ([] if s["residual"] is None else [total])


def _plain_norm_backward(s, x, stats):
    g = s["d_out"].float()
    unit = (x.float() - stats[0][:, None]) * stats[1][:, None]
    gw = g * s["weight"].float()
    dx = gw - unit * (gw * unit).mean(1, keepdim=True)
    if not s["rms"]:
        dx = dx - gw.mean(1, keepdim=True)
    dx = dx * stats[1][:, None]
    if s["d_total"] is not None:
        dx = dx + s["d_total"].float()
    # sums over all tokens
    dweight = (g.double() * unit.double()).sum(0).to(s["weight"].dtype)
    return [dx.to(x.dtype), dweight] + ([] if s["rms"] else [g.double().sum(0).to(s["weight"].dtype)])


def _run_norm(s):
    forward = s["pass"] != "backward"
    x, outs = s["x"], []
    if own:
        import paper_2410_20305_b200 as psa
        stats = s["stats"]
        if forward:
            outs = list(psa.psa_norm(x, s["weight"], s["bias"], eps=s["eps"], rms=s["rms"], residual=s["residual"]))
            x, stats = outs[2] if len(outs) > 2 else x, outs[1]
        if s["pass"] != "forward":
            dx, dweight, dbias = psa.psa_norm_bwd(s["d_out"], x, s["weight"], stats, rms=s["rms"], d_total=s["d_total"],
                                                  with_bias=not s["rms"])
            outs += [dx, dweight] + ([] if s["rms"] else [dbias])
        return outs
    stats = s["stats"]
    if forward:
        outs = _plain_norm(s, x)
        x, stats = outs[2] if len(outs) > 2 else x, outs[1]
    if s["pass"] != "forward":
        outs = outs + _plain_norm_backward(s, x, stats)
    return outs


def _run_embed(s):
    if own:
        import paper_2410_20305_b200 as psa
        if s["pass"] == "forward":
            return psa.psa_embed(s["ids"], s["table"], scale=s["scale"])
        return psa.psa_embed_bwd(s["d_out"], s["ids"], s["vocab"], scale=s["scale"], dtype=DTYPES[s["grad"]])
    if s["pass"] == "forward":
        return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["table"].dtype)
    grad = torch.zeros((s["vocab"], s["hidden"]), dtype=torch.float32, device="cuda")
    grad.index_add_(0, s["ids"].long(), s["d_out"].float())
    return (grad * s["scale"]).to(DTYPES[s["grad"]])


def _run_ffn(s):
    x, w = s["x"], s["w"]
    if own:
        import paper_2410_20305_b200 as psa
        step = s["pass"] == "step"
        out, saved = psa.psa_ffn(x, *w, save=step)
        return [out, *psa.psa_ffn_bwd(s["d_out"], x, *w, saved)] if step else out
    wg, wu, wd = (t.float() for t in w)
    wide = x.float()
    gate, up = wide @ wg, wide @ wu
    sig = 1 / (1 + torch.exp(-gate))
    act = gate * sig
    h = act * up
    out = (h @ wd).to(x.dtype)
    if s["pass"] == "forward":
        return out
    g = s["d_out"].float()
    dh = g @ wd.t()
    dwd = (h.t() @ g).to(x.dtype)
    d_up = dh * act
    d_gate = dh * up * (sig * (1 + gate * (1 - sig)))
    dx = (d_gate @ wg.t() + d_up @ wu.t()).to(x.dtype)
    return [out, dx, (wide.t() @ d_gate).to(x.dtype), (wide.t() @ d_up).to(x.dtype), dwd]


def run(state):
    return {"norm": _run_norm, "embed": _run_embed, "ffn": _run_ffn}[state["op"]](state)


def work(case):
    """Bytes of every input read once and every output written once (a table's rows that occur, once each at most);
    flops of the products, and a handful per element elsewhere."""
    T, D = case["tokens"], case["hidden"]
    size = {"bf16": 2, "f32": 4}
    forward, backward = case["pass"] != "backward", case["pass"] != "forward"
    if case["op"] == "norm":
        e, w, res, row = size[case["x"]], size[case["weight"]], case["residual"], T * D
        bias = 1 if case["kind"] == "rms" else 2
        bytes_ = 0
        if forward:
            bytes_ += e * row * (4 if res else 2) + w * bias * D + 8 * T
        if backward:   # d_out, x, dx and, with a residual, its gradient; the parameters' gradients; what a forward left is read
            bytes_ += e * row * (4 if res else 3) + w * (1 + bias) * D + 8 * T
        return {"bytes": bytes_, "flops": row * (8 * forward + 14 * backward)}
    if case["op"] == "embed":
        e, vocab = size[case["x"]], case["vocab"]
        # distinct tokens among T with frequencies as 1 / rank: a token of rank r is missed with (1 - p_r)^T
        ranks = torch.arange(1, vocab + 1, dtype=torch.float64)
        p = torch.log1p(1 / ranks) / math.log(vocab + 1)
        distinct = min(T, int((1 - torch.exp(T * torch.log1p(-p))).sum()) + 1)
        if forward:
            return {"bytes": 4 * T + e * D * (distinct + T), "flops": T * D}
        return {"bytes": 4 * T + e * D * T + size[case["grad"]] * vocab * D, "flops": T * D + distinct * D}
    F = case["ffn"]
    bytes_, flops = 2 * (2 * T * D + 3 * D * F), 6 * T * D * F
    if backward:   # d_out read, dx and three gradients of weights written
        bytes_, flops = bytes_ + 2 * (2 * T * D + 3 * D * F), 3 * flops
    return {"bytes": bytes_, "flops": flops}


def _exact_norm(s):
    x, w, outs = s["x"].double(), s["weight"].double(), []
    if s["pass"] != "backward" and s["residual"] is not None:
        x = (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()
    mu = x.mean(dim=1, keepdim=True) * (0.0 if s["rms"] else 1.0)
    sigma = torch.sqrt(((x - mu) ** 2).sum(dim=1, keepdim=True) / x.shape[1] + s["eps"])
    unit = (x - mu) / sigma
    if s["pass"] != "backward":
        y = unit * w if s["bias"] is None else torch.addcmul(s["bias"].double(), unit, w)
        outs = [y, torch.cat([mu, 1 / sigma], dim=1).t()] + ([] if s["residual"] is None else [x])
    if s["pass"] != "forward":
        g = s["d_out"].double()
        v = g * w
        # the Jacobian of a row's normalisation is (I - 11'/n - uu'/n) / sigma, without 11'/n where no mean is taken off
        dx = v - unit * ((v * unit).sum(dim=1, keepdim=True) / x.shape[1])
        if not s["rms"]:
            dx = dx - v.sum(dim=1, keepdim=True) / x.shape[1]
        dx = dx / sigma
        if s["d_total"] is not None:
            dx = dx + s["d_total"].double()
        outs += [dx, torch.einsum("td,td->d", g, unit)] + ([] if s["rms"] else [g.sum(dim=0)])
    return outs


def _exact_embed(s):
    if s["pass"] == "forward":
        return torch.index_select(s["table"], 0, s["ids"].long()).double() * s["scale"]
    grad = torch.zeros((s["vocab"], s["hidden"]), dtype=torch.float64, device="cuda")
    return grad.index_put_((s["ids"].long(),), s["d_out"].double() * s["scale"], accumulate=True)


def _exact_ffn(s):
    x, wg, wu, wd = [t.double() for t in (s["x"], *s["w"])]
    a, b = torch.mm(x, wg), torch.mm(x, wu)
    z = torch.sigmoid(a)
    out = torch.mm(a * z * b, wd)
    if s["pass"] == "forward":
        return out
    g = s["d_out"].double()
    dwd = torch.mm((a * z * b).t(), g)
    dh = torch.mm(g, wd.t())
    db = dh * a * z
    da = dh * b * (z + a * z * (1 - z))
    return [out, torch.mm(da, wg.t()).addmm_(db, wu.t()), torch.mm(x.t(), da), torch.mm(x.t(), db), dwd]


def exact(case, seed):
    return {"norm": _exact_norm, "embed": _exact_embed, "ffn": _exact_ffn}[case["op"]](prepare(case, seed))
