"""Operators that complete a training step on the shared layout, for timing: summed log-probabilities of responses straight
from the hidden states and the output table, without logits; rotary positions of queries and keys in their various forms;
and the step between two sublayers whose output is normalised before it joins the residual stream.  Forward and backward.

A case is one call, or one forward and its backward, on a packed row of tokens.  Token counts, widths and vocabularies are
those of the package's workloads (workloads.py), of its tests, or lie between them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # ---- log-probabilities from hidden states
        # A prompt of one token and a response of one: one scored row against the whole table, which is read once.
        {"name": "logp-one-row", "op": "logp", "pass": "forward", "tokens": 2, "prompt": 1, "response": 1, "lengths": 0,
         "hidden": 4096, "vocab": 128256, "scale": 1.0},
        # The tiny configuration's vocabulary and width: launches.
        {"name": "logp-tiny-step", "op": "logp", "pass": "step", "tokens": 672, "prompt": 192, "response": 72, "lengths": 1,
         "hidden": 256, "vocab": 1024, "scale": 1.0},
        # A small model's step on a small odd pack of short samples; the vocabulary divides by nothing.
        {"name": "logp-ragged-step", "op": "logp", "pass": "step", "tokens": 1815, "prompt": 160, "response": 160, "lengths": 2,
         "hidden": 1032, "vocab": 50257, "scale": 0.5},
        # The frozen model's pass on long prompts with short responses: most rows score nothing.
        {"name": "logp-reference-long-prompt", "op": "logp", "pass": "forward", "tokens": 15154, "prompt": 2048, "response": 80,
         "lengths": 3, "hidden": 4096, "vocab": 128256, "scale": 1.0},
        # The last operation of a step of the benchmark's model on its pack, forward and backward.
        {"name": "logp-llama3-8b-step", "op": "logp", "pass": "step", "tokens": 16215, "prompt": 600, "response": 380,
         "lengths": 4, "hidden": 4096, "vocab": 128256, "scale": 1.0},
        # ---- rotary positions
        # One token of the benchmark's model: a launch's latency.
        {"name": "rotary-one-token", "op": "rotary", "tokens": 1, "q_heads": 32, "k_heads": 8, "head_dim": 128, "rotary": 128,
         "x": "bf16", "interleaved": False, "inverse": False, "fused": True, "scaling": "wavelength", "far": 0},
        # Queries and keys of the benchmark's pack where one projection left them, frequencies scaled by their wavelength.
        {"name": "rotary-llama3-8b", "op": "rotary", "tokens": 16215, "q_heads": 32, "k_heads": 8, "head_dim": 128, "rotary": 128,
         "x": "bf16", "interleaved": False, "inverse": False, "fused": True, "scaling": "wavelength", "far": 0},
        # Gradients in fp32 of a head of which a part turns, neighbours in pairs, at positions of a very long context.
        {"name": "rotary-part-of-head-backward", "op": "rotary", "tokens": 7965, "q_heads": 12, "k_heads": 3, "head_dim": 80,
         "rotary": 36, "x": "f32", "interleaved": True, "inverse": True, "fused": False, "scaling": "ramp", "far": 900000},
        # ---- norms before and after a block
        # One token through a frozen model.
        {"name": "block-norm-one-token", "op": "block", "pass": "forward", "tokens": 1, "hidden": 4096, "kind": "rms",
         "post": True, "gate": False, "residual_scale": 1.0, "x": "bf16", "weight": "bf16"},
        # Between the attention and the feed-forward block on the pack of the benchmark.
        {"name": "block-norm-llama3-8b", "op": "block", "pass": "forward", "tokens": 16215, "hidden": 4096, "kind": "rms",
         "post": True, "gate": False, "residual_scale": 1.0, "x": "bf16", "weight": "bf16"},
        # Gradients on the largest pack, with a gate for each channel and parameters kept in fp32.
        {"name": "block-norm-multi-turn-backward", "op": "block", "pass": "backward", "tokens": 31041, "hidden": 4096,
         "kind": "layer", "post": True, "gate": True, "residual_scale": 1.0, "x": "bf16", "weight": "f32"},
        # A width that fills no vector, an odd number of tokens, a gate without a norm in front of it.
        {"name": "block-norm-ragged-step", "op": "block", "pass": "step", "tokens": 5465, "hidden": 1237, "kind": "layer",
         "post": False, "gate": True, "residual_scale": 0.7, "x": "bf16", "weight": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = _drawn(rng)
    # no more work than the largest listed one of its kind has
    most = [work(c) for c in listed() if c["op"] == case["op"]]
    axis = "vocab" if case["op"] == "logp" else "tokens"
    while any(work(case)[unit] > max(w[unit] for w in most) for unit in ("bytes", "flops")):
        case[axis] = case[axis] * 2 // 3
    return case


def _drawn(rng):
    op = rng.choice(("logp", "logp", "rotary", "block"))
    if op == "logp":
        tokens = _log_uniform(rng, 2, 16000)
        return {"op": op, "pass": rng.choice(("forward", "backward", "step")), "tokens": tokens,
                "prompt": min(_log_uniform(rng, 1, 2048), max(1, tokens // 2)), "response": _log_uniform(rng, 1, 800), "lengths": rng.randrange(1 << 20),
                "hidden": 8 * _log_uniform(rng, 8, 512), "vocab": _log_uniform(rng, 300, 128256),
                "scale": rng.choice((1.0, 1.0, 0.5))}
    if op == "rotary":
        head = rng.choice((64, 72, 80, 96, 128, 128, 192, 256))
        kv = rng.choice((1, 2, 3, 4, 8))
        return {"op": op, "tokens": _log_uniform(rng, 1, 32768), "q_heads": kv * rng.choice((1, 2, 4)), "k_heads": kv,
                "head_dim": head, "rotary": head if rng.random() < 0.5 else 2 * rng.randint(4, head // 2),
                "x": rng.choice(("bf16", "bf16", "f32")), "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5,
                "fused": rng.random() < 0.5, "scaling": rng.choice(("none", "linear", "base", "wavelength", "ramp")),
                "far": rng.choice((0, 0, 100000, 900000))}
    x, weight = rng.choice((("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")))
    # a step in bf16 goes with parameters in bf16: its total is rounded to bf16 before the second norm, and a value at the
    # border of two roundings may go either way, which is an error of bf16 in the parameters' gradients
    return {"op": op, "pass": rng.choice(("forward", "backward") if x != weight else ("forward", "backward", "step")),
            "tokens": _log_uniform(rng, 1, 32768), "hidden": _log_uniform(rng, 64, 8192), "kind": rng.choice(("layer", "rms")),
            "post": rng.random() < 0.7, "gate": rng.random() < 0.5, "residual_scale": rng.choice((1.0, 1.0, 0.7)), "x": x,
            "weight": weight}


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=gen, device="cuda")
    return (t.mul_(std) if std != 1.0 else t).to(dtype)


def _samples(case):
    """(prompt, chosen, rejected) lengths of a pack of exactly case["tokens"] tokens."""
    rng = np.random.default_rng(case["lengths"])
    draw_one = lambda mean: int(rng.integers((mean + 1) // 2, 3 * mean // 2 + 1))  # noqa: E731
    left, out = case["tokens"], []
    while left:
        p, c, r = draw_one(case["prompt"]), draw_one(case["response"]), draw_one(case["response"])
        p = min(p, left)
        c = min(c, left - p)
        r = min(r, left - p - c)
        out.append((p, c, r))
        left -= p + c + r
    return out


def _labels(case):
    """Which row scores which token on the shared layout: (targets' rows of own labels [T] or -1, segments [T] or -1, forks
    as (row, token's row, segment)); a label is named by the row of the token that is scored."""
    T = case["tokens"]
    scored, segment, forks = np.full(T, -1, np.int64), np.full(T, -1, np.int64), []
    at = 0
    for s, (p, c, r) in enumerate(_samples(case)):
        for length, start, g in ((c, at + p, 2 * s), (r, at + p + c, 2 * s + 1)):
            rows = np.arange(start, start + length - 1)
            scored[rows], segment[rows] = rows + 1, g
            if length and p:      # the last prompt row scores the first token
                last = at + p - 1
                if segment[last] < 0:
                    scored[last], segment[last] = start, g
                else:
                    forks.append((last, start, g))
        at += p + c + r
    return scored, segment, np.array(forks, np.int64).reshape(-1, 3)


def _prepare_logp(case, s, gen):
    T, D, V = case["tokens"], case["hidden"], case["vocab"]
    scored, segment, forks = _labels(case)
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a)).cuda()  # noqa: E731
    tokens = torch.randint(0, V, (T,), generator=gen, device="cuda")
    own_rows = np.flatnonzero(segment >= 0)
    s["n_segments"] = 2 * len(_samples(case))
    s["targets"] = torch.where(dev(segment) >= 0, tokens[dev(np.maximum(scored, 0))], 0).to(torch.int32)
    s["segment_ids"] = dev(segment).to(torch.int32)
    s["fork_rows"], s["fork_segments"] = dev(forks[:, 0]).to(torch.int32), dev(forks[:, 2]).to(torch.int32)
    s["fork_targets"] = tokens[dev(forks[:, 1])].to(torch.int32)
    # the same labels one after the other: row, token and response
    s["label_rows"] = dev(np.concatenate([own_rows, forks[:, 0]]))
    s["label_tokens"] = tokens[dev(np.concatenate([scored[own_rows], forks[:, 1]]))]
    s["label_segments"] = dev(np.concatenate([segment[own_rows], forks[:, 2]]))
    # Logits of deviation 1.5, and the scored token's raised by 0 to 12: probabilities from 1e-6 to nearly 1.
    s["table"] = _normal(gen, V, D, std=1.5 * D ** -0.5 / case["scale"])
    hidden = torch.randn((T, D), generator=gen, device="cuda")
    lift = 12 * torch.rand(len(own_rows), generator=gen, device="cuda")[:, None] / 1.5
    towards = s["table"][s["label_tokens"][:len(own_rows)]].float()
    rows = s["label_rows"][:len(own_rows)]
    hidden[rows] += lift * towards / towards.norm(dim=1, keepdim=True)
    s["hidden"] = hidden.to(torch.bfloat16)
    # as the gradient of a mean over samples with a small temperature: chosen up, rejected down
    s["coef"] = torch.rand(s["n_segments"], generator=gen, device="cuda") * (0.1 / len(_samples(case)))
    s["coef"][1::2] *= -1
    if case["pass"] == "backward":       # what the forward pass left
        wide = s["table"].float()
        s["lse"] = torch.zeros(T, device="cuda")
        for rows in s["label_rows"].split(4096):
            s["lse"][rows] = torch.logsumexp(s["hidden"][rows].float() @ wide.t() * case["scale"], dim=1)
    return s


def _frequencies(case):
    """Radians per position of every pair, in 64 bits, and the factor of the rotated part."""
    r, theta, kind = case["rotary"], 500000.0, case["scaling"]
    i = torch.arange(r // 2, dtype=torch.float64)
    factor, length = 8.0, 8192.0
    if kind == "base":
        theta *= factor ** (r / (r - 2))
    f = theta ** (-2 * i / r)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "wavelength":
        low, high = 1.0, 4.0
        keep = ((length * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f * keep + f / factor * (1 - keep), 1.0
    if kind == "ramp":
        at = lambda turns: r * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        first, last = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        ramp = ((i - first) / max(last - first, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1
    return f, 1.0


def _prepare_rotary(case, s, gen):
    T, Hq, Hk, d, dtype = case["tokens"], case["q_heads"], case["k_heads"], case["head_dim"], DTYPES[case["x"]]
    if case["fused"]:      # one projection's output, values behind the keys
        all_heads = _normal(gen, T, (Hq + 2 * Hk) * d, dtype=dtype)
        s["q"] = all_heads[:, :Hq * d].view(T, Hq, d)
        s["k"] = all_heads[:, Hq * d:(Hq + Hk) * d].view(T, Hk, d)
    else:
        s["q"], s["k"] = _normal(gen, T, Hq, d, dtype=dtype), _normal(gen, T, Hk, d, dtype=dtype)
    # samples of a few hundred to a few thousand tokens
    at = torch.arange(T, device="cuda")
    s["positions"] = (at % int(torch.randint(300, 4000, (1,), generator=gen, device="cuda")) + case["far"]).to(torch.int32)
    radians, s["magnitude"] = _frequencies(case)
    s["radians"] = radians.cuda()
    if own:
        import paper_2410_20305_b200 as psa
        s["turns"], s["magnitude"] = psa.psa_rotary_frequencies(
            case["rotary"], theta=500000.0, scaling=None if case["scaling"] == "none" else case["scaling"], factor=8.0,
            original_length=8192, device="cuda")
    return s


def _prepare_block(case, s, gen):
    T, D, rms = case["tokens"], case["hidden"], case["kind"] == "rms"
    dtype, wtype = DTYPES[case["x"]], DTYPES[case["weight"]]
    s["rms"], s["eps"] = rms, 1e-5
    near_one = lambda: (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(wtype)  # noqa: E731
    s["x"], s["residual"] = _normal(gen, T, D, dtype=dtype), _normal(gen, T, D, std=2.0, dtype=dtype)
    s["weight"], s["bias"] = near_one(), None if rms else _normal(gen, D, std=0.2, dtype=wtype)
    s["post_weight"] = near_one() if case["post"] else None
    s["post_bias"] = _normal(gen, D, std=0.2, dtype=wtype) if case["post"] and not rms else None
    s["gate"] = _normal(gen, D, std=0.5, dtype=wtype) if case["gate"] else None
    s["d_out"], s["d_total"] = _normal(gen, T, D, dtype=dtype), _normal(gen, T, D, dtype=dtype)
    if case["pass"] == "backward":       # what the forward pass left
        _, s["total"], s["stats"] = _exact_block_forward(s)
        s["total"], s["stats"] = s["total"].to(dtype), s["stats"].float()
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"logp": _prepare_logp, "rotary": _prepare_rotary, "block": _prepare_block}[case["op"]](case, dict(case), gen)


def _plain_logits(s):
    rows = s["hidden"][s["label_rows"]].float()
    return rows, (rows @ s["table"].float().t()) * s["scale"]


def _run_logp(s):
    forward, backward = s["pass"] != "backward", s["pass"] != "forward"
    if own:
        import paper_2410_20305_b200 as psa
        labels = (s["targets"], s["segment_ids"])
        forks = (s["fork_rows"], s["fork_targets"], s["fork_segments"])
        outs, lse = [], s.get("lse")
        if forward:
            out, lse = psa.dpo_linear_logp(s["hidden"], s["table"], *labels, s["n_segments"], *forks, scale=s["scale"])
            outs = [out, lse]
        if backward:
            outs += psa.dpo_linear_logp_bwd(s["coef"], s["hidden"], s["table"], lse, *labels, *forks, scale=s["scale"])
        return outs
    at = s["label_rows"]
    rows, z = _plain_logits(s)
    outs = []
    if forward:
        top = z.max(dim=1, keepdim=True).values
        row_lse = top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))
        terms = z.gather(1, s["label_tokens"][:, None])[:, 0] - row_lse
        out = torch.zeros(s["n_segments"], dtype=torch.float64, device="cuda").index_add_(0, s["label_segments"], terms.double())
        lse = torch.zeros(s["tokens"], device="cuda")
        lse[at] = row_lse
        outs = [out.float(), lse]
    if backward:
        row_lse = (lse if forward else s["lse"])[at]
        c = s["coef"][s["label_segments"]][:, None] * s["scale"]
        d = z.sub_(row_lse[:, None]).exp_().mul_(-c)
        d.scatter_add_(1, s["label_tokens"][:, None], c)
        d_rows = d @ s["table"].float()
        d_hidden = torch.zeros((s["tokens"], s["hidden"].shape[1]), device="cuda").index_add_(0, at, d_rows)
        outs += [d_hidden.to(torch.bfloat16), (d.t() @ rows).to(torch.bfloat16)]
    return outs


def _plain_turn(s, x):
    r, sign = s["rotary"], -1.0 if s["inverse"] else 1.0
    angle = s["positions"].double()[:, None] * s["radians"]
    cos = (torch.cos(angle) * s["magnitude"]).float()[:, None]
    sin = (torch.sin(angle) * (sign * s["magnitude"])).float()[:, None]
    wide = x.float()
    out = wide.clone()
    if s["interleaved"]:
        a, b = wide[..., 0:r:2], wide[..., 1:r:2]
        out[..., 0:r:2], out[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = wide[..., :r // 2], wide[..., r // 2:r]
        out[..., :r // 2], out[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _run_rotary(s):
    if own:
        import paper_2410_20305_b200 as psa
        return psa.psa_rotary(s["q"], s["k"], s["positions"], s["turns"], magnitude=s["magnitude"], interleaved=s["interleaved"],
                              inverse=s["inverse"])
    return _plain_turn(s, s["q"]), _plain_turn(s, s["k"])


def _plain_unit(s, wide):
    """Rows normalised, their mean (0 in the RMS form) and the reciprocal of their deviation."""
    mean = torch.zeros_like(wide[:, 0]) if s["rms"] else wide.mean(1)
    centred = wide - mean[:, None]
    rstd = (centred.square().mean(1) + s["eps"]).rsqrt()
    return centred * rstd[:, None], mean, rstd


def _affine(unit, weight, bias):
    out = unit * weight.float()
    return out if bias is None else out + bias.float()


def _plain_block_forward(s):
    y, x = s["x"].float(), s["x"]
    mean1, rstd1 = torch.zeros_like(y[:, 0]), torch.ones_like(y[:, 0])
    if s["post_weight"] is not None:
        y, mean1, rstd1 = _plain_unit(s, y)
        y = _affine(y, s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        y = y * s["gate"].float()
    total = (s["residual"].float() * s["residual_scale"] + y).to(x.dtype)
    unit, mean2, rstd2 = _plain_unit(s, total.float())
    return _affine(unit, s["weight"], s["bias"]).to(x.dtype), total, torch.stack([mean1, rstd1, mean2, rstd2])


def _plain_unit_backward(s, g, unit, rstd):
    d = g - unit * (g * unit).mean(1, keepdim=True)
    if not s["rms"]:
        d = d - g.mean(1, keepdim=True)
    return d * rstd[:, None]


def _plain_block_backward(s, total, stats):
    """Gradients of x, residual, weight, bias, post_weight, post_bias and gate, as far as there are such parameters."""
    mean1, rstd1, mean2, rstd2 = stats
    over = lambda a: a.double().sum(0)  # noqa: E731
    wtype, g = s["weight"].dtype, s["d_out"].float()
    unit2 = (total.float() - mean2[:, None]) * rstd2[:, None]
    params = [over(g.double() * unit2.double())] + ([] if s["bias"] is None else [over(g)])
    d = _plain_unit_backward(s, g * s["weight"].float(), unit2, rstd2) + s["d_total"].float()
    d_residual = (d * s["residual_scale"]).to(s["x"].dtype)
    dy = d if s["gate"] is None else d * s["gate"].float()
    y, dx = s["x"].float(), dy
    if s["post_weight"] is not None:
        unit1 = (y - mean1[:, None]) * rstd1[:, None]
        params += [over(dy.double() * unit1.double())] + ([] if s["post_bias"] is None else [over(dy)])
        dx = _plain_unit_backward(s, dy * s["post_weight"].float(), unit1, rstd1)
        y = _affine(unit1, s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        params.append(over(d.double() * y.double()))
    return [dx.to(s["x"].dtype), d_residual] + [p.to(wtype) for p in params]


def _run_block(s):
    forward, backward = s["pass"] != "backward", s["pass"] != "forward"
    outs, total, stats = [], s.get("total"), s.get("stats")
    if own:
        import paper_2410_20305_b200 as psa
        around = dict(post_weight=s["post_weight"], gate=s["gate"], post_bias=s["post_bias"], residual_scale=s["residual_scale"],
                      rms=s["rms"])
        if forward:
            out, total, stats = psa.psa_block_norm(s["x"], s["residual"], s["weight"], bias=s["bias"], eps=s["eps"], **around)
            outs = [out, total, stats]
        if backward:
            grads = psa.psa_block_norm_bwd(s["d_out"], s["x"], total, s["weight"], stats, d_total=s["d_total"],
                                           with_bias=s["bias"] is not None, **around)
            outs += [g for g in grads if g is not None]
        return outs
    if forward:
        outs = list(_plain_block_forward(s))
        _, total, stats = outs
    return outs + (_plain_block_backward(s, total, stats) if backward else [])


def run(state):
    return {"logp": _run_logp, "rotary": _run_rotary, "block": _run_block}[state["op"]](state)


def work(case):
    """Bytes of every input read once and every output written once; flops of the products (the logits twice where there is a
    backward pass of its own or behind a forward pass, as they are not kept), and a handful per element elsewhere."""
    size = {"bf16": 2, "f32": 4}
    T = case["tokens"]
    if case["op"] == "logp":
        D, V = case["hidden"], case["vocab"]
        forward, backward = case["pass"] != "backward", case["pass"] != "forward"
        _, segment, forks = _labels(case)
        rows = int((segment >= 0).sum())
        bytes_ = 2 * D * (rows + V) + 8 * T + 12 * len(forks) + 4 * T      # and the rows' log-sums, of whichever pass
        flops = 2 * rows * V * D
        if backward:
            bytes_ += 2 * D * (T + V)
        return {"bytes": bytes_, "flops": flops * (forward + 3 * backward)}
    if case["op"] == "rotary":
        heads = T * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        return {"bytes": 2 * size[case["x"]] * heads + 4 * T + 8 * (case["rotary"] // 2), "flops": 4 * heads}
    D, e, w = case["hidden"], size[case["x"]], size[case["weight"]]
    bias = 1 if case["kind"] == "rms" else 2
    params = bias * (1 + case["post"]) + case["gate"]
    forward, backward = case["pass"] != "backward", case["pass"] != "forward"
    bytes_ = 0
    if forward:
        bytes_ += e * T * D * 4 + w * D * params + 16 * T
    if backward:      # d_out, d_total, x and total, the gradients of x and residual; what a forward left is read
        bytes_ += e * T * D * 6 + 2 * w * D * params + 16 * T
    return {"bytes": bytes_, "flops": T * D * (14 * forward + 26 * backward)}


def _exact_logp(s):
    h, w, scale = s["hidden"].double(), s["table"].double(), s["scale"]
    at, y, g = s["label_rows"], s["label_tokens"], s["label_segments"]
    logp = torch.mm(h.index_select(0, at), w.t()).mul_(scale)
    lse = torch.logsumexp(logp, dim=1)
    logp -= lse[:, None]
    outs = []
    if s["pass"] != "backward":
        picked = logp[torch.arange(len(at), device="cuda"), y]
        sums = [picked[g == k].sum() for k in range(s["n_segments"])]
        all_lse = torch.zeros(s["tokens"], dtype=torch.float64, device="cuda").index_put_((at,), lse)
        outs = [torch.stack(sums), all_lse]
    if s["pass"] != "forward":
        # d logp(y) / d logits = onehot(y) - softmax
        c = s["coef"].double()[g] * scale
        grad = torch.exp_(logp).neg_()
        grad[torch.arange(len(at), device="cuda"), y] += 1
        grad *= c[:, None]
        dh = torch.zeros_like(h).index_put_((at,), torch.mm(grad, w), accumulate=True)
        outs += [dh, torch.mm(grad.t(), h.index_select(0, at))]
    return outs


def _exact_rotary(s):
    r = s["rotary"]
    # a pair is a complex number that is turned by its angle
    turn = torch.polar(torch.full_like(s["radians"], s["magnitude"]).expand(s["tokens"], -1).contiguous(),
                       (-1 if s["inverse"] else 1) * torch.outer(s["positions"].double(), s["radians"]))[:, None]

    def turned(x):
        head, rest = x[..., :r].double(), x[..., r:].double()
        pairs = head.unflatten(-1, (r // 2, 2)) if s["interleaved"] else head.unflatten(-1, (2, r // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
        z = z.flatten(-2) if s["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, rest], dim=-1)

    return turned(s["q"]), turned(s["k"])


def _exact_norm(s, v):
    mu = v.mean(dim=1, keepdim=True) * (0.0 if s["rms"] else 1.0)
    sigma = torch.sqrt(((v - mu) ** 2).sum(dim=1, keepdim=True) / v.shape[1] + s["eps"])
    return (v - mu) / sigma, mu, sigma


def _exact_block_forward(s):
    opt = lambda t, other: other if t is None else t.double()  # noqa: E731
    y = s["x"].double()
    mu1, sigma1 = torch.zeros_like(y[:, :1]), torch.ones_like(y[:, :1])
    if s["post_weight"] is not None:
        y, mu1, sigma1 = _exact_norm(s, y)
        y = y * s["post_weight"].double() + opt(s["post_bias"], 0.0)
    total = torch.addcmul(s["residual"].double() * s["residual_scale"], y, opt(s["gate"], torch.ones((), dtype=torch.float64, device="cuda")))
    total = total.to(s["x"].dtype).double()      # what is normalised is what the residual stream holds
    unit, mu2, sigma2 = _exact_norm(s, total)
    out = unit * s["weight"].double() + opt(s["bias"], 0.0)
    return out, total, torch.cat([mu1, 1 / sigma1, mu2, 1 / sigma2], dim=1).t().contiguous()


def _exact_jacobian(s, v, unit, sigma):
    n = v.shape[1]
    d = v - unit * ((v * unit).sum(dim=1, keepdim=True) / n)
    return (d if s["rms"] else d - v.sum(dim=1, keepdim=True) / n) / sigma


def _exact_block(s):
    outs = []
    if s["pass"] != "backward":
        outs = list(_exact_block_forward(s))
        total = outs[1]
    else:
        total = s["total"].double()
    if s["pass"] != "forward":
        g = s["d_out"].double()
        unit2, _, sigma2 = _exact_norm(s, total)
        params = [torch.einsum("td,td->d", g, unit2)] + ([] if s["bias"] is None else [g.sum(dim=0)])
        ds = _exact_jacobian(s, g * s["weight"].double(), unit2, sigma2) + s["d_total"].double()
        gate = 1.0 if s["gate"] is None else s["gate"].double()
        y, dx = s["x"].double(), ds * gate
        if s["post_weight"] is not None:
            unit1, _, sigma1 = _exact_norm(s, y)
            params += [torch.einsum("td,td->d", dx, unit1)] + ([] if s["post_bias"] is None else [dx.sum(dim=0)])
            dx = _exact_jacobian(s, dx * s["post_weight"].double(), unit1, sigma1)
            y = unit1 * s["post_weight"].double() + (0.0 if s["post_bias"] is None else s["post_bias"].double())
        if s["gate"] is not None:
            params.append(torch.einsum("td,td->d", ds, y))
        outs += [dx, ds * s["residual_scale"]] + params
    return outs


def exact(case, seed):
    return {"logp": _exact_logp, "rotary": _exact_rotary, "block": _exact_block}[case["op"]](prepare(case, seed))
