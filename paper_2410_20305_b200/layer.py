"""One attention layer on the shared layout (Section 4.2: the full attention-layer benchmark):
query / key / value projections, rotary embedding on the position ids of Section 3.1,
psa_fwd, output projection, and the backward of all of it; a whole decoder layer around it
(norms, residual stream, gated feed-forward block), also with norms behind the sublayers; and a
decoder from token ids to the log-probabilities of the responses.

The projections are library GEMMs (torch.matmul, i.e. cuBLAS); all else is this library's
kernels.  Compositions for the layer-level measurement and for parity tests, not kernels of their own.
"""
from __future__ import annotations

from . import binding as B
from . import operators as O


class Rotary:
    """A rotary embedding in one of psa_rotary's forms, for the `rotary` of the layers below: rotary_dim, theta, scaling and what
    goes with it as psa_rotary_frequencies takes them."""

    def __init__(self, rotary_dim, theta=10000.0, interleaved=False, device="cuda", **scaling):
        self.turns, self.magnitude = O.psa_rotary_frequencies(rotary_dim, theta, device=device, **scaling)
        self.interleaved = interleaved

    def apply(self, q, k, position_ids, inverse=False):
        """Turns queries and keys in place."""
        O.psa_rotary(q, k, position_ids, self.turns, self.magnitude, self.interleaved, inverse, q_out=q, k_out=k)


class AttentionLayer:
    """Holds a plan, the position ids and the scratch of one pack; `forward` and `backward`
    run the layer for bf16 CUDA inputs x [T, hidden] and weights wq [hidden, Hq d],
    wk, wv [hidden, Hkv d], wo [Hq d, hidden].  `status` (optional): the int32 CUDA word in which
    psa_fwd and psa_bwd report a wait that gave up.  `rotary` (optional): a Rotary in the place of psa_rope with rope_theta."""

    def __init__(self, pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta=10000.0, status=None, rotary=None):
        import torch
        cu, P, C, R = pack_lengths
        self.plan = B.psa_plan(cu, P, C, R, n_q_heads, n_kv_heads, head_dim)
        self.pos = torch.as_tensor(B.psa_position_ids(cu, P, C, R)).to(device)
        self.neg = -self.pos
        self.ws = torch.empty(max(self.plan.bwd_workspace_bytes, 256), dtype=torch.uint8, device=device)
        self.theta = float(rope_theta)
        self.rotary = rotary
        self.status = status
        self.Hq, self.Hkv, self.d = n_q_heads, n_kv_heads, head_dim

    def forward(self, x, wq, wk, wv, wo):
        T = x.shape[0]
        q = (x @ wq).view(T, self.Hq, self.d)
        k = (x @ wk).view(T, self.Hkv, self.d)
        v = (x @ wv).view(T, self.Hkv, self.d)
        if self.rotary is None:
            B.psa_rope(q, self.pos, self.theta, out=q)
            B.psa_rope(k, self.pos, self.theta, out=k)
        else:
            self.rotary.apply(q, k, self.pos)
        o, lse = B.psa_fwd(self.plan, q, k, v, status=self.status)
        out = o.view(T, self.Hq * self.d) @ wo
        return out, (q, k, v, o, lse)

    def backward(self, x, wq, wk, wv, wo, saved, d_out):
        """Returns (dx, dwq, dwk, dwv, dwo) for the loss sum(out * d_out)."""
        q, k, v, o, lse = saved
        T = x.shape[0]
        d_o = (d_out @ wo.t()).view(T, self.Hq, self.d)
        dwo = o.view(T, self.Hq * self.d).t() @ d_out
        dq, dk, dv = B.psa_bwd(self.plan, d_o, q, k, v, o, lse, workspace=self.ws, status=self.status)
        # the gradient of a rotation is the inverse rotation
        if self.rotary is None:
            B.psa_rope(dq, self.neg, self.theta, out=dq)
            B.psa_rope(dk, self.neg, self.theta, out=dk)
        else:
            self.rotary.apply(dq, dk, self.pos, inverse=True)
        dq2, dk2, dv2 = dq.view(T, -1), dk.view(T, -1), dv.view(T, -1)
        # one sum for the three products: two additions of [T, hidden] matrices and two roundings less
        dx = dq2 @ wq.t()
        dx.addmm_(dk2, wk.t()).addmm_(dv2, wv.t())
        return dx, x.t() @ dq2, x.t() @ dk2, x.t() @ dv2, dwo


class DecoderLayer:
    """One pre-norm decoder layer on the shared layout: root-mean-square norm, AttentionLayer, norm, gated feed-forward block,
    with the residual stream around both (the layer whose attention and MLP Section 4.2 measures).  A weight is a dict with
    the keys of KEYS: norm1 and norm2 [hidden], wq, wk, wv, wo as in AttentionLayer, w_gate and w_up [hidden, ffn],
    w_down [ffn, hidden], all bf16.

    A layer takes the residual stream x and what is still to be added to it (`delta`, the feed-forward output of the layer
    before; None in the first one): the addition is part of its first norm, as that of the attention's output is of its second.
    `status` (optional): the int32 CUDA word in which all its calls report a wait that gave up."""

    KEYS = ("norm1", "wq", "wk", "wv", "wo", "norm2", "w_gate", "w_up", "w_down")

    def __init__(self, pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta=10000.0, eps=1e-5, status=None, rotary=None):
        self.attention = AttentionLayer(pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta, status, rotary)
        self.status = status
        self.eps = float(eps)

    def forward(self, x, w, delta=None):
        """Returns (residual stream, delta, what backward needs): the layer's output is the sum of the first two."""
        if delta is None:
            a, stats1 = B.psa_norm(x, w["norm1"], eps=self.eps, rms=True)
        else:
            a, stats1, x = B.psa_norm(x, w["norm1"], eps=self.eps, rms=True, residual=delta)
        attn, saved = self.attention.forward(a, w["wq"], w["wk"], w["wv"], w["wo"])
        b, stats2, mid = B.psa_norm(attn, w["norm2"], eps=self.eps, rms=True, residual=x)
        out, gate_up = B.psa_ffn(b, w["w_gate"], w["w_up"], w["w_down"], status=self.status)
        return mid, out, (x, a, stats1, saved, mid, b, stats2, gate_up)

    def backward(self, d_stream, d_delta, w, saved):
        """For the gradients of forward's first two results: (gradient of x, which is also delta's, dict of the weights'
        gradients).  Where the layer's output is their sum, both are the gradient of the output."""
        x, a, stats1, attn_saved, mid, b, stats2, gate_up = saved
        g = {}
        db, g["w_gate"], g["w_up"], g["w_down"] = B.psa_ffn_bwd(d_delta, b, w["w_gate"], w["w_up"], w["w_down"], gate_up,
                                                                          status=self.status)
        d_mid, g["norm2"], _ = B.psa_norm_bwd(db, mid, w["norm2"], stats2, rms=True, d_total=d_stream, status=self.status)
        da, g["wq"], g["wk"], g["wv"], g["wo"] = self.attention.backward(a, w["wq"], w["wk"], w["wv"], w["wo"], attn_saved, d_mid)
        dx, g["norm1"], _ = B.psa_norm_bwd(da, x, w["norm1"], stats1, rms=True, d_total=d_mid, status=self.status)
        return dx, g


class BlockNormLayer(DecoderLayer):
    """DecoderLayer whose sublayers' outputs are normalised, or scaled by a gate for each channel, or both, before they join the residual
    stream: beside DecoderLayer's, a weight has post1 and gate1 (the attention's output) and post2 and gate2 (the feed-forward
    block's), bf16 [hidden], each of which may be missing.  The stream itself is multiplied by residual_scale where an output joins it.

    The feed-forward block's output joins the stream in the layer behind (its first norm), with this layer's post2 and gate2:
    `before` there is this layer's weight."""

    def __init__(self, *args, residual_scale=1.0, **kwargs):
        super().__init__(*args, **kwargs)
        self.residual_scale = float(residual_scale)

    def join(self, delta, x, weight, w, n):
        """The stream x with sublayer n's output, and its norm: (norm, stream, statistics)."""
        return O.psa_block_norm(delta, x, weight, post_weight=w.get("post%d" % n), gate=w.get("gate%d" % n),
                                residual_scale=self.residual_scale, eps=self.eps, rms=True)

    def join_backward(self, d_norm, d_stream, delta, stream, weight, w, n, stats, g):
        """(gradient of delta, gradient of x, gradient of weight); those of post and gate go into the dict g."""
        d_delta, dx, dw, _, d_post, _, d_gate = O.psa_block_norm_bwd(
            d_norm, delta, stream, weight, stats, post_weight=w.get("post%d" % n), gate=w.get("gate%d" % n),
            residual_scale=self.residual_scale, rms=True, d_total=d_stream, status=self.status)
        g.update({k: d for k, d in (("post%d" % n, d_post), ("gate%d" % n, d_gate)) if d is not None})
        return d_delta, dx, dw

    def forward(self, x, w, delta=None, before=None):
        """Returns (residual stream, delta, what backward needs); delta joins the stream in the layer behind."""
        if delta is None:
            a, stats1 = B.psa_norm(x, w["norm1"], eps=self.eps, rms=True)
        else:
            a, x, stats1 = self.join(delta, x, w["norm1"], before, 2)
        attn, saved = self.attention.forward(a, w["wq"], w["wk"], w["wv"], w["wo"])
        b, mid, stats2 = self.join(attn, x, w["norm2"], w, 1)
        out, gate_up = B.psa_ffn(b, w["w_gate"], w["w_up"], w["w_down"], status=self.status)
        return mid, out, (x, delta, a, stats1, saved, attn, mid, b, stats2, gate_up)

    def backward(self, d_stream, d_delta, w, saved, before=None):
        """For the gradients of forward's first two results: (gradient of x, gradient of delta (None without one), dict of the
        weights' gradients, dict of those of the layer before's post2 and gate2)."""
        x, delta, a, stats1, attn_saved, attn, mid, b, stats2, gate_up = saved
        g, g_before = {}, {}
        db, g["w_gate"], g["w_up"], g["w_down"] = B.psa_ffn_bwd(d_delta, b, w["w_gate"], w["w_up"], w["w_down"], gate_up,
                                                                          status=self.status)
        d_attn, dx, g["norm2"] = self.join_backward(db, d_stream, attn, mid, w["norm2"], w, 1, stats2, g)
        da, g["wq"], g["wk"], g["wv"], g["wo"] = self.attention.backward(a, w["wq"], w["wk"], w["wv"], w["wo"], attn_saved, d_attn)
        if delta is None:
            dx, g["norm1"], _ = B.psa_norm_bwd(da, x, w["norm1"], stats1, rms=True, d_total=dx, status=self.status)
            return dx, None, g, g_before
        d_delta, dx, g["norm1"] = self.join_backward(da, dx, delta, x, w["norm1"], before, 2, stats1, g_before)
        return dx, d_delta, g, g_before


class PreferenceDecoder:
    """A decoder on one pack, from token ids to the summed log-probabilities of its responses, and back: token embedding, a
    BlockNormLayer for each weight of `layers`, the final norm, and dpo_linear_logp against the output table.  No logits are stored.

    params: a dict with table [vocab, hidden], layers (a list of weights, one at least), final [hidden], and head [vocab, hidden] or None, where
    the output table is the embedding's; all bf16.  labels: (targets, segment_ids, fork_rows, fork_targets, fork_segments) as
    logp_labels gives them, on the device."""

    def __init__(self, pack_lengths, n_q_heads, n_kv_heads, head_dim, device, embed_scale=1.0, logit_scale=1.0, eps=1e-5,
                 rope_theta=10000.0, rotary=None, residual_scale=1.0, status=None):
        self.layer = BlockNormLayer(pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta, eps, status, rotary,
                                    residual_scale=residual_scale)
        self.n_segments = 2 * len(pack_lengths[1])
        self.embed_scale, self.logit_scale, self.eps, self.status = float(embed_scale), float(logit_scale), float(eps), status

    def forward(self, params, token_ids, labels):
        """Returns (log-probabilities fp32 [2 n_samples], what backward needs)."""
        layers, head = params["layers"], params["table"] if params["head"] is None else params["head"]
        if not layers:
            raise ValueError("layers: one at least is needed")
        x, delta, saved, before = B.psa_embed(token_ids, params["table"], self.embed_scale, status=self.status), None, [], None
        for w in layers:
            x, delta, s = self.layer.forward(x, w, delta, before)
            saved.append(s)
            before = w
        y, stream, stats = self.layer.join(delta, x, params["final"], before, 2)
        logps, lse = O.dpo_linear_logp(y, head, *labels[:2], self.n_segments, *labels[2:], scale=self.logit_scale, status=self.status)
        return logps, (saved, delta, y, stream, stats, lse)

    def backward(self, coef, params, token_ids, labels, saved):
        """Gradients of sum(coef * log-probabilities), as a dict with the keys of params."""
        saved, delta, y, stream, stats, lse = saved
        layers, tied = params["layers"], params["head"] is None
        head, grads = params["table"] if tied else params["head"], [{} for _ in layers]
        dy, d_head = O.dpo_linear_logp_bwd(coef, y, head, lse, *labels, scale=self.logit_scale, status=self.status)
        d_delta, dx, d_final = self.layer.join_backward(dy, None, delta, stream, params["final"], layers[-1], 2, stats, grads[-1])
        for i in reversed(range(len(layers))):
            dx, d_delta, g, g_before = self.layer.backward(dx, d_delta, layers[i], saved[i], layers[i - 1] if i else None)
            grads[i].update(g)
            grads[i - 1].update(g_before)
        if tied:
            d_table = B.psa_embed_bwd(dx, token_ids, len(head), self.embed_scale, dtable=d_head, accumulate=True, status=self.status)
            return {"table": d_table, "layers": grads, "final": d_final, "head": None}
        d_table = B.psa_embed_bwd(dx, token_ids, len(params["table"]), self.embed_scale, status=self.status)
        return {"table": d_table, "layers": grads, "final": d_final, "head": d_head}
