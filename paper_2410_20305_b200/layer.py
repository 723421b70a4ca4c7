"""One attention layer on the shared layout (Section 4.2: the full attention-layer benchmark):
query / key / value projections, rotary embedding on the position ids of Section 3.1,
psa_fwd, output projection, and the backward of all of it; and a whole decoder layer around it
(norms, residual stream, gated feed-forward block).

The projections are library GEMMs (torch.matmul, i.e. cuBLAS); the rotary embedding, the
attention and its backward are this library's kernels.  A composition for the layer-level
measurement and its parity test, not a kernel of its own.
"""
from __future__ import annotations

from . import binding as B


class AttentionLayer:
    """Holds a plan, the position ids and the scratch of one pack; `forward` and `backward`
    run the layer for bf16 CUDA inputs x [T, hidden] and weights wq [hidden, Hq d],
    wk, wv [hidden, Hkv d], wo [Hq d, hidden].  `status` (optional): the int32 CUDA word in which
    psa_fwd and psa_bwd report a wait that gave up."""

    def __init__(self, pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta=10000.0, status=None):
        import torch
        cu, P, C, R = pack_lengths
        self.plan = B.psa_plan(cu, P, C, R, n_q_heads, n_kv_heads, head_dim)
        self.pos = torch.as_tensor(B.psa_position_ids(cu, P, C, R)).to(device)
        self.neg = -self.pos
        self.ws = torch.empty(max(self.plan.bwd_workspace_bytes, 256), dtype=torch.uint8, device=device)
        self.theta = float(rope_theta)
        self.status = status
        self.Hq, self.Hkv, self.d = n_q_heads, n_kv_heads, head_dim

    def forward(self, x, wq, wk, wv, wo):
        T = x.shape[0]
        q = (x @ wq).view(T, self.Hq, self.d)
        k = (x @ wk).view(T, self.Hkv, self.d)
        v = (x @ wv).view(T, self.Hkv, self.d)
        B.psa_rope(q, self.pos, self.theta, out=q)
        B.psa_rope(k, self.pos, self.theta, out=k)
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
        B.psa_rope(dq, self.neg, self.theta, out=dq)
        B.psa_rope(dk, self.neg, self.theta, out=dk)
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

    def __init__(self, pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta=10000.0, eps=1e-5, status=None):
        self.attention = AttentionLayer(pack_lengths, n_q_heads, n_kv_heads, head_dim, device, rope_theta, status)
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
