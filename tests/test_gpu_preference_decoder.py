"""A run of the operators as a training step uses them: token ids -> embedding -> two decoder layers with scaled rotary
positions and norms behind their sublayers -> final norm -> log-probabilities straight from the hidden states -> DPO loss, and all
the way back to the gradients of the tables and of every weight, against the same in 64 bits.

Every stage rounds to bf16 (2^-8 of the value at most).  The longest path to a gradient passes about 14 stages in each layer
forward and as many backward, 60 roundings in all; independent ones add up in the 2-norm to sqrt(60) 2^-8 / sqrt(3) = 1.8 % where
each enters with weight one.  The bound is 3 % of each gradient's norm."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import workloads as wl
from paper_2410_20305_b200.labels import logp_labels
from paper_2410_20305_b200.layer import AttentionLayer, BlockNormLayer, DecoderLayer, PreferenceDecoder, Rotary

pytestmark = pytest.mark.gpu

EPS, BETA = 1e-5, 0.1
f = wl.to_f64
dev = lambda a: torch.as_tensor(a).cuda()  # noqa: E731


def weights(hid, hq, hkv, d, ffn, seed, post, gate):
    bf = lambda shape, k, std, mean=0.0: (wl.bf16_normal(shape, seed * 20 + k, std).float() + mean).to(torch.bfloat16)  # noqa: E731
    std = hid ** -0.5
    w = {"norm1": bf((hid,), 1, 0.1, 1.0), "norm2": bf((hid,), 2, 0.1, 1.0), "wq": bf((hid, hq * d), 3, std), "wk": bf((hid, hkv * d), 4, std),
         "wv": bf((hid, hkv * d), 5, std), "wo": bf((hq * d, hid), 6, std), "w_gate": bf((hid, ffn), 7, std), "w_up": bf((hid, ffn), 8, std),
         "w_down": bf((ffn, hid), 9, ffn ** -0.5)}
    if post:
        w.update(post1=bf((hid,), 10, 0.1, 1.0), post2=bf((hid,), 11, 0.1, 1.0))
    if gate:
        w.update(gate1=bf((hid,), 12, 0.2, 0.8), gate2=bf((hid,), 13, 0.2, 0.8))
    return w


def oracle_attention(a, w, turn, mask, hq, hkv):
    T = len(a)
    d = w["wq"].shape[1] // hq
    q, k, v = (a @ w[n] for n in ("wq", "wk", "wv"))
    q, k, v = q.reshape(T, hq, d), k.reshape(T, hkv, d), v.reshape(T, hkv, d)
    rq, rk = turn(q), turn(k)
    o, _ = orc.attention_fwd(rq, rk, v, mask)
    return o.reshape(T, -1) @ w["wo"], (rq, rk, v, o)


def oracle_attention_bwd(a, w, saved, turn, mask, d_out):
    rq, rk, v, o = saved
    T = len(a)
    d_o = (d_out @ w["wo"].T).reshape(o.shape)
    dq, dk, dv = orc.attention_bwd(rq, rk, v, d_o, mask)
    dq, dk = turn(dq, inverse=True), turn(dk, inverse=True)
    g = {"wo": o.reshape(T, -1).T @ d_out}
    da = 0
    for n, x in (("wq", dq), ("wk", dk), ("wv", dv)):
        g[n] = a.T @ x.reshape(T, -1)
        da = da + x.reshape(T, -1) @ w[n].T
    return da, g


def oracle_join(delta, x, weight, w, n, scale):
    out, total, _ = orc.block_norm_fwd(delta, x, weight, None, w.get("post%d" % n), None, w.get("gate%d" % n), scale, EPS, True)
    return out, total


def oracle_join_bwd(d_norm, d_stream, delta, total, weight, w, n, scale, g):
    b = orc.block_norm_bwd(d_norm, delta, total, weight, w.get("post%d" % n), None, w.get("gate%d" % n), scale, EPS, True, d_stream)
    g.update({"%s%d" % (k, n): b["post_weight" if k == "post" else "gate"] for k in ("post", "gate") if "%s%d" % (k, n) in w})
    return b["x"], b["residual"], b["weight"]


@pytest.mark.parametrize("hq,hkv,d,ffn,vocab,tied,post,gate,scale,rotary", [
    (4, 2, 64, 696, 1000, True, True, False, 1.0, dict(rotary_dim=64, scaling="wavelength", factor=4.0, original_length=64)),
    (2, 2, 128, 520, 333, False, True, True, 0.9, dict(rotary_dim=48, interleaved=True, scaling="ramp", factor=2.0, original_length=128)),
    (3, 1, 64, 264, 517, False, False, True, 1.0, dict(rotary_dim=64, theta=500000.0))])
def test_a_step_from_token_ids_to_every_gradient(hq, hkv, d, ffn, vocab, tied, post, gate, scale, rotary):
    pack = wl.pack_from_lengths("step", [(90, 40, 60), (0, 33, 20), (129, 5, 31)], hq, hkv, d)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    T, hid, logit_scale = pack.total_tokens, hq * d, 0.5
    rng = np.random.default_rng(5)
    ids = rng.integers(0, vocab, size=T).astype(np.int32)
    params = {"table": wl.bf16_normal((vocab, hid), 91, hid ** -0.5), "layers": [weights(hid, hq, hkv, d, ffn, s, post, gate) for s in (1, 2)],
              "final": (1 + wl.bf16_normal((hid,), 93, 0.1).float()).to(torch.bfloat16),
              "head": None if tied else wl.bf16_normal((vocab, hid), 92, 4 * hid ** -0.5)}
    labels = logp_labels(ids, *lengths)
    targets, seg, fr, ft, fs = labels
    ref_logps = -6.0 * np.ones(2 * pack.n_samples) * np.maximum(1, np.bincount(seg[seg >= 0], minlength=2 * pack.n_samples))

    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    model = PreferenceDecoder(lengths, hq, hkv, d, "cuda", embed_scale=hid ** 0.5, logit_scale=logit_scale, eps=EPS, rotary=Rotary(**rotary),
                              residual_scale=scale, status=status)
    cuda = {k: [{n: t.cuda() for n, t in w.items()} for w in v] if k == "layers" else None if v is None else v.cuda() for k, v in params.items()}
    dl = [dev(a) for a in labels]
    logps, saved = model.forward(cuda, dev(ids), dl)
    loss, coef = B.dpo_loss(logps, dev(ref_logps.astype(np.float32)), BETA)
    grads = model.backward(coef, cuda, dev(ids), dl, saved)
    torch.cuda.synchronize()
    assert int(status.item()) == 0

    r = {k: [{n: f(t) for n, t in w.items()} for w in v] if k == "layers" else None if v is None else f(v) for k, v in params.items()}
    pos, mask = orc.position_ids(*lengths), orc.packed_mask(*lengths)
    radians, magnitude = orc.rotary_frequencies(**{k: v for k, v in rotary.items() if k != "interleaved"})
    turn = lambda x, **kw: orc.rotary(x, pos, radians, magnitude, rotary.get("interleaved", False), **kw)  # noqa: E731
    x, delta, kept, before = orc.embed_fwd(ids, r["table"], hid ** 0.5), None, [], None
    for w in r["layers"]:
        a, x = (orc.norm_fwd(x, w["norm1"], None, EPS, True)[0], x) if delta is None else oracle_join(delta, x, w["norm1"], before, 2, scale)
        attn, s = oracle_attention(a, w, turn, mask, hq, hkv)
        b, mid = oracle_join(attn, x, w["norm2"], w, 1, scale)
        out = orc.ffn_fwd(b, w["w_gate"], w["w_up"], w["w_down"])[0]
        kept.append((x, delta, a, s, attn, mid, b))
        x, delta, before = mid, out, w
    y, stream = oracle_join(delta, x, r["final"], before, 2, scale)
    head = r["table"] if tied else r["head"]
    rlogps, _ = orc.linear_logp(y, head, targets, seg, 2 * pack.n_samples, fr, ft, fs, scale=logit_scale)
    rloss, rcoef = orc.dpo_loss(rlogps, ref_logps, BETA)[:2]
    dy, d_head, _ = orc.linear_logp_grad(y, head, targets, seg, rcoef, fr, ft, fs, scale=logit_scale)
    rg = [{} for _ in r["layers"]]
    d_delta, dx, d_final = oracle_join_bwd(dy, None, delta, stream, r["final"], r["layers"][-1], 2, scale, rg[-1])
    for i in reversed(range(2)):
        w, g = r["layers"][i], rg[i]
        x, delta, a, s, attn, mid, b = kept[i]
        db, g["w_gate"], g["w_up"], g["w_down"] = orc.ffn_bwd(d_delta, b, w["w_gate"], w["w_up"], w["w_down"])
        d_attn, dx, g["norm2"] = oracle_join_bwd(db, dx, attn, mid, w["norm2"], w, 1, scale, g)
        da, ga = oracle_attention_bwd(a, w, s, turn, mask, d_attn)
        g.update(ga)
        if delta is None:
            dn, g["norm1"], _ = orc.norm_bwd(da, x, w["norm1"], EPS, True)
            dx = dx + dn
        else:
            d_delta, dx, g["norm1"] = oracle_join_bwd(da, dx, delta, x, w["norm1"], r["layers"][i - 1], 2, scale, rg[i - 1])
    d_table = orc.embed_bwd(dx, ids, vocab, hid ** 0.5)
    off = lambda a, b: np.linalg.norm(f(a) - b) / np.linalg.norm(b)  # noqa: E731
    far = {"logps": off(logps, rlogps), "final": off(grads["final"], d_final), "table": off(grads["table"], d_table + (d_head if tied else 0))}
    assert (grads["head"] is None) == tied
    if not tied:
        far["head"] = off(grads["head"], d_head)
    for i, (g, ref) in enumerate(zip(grads["layers"], rg)):
        assert sorted(g) == sorted(ref) == sorted(params["layers"][i])
        far.update({"%s of layer %d" % (k, i): off(g[k], ref[k]) for k in g})
    print({k: round(float(v), 4) for k, v in far.items()})
    want = float(np.asarray(rloss).reshape(-1)[0])
    assert abs(float(loss.item()) - want) <= 0.03 * abs(want)
    assert all(v <= 0.03 for v in far.values()), far


def test_a_layer_without_posts_gates_and_scale_is_a_decoder_layer():
    pack = wl.pack_from_lengths("one", [(60, 30, 40)], 4, 2, 64)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    w = {k: t.cuda() for k, t in weights(256, 4, 2, 64, 264, 3, False, False).items()}
    x, d = wl.bf16_normal((130, 256), 1, 1.0).cuda(), wl.bf16_normal((130, 256), 2, 1.0).cuda()
    plain, block = DecoderLayer(lengths, 4, 2, 64, "cuda"), BlockNormLayer(lengths, 4, 2, 64, "cuda")
    mid, out, s = plain.forward(x, w, d)
    mid2, out2, s2 = block.forward(x, w, d, {})
    dx, g = plain.backward(d, d, w, s)
    dx2, d_delta, g2, none = block.backward(d, d, w, s2, {})
    # the two round alike but for the order of a row's sums: rare neighbours in bf16
    near = lambda a, b: ((a.float() - b.float()).norm() / b.float().norm()).item() <= 2.0 ** -9  # noqa: E731
    assert near(mid2, mid) and near(out2, out) and near(dx2, dx) and torch.equal(dx2, d_delta) and none == {}
    assert sorted(g) == sorted(g2) and all(near(g2[k], g[k]) for k in g)


def test_a_layer_with_the_plain_rotary_is_one_with_psa_rope():
    pack = wl.pack_from_lengths("one", [(60, 30, 40)], 4, 2, 64)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    w = weights(256, 4, 2, 64, 264, 3, False, False)
    ws = [w[k].cuda() for k in ("wq", "wk", "wv", "wo")]
    x, d = wl.bf16_normal((130, 256), 1, 1.0).cuda(), wl.bf16_normal((130, 256), 2, 1.0).cuda()
    a, b = AttentionLayer(lengths, 4, 2, 64, "cuda"), AttentionLayer(lengths, 4, 2, 64, "cuda", rotary=Rotary(64))
    out, s = a.forward(x, *ws)
    out2, s2 = b.forward(x, *ws)
    near = lambda u, v: ((u.float() - v.float()).norm() / v.float().norm()).item() <= 2.0 ** -9  # noqa: E731
    assert near(out2, out) and all(near(u, v) for u, v in zip(b.backward(x, *ws, s2, d), a.backward(x, *ws, s, d)))


def test_gradients_follow_differences():
    """A direction through all parameters' gradients against the difference of the log-probabilities along it.

    A step along the gradient, of length h in each parameter's own units, changes the sum by h |g|^2 but for the second order and the
    roundings of both passes; with h such that the change is 2 % of |loss| or more, both stay below 15 % of it at this size."""
    pack = wl.pack_from_lengths("step", [(40, 30, 30)], 2, 1, 64)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    rng = np.random.default_rng(5)
    ids = rng.integers(0, 200, size=100).astype(np.int32)
    params = {"table": wl.bf16_normal((200, 128), 91, 0.1).cuda(), "layers": [{k: t.cuda() for k, t in weights(128, 2, 1, 64, 136, 1, True, True).items()}],
              "final": torch.ones(128, dtype=torch.bfloat16, device="cuda"), "head": wl.bf16_normal((200, 128), 92, 0.1).cuda()}
    labels = [dev(a) for a in logp_labels(ids, *lengths)]
    model = PreferenceDecoder(lengths, 2, 1, 64, "cuda", embed_scale=10.0)
    coef = torch.tensor([1.0, 0.5], device="cuda")
    value = lambda p: float((model.forward(p, dev(ids), labels)[0] * coef).sum())  # noqa: E731
    logps, saved = model.forward(params, dev(ids), labels)
    grads = model.backward(coef, params, dev(ids), labels, saved)
    g = grads["head"].float()
    step = 0.02 * abs(value(params)) / float((g * g).sum())
    moved = [dict(params, head=(params["head"].float() + s * step * g).to(torch.bfloat16)) for s in (1, -1)]
    real = [m["head"].float() - params["head"].float() for m in moved]
    want = float((g * (real[0] - real[1])).sum())
    got = value(moved[0]) - value(moved[1])
    assert abs(got - want) <= 0.15 * abs(want), (got, want)
