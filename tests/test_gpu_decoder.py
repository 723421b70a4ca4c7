"""A run of the operators as a training step uses them: token ids -> embedding -> two decoder layers -> final norm -> logits ->
log-probs -> DPO loss, and all the way back to the gradients of the table and of every weight, against the same in 64 bits.

Every stage rounds to bf16 (2^-8 of the value at most).  The longest path to a gradient passes about 12 stages in each layer
forward and as many backward, 50 roundings in all; independent ones add up in the 2-norm to sqrt(50) 2^-8 / sqrt(3) = 1.6 % where
each enters with weight one (the residual stream, which carries most of the signal, is rounded twice a layer).  The bound is 3 %
of each gradient's norm."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import workloads as wl
from paper_2410_20305_b200.labels import logp_labels
from paper_2410_20305_b200.layer import DecoderLayer

pytestmark = pytest.mark.gpu

EPS, BETA = 1e-5, 0.1


def weights(hid, hq, hkv, d, ffn, seed):
    bf = lambda shape, k, std, mean=0.0: (wl.bf16_normal(shape, seed * 20 + k, std).float() + mean).to(torch.bfloat16)  # noqa: E731
    std = hid ** -0.5
    return {"norm1": bf((hid,), 1, 0.1, 1.0), "norm2": bf((hid,), 2, 0.1, 1.0), "wq": bf((hid, hq * d), 3, std), "wk": bf((hid, hkv * d), 4, std),
            "wv": bf((hid, hkv * d), 5, std), "wo": bf((hq * d, hid), 6, std), "w_gate": bf((hid, ffn), 7, std), "w_up": bf((hid, ffn), 8, std),
            "w_down": bf((ffn, hid), 9, ffn ** -0.5)}


def oracle_layer_fwd(x, w, pos, mask, hq, hkv):
    a, _, _ = orc.norm_fwd(x, w["norm1"], None, EPS, True)
    attn, _ = orc.attention_layer_fwd(a, w["wq"], w["wk"], w["wv"], w["wo"], pos, mask, hq, hkv)
    mid = x + attn
    b, _, _ = orc.norm_fwd(mid, w["norm2"], None, EPS, True)
    return mid + orc.ffn_fwd(b, w["w_gate"], w["w_up"], w["w_down"])[0], (x, a, mid, b)


def oracle_layer_bwd(d_out, w, saved, pos, mask, hq, hkv):
    x, a, mid, b = saved
    g = {}
    db, g["w_gate"], g["w_up"], g["w_down"] = orc.ffn_bwd(d_out, b, w["w_gate"], w["w_up"], w["w_down"])
    dm, g["norm2"], _ = orc.norm_bwd(db, mid, w["norm2"], EPS, True)
    dm = dm + d_out
    ga = orc.attention_layer_bwd(a, w["wq"], w["wk"], w["wv"], w["wo"], pos, mask, hq, hkv, dm)
    g.update({k: ga["d" + k] for k in ("wq", "wk", "wv", "wo")})
    dx, g["norm1"], _ = orc.norm_bwd(ga["dx"], x, w["norm1"], EPS, True)
    return dx + dm, g


@pytest.mark.parametrize("hq,hkv,d,ffn,vocab", [(4, 2, 64, 696, 1000), (2, 2, 128, 520, 333)])
def test_a_step_from_token_ids_to_every_gradient(hq, hkv, d, ffn, vocab):
    pack = wl.pack_from_lengths("step", [(90, 40, 60), (0, 33, 20), (129, 5, 31)], hq, hkv, d)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    T, hid = pack.total_tokens, hq * d
    rng = np.random.default_rng(5)
    ids = rng.integers(0, vocab, size=T).astype(np.int32)
    table, head = wl.bf16_normal((vocab, hid), 91, hid ** -0.5), wl.bf16_normal((hid, vocab), 92, 2 * hid ** -0.5)
    final = (1 + wl.bf16_normal((hid,), 93, 0.1).float()).to(torch.bfloat16)
    ws = [weights(hid, hq, hkv, d, ffn, s) for s in (1, 2)]
    targets, seg, fr, ft, fs = logp_labels(ids, *lengths)
    ref_logps = -6.0 * np.ones(2 * pack.n_samples) * np.maximum(1, np.bincount(seg[seg >= 0], minlength=2 * pack.n_samples))

    dev = lambda a: torch.as_tensor(a).cuda()  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    layer = DecoderLayer(lengths, hq, hkv, d, "cuda", eps=EPS)
    cw = [{k: t.cuda() for k, t in w.items()} for w in ws]
    x, delta, saved = B.psa_embed(dev(ids), table.cuda(), scale=hid ** 0.5, status=status), None, []
    for w in cw:
        x, delta, s = layer.forward(x, w, delta)
        saved.append(s)
    y, stats, stream = B.psa_norm(x, final.cuda(), eps=EPS, rms=True, residual=delta)
    logits = torch.zeros((T, (vocab + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :vocab]
    logits.copy_(y @ head.cuda())
    forks = [dev(f) for f in (fr, ft, fs)]
    logps = B.dpo_logp(logits, dev(targets), dev(seg), 2 * pack.n_samples, *forks, status=status)
    loss, coef = B.dpo_loss(logps, dev(ref_logps.astype(np.float32)), BETA)
    dlogits = B.dpo_logp_bwd(logits, dev(targets), dev(seg), coef, *forks, status=status)
    dy, d_head = dlogits @ head.cuda().t(), y.t() @ dlogits
    d_stream, d_final, _ = B.psa_norm_bwd(dy, stream, final.cuda(), stats, rms=True, status=status)
    grads = []
    d_delta = d_stream
    for w, s in zip(reversed(cw), reversed(saved)):
        d_stream, g = layer.backward(d_stream, d_delta, w, s)
        d_delta = d_stream
        grads.insert(0, g)
    d_table = B.psa_embed_bwd(d_stream, dev(ids), vocab, scale=hid ** 0.5, dtype=torch.float32, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0

    f = wl.to_f64
    pos, mask = orc.position_ids(*lengths), orc.packed_mask(*lengths)
    rw = [{k: f(t) for k, t in w.items()} for w in ws]
    rx, rsaved = orc.embed_fwd(ids, f(table), hid ** 0.5), []
    for w in rw:
        rx, s = oracle_layer_fwd(rx, w, pos, mask, hq, hkv)
        rsaved.append(s)
    ry, _, _ = orc.norm_fwd(rx, f(final), None, EPS, True)
    rlogits = ry @ f(head)
    rlogps = orc.dpo_logp(rlogits, targets, seg, 2 * pack.n_samples, fr, ft, fs)
    rloss, rcoef = orc.dpo_loss(rlogps, ref_logps, BETA)[:2]
    rdl = orc.dpo_logp_grad(rlogits, targets, seg, rcoef, fr, ft, fs)
    rdy = rdl @ f(head).T
    rd, rd_final, _ = orc.norm_bwd(rdy, rx, f(final), EPS, True)
    rgrads = []
    for w, s in zip(reversed(rw), reversed(rsaved)):
        rd, g = oracle_layer_bwd(rd, w, s, pos, mask, hq, hkv)
        rgrads.insert(0, g)
    rd_table = orc.embed_bwd(rd, ids, vocab, hid ** 0.5)

    off = lambda a, b: np.linalg.norm(f(a) - b) / np.linalg.norm(b)  # noqa: E731
    far = {"logps": off(logps, rlogps), "head": off(d_head, ry.T @ rdl), "final": off(d_final, rd_final), "table": off(d_table, rd_table)}
    for i, (g, rg) in enumerate(zip(grads, rgrads)):
        far.update({"%s of layer %d" % (k, i): off(g[k], rg[k]) for k in DecoderLayer.KEYS})
    print({k: round(float(v), 4) for k, v in far.items()})
    assert abs(float(loss.item()) - float(np.asarray(rloss).reshape(-1)[0])) <= 0.03 * abs(float(np.asarray(rloss).reshape(-1)[0]))
    assert all(v <= 0.03 for v in far.values()), far


def test_gradients_of_a_layer_follow_differences():
    """Central differences of the oracle's layer confirm the gradients that the step above is held to."""
    pack = wl.pack_from_lengths("fd", [(5, 3, 4), (0, 2, 3)], 2, 1, 8)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    pos, mask = orc.position_ids(*lengths), orc.packed_mask(*lengths)
    rng = np.random.default_rng(0)
    x, d_out = rng.normal(size=(pack.total_tokens, 16)), rng.normal(size=(pack.total_tokens, 16))
    w = {k: wl.to_f64(t) for k, t in weights(16, 2, 1, 8, 24, 3).items()}
    out, saved = oracle_layer_fwd(x, w, pos, mask, 2, 1)
    dx, g = oracle_layer_bwd(d_out, w, saved, pos, mask, 2, 1)
    loss = lambda: (oracle_layer_fwd(x, w, pos, mask, 2, 1)[0] * d_out).sum()  # noqa: E731
    for array, grad in [(x, dx)] + [(w[k], g[k]) for k in DecoderLayer.KEYS]:
        for at in rng.choice(array.size, size=3, replace=False):
            at = np.unravel_index(at, array.shape)
            keep = array[at]
            array[at] = keep + 1e-5
            up = loss()
            array[at] = keep - 1e-5
            down = loss()
            array[at] = keep
            assert abs((up - down) / 2e-5 - grad[at]) <= 1e-6 * (1 + abs(grad[at]))


def test_two_captured_steps_share_nothing_but_the_allocator():
    """Two graphs of the same layer over different packs, replayed in turn, and one again after the other."""
    def make(lengths, seed):
        pack = wl.pack_from_lengths("g", lengths, 4, 2, 64)
        layer = DecoderLayer((pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len), 4, 2, 64, "cuda")
        w = {k: t.cuda() for k, t in weights(256, 4, 2, 64, 520, seed).items()}
        x = wl.bf16_normal((pack.total_tokens, 256), seed).cuda()
        d = wl.bf16_normal((pack.total_tokens, 256), seed + 50).cuda()

        def step():
            mid, delta, saved = layer.forward(x, w)
            dx, g = layer.backward(d, d, w, saved)
            return [mid, delta, dx] + [g[k] for k in DecoderLayer.KEYS]
        return step, x
    steps = [make([(60, 30, 20), (7, 40, 41)], 1), make([(200, 10, 20)], 2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for step, _ in steps:
            step()
    torch.cuda.synchronize()
    graphs, captured = [], []
    for step, _ in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):      # (a stream that the plans have been used on)
            captured.append(step())
        graphs.append(graph)
    for _, x in steps:
        x.mul_(0.5)
    want = [step() for step, _ in steps]
    for k in (0, 1, 0, 1, 1, 0):
        graphs[k].replay()
    torch.cuda.synchronize()
    # (psa_bwd adds dq with atomics, so what passes through it may differ in its last bits)
    for w_, c in zip(want, captured):
        for i, (a, b) in enumerate(zip(w_, c)):
            if i < 2:
                assert torch.equal(a, b), i
            else:
                assert (a.float() - b.float()).norm() <= 0.01 * a.float().norm(), i
