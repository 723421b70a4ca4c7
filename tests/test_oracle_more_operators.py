"""Pins of the oracle's log-probabilities from hidden states, rotary positions and norms around a block: the same written with
torch's library functions in float64 and differentiated by autograd, and by central differences; and the table of
frequencies, which the library makes on the host, against the oracle's."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O


def _t(a):
    return torch.tensor(a, dtype=torch.float64, requires_grad=True)


def scoring(seed=0, n=12, vocab=9, width=5):
    rng = np.random.default_rng(seed)
    h, w = rng.normal(size=(n, width)), rng.normal(size=(vocab, width))
    targets, seg = rng.integers(0, vocab, size=n), rng.integers(-1, 3, size=n)
    forks = np.array([2, 2, 7, n, -1]), np.array([0, 4, 8, 1, 1]), np.array([2, 0, 1, 0, 0])
    targets[5], seg[5], seg[6] = vocab, 1, 3      # a target and a response out of range
    return h, w, targets, seg, forks, rng.normal(size=3)


def test_linear_logp_matches_library_and_autograd():
    h, w, targets, seg, forks, coef = scoring()
    th, tw = _t(h), _t(w)
    logp = torch.log_softmax(0.7 * th @ tw.t(), dim=1)
    terms = {g: [] for g in range(3)}
    for t, y, g in [(t, targets[t], seg[t]) for t in range(len(h))] + list(zip(*forks)):
        if 0 <= t < len(h) and 0 <= y < len(w) and 0 <= g < 3:
            terms[g].append(logp[t, y])
    out = torch.stack([sum(terms[g], torch.zeros((), dtype=torch.float64)) for g in range(3)])
    got, lse = orc.linear_logp(h, w, targets, seg, 3, *forks, scale=0.7)
    assert np.allclose(got, out.detach().numpy(), atol=1e-12)
    scored = sorted({t for t, _, _ in orc._labels(len(h), len(w), 3, targets, seg, *forks)})
    want = torch.logsumexp(0.7 * th @ tw.t(), dim=1).detach().numpy()
    assert np.allclose(lse[scored], want[scored]) and not np.delete(lse, scored).any()
    (out * torch.tensor(coef)).sum().backward()
    dh, dw, _ = orc.linear_logp_grad(h, w, targets, seg, coef, *forks, scale=0.7)
    assert np.allclose(dh, th.grad.numpy(), atol=1e-12) and np.allclose(dw, tw.grad.numpy(), atol=1e-12)


def test_linear_logp_is_the_gather_of_stored_logits_and_follows_differences():
    h, w, targets, seg, forks, coef = scoring(1)
    targets, seg = np.minimum(targets, 8), np.where(seg == 3, -1, seg)
    keep = [a[:3] for a in forks]
    got, _ = orc.linear_logp(h, w, targets, seg, 3, *keep)
    assert np.allclose(got, orc.dpo_logp(h @ w.T, targets, seg, 3, *keep), atol=1e-12)
    dh, dw, dz = orc.linear_logp_grad(h, w, targets, seg, coef, *keep)
    assert np.allclose(dz, orc.dpo_logp_grad(h @ w.T, targets, seg, coef, *keep), atol=1e-12)
    for a, d, at in ((h, dh, (3, 2)), (w, dw, (4, 1)), (h, dh, (2, 0))):
        loss = []
        for step in (1e-5, -1e-5):
            moved = a.copy()
            moved[at] += step
            args = (moved, w) if a is h else (h, moved)
            loss.append(coef @ orc.linear_logp(*args, targets, seg, 3, *keep)[0])
        assert abs((loss[0] - loss[1]) / 2e-5 - d[at]) < 1e-7


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_keeps_lengths_turns_by_the_difference_of_positions_and_its_gradient_turns_back(interleaved):
    rng = np.random.default_rng(0)
    q, k, g = (rng.normal(size=(6, 2, 10)) for _ in range(3))
    radians, _ = orc.rotary_frequencies(8)
    pos = np.array([0, 1, 5, 100, 7, 3])
    turn = lambda x, p, **kw: orc.rotary(x, p, radians, 1.3, interleaved, **kw)  # noqa: E731
    rq = turn(q, pos)
    assert np.allclose(rq[0, :, :8], 1.3 * q[0, :, :8]) and np.array_equal(rq[..., 8:], q[..., 8:])
    assert np.allclose((rq[..., :8] ** 2).sum(-1), 1.69 * (q[..., :8] ** 2).sum(-1))
    a = (turn(q, pos)[..., :8] * turn(k, pos + 11)[..., :8]).sum(-1)
    b = (turn(q, pos * 0)[..., :8] * turn(k, pos * 0 + 11)[..., :8]).sum(-1)
    assert np.allclose(a, b)
    assert np.isclose((rq * g).sum(), (q * turn(g, pos, inverse=True)).sum())
    if not interleaved:
        whole, _ = orc.rotary_frequencies(10)
        assert np.allclose(orc.rotary(q, pos, whole), orc.rope(q, pos))


def test_frequencies_of_the_library_are_the_oracles():
    rng = np.random.default_rng(3)
    for i in range(200):
        r, kind = 2 * int(rng.integers(2, 129)), [None, "linear", "base", "wavelength", "ramp"][i % 5]
        theta, factor, length = float(np.exp(rng.uniform(np.log(100), np.log(1e7)))), float(rng.uniform(1, 64)), float(rng.integers(64, 65536))
        bounds = {} if i % 2 else {"low": float(rng.uniform(0.5, 2)), "high": float(rng.uniform(3, 40))}
        turns, magnitude = O.psa_rotary_frequencies(r, theta, kind, factor, length, **bounds)
        radians, want = orc.rotary_frequencies(r, theta, kind, factor, length, **bounds)
        got = turns.numpy().astype(np.float64) / 2.0 ** 64 * 2 * np.pi
        assert turns.shape == (r // 2,) and (turns > 0).all()
        # 53 bits, a power of theta's rounding times its exponent, and half a unit of 2^-64 turns
        assert (np.abs(got - radians) <= 2.0 ** -46 * radians + 2.0 ** -61).all(), (r, kind, theta)
        assert abs(magnitude - want) <= 2.0 ** -23 * want
    first = O.psa_rotary_frequencies(8, 10000.0)[0][0].item()
    assert abs(first / 2 ** 64 * 2 * np.pi - 1) < 1e-15      # pair 0 turns one radian per position


def test_scalings_do_what_they_are_for():
    plain, _ = orc.rotary_frequencies(64, 10000.0)
    for kind in ("linear", "base", "wavelength", "ramp"):
        f, m = orc.rotary_frequencies(64, 10000.0, kind, 4.0, 4096)
        assert np.allclose(f[-1], plain[-1] / 4) and (f <= plain * (1 + 1e-12)).all() and (np.diff(f) < 0).all()
        assert np.allclose(f[0], plain[0] / (4 if kind == "linear" else 1)) and (m > 1) == (kind == "ramp")
        same, _ = orc.rotary_frequencies(64, 10000.0, kind, 1.0, 4096)
        assert np.allclose(same, plain)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post,gate", [(True, True), (True, False), (False, True), (False, False)])
def test_block_norm_matches_library_and_autograd(rms, post, gate):
    rng = np.random.default_rng(2)
    n, d = 5, 7
    x, res, g, gt = (rng.normal(size=(n, d)) * 2 + 0.5 for _ in range(4))
    vec = lambda there: rng.normal(size=d) if there else None  # noqa: E731
    p = dict(weight=vec(True), bias=vec(not rms), post_weight=vec(post), post_bias=vec(post and not rms), gate=vec(gate))
    t = {k: None if v is None else _t(v) for k, v in p.items()}
    tx, tr = _t(x), _t(res)
    norm = lambda v, w, b: F.rms_norm(v, (d,), w, 1e-3) if rms else F.layer_norm(v, (d,), w, b, 1e-3)  # noqa: E731
    y = norm(tx, t["post_weight"], t["post_bias"]) if post else tx
    total = 0.6 * tr + (y * t["gate"] if gate else y)
    out = norm(total, t["weight"], t["bias"])
    ro, rt, stats = orc.block_norm_fwd(x, res, residual_scale=0.6, eps=1e-3, rms=rms, **p)
    assert np.allclose(ro, out.detach().numpy(), atol=1e-12) and np.allclose(rt, total.detach().numpy(), atol=1e-12)
    assert stats.shape == (4, n) and (post or (not stats[0].any() and (stats[1] == 1).all()))
    ((out * torch.tensor(g)).sum() + (total * torch.tensor(gt)).sum()).backward()
    q = {k: v for k, v in p.items() if k != "bias"}
    got = orc.block_norm_bwd(g, x, rt, residual_scale=0.6, eps=1e-3, rms=rms, d_total=gt, **q)
    assert np.allclose(got["x"], tx.grad.numpy(), atol=1e-11) and np.allclose(got["residual"], tr.grad.numpy(), atol=1e-11)
    for k, v in t.items():
        if v is not None:
            assert np.allclose(got[k], v.grad.numpy(), atol=1e-11), k
