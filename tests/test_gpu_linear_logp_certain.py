"""dpo_linear_logp and dpo_linear_logp_bwd where a token takes nearly all of a row's probability: the log-probability and the gradient
are then what is left for the others, 1 - p, and are held relative to that.

Bounds.  With z the label's logit and r = (1 - p) / p the sum of exp(z[v] - z) over the other tokens, a term is -log(1 + r).
The label's own product is taken by fp32 additions, width / 256 of them in a row and 11 that join threads at most: off by
(width / 256 + 11) 2^-24 of its sum of magnitudes.  Another token's logit comes from the tensor cores: off by width * 2^-23 of its own.  An
exponent's argument is rounded to 2^-22 of itself, the scale's division by log 2 counted, and 2^-16 covers the exponential and the sums.
r is off by the sum of these, relative to itself, the term by no more, and then by half a unit of 2^-40 and a rounding to fp32.
In the gradient the label's element c (1 - p) is taken from its own product and lse as fp32 holds it: off by p times the product's error, the
error of lse and 2^-23 of |z| and |lse|; the other elements as in test_gpu_linear_logp.py."""
import numpy as np
import pytest
import torch

from test_gpu_linear_logp import H8, both, f64, within

pytestmark = pytest.mark.gpu

NONE = [np.zeros(0, np.int32)] * 3


def certain(n, width, vocab, low, high, seed):
    """(hidden, table, targets): row t's token has the table's row along hidden[t], so long that 1 - p is about low .. high; the
    other rows of the table are short."""
    rng = np.random.default_rng(seed)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    hidden = bf(rng.normal(size=(n, width)))
    h = hidden.double().numpy()
    table = rng.normal(size=(vocab, width)) * 0.05 * width ** -0.5
    targets = rng.permutation(vocab)[:n].astype(np.int32)
    left = np.exp(np.linspace(np.log(low), np.log(high), n))
    table[targets] = h / (h ** 2).sum(1, keepdims=True) * np.log(vocab / left)[:, None]
    return hidden, bf(table), targets


def terms(hidden, table, rows, targets, scale):
    """Per label in 64 bits: z of every token, lse, 1 - p of the label, and the bounds of the label's product and of the others' logits."""
    h, w = f64(hidden)[rows], f64(table)
    z, size = scale * h @ w.T, scale * np.abs(h) @ np.abs(w).T
    at = np.arange(len(rows))
    own = z[at, targets]
    apart = z - own[:, None]
    apart[at, targets] = -np.inf
    r = np.exp(apart).sum(1)
    width = h.shape[1]
    e_own = (width / 256 + 11) * 2.0 ** -24 * size[at, targets]
    return z, own + np.log1p(r), r, e_own, width * 2.0 ** -23 * size


def logp_bound(z, r, e_own, e, at, targets):
    """Of a term -log1p(r)."""
    own = z[at, targets]
    rel = 2.0 ** -16 + e.max(1) + e_own + 2.0 ** -22 * (np.abs(z).max(1) + np.abs(own))
    return np.log1p(r) * 1.01 * rel + 2.0 ** -41 + 2.0 ** -24 * np.log1p(r)


@pytest.mark.parametrize("n,width,vocab,scale", [(200, 4096, 700, 1.0), (60, 64, 300, 1.0), (90, 1032, 2049, 0.5), (2500, 256, 3001, 1.0)])
def test_log_probabilities_near_zero(n, width, vocab, scale):
    hidden, table, targets = certain(n, width, vocab, 1e-8, 1e-1, n + width)
    if scale != 1.0:
        hidden = (hidden / scale).contiguous()
    seg = np.arange(n, dtype=np.int32)
    out, lse, _, _, status = both(hidden, table, targets, seg, NONE, np.ones(n, np.float32), scale=scale)
    at = np.arange(n)
    z, rl, r, e_own, e = terms(hidden, table, at, targets, scale)
    assert status == 0 and r.min() < 1e-7 and r.max() > 1e-2
    within("out", out, -np.log1p(r), logp_bound(z, r, e_own, e, at, targets))
    within("lse", lse, rl, e_own + np.log1p(r) * (2.0 ** -16 + e.max(1)) + 2.0 ** -22 * np.abs(rl))


def gradient(hidden, table, rows, targets, c, scale):
    """Rows of d_hidden per label in 64 bits and their bounds."""
    z, rl, r, e_own, e = terms(hidden, table, rows, targets, scale)
    w, at = f64(table), np.arange(len(rows))
    p = np.exp(z - rl[:, None])
    e_lse = e_own + np.log1p(r) * (2.0 ** -16 + e.max(1)) + 2.0 ** -23 * np.abs(rl)
    dz = -p
    dz[at, targets] = r / (1 + r)
    e_dz = 1.01 * p * (e + e_lse[:, None] + 2.0 ** -16) + 2.0 ** -22 * p
    e_dz[at, targets] = 1.01 * p[at, targets] * (e_own + e_lse + 2.0 ** -23 * (np.abs(z[at, targets]) + np.abs(rl))) + 2.0 ** -22 * np.abs(dz[at, targets])
    e_dz += H8 * np.abs(dz) + len(w) * 2.0 ** -23 * np.abs(dz)
    c = scale * c[:, None]
    ref = (c * dz) @ w
    return ref, np.abs(c) * e_dz @ np.abs(w) + H8 * np.abs(ref) + 1e-30


@pytest.mark.parametrize("n,width,vocab,scale", [(200, 4096, 700, 1.0), (60, 64, 300, 1.0), (90, 2056, 2049, 0.5)])
def test_gradients_of_log_probabilities_near_zero(n, width, vocab, scale):
    hidden, table, targets = certain(n, width, vocab, 1e-5, 1e-2, n + width)
    if scale != 1.0:
        hidden = (hidden / scale).contiguous()
    coef = np.random.default_rng(1).uniform(0.5, 2, size=n).astype(np.float32)
    _, _, dh, _, status = both(hidden, table, targets, np.arange(n, dtype=np.int32), NONE, coef, scale=scale)
    ref, tol = gradient(hidden, table, np.arange(n), targets, coef.astype(float), scale)
    assert status == 0
    within("d_hidden", dh, ref, tol)


@pytest.mark.parametrize("own", [True, False])
def test_forks_that_are_nearly_certain(own):
    """A row whose own label, or first fork, is improbable, and a later fork nearly certain: lse and the fork's gradient."""
    n, width, vocab = 120, 4096, 700
    hidden, table, sure = certain(n, width, vocab, 1e-5, 1e-2, 7)
    rng = np.random.default_rng(2)
    away = np.setdiff1d(np.arange(vocab), sure)[:n].astype(np.int32)
    coef = rng.uniform(0.5, 2, size=n + 1).astype(np.float32)
    coef[n] = 0      # of the improbable labels
    rows, seg = np.arange(n, dtype=np.int32), np.arange(n, dtype=np.int32)
    if own:
        labels, forks = (away, np.full(n, n, np.int32)), [rows, sure, seg]
    else:
        labels = (away, np.full(n, -1, np.int32))
        forks = [np.concatenate(a).astype(np.int32) for a in ((rows, rows), (away, sure), (np.full(n, n), seg))]
    out, lse, dh, _, status = both(hidden, table, *labels, forks, coef)
    z, rl, r, e_own, e = terms(hidden, table, rows, sure, 1.0)
    assert status == 0
    within("out", out[:n], -np.log1p(r), logp_bound(z, r, e_own, e, rows, sure))
    within("lse", lse, rl, e_own + np.log1p(r) * (2.0 ** -16 + e.max(1)) + 2.0 ** -22 * np.abs(rl))
    ref, tol = gradient(hidden, table, rows, sure, coef[:n].astype(float), 1.0)
    within("d_hidden", dh, ref, tol)


def test_a_label_with_nothing_beside_it():
    """A vocabulary of one token, other tokens of probability 0, and a label whose own logit is infinite."""
    rng = np.random.default_rng(3)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    hidden, table = bf(rng.uniform(0.5, 1, size=(40, 72))), bf(rng.normal(size=(300, 72)))
    seg = np.arange(40, dtype=np.int32)
    bound = (72 / 256 + 11) * 2.0 ** -24 * (f64(hidden) @ np.abs(f64(table)).T).max() + 2.0 ** -22 * 88
    out, lse, dh, dw, _ = both(hidden, table[:1].contiguous(), np.zeros(40, np.int32), seg, NONE, np.ones(40, np.float32))
    z = f64(hidden) @ f64(table).T
    assert not out.any() and np.abs(f64(lse) - z[:, 0]).max() <= bound
    assert np.abs(f64(dh)).max() <= 2 * bound * np.abs(f64(table)).max() and np.abs(f64(dw)).max() <= 40 * 2 * bound
    alone = torch.full_like(table, float("-inf"))
    alone[257] = table[257]
    out, lse, *_ = both(hidden, alone, np.full(40, 257, np.int32), seg, NONE, np.ones(40, np.float32))
    assert not out.any() and np.abs(f64(lse) - z[:, 257]).max() <= bound
    above = table.clone()
    above[257] = float("inf")
    out, lse, *_ = both(hidden, above, np.full(40, 257, np.int32), seg, NONE, np.ones(40, np.float32))
    assert out.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("width,vocab", [(4096, 4000), (1024, 3000), (8192, 1500)])
def test_log_probabilities_are_not_high_in_the_mean(width, vocab):
    """Ordinary rows.  The tensor cores cut off what is below a sum's last bit, which takes 2^-30 of a logit for each term in the mean and is given
    back; what that mean was measured to vary by, 15 %, is left: 0.15 width 2^-30 of the mean logit over the tokens as they are likely.  A
    single logit's cut-off scatters by half of the mean, which 500 labels and their tokens average to less than a tenth of that.
    What is rounded, to 2^-22 of lse at most in each of three places, is as often up as down and is allowed once."""
    n = 500
    rng = np.random.default_rng(width)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    hidden, table = bf(rng.normal(size=(n, width))), bf(rng.normal(size=(vocab, width)) * 3 * width ** -0.5)
    targets = rng.integers(0, vocab, size=n).astype(np.int32)
    out, lse, _, _, _ = both(hidden, table, targets, np.arange(n, dtype=np.int32), NONE, np.ones(n, np.float32))
    z = f64(hidden) @ f64(table).T
    rl = np.log(np.exp(z).sum(1))
    ro = z[np.arange(n), targets] - rl
    likely = (np.exp(z - rl[:, None]) * z).sum(1).mean()
    bound = 0.2 * width * 2.0 ** -30 * likely + 2.0 ** -22 * np.abs(rl).mean() / n ** 0.5
    error = (f64(out) - ro).mean(), (f64(lse) - rl).mean()
    print("mean error of the terms %.2e, of lse %.2e, bound %.2e" % (*error, bound))
    assert likely > 5 and abs(error[0]) <= bound and abs(error[1]) <= bound


@pytest.mark.parametrize("n,width,vocab,forked", [(300, 512, 2000, False), (40, 1032, 700, True), (2500, 64, 1500, False)])
def test_the_rounding_of_a_label_s_element_is_given_back_to_d_hidden(n, width, vocab, forked):
    """Responses' coefficients at which a label's element of dz, nearly all of its row, lies half way between two values of bf16: d_hidden has
    the error of its own rounding, uniform within 2^-8 of a value at most, and of the roundings of the other elements."""
    rng = np.random.default_rng(n)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    hidden, table = bf(rng.normal(size=(n, width))), bf(rng.normal(size=(vocab, width)) * 0.5 * width ** -0.5)
    targets, rows = rng.integers(0, vocab, size=n).astype(np.int32), np.arange(n, dtype=np.int32)
    coef = ((1 + 2.0 ** -8) * (1 + 1.0 / vocab) * rng.uniform(0.9995, 1.0005, size=n)).astype(np.float32)
    forks = NONE
    if forked:      # three more labels for each row, of the same responses
        forks = [np.tile(rows, 3), rng.integers(0, vocab, size=3 * n).astype(np.int32), np.tile(rows, 3)]
    _, _, dh, _, status = both(hidden, table, targets, rows, forks, coef)
    h, w = f64(hidden), f64(table)
    z = h @ w.T
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    ref, others = np.zeros_like(h), np.zeros_like(h)
    for t, y in zip(np.concatenate([rows, forks[0]]), np.concatenate([targets, forks[1]])):
        dz = -float(coef[t]) * p[t]
        others[t] += dz ** 2 @ w ** 2
        dz[y] += float(coef[t])
        ref[t] += dz @ w
    err = np.linalg.norm(f64(dh) - ref)
    bound = H8 / 3 ** 0.5 * np.sqrt((ref ** 2).sum() + others.sum()) + 2.0 ** -16 * np.linalg.norm(ref)
    print("%.3f of the bound" % (err / bound))
    assert status == 0 and err <= bound


@pytest.mark.parametrize("forked", [False, True])
def test_a_label_s_element_beyond_the_range_of_bf16(forked):
    """A coefficient that fp32 holds and bf16 does not: what reaches d_hidden is the label's infinity times its row of the table."""
    rng = np.random.default_rng(4)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    n, width, vocab = 20, 64, 3000
    hidden, table = bf(rng.normal(size=(n, width)) * 0.1), bf(rng.normal(size=(vocab, width)))
    targets, rows = rng.integers(0, vocab, size=n).astype(np.int32), np.arange(n, dtype=np.int32)
    coef = np.full(n, 3.401e38, np.float32)      # (1 - 1 / 3000 of it is nearer to the infinity of bf16 than to its largest number, 3.39e38)
    forks = [np.tile(rows, 2), np.tile(targets, 2), np.tile(rows, 2)] if forked else NONE
    _, _, dh, _, _ = both(hidden, table, targets, rows, forks, coef)
    w = f64(table)[targets]
    assert np.array_equal(f64(dh), np.sign(w) * np.inf)
