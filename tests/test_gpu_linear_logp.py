"""dpo_linear_logp and dpo_linear_logp_bwd against the oracle in 64 bits.

Bounds, per element.  A logit is a sum of `width` exact products in fp32: off by width * 2^-23 of the sum of magnitudes S (tensor
cores may cut off where an addition rounds), call it e.  An exponential's argument of magnitude up to 128 is rounded by 2^-18, the
exponential by 2^-22 of itself, and a row's sum passes 16 additions in a chunk, 4 chunks and vocab / 256 joins: with fewer than 100
joins the sum is off by 2^-16 of itself, so lse by max e + 2^-16 and a rounding.  dz = c (1[v = y] - p) is off by c p times what
its exponent is off by, by 2^-22 c, and by its rounding to bf16, 2^-8 of itself; d_hidden and d_table by the sums of that, by
n 2^-23 of the sum of magnitudes of n terms, and by their own rounding.  Those are bounds of the worst case; that errors do not
add up like that is held in the 2-norm, where dz's roundings, independent of one another, enter by the root of the sum of squares."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O

pytestmark = pytest.mark.gpu

H8 = 2.0 ** -8
f64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
dev = lambda a: torch.as_tensor(np.asarray(a)).cuda()  # noqa: E731
i32 = lambda a: dev(np.asarray(a, dtype=np.int32))  # noqa: E731


def inputs(n_rows, width, vocab, seed, live=0.6, n_segments=5, n_forks=3, spread=2.0, lift=True):
    rng = np.random.default_rng(seed)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    table = bf(rng.normal(size=(vocab, width)) * spread * width ** -0.5)
    targets = rng.integers(0, vocab, size=n_rows).astype(np.int32)
    seg = np.where(rng.random(n_rows) < live, rng.integers(0, n_segments, size=n_rows), -1).astype(np.int32)
    hidden = rng.normal(size=(n_rows, width))
    if lift:
        w = table.double().numpy()[targets]
        hidden += rng.uniform(0, 6, size=(n_rows, 1)) * w / np.maximum(np.linalg.norm(w, axis=1, keepdims=True), 1e-9)
    forks = [rng.integers(0, n, size=n_forks).astype(np.int32) if n else np.zeros(0, np.int32) for n in (n_rows, vocab, n_segments)]
    coef = rng.normal(size=n_segments).astype(np.float32)
    return bf(hidden), table, targets, seg, forks, coef


def both(hidden, table, targets, seg, forks, coef, scale=1.0, **kw):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = [i32(targets), i32(seg)]
    f = [i32(a) for a in forks]
    out, lse = O.dpo_linear_logp(hidden.cuda(), table.cuda(), *args, len(coef), *f, scale=scale, status=status, **kw)
    dh, dw = O.dpo_linear_logp_bwd(dev(coef), hidden.cuda(), table.cuda(), lse, *args, *f, scale=scale, status=status, **kw)
    torch.cuda.synchronize()
    return out, lse, dh, dw, int(status.item())


def within(name, got, ref, tol, norm=None):
    err = np.abs(f64(got) - ref)
    assert np.isfinite(err).all(), name
    worst = float((err / np.maximum(tol, 1e-300)).max(initial=0))
    share = float(np.linalg.norm(err) / max(norm, 1e-300)) if norm is not None else 0.0
    print("%s: %.3f of the bound, %.3f of the norm" % (name, worst, share))
    assert worst <= 1 and share <= 1, (name, worst, share)


def compare(hidden, table, targets, seg, forks, coef, scale, got):
    out, lse, dh, dw = got
    h, w, width, vocab = f64(hidden), f64(table), hidden.shape[1], table.shape[0]
    labels = orc._labels(len(h), vocab, len(coef), targets, seg, *forks)
    ro, rl = orc.linear_logp(h, w, targets, seg, len(coef), *forks, scale=scale)
    rdh, rdw, _ = orc.linear_logp_grad(h, w, targets, seg, coef, *forks, scale=scale)
    e = scale * width * 2.0 ** -23 * (np.abs(h) @ np.abs(w).T)
    z = scale * h @ w.T
    assert np.abs(z).max(initial=0) < 88 and vocab < 25600
    e_lse = e.max(1, initial=0) + 2.0 ** -16 + 2.0 ** -23 * np.abs(rl)
    scored = np.zeros(len(h), bool)
    e_out = 2.0 ** -23 * np.abs(ro)
    for t, y, g in labels:
        scored[t] = True
        e_out[g] += e[t, y] + e_lse[t]
    within("lse", lse, rl, np.where(scored, e_lse, 0) + 1e-300)
    within("out", out, ro, e_out + 1e-12)
    # one row of dz for each label, as the kernels round it
    rows = np.array([t for t, _, _ in labels], dtype=int)
    c = np.array([coef[g] for _, _, g in labels], dtype=np.float64) * scale
    p = np.exp(z[rows] - rl[rows][:, None])
    dz = -c[:, None] * p
    for i, (_, y, _) in enumerate(labels):
        dz[i, y] += c[i]
    e_dz = 1.01 * np.abs(c[:, None]) * p * (e[rows] + e_lse[rows][:, None] + 2.0 ** -16) + 2.0 ** -22 * np.abs(c[:, None]) + H8 * np.abs(dz)
    n = len(labels)
    gather = lambda a: np.stack([a[rows == t].sum(0) for t in range(len(h))]) if len(h) else np.zeros((0, a.shape[1]))  # noqa: E731
    norm = lambda *parts: np.sqrt(sum((q ** 2).sum() for q in parts))  # noqa: E731
    within("d_hidden", dh, rdh, H8 * np.abs(rdh) + gather((e_dz + vocab * 2.0 ** -23 * np.abs(dz)) @ np.abs(w)) + 1e-30,
           H8 * norm(rdh, np.sqrt(dz ** 2 @ w ** 2)) + 1e-30)
    within("d_table", dw, rdw, H8 * np.abs(rdw) + (e_dz + n * 2.0 ** -23 * np.abs(dz)).T @ np.abs(h[rows]) + 1e-30,
           H8 * norm(rdw, np.sqrt((dz ** 2).T @ h[rows] ** 2)) + 1e-30)


# one row, one column of the vocabulary, tile edges, ragged sizes, several tiles each way, split sums of d_hidden
SIZES = [(1, 8, 1), (1, 64, 300), (2, 8, 7), (3, 72, 255), (40, 64, 256), (41, 136, 257), (300, 264, 1000), (427, 256, 513), (700, 1032, 2049),
         (1000, 64, 5003), (129, 2056, 700), (5, 512, 20011)]


@pytest.mark.parametrize("n_rows,width,vocab", SIZES)
def test_against_the_oracle(n_rows, width, vocab):
    args = inputs(n_rows, width, vocab, n_rows + width + vocab, live=1.0 if n_rows < 4 else 0.6)
    for scale in (1.0, 0.3):
        *got, status = both(*args, scale=scale)
        assert status == 0
        compare(*args, scale, got)


def test_sizes_at_random():
    rng = np.random.default_rng(11)
    for i in range(12):
        n_rows, width, vocab = int(rng.integers(1, 900)), 8 * int(rng.integers(1, 70)), int(rng.integers(1, 3000))
        args = inputs(n_rows, width, vocab, i, live=float(rng.uniform(0.05, 1)), n_segments=int(rng.integers(1, 40)), n_forks=int(rng.integers(0, 30)))
        *got, status = both(*args)
        assert status == 0
        compare(*args, 1.0, got)


def test_labels_of_every_kind():
    """Rows without a label, forks on rows with and without one, several forks on a row, labels twice, and labels out of range,
    which are reported and leave the rest as it is."""
    hidden, table, targets, seg, _, coef = inputs(60, 64, 500, 3, live=0.5, n_segments=4)
    seg[10], seg[11], seg[12], seg[13] = 1, -1, -1, 0
    forks = [np.array(a, np.int32) for a in ([10, 11, 11, 12, 10, 10, 59], [5, 6, 7, 499, 5, 5, 0], [0, 1, 1, 3, 2, 2, 3])]
    *got, status = both(hidden, table, targets, seg, forks, coef)
    assert status == 0
    compare(hidden, table, targets, seg, forks, coef, 1.0, got)
    bad_t, bad_s = targets.copy(), seg.copy()
    bad_t[13], bad_s[14] = 500, 4
    bad = [np.append(a, b).astype(np.int32) for a, b in zip(forks, ([20, 21, 60, -1, 22], [-1, 3, 3, 3, 3], [0, 9, 0, 0, -1]))]
    *got, status = both(hidden, table, bad_t, bad_s, bad, coef)
    assert status == B.PSA_DEVSTAT_BAD_TARGET | B.PSA_DEVSTAT_BAD_SEGMENT
    compare(hidden, table, bad_t, bad_s, bad, coef, 1.0, got)


@pytest.mark.parametrize("n_rows,n_segments", [(0, 3), (5, 0), (300, 2), (0, 0)])
def test_nothing_is_scored(n_rows, n_segments):
    hidden, table, targets, seg, _, _ = inputs(n_rows, 72, 300, 1, n_segments=max(n_segments, 1))
    seg[:] = -1
    out, lse, dh, dw, status = both(hidden, table, targets, seg, [np.zeros(0, np.int32)] * 3, np.ones(n_segments, np.float32))
    assert status == 0 and out.shape == (n_segments,) and lse.shape == (n_rows,) and dh.shape == (n_rows, 72)
    assert not out.any() and not lse.any() and not dh.any() and not dw.any()


def test_probabilities_of_one_and_of_none():
    """One token takes all of the probability, or none of it that fp32 could hold."""
    rng = np.random.default_rng(0)
    table = torch.as_tensor(rng.normal(size=(700, 64)), dtype=torch.float32).to(torch.bfloat16)
    hidden = (table[:200] * 2).contiguous()
    targets = np.arange(200, dtype=np.int32)
    seg, none = np.zeros(200, np.int32), [np.zeros(0, np.int32)] * 3
    coef = np.ones(1, np.float32)
    z = 2.0 * f64(table[:200]) @ f64(table).T
    out, lse, dh, dw, _ = both(hidden, table, targets, seg, none, coef)
    ro, rl = orc.linear_logp(f64(hidden), f64(table), targets, seg, 1)
    e = 64 * 2.0 ** -23 * (2 * np.abs(f64(table[:200])) @ np.abs(f64(table)).T).max()
    assert abs(float(out[0]) - ro[0]) <= 200 * (2 * e + 2.0 ** -16) and ro[0] > -1e-3 and z.max() > 88
    assert np.abs(f64(lse) - rl).max() <= e + 2.0 ** -16 + 2.0 ** -23 * np.abs(rl).max()
    away = (targets + 300).astype(np.int32)
    out, *_ = both(hidden, table, away, seg, none, coef)
    ro, _ = orc.linear_logp(f64(hidden), f64(table), away, seg, 1)
    assert abs(float(out[0]) - ro[0]) <= 200 * (2 * e + 2.0 ** -16) + 2.0 ** -23 * abs(ro[0]) and ro[0] < -200 * 88


def test_rows_that_are_not_finite_stay_alone():
    hidden, table, targets, seg, forks, coef = inputs(300, 128, 700, 5, live=1.0, n_segments=2, n_forks=0)
    seg[:] = 0
    seg[7], seg[100] = 1, -1
    clean = both(hidden, table, targets, seg, forks, coef)
    dirty = hidden.clone()
    dirty[7, 3], dirty[100] = float("nan"), float("nan")
    got = both(dirty, table, targets, seg, forks, coef)
    rest = [i for i in range(300) if i != 7]
    assert torch.equal(got[0][:1], clean[0][:1]) and got[0][1].isnan() and got[1][7].isnan()
    assert torch.equal(got[1][rest], clean[1][rest]) and torch.equal(got[2][rest], clean[2][rest]) and got[2][7].isnan().all()
    infinite = hidden.clone()
    infinite[7, 3] = float("inf")
    got = both(infinite, table, targets, seg, forks, coef)
    assert got[0][1].isnan() and torch.equal(got[2][rest], clean[2][rest])


def test_the_same_inputs_give_the_same_bits_whatever_the_buffers_held():
    args = inputs(900, 264, 3001, 8, n_forks=40)
    first = both(*args)
    n, d, v, forks = 900, 264, 3001, 40
    need = max(B.load_library().dpo_linear_logp_workspace_bytes(n, forks, 5, v, d, b) for b in (0, 1))
    for fill in (0, 255, 127):
        ws = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
        again = both(*args, workspace=ws[:need])
        assert all(torch.equal(a, b) for a, b in zip(first[:4], again[:4]))
        assert bool((ws[need:] == fill).all())


def test_a_table_that_is_not_trained():
    args = inputs(200, 64, 900, 4)
    _, lse, dh, _, _ = both(*args)
    hidden, table, targets, seg, forks, coef = args
    got, none = O.dpo_linear_logp_bwd(dev(coef), hidden.cuda(), table.cuda(), lse, i32(targets), i32(seg), *[i32(f) for f in forks],
                                      with_table=False)
    assert none is None and torch.equal(got, dh)


def test_pieces_of_the_vocabulary():
    """More labels times tokens than one piece holds: 16100 rows, three pieces of 70001 tokens, the last of them ragged."""
    hidden, table, targets, seg, forks, coef = inputs(16100, 64, 70001, 9, live=0.4, n_segments=6, n_forks=20)
    out, lse, dh, dw, status = both(hidden, table, targets, seg, forks, coef)
    assert status == 0
    rows = dev(np.concatenate([np.flatnonzero(seg >= 0), forks[0]]).astype(np.int64))
    y = dev(np.concatenate([targets[seg >= 0], forks[1]]).astype(np.int64))
    g = dev(np.concatenate([seg[seg >= 0], forks[2]]).astype(np.int64))
    h, w = hidden.cuda().double(), table.cuda().double()
    ro, rl = torch.zeros(6, dtype=torch.float64, device="cuda"), torch.zeros(16100, dtype=torch.float64, device="cuda")
    rdh, rdw = torch.zeros_like(h), torch.zeros_like(w)
    for part in torch.arange(len(rows), device="cuda").split(2000):
        t, at = rows[part], torch.arange(len(part), device="cuda")
        z = h[t] @ w.t()
        l = torch.logsumexp(z, 1)
        rl[t] = l
        ro.index_add_(0, g[part], z[at, y[part]] - l)
        c = dev(coef).double()[g[part]]
        dz = torch.exp_(z - l[:, None]).mul_(-c[:, None])
        dz[at, y[part]] += c
        rdh.index_add_(0, t, dz @ w)
        rdw += dz.t() @ h[t]
    far = lambda a, b: ((a.double() - b).norm() / b.norm()).item()  # noqa: E731
    # (2-norms: a rounding to bf16 of dz and one of the result, 2^-8 / sqrt(3) each at most, with dz's error no larger than its share)
    assert far(out, ro) <= 1e-5 and far(lse, rl) <= 1e-6 and far(dh, rdh) <= 4.5e-3 and far(dw, rdw) <= 4.5e-3, (far(dh, rdh), far(dw, rdw))


def test_logits_of_minus_infinity_are_probabilities_of_none():
    """Table rows of -inf against hidden rows without a zero or a negative value: what the other tokens' probabilities are."""
    rng = np.random.default_rng(2)
    bf = lambda a: torch.as_tensor(a, dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    hidden, table = bf(rng.uniform(0.5, 1, size=(70, 64))), bf(rng.normal(size=(600, 64)))
    banned = [0, 5, 255, 256, 599] + list(range(300, 400))
    full = table.clone()
    full[banned] = float("-inf")
    rest = [v for v in range(600) if v not in banned]
    targets = np.array([rest[i % len(rest)] for i in range(70)], dtype=np.int32)
    targets[69] = 5
    seg = np.zeros(70, np.int32)
    seg[69] = 1
    out, lse = O.dpo_linear_logp(hidden.cuda(), full.cuda(), i32(targets), i32(seg), 2)
    where = {v: i for i, v in enumerate(rest)}
    ro, rl = orc.linear_logp(f64(hidden)[:69], f64(table)[rest], [where[v] for v in targets[:69]], np.zeros(69, int), 1)
    e = 64 * 2.0 ** -23 * (np.abs(f64(hidden)) @ np.abs(f64(table)).T).max() + 2.0 ** -16 + 2.0 ** -23 * np.abs(rl).max()
    assert np.abs(f64(lse)[:69] - rl).max() <= e and np.isfinite(f64(lse)).all()
    assert abs(float(out[0]) - ro[0]) <= 69 * 2 * e + 2.0 ** -23 * abs(ro[0]) and float(out[1]) == float("-inf")
