"""psa_block_norm and psa_block_norm_bwd against the oracle in 64 bits.

Tolerances, from the arithmetic: an output is rounded once, by at most half a step (eps / 2 of its type, relative).  Before
that, everything is fp32.  A sum over a row adds at most 32 terms in a thread and then 10 levels of a tree: 42 roundings of 2^-24, so
a mean is off by 2^-18 of the row's largest magnitude A at most, a deviation by 2^-18 relative, and u = (s - m) r by
E = 2^-18 (A + |m|) r + 2^-18 |u|.  What follows is carried through the formulas: the sum before its rounding, the second norm from
the sum that the kernel has written, ds, q and dx.  A sum over tokens adds at most T / 148 + 60 terms one after the other."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O

pytestmark = pytest.mark.gpu

P18, P22 = 2.0 ** -18, 2.0 ** -22
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.bfloat16, torch.float32), "f32": (torch.float32, torch.float32)}
f64 = lambda t: None if t is None else t.detach().cpu().double().numpy()  # noqa: E731
half = lambda t: torch.finfo(t).eps / 2  # noqa: E731


def normal(shape, seed, dtype, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def within(name, got, ref, tol):
    got = f64(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    worst = (np.abs(got - ref) / np.maximum(tol, 1e-300)).max() if ref.size else 0.0
    print("%s: %.3f of its tolerance" % (name, worst))
    assert worst <= 1, (name, worst)


def u_error(s, mean, rstd):
    big = np.abs(s).max(axis=1, keepdims=True, initial=0) + np.abs(mean)[:, None]
    return P18 * (big * rstd[:, None] + np.abs(s - mean[:, None]) * rstd[:, None])


def parameters(D, kind, rms, post, gate, seed):
    wt = TYPES[kind][1]
    p = {"weight": normal((D,), seed + 1, wt, 1.0, 0.3), "bias": None if rms else normal((D,), seed + 2, wt)}
    p["post_weight"] = normal((D,), seed + 3, wt, 1.0, 0.3) if post else None
    p["post_bias"] = normal((D,), seed + 4, wt) if post and not rms else None
    p["gate"] = normal((D,), seed + 5, wt, 0.3, 0.5) if gate else None
    return p


def stage_error(r, g, e_g, u, E, rms):
    """Error of r (g - u mean(g u) - mean(g)) in fp32 for g off by e_g and u by E."""
    mean = lambda a: a.mean(1, keepdims=True)  # noqa: E731
    a, one = np.abs(g), 0 if rms else 1
    fp32 = 2 * P18 * (a + np.abs(u) * mean(a * np.abs(u)) + one * mean(a)) + E * mean(a * np.abs(u)) + np.abs(u) * mean(a * E)
    return r[:, None] * (fp32 + 1.01 * (e_g + np.abs(u) * mean(e_g * np.abs(u)) + one * mean(e_g)))


def check(T, D, kind, rms, post, gate, scale=1.0, with_total=True, mean=0.0, seed=0):
    xt, wt = TYPES[kind]
    x, res = normal((T, D), seed, xt, mean), normal((T, D), seed + 6, xt, mean, 2.0)
    d_out, d_total = normal((T, D), seed + 7, xt), normal((T, D), seed + 8, xt) if with_total else None
    p = parameters(D, kind, rms, post, gate, seed)
    out, total, stats = O.psa_block_norm(x, res, eps=1e-5, rms=rms, residual_scale=scale, **p)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    around = {k: v for k, v in p.items() if k != "bias"}
    grads = O.psa_block_norm_bwd(d_out, x, total, stats=stats, rms=rms, residual_scale=scale, d_total=d_total, with_bias=not rms, status=status,
                                 **around)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    n = {k: f64(v) for k, v in p.items()}
    fx, fr, one = f64(x), f64(res), np.ones(D)
    _, r_total, r_stats = orc.block_norm_fwd(fx, fr, residual_scale=np.float32(scale), rms=rms, **n)
    pw, pb, gt = (one if n["post_weight"] is None else n["post_weight"]), (0 if n["post_bias"] is None else n["post_bias"]), \
        (one if n["gate"] is None else n["gate"])
    m1, r1 = r_stats[0], r_stats[1]
    u1 = (fx - m1[:, None]) * r1[:, None]
    E1 = u_error(fx, m1, r1) if post else np.zeros_like(fx)
    y = u1 * pw + pb
    e_total = np.abs(gt) * (E1 * np.abs(pw) + P22 * np.abs(u1 * pw) + P22 * np.abs(y)) + P22 * (np.abs(fr * scale) + np.abs(y * gt))
    within("total", total, r_total, half(xt) * np.abs(r_total) + 1.01 * e_total)
    # from here on from what was written
    s = f64(total)
    ref, m2, r2 = orc.norm_fwd(s, n["weight"], n["bias"], 1e-5, rms)
    E2 = u_error(s, m2, r2)
    within("out", out, ref, half(xt) * np.abs(ref) + E2 * np.abs(n["weight"]) + P22 * np.abs(ref) + (0 if rms else P22 * np.abs(n["bias"])))
    got = f64(stats)
    for k, (m, r, v) in enumerate(((m1, r1, fx), (m2, r2, s))):
        if k == 0 and not post:
            assert (got[0] == 0).all() and (got[1] == 1).all()
            continue
        top = np.abs(v).max(axis=1, initial=0)
        within("mean %d" % k, stats[2 * k], m, P18 * top + 1e-30)
        within("rstd %d" % k, stats[2 * k + 1], r, P18 * (1 + (np.abs(m) + top) * r * 2.0 ** -6) * r)
    g = orc.block_norm_bwd(f64(d_out), fx, s, n["weight"], n["post_weight"], n["post_bias"], n["gate"], np.float32(scale), 1e-5, rms, f64(d_total))
    u2, w = (s - m2[:, None]) * r2[:, None], n["weight"]
    e_ds = stage_error(r2, f64(d_out) * w, P22 * np.abs(f64(d_out) * w), u2, E2, rms) + (P22 * np.abs(f64(d_total)) if with_total else 0)
    ds = orc.norm_bwd(f64(d_out), s, w, 1e-5, rms)[0] + (f64(d_total) if with_total else 0)
    dx, d_res, dw, db, dpw, dpb, dgate = grads
    within("d_residual", d_res, g["residual"], half(xt) * np.abs(g["residual"]) + scale * (e_ds + P22 * np.abs(ds)))
    q = ds * gt * pw
    e_q = np.abs(gt * pw) * (e_ds + 2 * P22 * np.abs(ds))
    within("dx", dx, g["x"], half(xt) * np.abs(g["x"]) + (stage_error(r1, q, e_q, u1, E1, rms) if post else e_q))
    adds = (T / 148 + 60) * 2.0 ** -24
    done = lambda ref: half(wt) * np.abs(ref) + P22 * np.abs(ref)  # noqa: E731
    within("d_weight", dw, g["weight"], done(g["weight"]) + adds * np.abs(f64(d_out) * u2).sum(0) + (np.abs(f64(d_out)) * E2).sum(0))
    e_a = adds * np.abs(ds * u1).sum(0) + (e_ds * (np.abs(u1) + E1) + np.abs(ds) * E1).sum(0)
    e_c = adds * np.abs(ds).sum(0) + e_ds.sum(0)
    if rms:
        assert db is None and dpb is None
    else:
        within("d_bias", db, g["bias"], done(g["bias"]) + adds * np.abs(f64(d_out)).sum(0))
    if post:
        within("d_post_weight", dpw, g["post_weight"], done(g["post_weight"]) + np.abs(gt) * e_a + P22 * np.abs(g["post_weight"]))
        if not rms:
            within("d_post_bias", dpb, g["post_bias"], done(g["post_bias"]) + np.abs(gt) * e_c)
    else:
        assert dpw is None and dpb is None
    if gate:
        within("d_gate", dgate, g["gate"], done(g["gate"]) + np.abs(pw) * (e_a + P22 * np.abs((ds * u1).sum(0))) + np.abs(pb) * (e_c + P22 * np.abs(ds.sum(0))))
    else:
        assert dgate is None


FORMS = [(rms, post, gate) for rms in (False, True) for post, gate in ((True, False), (False, True), (True, True), (False, False))]


@pytest.mark.parametrize("rms,post,gate", FORMS)
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,D", [(1, 4096), (3, 1), (9, 7), (17, 64), (40, 127), (33, 129), (12, 256), (21, 520), (31, 1024), (300, 1237),
                                 (11, 2048), (13, 4096), (5, 4097), (170, 1000)])
def test_forward_and_backward(T, D, kind, rms, post, gate):
    check(T, D, kind, rms, post, gate, scale=1.0 if T % 2 else 0.7, with_total=T % 3 != 0, seed=T + D)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,D", [(4, 8192), (5, 8193), (3, 16384), (2, 16383), (9, 12000), (700, 96), (5000, 64), (20000, 24), (1300, 2047)])
def test_wide_and_many_rows(T, D, kind):
    check(T, D, kind, rms=T % 2 == 0, post=True, gate=D % 2 == 0, scale=0.5, seed=D)


@pytest.mark.parametrize("D", [256, 1000, 4096])
def test_rows_far_from_zero(D):
    check(50, D, "f32", False, True, True, mean=1000.0)


def test_no_tokens():
    p = parameters(40, "mixed", False, True, True, 0)
    x = torch.zeros((0, 40), dtype=torch.bfloat16, device="cuda")
    out, total, stats = O.psa_block_norm(x, x, **p)
    p.pop("bias")
    dx, dr, *dp = O.psa_block_norm_bwd(x, x, x, stats=stats, with_bias=True, **p)
    torch.cuda.synchronize()
    assert out.shape == total.shape == dx.shape == dr.shape == (0, 40) and stats.shape == (4, 0)
    assert len(dp) == 5 and not any(d.any() for d in dp)


@pytest.mark.parametrize("D", [129, 1237, 4096])
def test_in_place_and_rows_beyond_the_last(D):
    T, more = 201, 240
    p = parameters(D, "bf16", False, True, True, 3)
    x, res, d_out, d_total = (normal((more, D), k, torch.bfloat16) for k in range(4))
    want = O.psa_block_norm(x[:T].clone(), res[:T].clone(), **p)
    a, b = x.clone(), res.clone()
    a[T:], b[T:] = float("nan"), float("nan")
    out, total, stats = O.psa_block_norm(a[:T], b[:T], out=a[:T], total=b[:T], **p)
    assert all(torch.equal(u, v) for u, v in zip((out, total, stats), want))
    assert a[T:].isnan().all() and b[T:].isnan().all()
    p.pop("bias")
    grads = O.psa_block_norm_bwd(d_out[:T].clone(), x[:T].clone(), total.clone(), stats=stats, d_total=d_total[:T].clone(), **p)
    for places in (("d_out", "total"), ("x", "d_total"), ("total", "d_out"), ("d_total", "total")):
        t = {"d_out": d_out[:T].clone(), "x": x[:T].clone(), "total": total.clone(), "d_total": d_total[:T].clone()}
        again = O.psa_block_norm_bwd(**t, stats=stats, dx=t[places[0]], d_residual=t[places[1]], **p)
        torch.cuda.synchronize()
        assert again[0] is t[places[0]] and all(u is v is None or torch.equal(u, v) for u, v in zip(again, grads)), places


def test_in_place_of_wide_rows():
    p = parameters(12000, "bf16", True, True, False, 3)
    x, res, d_out, d_total = (normal((7, 12000), k, torch.bfloat16) for k in range(4))
    _, total, stats = O.psa_block_norm(x, res, rms=True, **p)
    p.pop("bias")
    grads = O.psa_block_norm_bwd(d_out.clone(), x.clone(), total.clone(), stats=stats, d_total=d_total.clone(), rms=True, **p)
    for places in (("d_out", "total"), ("x", "d_total"), ("total", "d_out"), ("d_total", "total")):
        t = {"d_out": d_out.clone(), "x": x.clone(), "total": total.clone(), "d_total": d_total.clone()}
        again = O.psa_block_norm_bwd(**t, stats=stats, rms=True, dx=t[places[0]], d_residual=t[places[1]], **p)
        assert all(u is v is None or torch.equal(u, v) for u, v in zip(again, grads)), places


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [96, 1237, 4096])
def test_rows_that_are_not_finite_stay_alone(D, bad):
    p = parameters(D, "bf16", False, True, True, 9)
    x, res = normal((60, D), 0, torch.bfloat16), normal((60, D), 1, torch.bfloat16)
    clean = O.psa_block_norm(x, res, **p)
    y = x.clone()
    y[31, D // 2] = bad
    got = O.psa_block_norm(y, res, **p)
    rest = [i for i in range(60) if i != 31]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(got[:2], clean[:2])) and got[0][31].isnan().all()
    p.pop("bias")
    a = O.psa_block_norm_bwd(res, x, clean[1], stats=clean[2], **p)
    b = O.psa_block_norm_bwd(res, y, got[1], stats=got[2], **p)
    assert all(torch.equal(u[rest], v[rest]) for u, v in zip(a[:2], b[:2])) and b[0][31].isnan().all()


def test_the_same_inputs_give_the_same_bits():
    for T, D in ((3000, 1237), (2000, 4096), (9000, 100)):
        p = parameters(D, "mixed", False, True, True, 9)
        x, res, g = (normal((T, D), k, torch.bfloat16) for k in range(3))
        _, total, stats = O.psa_block_norm(x, res, **p)
        q = {k: v for k, v in p.items() if k != "bias"}
        first = O.psa_block_norm_bwd(g, x, total, stats=stats, d_total=res, with_bias=True, **q)
        need = B.load_library().psa_block_norm_bwd_workspace_bytes(T, D)
        ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
        again = O.psa_block_norm_bwd(g, x, total, stats=stats, d_total=res, with_bias=True, workspace=ws[:need], **q)
        assert all(torch.equal(a, b) for a, b in zip(first, again)) and bool((ws[need:] == 255).all())


def test_without_a_norm_or_a_gate_it_is_psa_norm():
    x, res, g, dt = (normal((130, 520), k, torch.bfloat16) for k in range(4))
    w, b = normal((520,), 5, torch.bfloat16, 1.0), normal((520,), 6, torch.bfloat16)
    out, total, stats = O.psa_block_norm(x, res, w, bias=b)
    want = B.psa_norm(x, w, b, residual=res)
    assert torch.equal(total, want[2]) and (out.float() - want[0].float()).abs().max() <= 2.0 ** -6
    dx, dr, dw, db, *none = O.psa_block_norm_bwd(g, x, total, w, stats, d_total=dt, with_bias=True)
    wx, ww, wb = B.psa_norm_bwd(g, want[2], w, want[1], d_total=dt, with_bias=True)
    assert torch.equal(dx, dr) and (dx.float() - wx.float()).abs().max() <= 2.0 ** -5 and none == [None] * 3
