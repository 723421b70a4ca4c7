"""psa_norm and psa_norm_bwd against the oracle in 64 bits.

Tolerances, from the arithmetic: an output is rounded once, by at most half a step (eps / 2 of its type, relative).  Before
that, everything is fp32.  A sum over a row adds at most 32 terms in a thread and then 10 levels of a tree: 42 roundings of
2^-24, so the mean is off by 2^-18 of the row's largest magnitude A at most, the deviation by 2^-18 relative, and
u = (s - m) r by E = 2^-18 (A + |m|) r + 2^-18 |u|.  A sum over tokens adds at most T / 148 + 2 * 148 / 16 + 16 terms one after the
other."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

P18 = 2.0 ** -18
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.bfloat16, torch.float32), "f32": (torch.float32, torch.float32)}
f64 = lambda t: t if isinstance(t, np.ndarray) else t.detach().cpu().double().numpy()  # noqa: E731
half = lambda t: torch.finfo(t).eps / 2  # noqa: E731


def normal(shape, seed, dtype, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype)


def within(name, got, ref, tol):
    got = f64(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    worst = (np.abs(got - ref) / np.maximum(tol, 1e-300)).max() if ref.size else 0.0
    print("%s: %.3f of its tolerance" % (name, worst))
    assert worst <= 1, (name, worst)


def u_error(s, mean, rstd):
    big = np.abs(s).max(axis=1, keepdims=True) + np.abs(mean)[:, None]
    return P18 * (big * rstd[:, None] + np.abs(s - mean[:, None]) * rstd[:, None])


def check(T, D, kind, rms, residual, mean=0.0, seed=0):
    xt, wt = TYPES[kind]
    x, w = normal((T, D), seed, xt, mean), normal((D,), seed + 1, wt, 1.0, 0.3)
    b = None if rms else normal((D,), seed + 2, wt)
    res = normal((T, D), seed + 3, xt, mean, 2.0) if residual else None
    d_out, d_total = normal((T, D), seed + 4, xt), normal((T, D), seed + 5, xt) if residual else None
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    outs = B.psa_norm(dev(x), dev(w), dev(b), eps=1e-5, rms=rms, residual=dev(res))
    total = (x.float() + res.float()).to(xt) if residual else x
    if residual:
        assert torch.equal(outs[2].cpu(), total)      # one fp32 addition, rounded once
    dx, dw, db = B.psa_norm_bwd(dev(d_out), outs[2] if residual else dev(x), dev(w), outs[1], rms=rms, d_total=dev(d_total),
                                with_bias=not rms)
    torch.cuda.synchronize()
    s, ww, bb, g = f64(total), f64(w), None if rms else f64(b), f64(d_out)
    ref, m, r = orc.norm_fwd(s, ww, bb, 1e-5, rms)
    E = u_error(s, m, r)
    within("out", outs[0], ref, half(xt) * np.abs(ref) + E * np.abs(ww) + 2.0 ** -22 * np.abs(ref) + (0 if rms else 2.0 ** -22 * np.abs(bb)))
    stats = f64(outs[1])
    within("mean", stats[0], m, P18 * np.abs(s).max(axis=1)) if not rms else None
    within("rstd", stats[1], r, P18 * (1 + (np.abs(m) + np.abs(s).max(axis=1)) * r * 2.0 ** -6) * r)
    rdx, rdw, rdb = orc.norm_bwd(g, s, ww, 1e-5, rms)
    if d_total is not None:
        rdx = rdx + f64(d_total)
    u = (s - m[:, None]) * r[:, None]
    gw = np.abs(g * ww)
    gu, g1 = (gw * np.abs(u)).mean(1, keepdims=True), 0 if rms else gw.mean(1, keepdims=True)
    ge = (gw * E).mean(1, keepdims=True)
    fp32 = r[:, None] * (2 * P18 * (gw + np.abs(u) * gu + g1) + E * gu + np.abs(u) * ge)
    within("dx", dx, rdx, half(xt) * np.abs(rdx) + fp32 + (0 if d_total is None else 2.0 ** -22 * np.abs(f64(d_total))))
    adds = (T / 148 + 60) * 2.0 ** -24
    within("dweight", dw, rdw, half(wt) * np.abs(rdw) + adds * (np.abs(g * u)).sum(0) + (np.abs(g) * E).sum(0))
    if not rms:
        within("dbias", db, rdb, half(wt) * np.abs(rdb) + adds * np.abs(g).sum(0))
    else:
        assert db is None


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,D", [(1, 4096), (3, 1), (5, 2), (9, 7), (17, 64), (40, 127), (8, 128), (33, 129), (12, 256), (21, 520),
                                 (31, 1024), (7, 1032), (300, 1237), (11, 2048), (13, 4096), (5, 4097), (4, 8192), (3, 16384),
                                 (2, 16383), (700, 96)])
def test_forward_and_backward(T, D, kind, rms):
    check(T, D, kind, rms, residual=(T + D) % 2 == 0, seed=T + D)


@pytest.mark.parametrize("D", [256, 1000, 4096])
def test_rows_far_from_zero(D):
    check(50, D, "f32", False, True, mean=1000.0)


def test_many_rows_take_every_loop():
    check(3001, 640, "bf16", False, True)
    check(2500, 72, "mixed", True, True)


def test_no_tokens():
    x, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    out, stats = B.psa_norm(x, w, w)
    dx, dw, db = B.psa_norm_bwd(x, x, w, stats, with_bias=True, dweight=torch.full_like(w, 7.0), dbias=torch.full_like(w, 7.0))
    assert out.shape == dx.shape == (0, 64) and not dw.any() and not db.any()


def test_a_bad_row_stays_alone_and_constant_rows_are_finite():
    x = normal((6, 200), 3, torch.bfloat16).cuda()
    w = torch.ones(200, dtype=torch.bfloat16, device="cuda")
    clean, stats = B.psa_norm(x, w)
    y = x.clone()
    y[1, 5], y[3, 7] = float("nan"), float("inf")
    out, _ = B.psa_norm(y, w)
    rows = [0, 2, 4, 5]
    assert torch.equal(out[rows], clean[rows]) and out[1].isnan().all() and out[3].isnan().any()
    flat = torch.full((2, 200), 3.0, dtype=torch.bfloat16, device="cuda")
    out, stats = B.psa_norm(flat, w)
    dx, _, _ = B.psa_norm_bwd(flat, flat, w, stats)
    assert not out.any() and torch.isfinite(dx).all()


def test_in_place_results_are_the_same():
    x, r, w = (normal(s, i, torch.bfloat16).cuda() for i, s in enumerate(((70, 512), (70, 512), (512,))))
    out, stats, total = B.psa_norm(x, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    out2, stats2, total2 = B.psa_norm(x2, w, residual=r2, out=x2, total=r2)
    assert torch.equal(out, out2) and torch.equal(total, total2) and torch.equal(stats, stats2)
    dx, dw, _ = B.psa_norm_bwd(x, total, w, stats, d_total=r)
    g = x.clone()
    dx2, dw2, _ = B.psa_norm_bwd(g, total, w, stats, d_total=r, dx=g)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_the_same_bits_again_on_another_stream_and_in_a_graph():
    x, w = normal((900, 768), 1, torch.bfloat16).cuda(), normal((768,), 2, torch.bfloat16).cuda()
    g = normal((900, 768), 3, torch.bfloat16).cuda()

    def both(**kw):
        out, stats = B.psa_norm(x, w, w, **kw)
        return (out, stats) + B.psa_norm_bwd(g, x, w, stats, with_bias=True, **kw)
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    x.mul_(2)
    want = both()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, captured))


def test_rows_behind_the_last_token_are_left_as_they_were():
    x, w = normal((64, 130), 1, torch.float32).cuda(), torch.ones(130, device="cuda")
    out, dx = torch.full((64, 130), 5.0, device="cuda"), torch.full((64, 130), 5.0, device="cuda")
    _, stats = B.psa_norm(x[:37], w, out=out[:37])
    B.psa_norm_bwd(x[:37], x[:37], w, stats, dx=dx[:37])
    torch.cuda.synchronize()
    assert (out[37:] == 5).all() and (dx[37:] == 5).all()
