"""psa_ffn and psa_ffn_bwd.

Whole numbers first: with G = 64 in every element the sigmoid is 1 to the last bit, silu(G) = 64, and with small whole numbers
elsewhere every product is exact and every sum below 2^24, so each output is the exact value rounded to bf16 and has to be
equal bit by bit, whatever the order of the sums: an index or a stage that is wrong cannot hide in a tolerance.

Then N(0, 1) inputs against the oracle in 64 bits.  What is rounded to bf16 on the way (G and U for the backward, H, dG, dU) is
off by at most 2^-8 relative, every sum of n products by n 2^-24 of the sum of their magnitudes; the bounds below follow these
through the formulas.  They are bounds of the worst case, in which errors add up; that they do not is held in the 2-norm: a
product's error from independent roundings of its terms is 2^-8 of the root of the sum of the terms' squares, or less."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

H8 = 2.0 ** -8
f64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
bf16 = lambda a: torch.as_tensor(a).to(torch.bfloat16)  # noqa: E731
rounded = lambda a: f64(bf16(torch.as_tensor(a, dtype=torch.float32)))  # noqa: E731

# A few tokens, one tile and less, tile edges, several tiles, split sums, and sizes beyond the rule for the large tiles.
SIZES = [(1, 8, 8), (1, 64, 128), (2, 72, 200), (31, 128, 64), (64, 136, 520), (127, 64, 64), (128, 128, 128), (129, 200, 72),
         (300, 264, 392), (1, 2048, 4096), (3, 1032, 264), (4, 2056, 520), (5, 4096, 1032), (130, 1024, 2048), (1000, 512, 1024), (2300, 64, 128), (2048, 1024, 2056),
         (1803, 1544, 2816), (2900, 1800, 520)]


def whole_numbers(T, D, F, seed):
    rng = np.random.default_rng(seed)
    some = lambda shape, share: (rng.integers(-1, 2, size=shape) * (rng.random(shape) < share)).astype(np.float32)  # noqa: E731
    x = some((T, D), 0.5)
    x[:, 0] = 1
    wg = np.zeros((D, F), np.float32)
    wg[0] = 64
    return x, wg, some((D, F), min(0.5, 40 / D)), some((F, D), min(0.5, 200 / F)), some((T, D), min(0.5, 300 / D))


@pytest.mark.parametrize("T,D,F", SIZES)
def test_whole_numbers_are_exact(T, D, F):
    x, wg, wu, wd, g = whole_numbers(T, D, F, T + D + F)
    dev = [bf16(a).cuda() for a in (x, wg, wu, wd)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, saved = B.psa_ffn(*dev, status=status)
    bare, none = B.psa_ffn(*dev, save=False, status=status)
    grads = B.psa_ffn_bwd(bf16(g).cuda(), *dev, saved, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and none is None and torch.equal(out, bare)
    x, wg, wu, wd, g = (torch.as_tensor(a).cuda().double() for a in (x, wg, wu, wd, g))
    r = lambda a: a.float().to(torch.bfloat16)  # noqa: E731
    up = x @ wu
    h = 64 * up
    dh = g @ wd.t()
    d_gate, d_up = r(dh * up).double(), r(dh * 64).double()
    assert up.abs().max() <= 256 and (h.abs() @ wd.abs()).max() < 2 ** 24
    assert (d_gate.abs() @ wg.abs().t() + d_up.abs() @ wu.abs().t()).max() < 2 ** 24
    assert (x.abs().t() @ d_gate.abs()).max() < 2 ** 24 and (x.abs().t() @ d_up.abs()).max() < 2 ** 24 and (h.abs().t() @ g.abs()).max() < 2 ** 24
    for name, got, want in (("gate", saved[0], torch.full_like(h, 64)), ("up", saved[1], up), ("out", out, h @ wd),
                            ("dx", grads[0], d_gate @ wg.t() + d_up @ wu.t()), ("dw_gate", grads[1], x.t() @ d_gate),
                            ("dw_up", grads[2], x.t() @ d_up), ("dw_down", grads[3], h.t() @ g)):
        assert torch.equal(got, r(want)), (name, (got.double() - want).abs().max().item())


def within(name, got, ref, tol, norm):
    err = np.abs(f64(got) - ref)
    assert np.isfinite(err).all()
    worst, share = float((err / np.maximum(tol, 1e-300)).max()), float(np.linalg.norm(err) / norm)
    print("%s: %.3f of the bound, %.3f of the norm" % (name, worst, share))
    assert worst <= 1 and share <= 1, (name, worst, share)


@pytest.mark.parametrize("T,D,F", [(1, 64, 128), (37, 200, 136), (150, 256, 696), (260, 520, 1032), (1100, 512, 1288)])
def test_against_the_oracle(T, D, F):
    rng = np.random.default_rng(T)
    x, g = rounded(rng.normal(size=(T, D))), rounded(rng.normal(size=(T, D)))
    wg, wu, wd = (rounded(rng.normal(size=s) * s[0] ** -0.5) for s in ((D, F), (D, F), (F, D)))
    dev = [bf16(a).cuda() for a in (x, wg, wu, wd)]
    out, saved = B.psa_ffn(*dev)
    grads = B.psa_ffn_bwd(bf16(g).cuda(), *dev, saved)
    torch.cuda.synchronize()
    ro, gate, up, h = orc.ffn_fwd(x, wg, wu, wd)
    rdx, rdwg, rdwu, rdwd = orc.ffn_bwd(g, x, wg, wu, wd)
    eps = 2.0 ** -24
    s = 1 / (1 + np.exp(-gate))
    act, slope = gate * s, s * (1 + gate * (1 - s))          # silu and its derivative, at most 1.1 in magnitude
    sums = lambda a, b: np.abs(a) @ np.abs(b)  # noqa: E731
    e_gate, e_up = (D + 8) * eps * sums(x, wg), (D + 8) * eps * sums(x, wu)      # before rounding
    e_h = 1.1 * e_gate * np.abs(up) + np.abs(act) * e_up + 2.0 ** -20 * np.abs(h) + H8 * np.abs(h)
    norm = lambda *parts: np.sqrt(sum((p ** 2).sum() for p in parts))  # noqa: E731
    root = lambda a, b: np.sqrt((a ** 2) @ (b ** 2))  # noqa: E731
    within("out", out, ro, H8 * np.abs(ro) + e_h @ np.abs(wd) + F * eps * sums(h, wd), H8 * norm(ro, root(h, wd)))
    within("gate", saved[0], gate, H8 * np.abs(gate) + 1.01 * e_gate, H8 * norm(gate))
    within("up", saved[1], up, H8 * np.abs(up) + 1.01 * e_up, H8 * norm(up))
    # from here on with G and U as they were kept: off by r_gate, r_up (the second derivative of silu is 0.5 at most)
    r_gate, r_up = H8 * np.abs(gate) + 1.01 * e_gate, H8 * np.abs(up) + 1.01 * e_up
    dh = g @ wd.T
    e_dh = (D + 8) * eps * sums(g, wd.T)
    d_up, d_gate = dh * act, dh * up * slope
    tiny = 2.0 ** -20
    e_du = (H8 + tiny) * np.abs(d_up) + 1.02 * (e_dh * (np.abs(act) + 1.1 * r_gate) + np.abs(dh) * 1.1 * r_gate)
    e_dg = (H8 + tiny) * np.abs(d_gate) + 1.02 * (1.1 * e_dh * (np.abs(up) + r_up) + np.abs(dh) * (1.1 * r_up + 0.5 * np.abs(up) * r_gate))
    e_h2 = (H8 + tiny) * np.abs(h) + 1.02 * (1.1 * r_gate * (np.abs(up) + r_up) + np.abs(act) * r_up)
    # an element of dU, dG or H is off by three roundings, of G, of U and its own, each independent of the others
    v_du = np.sqrt(d_up ** 2 + (dh * slope * gate) ** 2)
    v_dg = np.sqrt(2 * d_gate ** 2 + (dh * up * 0.5 * gate) ** 2)
    v_h = np.sqrt(2 * h ** 2 + (slope * gate * up) ** 2)
    within("dx", grads[0], rdx, H8 * np.abs(rdx) + e_dg @ np.abs(wg.T) + e_du @ np.abs(wu.T) + 2 * F * eps * (sums(d_gate, wg.T) + sums(d_up, wu.T)),
           H8 * norm(rdx, root(v_dg, wg.T), root(v_du, wu.T)))
    within("dw_gate", grads[1], rdwg, H8 * np.abs(rdwg) + np.abs(x.T) @ e_dg + T * eps * sums(x.T, d_gate), H8 * norm(rdwg, root(x.T, v_dg)))
    within("dw_up", grads[2], rdwu, H8 * np.abs(rdwu) + np.abs(x.T) @ e_du + T * eps * sums(x.T, d_up), H8 * norm(rdwu, root(x.T, v_du)))
    within("dw_down", grads[3], rdwd, H8 * np.abs(rdwd) + e_h2.T @ np.abs(g) + T * eps * sums(h.T, g), H8 * norm(rdwd, root(v_h.T, g)))


def small(T=200, D=128, F=264, seed=0):
    gen = torch.Generator().manual_seed(seed)
    make = lambda *s: (torch.randn(s, generator=gen) * s[0] ** -0.5).to(torch.bfloat16).cuda()  # noqa: E731
    return torch.randn((T, D), generator=gen).to(torch.bfloat16).cuda(), make(D, F), make(D, F), make(F, D)


def test_no_tokens():
    x, *w = small(T=0)
    out, saved = B.psa_ffn(x, *w)
    dx, *dw = B.psa_ffn_bwd(x, x, *w, saved, dw_up=torch.full_like(w[1], 3.0))
    assert out.shape == dx.shape == (0, 128) and not any(d.any() for d in dw)


def test_saturated_gates_and_a_bad_row():
    x, wg, wu, wd = small()
    big, _ = B.psa_ffn(x * 512, wg, wu, wd)                    # gates of some hundreds, of either sign
    ref = orc.ffn_fwd(f64(x * 512), f64(wg), f64(wu), f64(wd))[0]
    assert np.linalg.norm(f64(big) - ref) <= H8 * 1.5 * np.linalg.norm(ref)
    clean, saved = B.psa_ffn(x, wg, wu, wd)
    y = x.clone()
    y[130, 3] = float("nan")
    out, saved_y = B.psa_ffn(y, wg, wu, wd)
    rest = [i for i in range(200) if i != 130]
    assert torch.equal(out[rest], clean[rest]) and out[130].isnan().all()
    dx = B.psa_ffn_bwd(x, y, wg, wu, wd, saved_y)[0]
    assert torch.equal(dx[rest], B.psa_ffn_bwd(x, x, wg, wu, wd, saved)[0][rest]) and dx[130].isnan().all()


def test_rows_behind_the_last_token_are_neither_read_nor_written():
    x, wg, wu, wd = small(T=256)
    want, saved = B.psa_ffn(x[:201].clone(), wg, wu, wd)
    wgrads = B.psa_ffn_bwd(x[:201].clone(), x[:201].clone(), wg, wu, wd, saved)
    x[201:] = float("nan")
    out, gate, up, dx = (torch.full((256, n), 5.0, dtype=torch.bfloat16, device="cuda") for n in (128, 264, 264, 128))
    B.psa_ffn(x[:201], wg, wu, wd, out=out[:201], gate=gate[:201], up=up[:201])
    gate[201:], up[201:] = float("nan"), float("nan")
    grads = B.psa_ffn_bwd(x[:201], x[:201], wg, wu, wd, (gate[:201], up[:201]), dx=dx[:201])
    torch.cuda.synchronize()
    assert torch.equal(out[:201], want) and (out[201:] == 5).all() and (dx[201:] == 5).all()
    assert all(torch.equal(a, b) for a, b in zip(grads, wgrads))


def test_the_same_bits_again_on_two_streams_at_once_and_in_a_graph():
    a, b = small(seed=1), small(T=321, seed=2)

    def step(args, **kw):
        out, saved = B.psa_ffn(*args, **kw)
        return (out,) + B.psa_ffn_bwd(args[0], *args, saved, **kw)
    want = [step(a), step(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [step(args, stream=s.cuda_stream) for args, s in zip((a, b), streams)]
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(w, g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(a)
    a[0].mul_(-0.5)
    want = step(a)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, captured))
