"""The log-probabilities from hidden states, the rotary positions and the norms around a block through both routes of the binding,
on other streams, from several host threads, and captured into CUDA graphs that share a workspace."""
import threading

import numpy as np
import pytest
import torch

from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def normal(*shape, dtype=BF, seed=None):
    g = torch.Generator().manual_seed(sum(shape) if seed is None else seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def make(T=300, D=264, V=700, seed=0):
    rng = np.random.default_rng(seed)
    i = lambda hi, n: torch.as_tensor(rng.integers(-1 if hi == 4 else 0, hi, size=n).astype(np.int32)).cuda()  # noqa: E731
    s = dict(h=normal(T, D, seed=seed), w=normal(V, D, seed=seed + 1) * 0.05, y=i(V, T), g=i(4, T), forks=[i(T, 9), i(V, 9), i(4, 9)],
             coef=normal(4, dtype=F32), q=normal(T, 6, 64, seed=seed + 2), k=normal(T, 2, 64, seed=seed + 3), pos=i(5000, T), x=normal(T, D, seed=seed + 4),
             r=normal(T, D, seed=seed + 5), d=normal(T, D, seed=seed + 6), p=[normal(D, seed=seed + 7 + j) for j in range(5)])
    s["turns"] = O.psa_rotary_frequencies(48, device="cuda")[0]
    s["lse"] = O.dpo_linear_logp(s["h"], s["w"], s["y"], s["g"], 4, *s["forks"])[1]
    s["total"], s["stats"] = O.psa_block_norm(s["x"], s["r"], *s["p"])[1:]
    return s


def calls(s):
    st = torch.zeros(1, dtype=I32, device="cuda")
    w, b, pw, pb, gate = s["p"]
    return {
        "logp": (lambda **k: O.dpo_linear_logp(s["h"], s["w"], s["y"], s["g"], 4, *s["forks"], **k),
                 lambda n: n.linear_logp(s["h"], s["w"], s["y"], s["g"], *s["forks"], 4, 1.0, None, st)),
        "logp_bwd": (lambda **k: O.dpo_linear_logp_bwd(s["coef"], s["h"], s["w"], s["lse"], s["y"], s["g"], *s["forks"], scale=0.5, **k),
                     lambda n: n.linear_logp_bwd(s["coef"], s["h"], s["w"], s["lse"], s["y"], s["g"], *s["forks"], 0.5, True, None, None)),
        "logp_bwd frozen": (lambda **k: O.dpo_linear_logp_bwd(s["coef"], s["h"], s["w"], s["lse"], s["y"], s["g"], with_table=False, **k),
                            lambda n: n.linear_logp_bwd(s["coef"], s["h"], s["w"], s["lse"], s["y"], s["g"], None, None, None, 1.0, False, None, st)),
        "rotary": (lambda **k: O.psa_rotary(s["q"], s["k"], s["pos"], s["turns"], 1.5, True, True, **k),
                   lambda n: n.rotary(s["q"], s["k"], s["pos"], s["turns"], 1.5, True, True)),
        "rotary q": (lambda **k: O.psa_rotary(s["q"].transpose(0, 1).contiguous().transpose(0, 1), None, s["pos"], s["turns"], **k),
                     lambda n: n.rotary(s["q"], None, s["pos"], s["turns"], 1.0, False, False)),
        "block": (lambda **k: O.psa_block_norm(s["x"], s["r"], w, b, pw, pb, gate, 0.7, **k),
                  lambda n: n.block_norm(s["x"], s["r"], w, b, pw, pb, gate, 0.7, 1e-5, False)),
        "block_bwd": (lambda **k: O.psa_block_norm_bwd(s["d"], s["x"], s["total"], w, s["stats"], pw, pb, gate, 0.7, d_total=s["r"], with_bias=True, **k),
                      lambda n: n.block_norm_bwd(s["d"], s["x"], s["total"], w, None, pw, pb, gate, s["stats"], 0.7, False, s["r"], True, None, st)),
        "block_bwd rms": (lambda **k: O.psa_block_norm_bwd(s["d"], s["x"], s["total"], w, s["stats"], gate=gate, rms=True, **k),
                          lambda n: n.block_norm_bwd(s["d"], s["x"], s["total"], w, None, None, None, gate, s["stats"], 1.0, True, None, False, None, None)),
    }


NAMES = ("logp", "logp_bwd", "logp_bwd frozen", "rotary", "rotary q", "block", "block_bwd", "block_bwd rms")


def flat(v):
    return [t for t in v if t is not None]


def same(a, b):
    return len(a) == len(b) and all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
def test_both_routes_give_the_same_bits(name):
    call, native = calls(make())[name]
    B.load_library()
    assert B._native is not None
    want = flat(call(stream=torch.cuda.current_stream().cuda_stream))
    assert same(flat(call()), want) and same(flat(native(B._native)), want)


def test_the_compiled_route_leaves_what_it_does_not_know():
    n, s = B._native, make(T=6, D=40, V=50)
    h, w, y, g, f = s["h"], s["w"], s["y"], s["g"], s["forks"]
    for a in ((h.cpu(), w, y, g, *f, 4, 1.0, None, None), (h.float(), w, y, g, *f, 4, 1.0, None, None), (h, w.t(), y, g, *f, 4, 1.0, None, None),
              (h, w, y.long(), g, *f, 4, 1.0, None, None), (h, w, y, g, f[0], None, None, 4, 1.0, None, None), (h, w, y, g, None, f[1], None, 4, 1.0, None, None),
              (h, w, y, g, f[0], f[1][:3], f[2], 4, 1.0, None, None), (h, w, y, g, *f, -1, 1.0, None, None), (h, w, y, g, *f, 4, 1, None, None),
              (h, w, y, g, *f, 4, 1.0, torch.empty(64, dtype=torch.uint8, device="cuda"), None), (h, w, y, g, *f, 4, 1.0, None, y.cpu())):
        assert n.linear_logp(*a) is None
    assert n.linear_logp_bwd(s["coef"].half(), h, w, s["lse"], y, g, *f, 1.0, True, None, None) is None
    assert n.linear_logp_bwd(s["coef"], h, w, s["lse"][:5], y, g, *f, 1.0, True, None, None) is None
    assert type(n.linear_logp(h, w, y, g, *f, 4, -1.0, None, None)) is int
    q, k, pos, t = s["q"], s["k"], s["pos"], s["turns"]
    for a in ((q, k[:5], pos, t, 1.0, False, False), (q, k.float(), pos, t, 1.0, False, False), (q, k, pos.long(), t, 1.0, False, False),
              (q, k, pos, t.int(), 1.0, False, False), (q.transpose(1, 2), None, pos, t, 1.0, False, False), (q, k, pos, t, 1, False, False), (q.half(), None, pos, t, 1.0, False, False)):
        assert n.rotary(*a) is None
    x, r, p = s["x"], s["r"], s["p"]
    for a in ((x, None, *p, 1.0, 1e-5, False), (x, r, *p, 1.0, 1e-5, True), (x, r, p[0], None, None, p[1], None, 1.0, 1e-5, False), (x, r[:5], *p, 1.0, 1e-5, False),
              (x, r, p[0].half(), *p[1:], 1.0, 1e-5, False)):
        assert n.block_norm(*a) is None
    for bad in (lambda: O.dpo_linear_logp(normal(6, 36), normal(50, 36), y, g, 4), lambda: O.dpo_linear_logp(h, w, y, g, 4, scale=0.0),
                lambda: O.psa_block_norm(normal(1, 16385), normal(1, 16385), normal(16385))):
        with pytest.raises(B.PsaError):
            bad()


@pytest.mark.parametrize("name", NAMES)
def test_on_a_stream_of_its_own(name):
    s = make()
    call, _ = calls(s)[name]
    want = flat(call())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = flat(call())
    by_handle = flat(call(stream=side.cuda_stream))
    side.synchronize()
    assert same(got, want) and same(by_handle, want)


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed_with_other_inputs(name):
    """Two graphs of the call, replayed in turn with other contents of the same inputs, while eager calls come between."""
    s, other = make(seed=0), make(seed=50)
    call, _ = calls(s)[name]
    eager = [flat(calls(v)[name][0]()) for v in (s, other)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(flat(call()))
        graphs.append(g)
    first = {k: v.clone() if torch.is_tensor(v) else [t.clone() for t in v] for k, v in s.items()}
    for source, want in ((other, eager[1]), (first, eager[0])):
        for k, v in s.items():
            for a, b in zip([v] if torch.is_tensor(v) else v, [source[k]] if torch.is_tensor(v) else source[k]):
                a.copy_(b)
        for g, out in zip(graphs, outs):
            g.replay()
            calls(other)[name][0]()
            torch.cuda.synchronize()
            assert same(out, want)


def test_two_graphs_that_share_a_workspace():
    s = make()
    lib = B.load_library()
    ws = torch.empty(max(lib.dpo_linear_logp_workspace_bytes(300, 9, 4, 700, 264, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    c = calls(s)
    want = [flat(c[n][0]()) for n in ("logp", "logp_bwd")]
    graphs, outs = [], []
    for n in ("logp", "logp_bwd"):
        c[n][0](workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(flat(c[n][0](workspace=ws)))
        graphs.append(g)
    for _ in range(3):      # one behind the other on one stream, each leaves the workspace as it likes
        for g in graphs:
            g.replay()
    ws.fill_(255)
    for g in reversed(graphs):
        g.replay()
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, want))


def test_several_host_threads_on_streams_of_their_own():
    sets = [make(T=200 + 37 * i, seed=10 * i) for i in range(4)]
    wants = [[flat(calls(s)[n][0]()) for n in NAMES] for s in sets]
    torch.cuda.synchronize()
    bad = []

    def work(s, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                c = calls(s)
                for _ in range(5):
                    for n, w in zip(NAMES, want):
                        got = flat(c[n][0]())
                        torch.cuda.current_stream().synchronize()
                        if not same(got, w):
                            bad.append(n)
        except Exception as e:      # noqa: BLE001
            bad.append(repr(e))
    threads = [threading.Thread(target=work, args=a) for a in zip(sets, wants)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert bad == []


def test_calls_one_behind_the_other_read_what_the_one_before_wrote():
    """The chain of a step, without a wait between its calls, as often as it takes for an early start to show: each call's
    inputs are the outputs of the call before, and all of them change every time."""
    T, D, V = 1500, 512, 900
    s = make(T=T, D=D, V=V)

    def chain(x, wait):
        out = []
        for _ in range(3):
            y, total, stats = O.psa_block_norm(x, s["r"], *s["p"])
            wait()
            q, _ = O.psa_rotary(y.view(T, 8, 64), None, s["pos"], s["turns"])
            wait()
            logps, lse = O.dpo_linear_logp(q.view(T, D), s["w"], s["y"], s["g"], 4, *s["forks"])
            wait()
            dq, dw = O.dpo_linear_logp_bwd(logps, q.view(T, D), s["w"], lse, s["y"], s["g"], *s["forks"])
            wait()
            dy, _ = O.psa_rotary(dq.view(T, 8, 64), None, s["pos"], s["turns"], inverse=True)
            wait()
            w, _, pw, pb, gate = s["p"]
            dx, dr, *params = O.psa_block_norm_bwd(dy.view(T, D), x, total, w, stats, pw, pb, gate, d_total=dq, with_bias=True)
            wait()
            out += [y, total, stats, q, logps, lse, dq, dw, dy, dx, dr, *params]
            x = dx
        return out
    for seed in range(4):
        x = normal(T, D, seed=seed)
        want = chain(x, torch.cuda.synchronize)
        got = chain(x, lambda: None)
        torch.cuda.synchronize()
        assert same(flat(got), flat(want))
