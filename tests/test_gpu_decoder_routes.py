"""The normalisation, the embedding and the feed-forward block through both routes of the binding: the same bits, and what the
compiled route does not take is refused or done by the other one."""
import pytest
import torch

from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def normal(*shape, dtype=BF):
    return torch.randn(*shape, device="cuda").to(dtype)


@pytest.fixture(scope="module")
def calls():
    torch.manual_seed(0)
    x, r, w = normal(70, 136), normal(70, 136), normal(136)
    ids = torch.randint(0, 50, (70,), device="cuda", dtype=I32)
    wg, wu, wd = normal(136, 264), normal(136, 264), normal(264, 136)
    stats = B.psa_norm(x, w)[1]
    saved = B.psa_ffn(x, wg, wu, wd)[1]
    status = torch.zeros(1, dtype=I32, device="cuda")
    return {
        "norm": (lambda **k: B.psa_norm(x, w, w, residual=r, **k), lambda n: n.norm(x, w, w, 1e-5, False, r)),
        "norm rms": (lambda **k: B.psa_norm(x, w, rms=True, **k), lambda n: n.norm(x, w, None, 1e-5, True, None)),
        "norm_bwd": (lambda **k: B.psa_norm_bwd(r, x, w, stats, d_total=r, with_bias=True, **k),
                     lambda n: n.norm_bwd(r, x, w, stats, False, r, True, None, status)),
        "embed": (lambda **k: B.psa_embed(ids, wg, scale=3.0, **k), lambda n: n.embed(ids, wg, 3.0, status)),
        "embed_bwd": (lambda **k: B.psa_embed_bwd(x, ids, 50, scale=3.0, **k), lambda n: n.embed_bwd(x, ids, 50, 3.0, False, None, None)),
        "embed_bwd f32": (lambda **k: B.psa_embed_bwd(x, ids, 50, scale=3.0, dtype=F32, **k),
                          lambda n: n.embed_bwd(x, ids, 50, 3.0, True, None, None)),
        "ffn": (lambda **k: B.psa_ffn(x, wg, wu, wd, **k), lambda n: n.ffn(x, wg, wu, wd, True, None, None)),
        "ffn only": (lambda **k: B.psa_ffn(x, wg, wu, wd, save=False, **k), lambda n: n.ffn(x, wg, wu, wd, False, None, None)),
        "ffn_bwd": (lambda **k: B.psa_ffn_bwd(r, x, wg, wu, wd, saved, **k), lambda n: n.ffn_bwd(r, x, wg, wu, wd, *saved, None, status)),
    }


def flat(v):
    if isinstance(v, torch.Tensor):
        return [v]
    return [t for u in v if u is not None for t in flat(u)]


NAMES = ("norm", "norm rms", "norm_bwd", "embed", "embed_bwd", "embed_bwd f32", "ffn", "ffn only", "ffn_bwd")


@pytest.mark.parametrize("name", NAMES)
def test_both_routes_give_the_same_bits(calls, name):
    call, native = calls[name]
    B.load_library()
    assert B._native is not None
    want = flat(call(stream=torch.cuda.current_stream().cuda_stream))
    for got in (flat(call()), flat(native(B._native))):
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_compiled_route_leaves_what_it_does_not_know():
    n = B._native
    x, w, ids = normal(6, 40), normal(40), torch.zeros(6, dtype=I32, device="cuda")
    wg, wd, st = normal(40, 24), normal(24, 40), torch.zeros(2, 6, device="cuda")
    cpu = x.cpu()
    for args in ((cpu, w, None, 1e-5, False, None), (x, w[:39], None, 1e-5, False, None), (x, w, w, 1e-5, True, None),
                 (x, w, None, 1e-5, 0, None), (x.t(), w, None, 1e-5, False, None), (x, w, None, 1e-5, False, x[:5]),
                 (x.float(), w, None, 1e-5, False, None), (x.half(), w, None, 1e-5, False, None), (x, w, None, 1, False, None)):
        assert n.norm(*args) is None
    assert n.norm_bwd(x, x, w, st[:, :5], False, None, False, None, None) is None
    assert n.norm_bwd(x, x, w, st, True, None, True, None, None) is None
    assert n.norm_bwd(x, x, w, st, False, None, False, torch.empty(8, dtype=torch.uint8, device="cuda"), None) is None
    assert n.norm_bwd(x, x, w, st, False, None, False, None, torch.zeros(1, dtype=I32)) is None
    assert n.embed(ids.long(), wd, 1.0, None) is None and n.embed(ids, wd[:, ::2], 1.0, None) is None
    assert n.embed_bwd(x, ids[:5], 9, 1.0, False, None, None) is None and n.embed_bwd(x, ids, 0, 1.0, False, None, None) is None
    assert n.ffn(x, wg, wg, wd.t(), True, None, None) is None and n.ffn(x, wg, wg[:, :16], wd, True, None, None) is None
    assert n.ffn(None, wg, wg, wd, True, None, None) is None
    assert n.ffn_bwd(x, x, wg, wg, wd, None, x, None, None) is None
    assert type(n.ffn(normal(6, 36), normal(36, 24), normal(36, 24), normal(24, 36), True, None, None)) is int
    for call in (lambda: B.psa_ffn(normal(6, 36), normal(36, 24), normal(36, 24), normal(24, 36)),
                 lambda: B.psa_norm(normal(1, 16385), normal(16385)), lambda: B.psa_embed_bwd(x, ids, (1 << 24) + 1)):
        with pytest.raises(B.PsaError):
            call()
    for call in (lambda: B.psa_ffn(x, wg, wg, wd.t()), lambda: B.psa_norm(x, w, w, rms=True), lambda: B.psa_embed(ids.long(), wd),
                 lambda: B.psa_norm_bwd(x, x, w, st, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
                 lambda: B.psa_norm(cpu, w.cpu())):
        with pytest.raises(ValueError):
            call()


def test_a_workspace_of_the_caller_is_used_and_may_be_reused():
    x, w = normal(300, 264), normal(264)
    g = normal(300, 264)
    stats = B.psa_norm(x, w)[1]
    lib = B.load_library()
    ws = torch.empty(lib.psa_norm_bwd_workspace_bytes(300, 264), dtype=torch.uint8, device="cuda")
    want = B.psa_norm_bwd(g, x, w, stats)
    for _ in range(2):
        ws.fill_(255)
        assert all(torch.equal(a, b) for a, b in zip(want[:2], B.psa_norm_bwd(g, x, w, stats, workspace=ws)))
    wg, wu, wd = normal(264, 400), normal(264, 400), normal(400, 264)
    out, saved = B.psa_ffn(x, wg, wu, wd)
    ws = torch.empty(lib.psa_ffn_workspace_bytes(300, 264, 400, 1), dtype=torch.uint8, device="cuda")
    want = B.psa_ffn_bwd(g, x, wg, wu, wd, saved)
    for _ in range(2):
        ws.fill_(255)
        assert torch.equal(out, B.psa_ffn(x, wg, wu, wd, workspace=ws)[0])
        assert all(torch.equal(a, b) for a, b in zip(want, B.psa_ffn_bwd(g, x, wg, wu, wd, saved, workspace=ws)))
    ids = torch.randint(0, 90, (300,), device="cuda", dtype=I32)
    ws = torch.empty(lib.psa_embed_bwd_workspace_bytes(300, 90, 264), dtype=torch.uint8, device="cuda")
    want = B.psa_embed_bwd(g, ids, 90)
    for _ in range(2):
        ws.fill_(255)
        assert torch.equal(want, B.psa_embed_bwd(g, ids, 90, workspace=ws))
