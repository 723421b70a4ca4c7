"""Calls of the normalisation, the embedding and the feed-forward block that are refused before anything is launched: by the
binding (host tensors that say they are on a GPU stand in for device ones), by the C entry points, and where the library
itself has no GPU."""
import ctypes as C

import pytest
import torch

from paper_2410_20305_b200 import binding as B

BF, F32 = torch.bfloat16, torch.float32
OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 3, 4


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def dev(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def reached(monkeypatch):
    """The library, whose calls are written down and not made (sizes of workspaces come from the real one)."""
    real, calls = B.load_library(), []

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_bytes") else (lambda *a: calls.append(name) or 0)
    monkeypatch.setattr(B, "load_library", Library)
    return calls


def norm(**change):
    a = dict(x=dev(6, 40), weight=dev(40), bias=dev(40), residual=dev(6, 40), out=dev(6, 40), total=dev(6, 40), stats=dev(2, 6, dtype=F32))
    a.update(change)
    return B.psa_norm(stream=0, **a)


def norm_bwd(**change):
    a = dict(d_out=dev(6, 40), x=dev(6, 40), weight=dev(40), stats=dev(2, 6, dtype=F32), d_total=dev(6, 40), with_bias=True, dx=dev(6, 40),
             dweight=dev(40), dbias=dev(40), workspace=dev(1 << 14, dtype=torch.uint8), status=dev(1, dtype=torch.int32))
    a.update(change)
    return B.psa_norm_bwd(stream=0, **a)


def embed(**change):
    a = dict(token_ids=dev(6, dtype=torch.int32), table=dev(9, 40), out=dev(6, 40), status=dev(1, dtype=torch.int32))
    a.update(change)
    return B.psa_embed(stream=0, **a)


def embed_bwd(**change):
    a = dict(d_out=dev(6, 40), token_ids=dev(6, dtype=torch.int32), vocab=9, dtable=dev(9, 40, dtype=F32),
             workspace=dev(1 << 16, dtype=torch.uint8), status=dev(1, dtype=torch.int32))
    a.update(change)
    return B.psa_embed_bwd(stream=0, **a)


def ffn(**change):
    a = dict(x=dev(6, 40), w_gate=dev(40, 24), w_up=dev(40, 24), w_down=dev(24, 40), out=dev(6, 40), gate=dev(6, 24), up=dev(6, 24),
             workspace=dev(1 << 12, dtype=torch.uint8), status=dev(1, dtype=torch.int32))
    a.update(change)
    return B.psa_ffn(stream=0, **a)


def ffn_bwd(**change):
    a = dict(d_out=dev(6, 40), x=dev(6, 40), w_gate=dev(40, 24), w_up=dev(40, 24), w_down=dev(24, 40), saved=(dev(6, 24), dev(6, 24)),
             dx=dev(6, 40), dw_gate=dev(40, 24), dw_up=dev(40, 24), dw_down=dev(24, 40), workspace=dev(1 << 13, dtype=torch.uint8))
    a.update(change)
    return B.psa_ffn_bwd(stream=0, **a)


HOST = torch.zeros
X = dev(6, 40)
CALLS = {"psa_norm": norm, "psa_norm_bwd": norm_bwd, "psa_embed": embed, "psa_embed_bwd": embed_bwd, "psa_ffn": ffn, "psa_ffn_bwd": ffn_bwd}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_well_formed_calls_reach_the_library(name, reached):
    CALLS[name]()
    assert reached == [name]


@pytest.mark.parametrize("name,change", [
    ("psa_norm", dict(x=dev(240))), ("psa_norm", dict(x=dev(6, 40, dtype=torch.float16))), ("psa_norm", dict(x=HOST(6, 40, dtype=BF))),
    ("psa_norm", dict(weight=dev(39))), ("psa_norm", dict(bias=dev(40, dtype=F32))), ("psa_norm", dict(rms=True)),
    ("psa_norm", dict(residual=dev(5, 40))), ("psa_norm", dict(residual=None)), ("psa_norm", dict(out=dev(6, 41))),
    ("psa_norm", dict(total=dev(6, 40, dtype=F32))), ("psa_norm", dict(stats=dev(6, 2, dtype=F32))),
    ("psa_norm", dict(x=dev(40, 6).t())), ("psa_norm", dict(x=dev(6, 40, dtype=F32))),
    ("psa_norm", dict(out=X, total=X)), ("psa_norm", dict(eps="a")),
    ("psa_norm_bwd", dict(d_out=dev(6, 39))), ("psa_norm_bwd", dict(stats=dev(2, 5, dtype=F32))), ("psa_norm_bwd", dict(rms=True)),
    ("psa_norm_bwd", dict(dweight=dev(40, dtype=F32))), ("psa_norm_bwd", dict(d_total=HOST(6, 40, dtype=BF))),
    ("psa_norm_bwd", dict(workspace=dev(64, dtype=torch.uint8))), ("psa_norm_bwd", dict(status=HOST(1, dtype=torch.int32))),
    ("psa_norm_bwd", dict(workspace=dev(1, dtype=torch.uint8).expand(1 << 14))),
    ("psa_embed", dict(token_ids=dev(6, dtype=torch.int64))), ("psa_embed", dict(token_ids=dev(6, 1, dtype=torch.int32))),
    ("psa_embed", dict(table=dev(9, 40, dtype=torch.float16))), ("psa_embed", dict(out=dev(6, 40, dtype=F32))),
    ("psa_embed", dict(table=dev(40, 9).t())), ("psa_embed", dict(token_ids=dev(12, dtype=torch.int32)[::2])),
    ("psa_embed_bwd", dict(token_ids=dev(5, dtype=torch.int32))), ("psa_embed_bwd", dict(dtable=dev(8, 40, dtype=F32))),
    ("psa_embed_bwd", dict(dtable=None, accumulate=True)), ("psa_embed_bwd", dict(d_out=dev(6, 40, dtype=F32), dtable=dev(9, 40))),
    ("psa_embed_bwd", dict(dtype=BF)), ("psa_embed_bwd", dict(workspace=dev(64, dtype=torch.uint8))), ("psa_embed_bwd", dict(vocab=8)),
    ("psa_ffn", dict(x=dev(6, 40, dtype=F32))), ("psa_ffn", dict(w_up=dev(24, 40))), ("psa_ffn", dict(w_down=dev(40, 24))),
    ("psa_ffn", dict(w_down=dev(40, 24).t())), ("psa_ffn", dict(gate=None, save=False)), ("psa_ffn", dict(out=HOST(6, 40, dtype=BF))),
    ("psa_ffn", dict(x=X, out=X)), ("psa_ffn", dict(gate=dev(6, 24), up=dev(6, 23))), ("psa_ffn", dict(workspace=dev(32, dtype=torch.uint8))),
    ("psa_ffn_bwd", dict(d_out=dev(5, 40))), ("psa_ffn_bwd", dict(saved=(dev(6, 24), dev(6, 40)))), ("psa_ffn_bwd", dict(d_out=X, dx=X)),
    ("psa_ffn_bwd", dict(dw_down=dev(40, 24))), ("psa_ffn_bwd", dict(workspace=dev(1 << 9, dtype=torch.uint8))), ("psa_ffn_bwd", dict(saved=None)),
])
def test_malformed_calls_do_not(name, change, reached):
    with pytest.raises((ValueError, TypeError)):
        CALLS[name](**change)
    assert reached == []


def test_results_may_take_the_place_of_some_inputs(reached):
    x, r = dev(6, 40), dev(6, 40)
    norm(x=x, residual=r, out=x, total=r)
    norm(x=x, residual=r, out=r, total=x)
    norm_bwd(d_out=x, dx=x)
    norm_bwd(d_total=x, dx=x)
    assert len(reached) == 4
    whole = dev(7, 40)
    with pytest.raises(ValueError):      # a row further on is another place
        norm(x=whole[:6], out=whole[1:])
    with pytest.raises(ValueError):
        norm(out=x, total=x)


def test_the_c_entry_points_check_before_any_launch():
    lib = B.load_library()
    buf = C.create_string_buffer(4096)
    p = (C.addressof(buf) + 255) // 256 * 256
    bf, f32 = B.PSA_DTYPE_BF16, B.PSA_DTYPE_F32

    def fwd(x=p, res=None, w=p, b=None, dt=bf, wt=bf, T=2, D=16, eps=1e-5, rms=0, out=p, total=None, stats=p):
        return lib.psa_norm(x, res, w, b, dt, wt, T, D, eps, rms, out, total, stats, None)
    assert fwd(T=0, x=None, w=None, out=None, stats=None) == OK
    for change in (dict(x=None), dict(w=None), dict(out=None), dict(stats=None), dict(T=-1), dict(D=0), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(rms=1, b=p), dict(res=p), dict(total=p), dict(dt=f32), dict(dt=7), dict(wt=2)):
        assert fwd(**change) == INVALID, change
    assert fwd(D=16385) == UNSUPPORTED and fwd(T=1 << 31) == UNSUPPORTED
    assert fwd(x=p + 8) == ALIGNMENT and fwd(w=p + 2) == ALIGNMENT and fwd(stats=p + 4) == ALIGNMENT

    def bwd(g=p, x=p, w=p, stats=p, dtot=None, dt=bf, wt=bf, T=2, D=16, rms=0, dx=p, dw=p, db=None, ws=p):
        return lib.psa_norm_bwd(g, x, w, stats, dtot, dt, wt, T, D, rms, dx, dw, db, ws, None, None)
    for change in (dict(g=None), dict(x=None), dict(stats=None), dict(dx=None), dict(dw=None), dict(ws=None), dict(rms=1, db=p), dict(T=-1)):
        assert bwd(**change) == INVALID, change
    assert bwd(D=20000) == UNSUPPORTED and bwd(ws=p + 8) == ALIGNMENT and bwd(dtot=p + 2) == ALIGNMENT

    def emb(ids=p, table=p, dt=bf, T=2, V=3, D=8, out=p):
        return lib.psa_embed(ids, table, dt, T, V, D, 1.0, out, None, None)
    assert emb(T=0, ids=None, table=None, out=None) == OK
    for change in (dict(ids=None), dict(table=None), dict(out=None), dict(T=-1), dict(V=0), dict(D=0), dict(dt=9)):
        assert emb(**change) == INVALID, change
    assert emb(T=(1 << 24) + 1) == UNSUPPORTED and emb(V=(1 << 24) + 1) == UNSUPPORTED and emb(D=(1 << 20) + 1) == UNSUPPORTED
    assert emb(table=p + 4) == ALIGNMENT and emb(ids=p + 2) == ALIGNMENT

    def embb(g=p, ids=p, dt=bf, gt=bf, T=2, V=3, D=8, dtable=p, ws=p):
        return lib.psa_embed_bwd(g, ids, dt, gt, T, V, D, 1.0, 0, dtable, ws, None, None)
    for change in (dict(g=None), dict(ids=None), dict(dtable=None), dict(ws=None), dict(dt=f32, gt=bf), dict(gt=5), dict(V=-1)):
        assert embb(**change) == INVALID, change
    assert embb(dtable=p + 8) == ALIGNMENT and embb(D=1 << 21) == UNSUPPORTED

    def f(x=p, wg=p, wu=p, wd=p, T=2, D=16, F=24, out=p, gate=None, up=None, ws=p):
        return lib.psa_ffn(x, wg, wu, wd, T, D, F, out, gate, up, ws, None, None)
    assert f(T=0, x=None, out=None, ws=None) == OK
    for change in (dict(x=None), dict(wu=None), dict(out=None), dict(ws=None), dict(gate=p), dict(up=p), dict(T=-1), dict(D=0), dict(F=-8)):
        assert f(**change) == INVALID, change
    for change in (dict(D=12), dict(F=20), dict(D=1 << 21), dict(T=1 << 31)):
        assert f(**change) == UNSUPPORTED, change
    assert f(wd=p + 8) == ALIGNMENT and f(gate=p + 2, up=p) == ALIGNMENT

    def fb(g=p, x=p, wg=p, wu=p, wd=p, gate=p, up=p, T=2, D=16, F=24, dx=p, dg=p, du=p, dd=p, ws=p):
        return lib.psa_ffn_bwd(g, x, wg, wu, wd, gate, up, T, D, F, dx, dg, du, dd, ws, None, None)
    for change in (dict(g=None), dict(gate=None), dict(dx=None), dict(dg=None), dict(dd=None), dict(ws=None), dict(T=-2)):
        assert fb(**change) == INVALID, change
    assert fb(D=4) == UNSUPPORTED and fb(up=p + 4) == ALIGNMENT and fb(du=p + 8) == ALIGNMENT


def test_workspaces_grow_with_the_call_and_are_0_for_what_is_refused():
    lib = B.load_library()
    assert lib.psa_ffn_workspace_bytes(100, 64, 128, 0) >= 100 * 128 * 2 and lib.psa_ffn_workspace_bytes(100, 64, 128, 1) >= 3 * 100 * 128 * 2
    assert lib.psa_ffn_workspace_bytes(100, 63, 128, 0) == 0 and lib.psa_ffn_workspace_bytes(-1, 64, 128, 0) == 0
    assert lib.psa_norm_bwd_workspace_bytes(1000, 0) == 0 and lib.psa_norm_bwd_workspace_bytes(1000, 16385) == 0
    assert lib.psa_norm_bwd_workspace_bytes(1, 100) >= 800
    assert lib.psa_embed_bwd_workspace_bytes(10, 0, 8) == 0 and lib.psa_embed_bwd_workspace_bytes(10, 100, 8) >= 4 * 100 + 8 * 10
    # beyond 32 bits
    assert lib.psa_ffn_workspace_bytes(1 << 20, 4096, 14336, 1) > 3 * (1 << 20) * 14336 * 2 - 1
    assert lib.psa_embed_bwd_workspace_bytes(1 << 24, 1 << 24, 4096) > (1 << 32)
