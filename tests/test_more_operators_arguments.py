"""Calls of the log-probabilities from hidden states, the rotary positions and the norms around a block that are refused before
anything is launched: by the binding (host tensors that say they are on a GPU stand in for device ones), and by the C
entry points."""
import ctypes as C

import pytest
import torch

from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O

BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
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


FORKS = dict(fork_rows=dev(2, dtype=I32), fork_targets=dev(2, dtype=I32), fork_segments=dev(2, dtype=I32))


def logp(**change):
    a = dict(hidden=dev(6, 40), table=dev(9, 40), targets=dev(6, dtype=I32), segment_ids=dev(6, dtype=I32), n_segments=3, **FORKS,
             out=dev(3, dtype=F32), lse=dev(6, dtype=F32), workspace=dev(1 << 16, dtype=torch.uint8), status=dev(1, dtype=I32))
    a.update(change)
    return O.dpo_linear_logp(stream=0, **a)


def logp_bwd(**change):
    a = dict(coef=dev(3, dtype=F32), hidden=dev(6, 40), table=dev(9, 40), lse=dev(6, dtype=F32), targets=dev(6, dtype=I32),
             segment_ids=dev(6, dtype=I32), **FORKS, d_hidden=dev(6, 40), d_table=dev(9, 40), workspace=dev(1 << 22, dtype=torch.uint8),
             status=dev(1, dtype=I32))
    a.update(change)
    return O.dpo_linear_logp_bwd(stream=0, **a)


def rotary(**change):
    a = dict(q=dev(6, 4, 16), k=dev(6, 2, 16), position_ids=dev(6, dtype=I32), turns=dev(4, dtype=I64), q_out=dev(6, 4, 16), k_out=dev(6, 2, 16))
    a.update(change)
    return O.psa_rotary(stream=0, **a)


def block(**change):
    a = dict(x=dev(6, 40), residual=dev(6, 40), weight=dev(40), bias=dev(40), post_weight=dev(40), post_bias=dev(40), gate=dev(40),
             out=dev(6, 40), total=dev(6, 40), stats=dev(4, 6, dtype=F32))
    a.update(change)
    return O.psa_block_norm(stream=0, **a)


def block_bwd(**change):
    a = dict(d_out=dev(6, 40), x=dev(6, 40), total=dev(6, 40), weight=dev(40), stats=dev(4, 6, dtype=F32), post_weight=dev(40),
             post_bias=dev(40), gate=dev(40), d_total=dev(6, 40), with_bias=True, dx=dev(6, 40), d_residual=dev(6, 40),
             workspace=dev(1 << 16, dtype=torch.uint8), status=dev(1, dtype=I32))
    a.update(change)
    return O.psa_block_norm_bwd(stream=0, **a)


HOST = torch.zeros
X = dev(6, 40)
HEADS = dev(6, 4, 16)
CALLS = {"dpo_linear_logp": logp, "dpo_linear_logp_bwd": logp_bwd, "psa_rotary": rotary, "psa_block_norm": block, "psa_block_norm_bwd": block_bwd}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_well_formed_calls_reach_the_library(name, reached):
    CALLS[name]()
    assert reached == [name]


@pytest.mark.parametrize("name,change", [
    ("dpo_linear_logp", dict(hidden=dev(240))), ("dpo_linear_logp", dict(hidden=dev(6, 40, dtype=F32))), ("dpo_linear_logp", dict(hidden=HOST(6, 40, dtype=BF))),
    ("dpo_linear_logp", dict(hidden=dev(40, 6).t())), ("dpo_linear_logp", dict(table=dev(9, 48))), ("dpo_linear_logp", dict(table=dev(40, 9).t())),
    ("dpo_linear_logp", dict(targets=dev(5, dtype=I32))), ("dpo_linear_logp", dict(targets=dev(6, dtype=I64))), ("dpo_linear_logp", dict(segment_ids=dev(6, 1, dtype=I32))),
    ("dpo_linear_logp", dict(fork_rows=None)), ("dpo_linear_logp", dict(fork_targets=dev(3, dtype=I32))), ("dpo_linear_logp", dict(n_segments=-1)),
    ("dpo_linear_logp", dict(out=dev(4, dtype=F32))), ("dpo_linear_logp", dict(out=dev(3))), ("dpo_linear_logp", dict(lse=dev(5, dtype=F32))),
    ("dpo_linear_logp", dict(workspace=dev(1 << 8, dtype=torch.uint8))), ("dpo_linear_logp", dict(status=HOST(1, dtype=I32))), ("dpo_linear_logp", dict(scale="a")),
    ("dpo_linear_logp", dict(n_segments=6, out=(o := dev(6, dtype=F32)), lse=o)),
    ("dpo_linear_logp_bwd", dict(coef=dev(3))), ("dpo_linear_logp_bwd", dict(coef=dev(3, 1, dtype=F32))), ("dpo_linear_logp_bwd", dict(lse=dev(7, dtype=F32))),
    ("dpo_linear_logp_bwd", dict(d_hidden=dev(6, 39))), ("dpo_linear_logp_bwd", dict(d_table=dev(9, 40, dtype=F32))), ("dpo_linear_logp_bwd", dict(with_table=False)),
    ("dpo_linear_logp_bwd", dict(hidden=X, d_hidden=X)), ("dpo_linear_logp_bwd", dict(workspace=dev(1 << 10, dtype=torch.uint8))),
    ("psa_rotary", dict(q=dev(6, 64))), ("psa_rotary", dict(q=dev(6, 4, 16, dtype=torch.float16))), ("psa_rotary", dict(q=HOST(6, 4, 16, dtype=BF))),
    ("psa_rotary", dict(k=dev(5, 2, 16))), ("psa_rotary", dict(k=dev(6, 2, 32))), ("psa_rotary", dict(k=dev(6, 2, 16, dtype=F32))), ("psa_rotary", dict(k=None)),
    ("psa_rotary", dict(turns=dev(9, dtype=I64))), ("psa_rotary", dict(turns=dev(4, dtype=I32))), ("psa_rotary", dict(turns=dev(4, 1, dtype=I64))),
    ("psa_rotary", dict(position_ids=dev(7, dtype=I32))), ("psa_rotary", dict(position_ids=dev(6, dtype=I64))), ("psa_rotary", dict(q=dev(6, 16, 4).transpose(1, 2))),
    ("psa_rotary", dict(q_out=dev(6, 4, 17)[..., :15])), ("psa_rotary", dict(q_out=dev(1, 4, 16).expand(6, 4, 16))), ("psa_rotary", dict(q_out=dev(6, 1, 16).expand(6, 4, 16))),
    ("psa_rotary", dict(q=HEADS, q_out=HEADS[:, [0, 1, 2, 3]].as_strided((6, 4, 16), (64, 15, 1)))), ("psa_rotary", dict(q=(w := dev(7, 4, 16))[:6], q_out=w[1:])),
    ("psa_rotary", dict(q=(w2 := dev(6, 6, 16))[:, :4], k_out=w2[:, 2:4])), ("psa_rotary", dict(q_out=(w3 := dev(6, 6, 16))[:, :4], k_out=w3[:, 3:5])),
    ("psa_block_norm", dict(residual=None)), ("psa_block_norm", dict(residual=dev(5, 40))), ("psa_block_norm", dict(rms=True)), ("psa_block_norm", dict(post_weight=None)),
    ("psa_block_norm", dict(gate=dev(40, dtype=F32))), ("psa_block_norm", dict(gate=dev(1))), ("psa_block_norm", dict(x=dev(6, 40, dtype=F32))), ("psa_block_norm", dict(stats=dev(2, 6, dtype=F32))),
    ("psa_block_norm", dict(out=X, total=X)), ("psa_block_norm", dict(x=dev(40, 6).t())), ("psa_block_norm", dict(eps=None)),
    ("psa_block_norm_bwd", dict(total=dev(6, 41))), ("psa_block_norm_bwd", dict(rms=True)), ("psa_block_norm_bwd", dict(post_weight=None)), ("psa_block_norm_bwd", dict(d_total=HOST(6, 40, dtype=BF))),
    ("psa_block_norm_bwd", dict(x=X, d_residual=X)), ("psa_block_norm_bwd", dict(dx=X, d_residual=X)), ("psa_block_norm_bwd", dict(workspace=dev(64, dtype=torch.uint8))),
    ("psa_block_norm_bwd", dict(stats=dev(6, 4, dtype=F32))),
])
def test_malformed_calls_do_not(name, change, reached):
    with pytest.raises((ValueError, TypeError)):
        CALLS[name](**change)
    assert reached == []


def test_results_may_take_the_place_of_some_inputs(reached):
    x, r = dev(6, 40), dev(6, 40)
    block(x=x, residual=r, out=x, total=r)
    block(x=x, residual=r, out=r, total=x)
    block_bwd(d_out=x, d_total=r, dx=x, d_residual=r)
    block_bwd(x=x, total=r, dx=x, d_residual=r)
    fused = dev(6, 8 * 16)
    q, k = fused[:, :64].view(6, 4, 16), fused[:, 64:96].view(6, 2, 16)
    rotary(q=q, k=k, q_out=q, k_out=k)
    rotary(q=q, k=k)
    rotary(q_out=q, k_out=k)
    rotary(q=dev(1, 4, 16).expand(6, 4, 16), k=None, k_out=None)
    assert len(reached) == 8


@pytest.mark.parametrize("change", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=1026), dict(theta=1.0), dict(theta=float("nan")),
                                    dict(scaling="linear", factor=0.5), dict(scaling="base", rotary_dim=2, factor=2.0), dict(scaling="wavelength", factor=2.0),
                                    dict(scaling="wavelength", factor=2.0, original_length=100, low=4.0, high=4.0),
                                    dict(scaling="ramp", factor=float("inf"), original_length=100), dict(scaling="other"), dict(rotary_dim=-2)])
def test_frequencies_that_do_not_exist(change):
    a = dict(rotary_dim=8)
    a.update(change)
    with pytest.raises((ValueError, B.PsaError)):
        O.psa_rotary_frequencies(**a)


def test_the_c_entry_points_check_before_any_launch():
    lib = B.load_library()
    buf = C.create_string_buffer(4096)
    p = (C.addressof(buf) + 255) // 256 * 256
    bf, f32 = B.PSA_DTYPE_BF16, B.PSA_DTYPE_F32

    def lp(h=p, w=p, n=2, V=3, D=16, scale=1.0, y=p, g=p, fr=None, ft=None, fg=None, nf=0, ns=2, out=p, lse=p, ws=p):
        return lib.dpo_linear_logp(h, w, n, V, D, scale, y, g, fr, ft, fg, nf, ns, out, lse, ws, None, None)
    for change in (dict(h=None), dict(w=None), dict(y=None), dict(g=None), dict(out=None), dict(lse=None), dict(ws=None), dict(nf=1), dict(n=-1),
                   dict(V=0), dict(D=0), dict(ns=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert lp(**change) == INVALID, change
    for change in (dict(D=12), dict(D=1 << 21), dict(V=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(n=1 << 22, V=(1 << 23) + 1)):
        assert lp(**change) == UNSUPPORTED, change
    assert lp(h=p + 8) == ALIGNMENT and lp(w=p + 2) == ALIGNMENT and lp(ws=p + 4) == ALIGNMENT

    def lpb(c=p, h=p, w=p, lse=p, n=2, V=3, D=16, scale=1.0, y=p, g=p, nf=0, ns=2, dh=p, dw=p, ws=p):
        return lib.dpo_linear_logp_bwd(c, h, w, lse, n, V, D, scale, y, g, None, None, None, nf, ns, dh, dw, ws, None, None)
    for change in (dict(c=None), dict(h=None), dict(w=None), dict(lse=None), dict(dh=None), dict(ws=None), dict(nf=2), dict(V=-1)):
        assert lpb(**change) == INVALID, change
    assert lpb(D=20) == UNSUPPORTED and lpb(dh=p + 8) == ALIGNMENT and lpb(dw=p + 2) == ALIGNMENT

    def rot(q=p, k=p, qo=p, ko=p, pos=p, turns=p, dt=bf, T=2, Hq=2, Hk=1, d=16, r=8, inter=0):
        return lib.psa_rotary(q, k, qo, ko, pos, turns, dt, T, Hq, Hk, d, r, None, inter, 0, 1.0, None)
    assert rot(T=0, q=None, qo=None, pos=None) == OK
    for change in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None), dict(turns=None), dict(T=-1), dict(Hq=0), dict(Hk=-1),
                   dict(d=0), dict(r=7), dict(r=18), dict(r=0), dict(dt=4)):
        assert rot(**change) == INVALID, change
    assert rot(d=1026) == UNSUPPORTED and rot(T=1 << 31) == UNSUPPORTED and rot(Hq=70000) == UNSUPPORTED
    assert rot(q=p + 1) == ALIGNMENT and rot(q=p + 2, dt=f32) == ALIGNMENT and rot(q=p + 2, inter=1) == ALIGNMENT

    def fwd(x=p, res=p, w=p, b=None, pw=None, pb=None, g=None, dt=bf, wt=bf, T=2, D=16, eps=1e-5, rms=0, out=p, total=p, stats=p):
        return lib.psa_block_norm(x, res, w, b, pw, pb, g, 1.0, dt, wt, T, D, eps, rms, out, total, stats, None)
    assert fwd(T=0, x=None, res=None, w=None, out=None, total=None, stats=None) == OK
    for change in (dict(x=None), dict(res=None), dict(w=None), dict(out=None), dict(total=None), dict(stats=None), dict(T=-1), dict(D=0), dict(eps=-1.0),
                   dict(rms=1, b=p), dict(rms=1, pw=p, pb=p), dict(pb=p), dict(dt=f32), dict(dt=7), dict(wt=2)):
        assert fwd(**change) == INVALID, change
    assert fwd(D=16385) == UNSUPPORTED and fwd(T=1 << 31) == UNSUPPORTED
    assert fwd(x=p + 8) == ALIGNMENT and fwd(g=p + 2) == ALIGNMENT and fwd(stats=p + 4) == ALIGNMENT

    def bwd(g=p, x=p, s=p, w=p, pw=p, pb=None, gate=p, stats=p, dtot=None, dt=bf, wt=bf, T=2, D=16, rms=0, dx=p, dr=p, dw=p, db=None, dpw=p, dpb=None, dg=p, ws=p):
        return lib.psa_block_norm_bwd(g, x, s, w, pw, pb, gate, 1.0, stats, dtot, dt, wt, T, D, rms, dx, dr, dw, db, dpw, dpb, dg, ws, None, None)
    for change in (dict(g=None), dict(x=None), dict(s=None), dict(stats=None), dict(dx=None), dict(dr=None), dict(dw=None), dict(ws=None), dict(rms=1, db=p),
                   dict(dpw=None), dict(dg=None), dict(pw=None), dict(gate=None), dict(T=-1), dict(pw=None, dpw=None, dpb=p)):
        assert bwd(**change) == INVALID, change
    assert bwd(D=20000) == UNSUPPORTED and bwd(ws=p + 8) == ALIGNMENT and bwd(dtot=p + 2) == ALIGNMENT and bwd(dr=p + 8) == ALIGNMENT


def test_workspaces_grow_with_the_call_and_are_0_for_what_is_refused():
    lib = B.load_library()
    need = lib.dpo_linear_logp_workspace_bytes
    assert need(100, 5, 4, 1000, 63, 0) == 0 and need(-1, 0, 4, 1000, 64, 0) == 0 and need(100, 0, 4, 0, 64, 1) == 0
    assert need(1000, 5, 4, 1000, 64, 0) >= 1005 * 64 * 2 and need(1000, 5, 4, 1000, 64, 1) >= 1005 * (64 * 2 + 1000 * 2 + 64 * 4)
    # dz of a piece stays within 1 GiB, whatever the vocabulary, and beyond 32 bits in all
    rows = 16384 * (4096 * 2 + 4096 * 4)
    assert need(16384, 0, 4, 1 << 20, 4096, 1) <= (1 << 30) + rows + (1 << 20) and need(1 << 20, 0, 4, 128256, 4096, 1) > (1 << 32)
    blocks = lib.psa_block_norm_bwd_workspace_bytes
    assert blocks(1000, 0) == 0 and blocks(1000, 16385) == 0 and blocks(1, 100) >= 4 * 400
