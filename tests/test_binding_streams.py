"""Which stream the results that a call makes are allocated on, checked without a GPU: host tensors that say they are on one,
the library's calls and torch's streams replaced by stand-ins that write down what is done with them."""
import contextlib
import inspect

import pytest
import torch

from paper_2410_20305_b200 import binding as B

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def dev(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


class Plan:
    _h, _key, total_tokens, n_q_heads, n_kv_heads, head_dim, bwd_workspace_bytes = None, None, 6, 2, 1, 64, 256


Q, KV, LSE, WS = dev(6, 2, 64), dev(6, 1, 64), dev(2, 6, dtype=F32), dev(1 << 16, dtype=U8)
X, W, STATS, IDS = dev(6, 40), dev(40), dev(2, 6, dtype=F32), dev(6, dtype=I32)
LOGITS, LOGPS = dev(6, 40, dtype=F32), dev(4, dtype=F32)
CALLS = {
    "psa_fwd": lambda **k: B.psa_fwd(Plan, Q, KV, KV, **k),
    "psa_bwd": lambda **k: B.psa_bwd(Plan, Q, Q, KV, KV, Q, LSE, workspace=WS, **k),
    "psa_bwd_f32": lambda **k: B.psa_bwd_f32(Plan, Q, Q, KV, KV, Q, LSE, workspace=WS, **k),
    "dpo_logp": lambda **k: B.dpo_logp(LOGITS, IDS, IDS, 2, scratch=dev(3, dtype=torch.float64), **k),
    "dpo_logp_bwd": lambda **k: B.dpo_logp_bwd(LOGITS, IDS, IDS, dev(2, dtype=F32), **k),
    "dpo_loss": lambda **k: B.dpo_loss(LOGPS, LOGPS, 0.1, **k),
    "simpo_loss": lambda **k: B.simpo_loss(LOGPS, dev(4, dtype=I32), 0.1, 0.2, **k),
    "orpo_loss": lambda **k: B.orpo_loss(LOGPS, dev(4, dtype=I32), 0.1, **k),
    "psa_rope": lambda **k: B.psa_rope(Q, IDS, **k),
    "psa_norm": lambda **k: B.psa_norm(X, W, W, residual=X, **k),
    "psa_norm_bwd": lambda **k: B.psa_norm_bwd(X, X, W, STATS, with_bias=True, workspace=WS, **k),
    "psa_embed": lambda **k: B.psa_embed(IDS, dev(9, 40), **k),
    "psa_embed_bwd": lambda **k: B.psa_embed_bwd(X, IDS, 9, workspace=WS, **k),
    "psa_ffn": lambda **k: B.psa_ffn(X, dev(40, 24), dev(40, 24), dev(24, 40), workspace=WS, **k),
    "psa_ffn_bwd": lambda **k: B.psa_ffn_bwd(X, X, dev(40, 24), dev(40, 24), dev(24, 40), (dev(6, 24), dev(6, 24)), workspace=WS, **k),
}


def flat(v):
    return [v] if isinstance(v, torch.Tensor) else [t for u in v if u is not None for t in flat(u)]


@pytest.fixture
def made(monkeypatch):
    """Addresses of the tensors allocated, with the stream that was current, and of those recorded on a stream."""
    real = B.load_library()
    current, allocated, recorded = ["current"], {}, {}

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_bytes") else (lambda *a: 0)

    @contextlib.contextmanager
    def stream_of(s):
        current.append(s)
        yield
        current.pop()

    def noted(make):
        def call(*a, **k):
            t = make(*a, **k).as_subclass(OnDevice)
            allocated[t.data_ptr()] = current[-1]
            return t
        return call
    monkeypatch.setattr(B, "load_library", Library)
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(B, "_stream", lambda s: 7 if s is None else int(s))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s, device=None: "stream %d" % s)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.cuda, "stream", stream_of)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.setdefault(t.data_ptr(), s), raising=False)
    for name in ("empty", "empty_like", "empty_strided"):
        monkeypatch.setattr(torch, name, noted(getattr(torch, name)))
    return allocated, recorded


def test_every_call_with_a_stream_is_here():
    """psa_step_host and psa_bwd_static_scratch make no results, the others no tensors."""
    names = {n for n, f in vars(B).items() if inspect.isfunction(f) and not n.startswith("_") and "stream" in inspect.signature(f).parameters}
    assert names - set(CALLS) == {"psa_plan", "psa_step_host", "psa_bwd_static_scratch", "psa_selftest_wait_expiry", "psa_selftest_bounds"}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("handle,owner", [(12, "stream 12"), (0, "default"), (1, "default")])
def test_results_belong_to_the_calls_stream_and_are_kept_for_the_current_one(name, handle, owner, made):
    allocated, recorded = made
    results = flat(CALLS[name](stream=handle))
    assert len(results) >= 1
    for t in results:
        assert allocated[t.data_ptr()] == owner and recorded[t.data_ptr()] == "current"


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream", [None, 7])
def test_results_on_the_current_stream_are_plain_ones(name, stream, made):
    allocated, recorded = made
    assert all(allocated[t.data_ptr()] == "current" for t in flat(CALLS[name](stream=stream))) and not recorded
