"""Status words of the decoder's operators that lie on another GPU than the call: kernels add to them, so they are refused as
the other tensors are.  (Host tensors that say where they are stand in for those of two GPUs.)"""
import pytest
import torch

from paper_2410_20305_b200 import binding as B

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def dev(*shape, dtype=BF, gpu=0):
    cls = type("OnDevice", (torch.Tensor,), {"is_cuda": property(lambda self: True), "device": property(lambda self: torch.device("cuda", gpu))})
    return torch.zeros(*shape, dtype=dtype).as_subclass(cls)


@pytest.fixture
def reached(monkeypatch):
    """The library, whose calls are written down and not made (sizes of workspaces come from the real one)."""
    real, calls = B.load_library(), []

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_bytes") else (lambda *a: calls.append(name) or 0)
    monkeypatch.setattr(B, "load_library", Library)
    monkeypatch.setattr(B, "_native", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return calls


WS = dev(1 << 16, dtype=torch.uint8)
X, W, IDS, WG, WD = dev(6, 40), dev(40), dev(6, dtype=I32), dev(40, 24), dev(24, 40)
CALLS = {
    "psa_norm_bwd": lambda s: B.psa_norm_bwd(X, X, W, dev(2, 6, dtype=F32), dx=dev(6, 40), dweight=dev(40), workspace=WS, status=s, stream=0),
    "psa_embed": lambda s: B.psa_embed(IDS, X, out=dev(6, 40), status=s, stream=0),
    "psa_embed_bwd": lambda s: B.psa_embed_bwd(X, IDS, 9, dtable=dev(9, 40), workspace=WS, status=s, stream=0),
    "psa_ffn": lambda s: B.psa_ffn(X, WG, WG, WD, out=dev(6, 40), gate=dev(6, 24), up=dev(6, 24), workspace=WS, status=s, stream=0),
    "psa_ffn_bwd": lambda s: B.psa_ffn_bwd(X, X, WG, WG, WD, (dev(6, 24), dev(6, 24)), dx=dev(6, 40), dw_gate=dev(40, 24), dw_up=dev(40, 24),
                                           dw_down=dev(24, 40), workspace=WS, status=s, stream=0),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_status_word_on_another_gpu_is_refused(name, reached):
    CALLS[name](dev(1, dtype=I32))
    CALLS[name](None)
    CALLS[name](dev(0, dtype=I32, gpu=1))      # an empty tensor is no status word
    assert reached == [name] * 3
    with pytest.raises(ValueError, match="status"):
        CALLS[name](dev(1, dtype=I32, gpu=1))
    assert reached == [name] * 3
