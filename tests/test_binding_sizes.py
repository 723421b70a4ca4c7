"""Sizes that the library takes as 32-bit numbers: a wider tensor is refused, where its size modulo 2^32 would pass.  (Tensors
of a few elements that say they have the shape stand in for those of 8 GB and more.)"""
import pytest
import torch

from paper_2410_20305_b200 import binding as B

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
WIDE = 2 ** 32 + 40      # 40 in the lower 32 bits


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)


def dev(*shape, dtype=BF):
    t = torch.zeros([40 if n == WIDE else n for n in shape], dtype=dtype)
    cls = type("Wide", (OnDevice,), {"shape": property(lambda self: torch.Size(shape)), "dim": lambda self: len(shape)})
    return t.as_subclass(cls)


@pytest.fixture
def reached(monkeypatch):
    """The library, whose calls are written down and not made (sizes of workspaces come from the real one)."""
    real, calls = B.load_library(), []

    class Library:
        def __getattr__(self, name):
            if name == "psa_status_string":
                return real.psa_status_string
            return getattr(real, name) if name.endswith("_bytes") else (lambda *a: calls.append(name) or 0)
    monkeypatch.setattr(B, "load_library", Library)
    monkeypatch.setattr(B, "_native", None)
    return calls


WS = torch.zeros(1 << 16, dtype=torch.uint8).as_subclass(OnDevice)
CALLS = {
    "psa_norm": lambda D, F: B.psa_norm(dev(6, D), dev(D), out=dev(6, D), stats=dev(2, 6, dtype=F32), stream=0),
    "psa_norm_bwd": lambda D, F: B.psa_norm_bwd(dev(6, D), dev(6, D), dev(D), dev(2, 6, dtype=F32), dx=dev(6, D), dweight=dev(D), workspace=WS,
                                                stream=0),
    "psa_embed": lambda D, F: B.psa_embed(dev(6, dtype=I32), dev(9, D), out=dev(6, D), stream=0),
    "psa_embed_bwd": lambda D, F: B.psa_embed_bwd(dev(6, D), dev(6, dtype=I32), 9, dtable=dev(9, D), workspace=WS, stream=0),
    "psa_ffn": lambda D, F: B.psa_ffn(dev(6, D), dev(D, F), dev(D, F), dev(F, D), out=dev(6, D), gate=dev(6, F), up=dev(6, F), workspace=WS,
                                      stream=0),
    "psa_ffn_bwd": lambda D, F: B.psa_ffn_bwd(dev(6, D), dev(6, D), dev(D, F), dev(D, F), dev(F, D), (dev(6, F), dev(6, F)), dx=dev(6, D),
                                              dw_gate=dev(D, F), dw_up=dev(D, F), dw_down=dev(F, D), workspace=WS, stream=0),
    "psa_rope": lambda D, F: B.psa_rope(dev(6, D, 16), dev(6, dtype=I32), out=dev(6, D, 16), stream=0),
}


@pytest.mark.parametrize("name,D,F", [(n, WIDE, 24) for n in sorted(CALLS)] + [("psa_ffn", 24, WIDE), ("psa_ffn_bwd", 24, WIDE)])
def test_a_width_beyond_32_bits_is_refused(name, D, F, reached):
    CALLS[name](40, 24)
    assert reached == [name]
    with pytest.raises(B.PsaError) as e:
        CALLS[name](D, F)
    assert e.value.code == 3 and reached == [name]
