"""The status word of a layer: a bounded wait that gives up in one of its calls is reported there and nowhere else, so every
call that can report has to get it.  Checked without a GPU: the binding's calls are replaced by stand-ins that return
zeros of the right shape and write down what they were given."""
import inspect

import numpy as np
import pytest
import torch

from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import layer as L

T, HQ, HKV, D, FFN = 6, 2, 1, 64, 24
HID = HQ * D
BF = torch.bfloat16


class Binding:
    """The calls that layers make; `given` holds the status of each one that takes a status."""

    def __init__(self):
        self.given = []

    def __getattr__(self, name):
        def call(*a, **k):
            if "status" in inspect.signature(getattr(B, name)).parameters:
                self.given.append((name, k.get("status")))
            like = torch.zeros_like
            if name == "psa_plan":
                return type("Plan", (), {"bwd_workspace_bytes": 256})()
            if name == "psa_position_ids":
                return np.zeros(T, dtype=np.int32)
            if name == "psa_rope":
                return k["out"]
            if name == "psa_fwd":
                return like(a[1]), torch.zeros(HQ, T)
            if name == "psa_bwd":
                return like(a[2]), like(a[3]), like(a[4])
            if name == "psa_norm":
                return (like(a[0]), torch.zeros(2, T)) + ((like(a[0]),) if k.get("residual") is not None else ())
            if name == "psa_norm_bwd":
                return like(a[0]), like(a[2]), None
            if name == "psa_ffn":
                return like(a[0]), (torch.zeros(T, FFN, dtype=BF),) * 2
            assert name == "psa_ffn_bwd", name
            return tuple(like(t) for t in a[1:5])
        return call


def weights():
    z = lambda *s: torch.zeros(*s, dtype=BF)  # noqa: E731
    return {"norm1": z(HID), "norm2": z(HID), "wq": z(HID, HID), "wk": z(HID, HKV * D), "wv": z(HID, HKV * D), "wo": z(HID, HID),
            "w_gate": z(HID, FFN), "w_up": z(HID, FFN), "w_down": z(FFN, HID)}


@pytest.mark.parametrize("status", [None, torch.zeros(1, dtype=torch.int32)])
def test_every_call_of_a_decoder_layer_gets_its_status(status, monkeypatch):
    fake = Binding()
    monkeypatch.setattr(L, "B", fake)
    layer = L.DecoderLayer(([0, T], [2], [2], [2]), HQ, HKV, D, "cpu", status=status)
    x, w = torch.zeros(T, HID, dtype=BF), weights()
    _, out, saved = layer.forward(x, w)
    layer.forward(x, w, out)
    layer.backward(x, x, w, saved)
    assert all(s is status for _, s in fake.given)
    assert [n for n, _ in fake.given] == ["psa_fwd", "psa_ffn"] * 2 + ["psa_ffn_bwd", "psa_norm_bwd", "psa_bwd", "psa_norm_bwd"]


@pytest.mark.parametrize("status", [None, torch.zeros(1, dtype=torch.int32)])
def test_every_call_of_an_attention_layer_gets_its_status(status, monkeypatch):
    fake = Binding()
    monkeypatch.setattr(L, "B", fake)
    layer = L.AttentionLayer(([0, T], [2], [2], [2]), HQ, HKV, D, "cpu", status=status)
    x, w = torch.zeros(T, HID, dtype=BF), weights()
    ws = [w[k] for k in ("wq", "wk", "wv", "wo")]
    _, saved = layer.forward(x, *ws)
    layer.backward(x, *ws, saved, x)
    assert fake.given == [("psa_fwd", status), ("psa_bwd", status)]
