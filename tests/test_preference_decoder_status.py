"""The status word of a PreferenceDecoder and its layers: every call that can report a wait that gave up gets it.  Checked
without a GPU: the calls are replaced by stand-ins that return zeros of the right shape and write down what they were given."""
import inspect

import numpy as np
import pytest
import torch

from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import layer as L
from paper_2410_20305_b200 import operators as O

T, HQ, HKV, D, FFN, V = 6, 2, 1, 64, 24, 9
HID = HQ * D
BF = torch.bfloat16


def results(name, a, k):
    like = torch.zeros_like
    z = lambda *s: torch.zeros(*s, dtype=BF)  # noqa: E731
    return {
        "psa_plan": lambda: type("Plan", (), {"bwd_workspace_bytes": 256})(),
        "psa_position_ids": lambda: np.zeros(T, dtype=np.int32),
        "psa_rope": lambda: k["out"],
        "psa_rotary": lambda: (k["q_out"], k["k_out"]),
        "psa_rotary_frequencies": lambda: (torch.zeros(D // 2, dtype=torch.int64), 1.0),
        "psa_fwd": lambda: (like(a[1]), torch.zeros(HQ, T)),
        "psa_bwd": lambda: (like(a[2]), like(a[3]), like(a[4])),
        "psa_norm": lambda: (like(a[0]), torch.zeros(2, T)),
        "psa_norm_bwd": lambda: (like(a[0]), like(a[2]), None),
        "psa_block_norm": lambda: (like(a[0]), like(a[0]), torch.zeros(4, T)),
        "psa_block_norm_bwd": lambda: (like(a[0]), like(a[0]), like(a[3]), None, *(
            None if p is None else like(p) for p in (k["post_weight"], None, k["gate"]))),
        "psa_ffn": lambda: (like(a[0]), (z(T, FFN), z(T, FFN))),
        "psa_ffn_bwd": lambda: tuple(like(t) for t in a[1:5]),
        "psa_embed": lambda: z(T, HID),
        "psa_embed_bwd": lambda: z(V, HID),
        "dpo_linear_logp": lambda: (torch.zeros(2), torch.zeros(T)),
        "dpo_linear_logp_bwd": lambda: (like(a[1]), like(a[2])),
    }[name]()


class Calls:
    def __init__(self, module, given):
        self.module, self.given = module, given

    def __getattr__(self, name):
        def call(*a, **k):
            if "status" in inspect.signature(getattr(self.module, name)).parameters:
                self.given.append((name, k.get("status")))
            return results(name, a, k)
        return call


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("status", [None, torch.zeros(1, dtype=torch.int32)])
def test_every_call_of_a_preference_decoder_gets_its_status(status, tied, monkeypatch):
    given = []
    monkeypatch.setattr(L, "B", Calls(B, given))
    monkeypatch.setattr(L, "O", Calls(O, given))
    z = lambda *s: torch.zeros(*s, dtype=BF)  # noqa: E731
    w = {"norm1": z(HID), "norm2": z(HID), "wq": z(HID, HID), "wk": z(HID, HKV * D), "wv": z(HID, HKV * D), "wo": z(HID, HID),
         "w_gate": z(HID, FFN), "w_up": z(HID, FFN), "w_down": z(FFN, HID), "post1": z(HID), "gate2": z(HID)}
    params = {"table": z(V, HID), "layers": [w, dict(w)], "final": z(HID), "head": None if tied else z(V, HID)}
    decoder = L.PreferenceDecoder(([0, T], [2], [2], [2]), HQ, HKV, D, "cpu", status=status, rotary=L.Rotary(D, device="cpu"))
    ids = torch.zeros(T, dtype=torch.int32)
    labels = (ids, ids, None, None, None)
    logps, saved = decoder.forward(params, ids, labels)
    grads = decoder.backward(logps, params, ids, labels, saved)
    assert all(s is status for _, s in given)
    forward = ["psa_embed"] + ["psa_fwd", "psa_ffn"] * 2 + ["dpo_linear_logp"]
    layer = ["psa_ffn_bwd", "psa_block_norm_bwd", "psa_bwd"]
    assert [n for n, _ in given] == forward + ["dpo_linear_logp_bwd", "psa_block_norm_bwd"] + layer + ["psa_block_norm_bwd"] + layer + [
        "psa_norm_bwd", "psa_embed_bwd"]
    assert [set(g) for g in grads["layers"]] == [set(w)] * 2 and (grads["head"] is None) == tied
