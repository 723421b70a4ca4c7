"""A decoder layer with a status word: its calls run as without one, and none of its waits gives up."""
import pytest
import torch

from paper_2410_20305_b200 import workloads as wl
from paper_2410_20305_b200.layer import DecoderLayer

pytestmark = pytest.mark.gpu


def test_a_layer_reports_into_its_status_word_and_computes_the_same():
    pack = wl.pack_from_lengths("status", [(90, 40, 60), (0, 33, 20)], 4, 2, 64)
    lengths = (pack.cu_seqlens, pack.prefix_len, pack.chosen_len, pack.rejected_len)
    T, hid, ffn = pack.total_tokens, 256, 520
    shapes = {"norm1": (hid,), "norm2": (hid,), "wq": (hid, hid), "wk": (hid, 128), "wv": (hid, 128), "wo": (hid, hid),
              "w_gate": (hid, ffn), "w_up": (hid, ffn), "w_down": (ffn, hid)}
    w = {k: wl.bf16_normal(s, i, 0.06).cuda() for i, (k, s) in enumerate(shapes.items())}
    x, d = wl.bf16_normal((T, hid), 20).cuda(), wl.bf16_normal((T, hid), 21).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = []
    for word in (None, status):
        layer = DecoderLayer(lengths, 4, 2, 64, "cuda", status=word)
        mid, delta, saved = layer.forward(x, w)
        _, g = layer.backward(d, d, w, saved)
        got.append([mid, delta, g["w_gate"], g["w_up"], g["w_down"], g["norm2"], g["wo"]])     # (what dq's unordered adds do not reach)
    assert int(status.item()) == 0
    assert all(torch.equal(a, b) for a, b in zip(*got))
