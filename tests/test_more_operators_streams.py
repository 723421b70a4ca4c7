"""Which stream the results of operators.py's calls are allocated on, as test_binding_streams.py checks it for binding.py's."""
import inspect

import pytest
import torch
from test_binding_streams import dev, flat, made  # noqa: F401  (the fixture)

from paper_2410_20305_b200 import operators as O

F32, I32, I64, U8 = torch.float32, torch.int32, torch.int64, torch.uint8
X, W, IDS, WS = dev(6, 40), dev(40), dev(6, dtype=I32), dev(1 << 22, dtype=U8)
CALLS = {
    "dpo_linear_logp": lambda **k: O.dpo_linear_logp(X, dev(9, 40), IDS, IDS, 3, workspace=WS, **k),
    "dpo_linear_logp_bwd": lambda **k: O.dpo_linear_logp_bwd(dev(3, dtype=F32), X, dev(9, 40), dev(6, dtype=F32), IDS, IDS, workspace=WS, **k),
    "psa_rotary": lambda **k: O.psa_rotary(dev(6, 2, 64), dev(6, 1, 64), IDS, dev(20, dtype=I64), **k),
    "psa_block_norm": lambda **k: O.psa_block_norm(X, X, W, W, W, W, W, **k),
    "psa_block_norm_bwd": lambda **k: O.psa_block_norm_bwd(X, X, X, W, dev(4, 6, dtype=F32), W, W, W, with_bias=True, workspace=WS, **k),
}


def test_every_call_with_a_stream_is_here():
    names = {n for n, f in vars(O).items() if inspect.isfunction(f) and not n.startswith("_") and "stream" in inspect.signature(f).parameters}
    assert names == set(CALLS)


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("handle,owner", [(12, "stream 12"), (0, "default"), (1, "default")])
def test_results_belong_to_the_calls_stream_and_are_kept_for_the_current_one(name, handle, owner, made):  # noqa: F811
    allocated, recorded = made
    results = flat(CALLS[name](stream=handle))
    assert len(results) >= 2
    for t in results:
        assert allocated[t.data_ptr()] == owner and recorded[t.data_ptr()] == "current"


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream", [None, 7])
def test_results_on_the_current_stream_are_plain_ones(name, stream, made):  # noqa: F811
    allocated, recorded = made
    assert all(allocated[t.data_ptr()] == "current" for t in flat(CALLS[name](stream=stream))) and not recorded
