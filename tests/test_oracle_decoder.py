"""Pins of the oracle's normalisation, embedding and feed-forward block: the same written with torch's library functions in
float64 and differentiated by autograd, and by central differences."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import psa_oracle as orc


def _t(a):
    return torch.tensor(a, dtype=torch.float64, requires_grad=True)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("hidden", [1, 2, 7, 32])
def test_norm_matches_library_and_autograd(rms, hidden):
    rng = np.random.default_rng(hidden)
    x, w, b, g = rng.normal(size=(5, hidden)) * 3 + 1, rng.normal(size=hidden), rng.normal(size=hidden), rng.normal(size=(5, hidden))
    tx, tw, tb = _t(x), _t(w), _t(b)
    out, mean, rstd = orc.norm_fwd(x, w, None if rms else b, 1e-3, rms)
    ref = F.rms_norm(tx, (hidden,), tw, 1e-3) if rms else F.layer_norm(tx, (hidden,), tw, tb, 1e-3)
    assert np.allclose(out, ref.detach().numpy(), atol=1e-12)
    (ref * torch.tensor(g)).sum().backward()
    dx, dw, db = orc.norm_bwd(g, x, w, 1e-3, rms)
    assert np.allclose(dx, tx.grad.numpy(), atol=1e-11) and np.allclose(dw, tw.grad.numpy(), atol=1e-11)
    if not rms:
        assert np.allclose(db, tb.grad.numpy(), atol=1e-12) and np.allclose(mean, x.mean(1))
    assert np.allclose(rstd, 1 / np.sqrt((x ** 2).mean(1) - mean ** 2 + 1e-3))


def test_embedding_matches_library_and_autograd():
    rng = np.random.default_rng(0)
    ids, table, g = rng.integers(0, 6, size=20), rng.normal(size=(9, 4)), rng.normal(size=(20, 4))
    tt = _t(table)
    ref = F.embedding(torch.tensor(ids), tt) * 2.5
    (ref * torch.tensor(g)).sum().backward()
    assert np.allclose(orc.embed_fwd(ids, table, 2.5), ref.detach().numpy())
    assert np.allclose(orc.embed_bwd(g, ids, 9, 2.5), tt.grad.numpy())
    assert not orc.embed_fwd([9, -1], table).any() and not orc.embed_bwd(g[:2], [9, -1], 9).any()


def test_feed_forward_matches_library_autograd_and_differences():
    rng = np.random.default_rng(1)
    shapes = [(5, 6), (6, 8), (6, 8), (8, 6)]
    args = [rng.normal(size=s) for s in shapes]
    g = rng.normal(size=(5, 6))
    ts = [_t(a) for a in args]
    ref = (F.silu(ts[0] @ ts[1]) * (ts[0] @ ts[2])) @ ts[3]
    (ref * torch.tensor(g)).sum().backward()
    assert np.allclose(orc.ffn_fwd(*args)[0], ref.detach().numpy(), atol=1e-12)
    grads = orc.ffn_bwd(g, *args)
    for got, t in zip(grads, ts):
        assert np.allclose(got, t.grad.numpy(), atol=1e-11)
    step = 1e-5
    for k, at in ((0, (2, 3)), (1, (1, 5)), (2, (4, 0)), (3, (7, 2))):
        loss = []
        for sign in (1, -1):
            moved = [a.copy() for a in args]
            moved[k][at] += sign * step
            loss.append((orc.ffn_fwd(*moved)[0] * g).sum())
        assert abs((loss[0] - loss[1]) / (2 * step) - grads[k][at]) < 1e-6
