"""dpo_linear_logp and dpo_linear_logp_bwd with many labels: responses of millions of tokens, and forks by the hundred and by the million."""
import numpy as np
import pytest
import torch

from paper_2410_20305_b200 import operators as O
from test_gpu_linear_logp import both, compare, inputs

pytestmark = pytest.mark.gpu

i32s = lambda n, v: torch.full((n,), v, dtype=torch.int32, device="cuda")  # noqa: E731


def test_a_response_of_more_than_2_23_tokens():
    """Terms a little below 0: each is -1 and nearly a whole unit of the fixed-point rest."""
    n = (1 << 23) + (1 << 22)
    hidden = torch.ones((n, 8), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((2, 8), dtype=torch.bfloat16, device="cuda")
    table[1] = 1.0
    out, lse = O.dpo_linear_logp(hidden, table, i32s(n, 1), i32s(n, 0), 1)
    term = -np.log1p(np.exp(-8.0))
    # a term: an exponential's 2^-16 as in test_gpu_linear_logp.py, half a unit of 2^-40; the sum rounded once
    assert abs(float(out[0]) / (n * term) - 1) <= 2.0 ** -16 + 2.0 ** -41 / -term + 2.0 ** -24
    assert bool(((lse - (8.0 - term)).abs() <= 2.0 ** -16).all())


def test_a_response_of_as_many_tokens_as_there_may_be():
    """2^24 rows and as many forks in one response."""
    n = 1 << 24
    hidden = torch.ones((n, 8), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((2, 8), dtype=torch.bfloat16, device="cuda")
    table[1] = 1.0
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    out, lse = O.dpo_linear_logp(hidden, table, i32s(n, 1), i32s(n, 0), 1, rows, i32s(n, 1), i32s(n, 0))
    term = -np.log1p(np.exp(-8.0))
    assert abs(float(out[0]) / (2 * n * term) - 1) <= 2.0 ** -16 + 2.0 ** -41 / -term + 2.0 ** -24
    assert bool(((lse - (8.0 - term)).abs() <= 2.0 ** -16).all())


@pytest.mark.parametrize("n_rows,n_forks,live", [(5, 700, 0.5), (300, 2000, 0.5), (1, 300, 0.0), (40, 90, 1.0)])
def test_many_forks_on_a_row(n_rows, n_forks, live):
    hidden, table, targets, seg, forks, coef = inputs(n_rows, 264, 513, n_forks, live=live, n_segments=9, n_forks=n_forks)
    *got, status = both(hidden, table, targets, seg, forks, coef)
    assert status == 0
    compare(hidden, table, targets, seg, forks, coef, 1.0, got)
    again = both(hidden, table, targets, seg, forks, coef)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def seconds(call):
    call()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    got = call()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) * 1e-3, got


def test_time_grows_with_the_number_of_forks_not_with_its_square():
    """A million labels as forks of as many rows, against the same labels as the rows' own.  (Looking through all forks for each
    takes a hundred times as long.)"""
    n, width, vocab = 1 << 20, 8, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    hidden = torch.randn((n, width), generator=gen, device="cuda").to(torch.bfloat16)
    table = torch.randn((vocab, width), generator=gen, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.randint(0, 7, (n,), generator=gen, device="cuda", dtype=torch.int32)
    rows = torch.randperm(n, generator=gen, device="cuda").to(torch.int32)
    coef = torch.randn(7, generator=gen, device="cuda")
    at = rows.long()
    own = (y, g)
    forked = (i32s(n, 0), i32s(n, -1), rows, y[at].contiguous(), g[at].contiguous())
    results = {}
    for name, labels in (("own", own), ("forked", forked)):
        t, (out, lse) = seconds(lambda: O.dpo_linear_logp(hidden, table, *labels[:2], 7, *labels[2:]))
        u, (dh, dw) = seconds(lambda: O.dpo_linear_logp_bwd(coef, hidden, table, lse, *labels))
        results[name] = (t, u, out, lse, dh)
        print(name, "forward %.1f ms, backward %.1f ms" % (1e3 * t, 1e3 * u))
    a, b = results["own"], results["forked"]
    assert b[0] <= 10 * a[0] and b[1] <= 10 * a[1], (a[:2], b[:2])
    # (each label's own arithmetic is the same)
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])
