"""The decoder's operators called from two host threads at once, each on a stream of its own."""
import threading

import pytest
import torch

from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_norm_gradients_of_two_widths_at_once():
    """Both widths run the same kernel with different amounts of shared memory."""
    sets = []
    for T, D in ((300, 2816), (400, 8192)):
        x, g, w = (torch.randn(s, device="cuda").to(BF) for s in ((T, D), (T, D), (D,)))
        stats = B.psa_norm(x, w, w)[1]
        sets.append((g, x, w, stats, B.psa_norm_bwd(g, x, w, stats, d_total=g, with_bias=True)))
    torch.cuda.synchronize()
    wrong = []

    def work(first):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for i in range(300):
                g, x, w, stats, want = sets[(first + i) % 2]
                try:
                    got = B.psa_norm_bwd(g, x, w, stats, d_total=g, with_bias=True)
                    if not all(torch.equal(a, b) for a, b in zip(want, got)):
                        wrong.append("call %d: other bits" % i)
                except B.PsaError as e:
                    wrong.append("call %d: %s" % (i, e))
        stream.synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:5]
