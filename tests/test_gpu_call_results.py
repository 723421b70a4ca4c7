"""Results that a call on a stream other than the current one allocates: no block that the current stream's work may still use,
and none that is given away while the current stream's work on the result is under way."""
import pytest
import torch

from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
T, D = 5000, 4000        # 40 MB a tensor


def normal(*shape, dtype=BF):
    return torch.randn(*shape, device="cuda").to(dtype)


def flat(v):
    return [v] if isinstance(v, torch.Tensor) else [t for u in v if u is not None for t in flat(u)]


def calls():
    x, w, ids = normal(T, D), normal(D), torch.randint(0, T, (T,), device="cuda", dtype=torch.int32)
    wg, wd = normal(D, 64), normal(64, D)
    stats = B.psa_norm(x, w)[1]
    saved = B.psa_ffn(x, wg, wg, wd)[1]
    return {"psa_norm": lambda **k: B.psa_norm(x, w, residual=x, **k), "psa_norm_bwd": lambda **k: B.psa_norm_bwd(x, x, w, stats, **k),
            "psa_embed": lambda **k: B.psa_embed(ids, x, **k), "psa_embed_bwd": lambda **k: B.psa_embed_bwd(x, ids, T, **k),
            "psa_ffn": lambda **k: B.psa_ffn(x, wg, wg, wd, **k), "psa_ffn_bwd": lambda **k: B.psa_ffn_bwd(x, x, wg, wg, wd, saved, **k),
            "psa_rope": lambda **k: B.psa_rope(x.view(T, -1, 80), ids, **k)}


@pytest.mark.parametrize("name", ["psa_norm", "psa_norm_bwd", "psa_embed", "psa_embed_bwd", "psa_ffn", "psa_ffn_bwd", "psa_rope"])
def test_blocks_of_the_current_stream_are_not_taken_and_results_are_kept_for_it(name):
    call = calls()[name]
    want = flat(call())
    side = torch.cuda.Stream()
    a = normal(8192, 8192)
    (a @ a).add_(1)                            # (a kernel's first launch loads it, which takes as long as the work below)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):              # enough blocks that no allocation below waits for the device
        spare = [torch.empty((T, D), dtype=BF, device="cuda") for _ in range(8)]
    del spare
    freed = [torch.empty((T, D), dtype=BF, device="cuda") for _ in range(4)]
    for _ in range(40):
        a @ a                                  # the current stream is busy, and may still use what is dropped now
    taken = {t.data_ptr() for t in freed}
    del freed
    got = flat(call(stream=side.cuda_stream))
    assert not taken & {t.data_ptr() for t in got}
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(want, got))
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(100):
        a @ a                                  # 60 ms and more
    large = [t for t in got if t.numel() == T * D]
    for t in large:
        t.add_(1)
    kept = {t.data_ptr() for t in large}
    assert kept
    done = torch.cuda.Event()
    done.record()
    del got, large, t
    with torch.cuda.stream(side):
        new = [torch.empty((T, D), dtype=BF, device="cuda") for _ in range(4)]
    at = {t.data_ptr() for t in new}
    assert done.query() or not kept & at       # (done: the host was held up for longer than that, and they may be)
    torch.cuda.synchronize()
