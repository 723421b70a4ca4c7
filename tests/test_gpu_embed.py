"""psa_embed and psa_embed_bwd against the oracle in 64 bits.  The forward is one fp32 product, rounded once.  The backward
adds the n rows of an id in fp32: in runs of 32, then the runs, so at most 32 + n / 32 roundings of 2^-24 follow one another;
then one product, one addition where the gradient accumulates, and the rounding to its type."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.bfloat16, torch.float32), "f32": (torch.float32, torch.float32)}
f64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
half = lambda t: torch.finfo(t).eps / 2  # noqa: E731


def ids_of(T, vocab, seed, how):
    rng = np.random.default_rng(seed)
    if how == "text":
        return np.minimum(((vocab + 1) ** rng.random(T) - 1).astype(np.int64), vocab - 1).astype(np.int32)
    if how == "one":
        return np.full(T, vocab // 2, dtype=np.int32)
    if how == "ends":
        return rng.choice([0, vocab - 1], size=T).astype(np.int32)
    return rng.integers(0, vocab, size=T).astype(np.int32)


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def check_bwd(T, vocab, D, kind, how, accumulate=False, seed=0):
    xt, gt = TYPES[kind]
    ids, d_out = ids_of(T, vocab, seed, how), normal((T, D), seed + 1, xt)
    old = normal((vocab, D), seed + 2, gt)
    given = old.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = B.psa_embed_bwd(d_out.cuda(), torch.as_tensor(ids).cuda(), vocab, scale=1.5, dtable=given, accumulate=accumulate, status=status)
    assert got is given and int(status.item()) == 0
    ref = orc.embed_bwd(f64(d_out), ids, vocab, 1.5)
    size = orc.embed_bwd(np.abs(f64(d_out)), ids, vocab, 1.5)
    n = np.bincount(ids, minlength=vocab)[:, None]
    adds = (34 + n / 32) * 2.0 ** -24
    if accumulate:
        ref, size = ref + f64(old), size + np.abs(f64(old))
        untouched = n[:, 0] == 0
        assert torch.equal(got.cpu()[untouched], old[untouched])
    tol = half(gt) * np.abs(ref) + adds * size
    bad = np.abs(f64(got) - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(f64(got) - ref).max())


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,vocab,D", [(1, 1, 1), (1, 300, 8), (31, 5, 3), (32, 64, 16), (33, 31, 10), (65, 1000, 64), (257, 33, 130),
                                       (1000, 2000, 96), (500, 4737, 24)])
def test_gradient(T, vocab, D, kind):
    check_bwd(T, vocab, D, kind, "any", seed=T)
    check_bwd(T, vocab, D, kind, "text", accumulate=True, seed=T + 1)


@pytest.mark.parametrize("how", ["one", "ends", "text"])
@pytest.mark.parametrize("T,vocab,D", [(96, 7, 8), (2048, 151600, 8), (3333, 400, 20), (8200, 152000, 2)])
def test_gradient_of_frequent_tokens(T, vocab, D, how):
    check_bwd(T, vocab, D, "mixed", how, seed=T)


def test_wide_rows_take_every_slice():
    check_bwd(70, 40, 5001, "bf16", "any")
    check_bwd(70, 40, 4104, "f32", "any", accumulate=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,vocab,D", [(1, 1, 1), (1, 50, 4096), (3, 9, 2), (100, 77, 33), (513, 300, 72), (40, 1000, 4104)])
def test_forward(T, vocab, D, dtype):
    ids, table = ids_of(T, vocab, T, "any"), normal((vocab, D), 5, dtype)
    for scale in (1.0, D ** 0.5):
        got = B.psa_embed(torch.as_tensor(ids).cuda(), table.cuda(), scale=scale)
        ref = orc.embed_fwd(ids, f64(table), np.float32(scale))
        assert (np.abs(f64(got) - ref) <= (half(dtype) + 2.0 ** -23) * np.abs(ref)).all()


def test_bad_ids_are_reported_and_give_nothing():
    table, d_out = normal((10, 16), 1, torch.float32).cuda(), normal((6, 16), 2, torch.float32).cuda()
    ids = torch.tensor([3, -1, 10, 9, 2147483647, 0], dtype=torch.int32, device="cuda")
    for call in (lambda s: B.psa_embed(ids, table, status=s), lambda s: B.psa_embed_bwd(d_out, ids, 10, status=s)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = call(status)
        assert int(status.item()) == B.PSA_DEVSTAT_BAD_TARGET
        call(None)
        if got.shape[0] == 6:
            assert not got[[1, 2, 4]].any() and torch.equal(got[[0, 3, 5]], table[[3, 9, 0]])
        else:
            want = torch.zeros_like(table)
            want[[3, 9, 0]] = d_out[[0, 3, 5]]
            assert torch.equal(got, want)


def test_no_tokens():
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    assert B.psa_embed(ids, torch.ones((4, 8), device="cuda")).shape == (0, 8)
    dtable = torch.full((40, 8), 3.0, device="cuda")
    B.psa_embed_bwd(torch.empty((0, 8), device="cuda"), ids, 40, dtable=dtable, accumulate=True)
    assert (dtable == 3).all()
    B.psa_embed_bwd(torch.empty((0, 8), device="cuda"), ids, 40, dtable=dtable)
    assert not dtable.any()


def test_the_same_bits_again_and_in_a_graph():
    ids = torch.as_tensor(ids_of(4000, 500, 3, "text")).cuda()
    d_out = normal((4000, 264), 4, torch.bfloat16).cuda()
    want = B.psa_embed_bwd(d_out, ids, 500, dtype=torch.float32)
    for _ in range(3):
        assert torch.equal(want, B.psa_embed_bwd(d_out, ids, 500, dtype=torch.float32))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.psa_embed_bwd(d_out, ids, 500, dtype=torch.float32)
    ids.copy_(ids.flip(0))
    want = B.psa_embed_bwd(d_out, ids, 500, dtype=torch.float32)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want, got)
