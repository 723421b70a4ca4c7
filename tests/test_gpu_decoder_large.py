"""The normalisation, the embedding and the feed-forward block where an element's offset passes 32 bits, where rows that start
anywhere are replaced in place, and with sizes that take every number of parts of a split sum.

A row's result depends on that row alone, so the rows of a long tensor must have the bits of a call with just these rows;
sums over tokens have few terms that are not 0, or whole numbers whose sums fp32 holds, and are exact."""
import pytest
import torch

from paper_2410_20305_b200 import binding as B
from test_gpu_embed import check_bwd as check_embed_bwd
from test_gpu_ffn import test_whole_numbers_are_exact as whole_numbers_are_exact

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def rows_to_look_at(T, width):
    at = 2 ** 31 // width
    return torch.tensor([0, 1, at - 1, at, at + 1, 2 * at % T, T - 2, T - 1], device="cuda")


# both where a row is whole vectors and where it starts anywhere (a multiple of 8 rows from the first one keeps its place)
@pytest.mark.parametrize("D", [8200, 8196])
def test_norm_of_more_than_2_31_elements(D):
    T = 262200
    assert T * D > 2 ** 31
    x, g = (torch.empty((T, D), dtype=BF, device="cuda").normal_() for _ in range(2))
    w = torch.empty(D, dtype=BF, device="cuda").normal_()
    g[:-1] = 0
    out, stats = B.psa_norm(x, w, w)
    dx, dw, db = B.psa_norm_bwd(g, x, w, stats, with_bias=True)
    few = rows_to_look_at(T, D)
    for first in (few // 8 * 8).tolist():
        part = slice(first, min(first + 8, T))
        po, ps = B.psa_norm(x[part].clone(), w, w)
        assert torch.equal(out[part], po) and torch.equal(stats[:, part], ps)
    part = slice((T - 1) // 8 * 8, T)
    pdx, pdw, pdb = B.psa_norm_bwd(g[part].clone(), x[part].clone(), w, ps, with_bias=True)
    assert torch.equal(dx[part], pdx) and torch.equal(dw, pdw) and torch.equal(db, pdb)
    assert not dx[:-1].any() and torch.equal(db, g[-1])


def test_embedding_from_a_table_of_more_than_2_31_elements():
    V, D = 16_000_000, 136
    assert V * D > 2 ** 31
    table = torch.empty((V, D), dtype=BF, device="cuda").normal_()
    ids = rows_to_look_at(V, D).int()
    out = B.psa_embed(ids, table, 2.0)
    assert torch.equal(out, table[ids.long()] * 2)
    grad = B.psa_embed_bwd(out, ids, V, 0.5)
    want = table.zero_()
    want[ids.long()] = out * 0.5
    assert torch.equal(grad, want)


def test_embedding_of_more_than_2_31_elements():
    T, V, D = 2 ** 24, 50, 136
    assert T * D > 2 ** 31
    ids = torch.arange(T, device="cuda", dtype=torch.int32) * 7 % V
    table = torch.empty((V, D), dtype=BF, device="cuda").normal_()
    out = B.psa_embed(ids, table)
    assert torch.equal(out[-1000:], table[ids[-1000:].long()]) and torch.equal(out[2 ** 31 // D - 9:][:20], table[ids[2 ** 31 // D - 9:][:20].long()])
    grad = B.psa_embed_bwd(out.fill_(1), ids, V, dtype=F32)
    assert torch.equal(grad, torch.bincount(ids, minlength=V).float()[:, None].expand(V, D))


def test_ffn_of_more_than_2_31_elements():
    T, D, F = 524_000, 64, 4104
    assert T * F > 2 ** 31
    some = lambda shape, share: (torch.randint(-1, 2, shape, device="cuda") * (torch.rand(shape, device="cuda") < share)).to(BF)  # noqa: E731
    x, wu, wd, g = some((T, D), 0.5), some((D, F), 0.5), some((F, D), 0.05), some((T, D), 0.5)
    x[:, 0] = 1
    wg = torch.zeros((D, F), dtype=BF, device="cuda")
    wg[0] = 64                                       # silu(64) is 64 to the last bit: all products and sums are exact
    few = torch.cat([rows_to_look_at(T, F), torch.arange(T - 300, T - 2, device="cuda")])
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[few] = False
    g[rest] = 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, saved = B.psa_ffn(x, wg, wu, wd, status=status)
    grads = B.psa_ffn_bwd(g, x, wg, wu, wd, saved, status=status)
    assert int(status.item()) == 0
    r = lambda a: a.float().to(BF)  # noqa: E731
    xs, gs, wgd, wud, wdd = (t.double() for t in (x[few], g[few], wg, wu, wd))
    up = xs @ wud
    h, dh = 64 * up, gs @ wdd.t()
    d_gate, d_up = r(dh * up).double(), r(dh * 64).double()
    for got, want in ((saved[0][few], torch.full_like(h, 64)), (saved[1][few], up), (out[few], h @ wdd),
                      (grads[0][few], d_gate @ wgd.t() + d_up @ wud.t())):
        assert torch.equal(got, r(want))
    unique = torch.unique(few, return_inverse=True)[1]      # a row named twice counts once
    once = torch.zeros(len(few), 1, dtype=torch.float64, device="cuda")
    seen = set()
    for i, u in enumerate(unique.tolist()):
        once[i] = float(u not in seen)
        seen.add(u)
    for got, want in zip(grads[1:], ((xs * once).t() @ d_gate, (xs * once).t() @ d_up, (h * once).t() @ gs)):
        assert torch.equal(got, r(want))
    assert not grads[0][rest].any()


# parts of K: 2 of the second product, 2 of dX alone, 2 of the last products in one launch, and the weights' gradients without dX
@pytest.mark.parametrize("T,D,F", [(40, 4096, 2056), (300, 4096, 4104), (1, 64, 1032), (400, 64, 4104)])
def test_every_number_of_parts(T, D, F):
    whole_numbers_are_exact(T, D, F)


@pytest.mark.parametrize("T,D,dtype", [(3000, 1237, BF), (2999, 2047, BF), (1500, 2047, F32), (3001, 300, BF), (900, 5001, BF),
                                       (40, 16383, F32)])
def test_rows_that_start_anywhere_in_place(T, D, dtype):
    x, r, g = (torch.empty((T, D), device="cuda").normal_().to(dtype) for _ in range(3))
    w = torch.empty(D, device="cuda").normal_().to(dtype)
    out, stats, total = B.psa_norm(x, w, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    got, stats2, total2 = B.psa_norm(x2, w, w, residual=r2, out=x2, total=r2)
    assert got is x2 and torch.equal(out, x2) and torch.equal(total, r2) and torch.equal(stats, stats2)
    dx, dw, db = B.psa_norm_bwd(g, total, w, stats, d_total=r, with_bias=True)
    for place in range(3):
        given = [g.clone(), total.clone(), r.clone()]
        dx2, dw2, db2 = B.psa_norm_bwd(given[0], given[1], w, stats, d_total=given[2], with_bias=True, dx=given[place])
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("D", [201, 1237, 4095])
def test_a_bad_row_beside_rows_that_share_its_vectors(D):
    x, g = (torch.empty((2000, D), device="cuda").normal_().to(BF) for _ in range(2))
    w = torch.ones(D, dtype=BF, device="cuda")
    clean, stats = B.psa_norm(x, w, w)
    dx, _, _ = B.psa_norm_bwd(g, x, w, stats, with_bias=True)
    bad = torch.zeros(2000, dtype=torch.bool, device="cuda")
    bad[3::50] = True
    x2, g2 = x.clone(), g.clone()
    x2[bad], g2[bad] = float("nan"), float("inf")
    out, stats2 = B.psa_norm(x2, w, w)
    dx2, _, _ = B.psa_norm_bwd(g2, x2, w, stats2, with_bias=True)
    assert torch.equal(out[~bad], clean[~bad]) and torch.equal(dx2[~bad], dx[~bad])
    assert out[bad].isnan().all() and dx2[bad].isnan().all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,D", [(701, 4099), (35, 9001), (100, 2305)])
def test_ranges_of_absent_ids_in_wide_rows_that_start_anywhere(V, D, dtype):
    ids = torch.tensor([0, 1, 7, 15, 16, 33, V - 2], dtype=torch.int32, device="cuda")
    d_out = torch.empty((7, D), device="cuda").normal_().to(BF)
    padded = torch.full((V + 1, D), 5.0, dtype=dtype, device="cuda")
    B.psa_embed_bwd(d_out, ids, V, dtable=padded[:V])
    # (V - 2 is 33 again in one case: the fp32 sum of two values, in either order, rounded once more)
    want = torch.zeros((V, D), device="cuda").index_add_(0, ids.long(), d_out.float()).to(dtype)
    assert torch.equal(padded[:V], want) and (padded[V:] == 5).all()


# (runs of 32 sorted tokens; test_gpu_embed's tensors are short enough for runs of 16)
@pytest.mark.parametrize("kind", ["bf16", "mixed", "f32"])
@pytest.mark.parametrize("T,V,D,how", [(9000, 3000, 1001, "text"), (20000, 64, 424, "any"), (8400, 5, 1024, "one")])
def test_gradient_in_long_runs(T, V, D, how, kind):
    check_embed_bwd(T, V, D, kind, how, accumulate=D == 424, seed=T)
