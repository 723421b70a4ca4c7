"""psa_block_norm_bwd in place, where what is written over an input is not finite: the results are those of outputs that lie apart; and
how psa_block_norm rounds the scaled residual."""
import pytest
import torch

from paper_2410_20305_b200 import operators as O

pytestmark = pytest.mark.gpu


def normal(shape, seed, dtype, mean=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") + mean).to(dtype)


@pytest.mark.parametrize("T,D,dtype", [(300, 12288, torch.bfloat16), (300, 8200, torch.bfloat16), (150, 9001, torch.float32), (200, 8192, torch.bfloat16),
                                       (300, 4096, torch.bfloat16), (300, 1237, torch.bfloat16)])
def test_a_gradient_of_the_residual_that_overflows_over_an_input(T, D, dtype):
    """residual_scale takes d_residual out of the type's range; dx does not depend on it."""
    x, res, d_out, d_total = (normal((T, D), k, dtype) for k in range(4))
    w, post, gate = (normal((D,), 5 + k, dtype, mean=1.0) for k in range(3))
    _, total, stats = O.psa_block_norm(x, res, w, post_weight=post, gate=gate, rms=True)
    kw = dict(post_weight=post, gate=gate, rms=True, residual_scale=3e38)
    want = O.psa_block_norm_bwd(d_out.clone(), x, total.clone(), w, stats, d_total=d_total.clone(), **kw)
    torch.cuda.synchronize()
    assert want[1].isinf().any() and not want[0].isnan().any()
    for place in ("d_out", "total", "d_total"):
        t = {"d_out": d_out.clone(), "total": total.clone(), "d_total": d_total.clone()}
        got = O.psa_block_norm_bwd(x=x, weight=w, stats=stats, d_residual=t[place], **t, **kw)
        torch.cuda.synchronize()
        same = [a is b is None or bool(((a == b) | (a.isnan() & b.isnan())).all()) for a, b in zip(got, want)]
        assert all(same), (place, same)


@pytest.mark.parametrize("D", [100, 1237, 4096])
@pytest.mark.parametrize("scale", [0.7, 0.3, 1.0])
def test_the_scaled_residual_is_rounded_before_the_block_joins_it(scale, D):
    """Of a scale that fp32 does not hold, what was added to it goes with the rounding of the product, so that sums of few digits which
    lie half way between two values of bf16 go the way that they go as written: the sum is that of products and a sum rounded to fp32 each."""
    T = 700
    x, res, w = normal((T, D), 1, torch.bfloat16), (2 * normal((T, D), 2, torch.float32)).to(torch.bfloat16), normal((D,), 3, torch.bfloat16, 1.0)
    gate = (0.5 * normal((D,), 4, torch.float32)).to(torch.bfloat16)
    _, total, _ = O.psa_block_norm(x, res, w, gate=gate, residual_scale=scale)
    assert torch.equal(total, (res.float() * scale + x.float() * gate.float()).to(torch.bfloat16))
