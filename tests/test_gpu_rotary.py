"""psa_rotary against the oracle in 64 bits.

Tolerances: a fraction of a turn is exact to 2^-33, becomes an fp32 number of at most 1/2 (off by 2^-26 of a turn, 2^-23.3 rad), and
its sine and cosine are off by 2^-23 more; two products, a sum and the magnitude round by 2^-24 each: 2^-21 of (|a| + |b|) times
the magnitude covers all, then half a step of the output's type."""
import numpy as np
import pytest
import torch

from oracle import psa_oracle as orc
from paper_2410_20305_b200 import binding as B
from paper_2410_20305_b200 import operators as O

pytestmark = pytest.mark.gpu

f64 = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
half = lambda t: torch.finfo(t).eps / 2  # noqa: E731
SCALINGS = [None, "linear", "base", "wavelength", "ramp"]


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def tables(r, scaling=None, theta=10000.0):
    turns, magnitude = O.psa_rotary_frequencies(r, theta, scaling, factor=8.0, original_length=2048, device="cuda")
    return turns, magnitude, orc.rotary_frequencies(r, theta, scaling, 8.0, 2048)


def within(name, got, x, pos, radians, magnitude, **kw):
    ref = orc.rotary(f64(x), pos, radians, magnitude, **kw)
    n = len(radians)
    a = np.abs(f64(x))
    size = np.zeros_like(a)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if kw.get("interleaved") else (slice(0, n), slice(n, 2 * n))
    size[..., first] = size[..., second] = a[..., first] + a[..., second]
    tol = np.where(size > 0, half(got.dtype) * np.abs(ref), 0) + magnitude * 2.0 ** -21 * size
    worst = (np.abs(f64(got) - ref) / np.maximum(tol, 1e-300)).max(initial=0)
    print("%s: %.3f of its tolerance" % (name, worst))
    assert worst <= 1, (name, worst)


def positions(T, seed, far=0):
    rng = np.random.default_rng(seed)
    return (rng.integers(0, 5000, size=T) + far).astype(np.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,d,r", [(1, 32, 8, 128, 128), (1, 1, 1, 2, 2), (3, 2, 1, 6, 4), (7, 3, 3, 80, 20), (50, 4, 2, 64, 64), (33, 5, 1, 96, 36),
                                         (300, 32, 8, 128, 128), (1000, 7, 1, 72, 66), (17, 2, 2, 256, 192), (5, 3, 2, 1024, 1024),
                                         (4000, 9, 3, 66, 66), (13, 2, 2, 7, 6)])
def test_against_the_oracle(T, Hq, Hk, d, r, interleaved, dtype):
    scaling = SCALINGS[(T + r) % 5] if r > 2 else None
    turns, magnitude, (radians, m) = tables(r, scaling)
    q, k, pos = normal((T, Hq, d), 1, dtype), normal((T, Hk, d), 2, dtype), positions(T, 3)
    odd_pair = interleaved and d % 2      # pairs of such heads start at odd elements: refused
    for inverse in (False, True):
        if odd_pair:
            with pytest.raises(B.PsaError) as e:
                O.psa_rotary(q, k, torch.as_tensor(pos).cuda(), turns, magnitude, interleaved, inverse)
            assert e.value.code == 4
            continue
        yq, yk = O.psa_rotary(q, k, torch.as_tensor(pos).cuda(), turns, magnitude, interleaved, inverse)
        within("q", yq, q, pos, radians, m, interleaved=interleaved, inverse=inverse)
        within("k", yk, k, pos, radians, m, interleaved=interleaved, inverse=inverse)


@pytest.mark.parametrize("scaling", SCALINGS)
def test_positions_near_and_far(scaling):
    """Angles are exact for any position: the fp32 product of position and frequency is off by whole turns at the last of these."""
    turns, magnitude, (radians, m) = tables(64, scaling, 500000.0)
    pos = np.array([0, 1, -1, 2, 4095, 10 ** 5, 10 ** 6 + 1, -10 ** 6, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], np.int32)
    q = normal((len(pos), 2, 64), 1, torch.float32)
    y, none = O.psa_rotary(q, None, torch.as_tensor(pos).cuda(), turns, magnitude)
    # 2^31 positions times a frequency that is exact to 2^-53 of itself are off by 2^-22 rad at most
    exact = f64(turns.cpu()) / 2.0 ** 64 * 2 * np.pi
    assert none is None and np.abs(exact / radians - 1).max() < 1e-12
    turned = np.mod(np.asarray(pos, dtype=object)[:, None] * np.array([int(t) for t in turns.cpu()], dtype=object), 2 ** 64)
    angle = turned.astype(np.float64) / 2.0 ** 64 * 2 * np.pi
    z = (f64(q)[..., :32] + 1j * f64(q)[..., 32:]) * (m * np.exp(1j * angle))[:, None]
    size = np.abs(f64(q)[..., :32]) + np.abs(f64(q)[..., 32:])
    for got, ref in ((f64(y)[..., :32], z.real), (f64(y)[..., 32:], z.imag)):
        assert (np.abs(got - ref) <= 2.0 ** -24 * np.abs(ref) + m * 2.0 ** -21 * size).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_whole_head_in_halves_is_psa_rope(dtype):
    q, pos = normal((200, 4, 128), 1, torch.bfloat16), positions(200, 2)
    turns, magnitude = O.psa_rotary_frequencies(128, device="cuda")
    want = B.psa_rope(q, torch.as_tensor(pos).cuda())
    got, _ = O.psa_rotary(q.to(dtype), None, torch.as_tensor(pos).cuda(), turns, magnitude)
    # psa_rope's angle is an fp32 product: 5000 * (2^-24 + the 2^-22 of its frequency's power) rad
    assert (got.float() - want.float()).abs().max() <= 2.0 ** -8 * 8 + 2 * 5 * 5000 * 2.0 ** -22


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_views_of_one_projection_in_place_and_apart(dtype, interleaved):
    T, Hq, Hk, d, r = 130, 6, 2, 64, 48
    fused = normal((T + 3, (Hq + 2 * Hk) * d), 1, dtype)
    turns, magnitude, (radians, m) = tables(r, "ramp")
    pos = positions(T, 5)
    dp = torch.as_tensor(pos).cuda()
    views = lambda f: (f[:T, :Hq * d].view(T, Hq, d), f[:T, Hq * d:(Hq + Hk) * d].view(T, Hk, d))  # noqa: E731
    q, k = views(fused)
    yq, yk = O.psa_rotary(q, k, dp, turns, magnitude, interleaved)
    assert yq.is_contiguous() and yk.is_contiguous()
    within("q", yq, q, pos, radians, m, interleaved=interleaved)
    within("k", yk, k, pos, radians, m, interleaved=interleaved)
    twin = fused.clone()
    q2, k2 = views(twin)
    assert O.psa_rotary(q2, k2, dp, turns, magnitude, interleaved, q_out=q2, k_out=k2)[0] is q2
    assert torch.equal(q2, yq) and torch.equal(k2, yk)
    assert torch.equal(twin[:, (Hq + Hk) * d:], fused[:, (Hq + Hk) * d:]) and torch.equal(twin[T:], fused[T:])
    # into another fused buffer, heads outermost, tokens apart, every second token, and one side in place
    other = torch.zeros_like(fused)
    q3, k3 = views(other)
    O.psa_rotary(q, k, dp, turns, magnitude, interleaved, q_out=q3, k_out=k3)
    assert torch.equal(q3, yq) and torch.equal(k3, yk) and not other[:, (Hq + Hk) * d:].any() and not other[T:].any()
    heads_first = torch.zeros((Hq, T, d), dtype=dtype, device="cuda").transpose(0, 1)
    O.psa_rotary(q, None, dp, turns, magnitude, interleaved, q_out=heads_first)
    assert torch.equal(heads_first, yq)
    wide = torch.zeros((2 * T, Hq, d + 8), dtype=dtype, device="cuda")
    O.psa_rotary(q.transpose(0, 1).contiguous().transpose(0, 1), k, dp, turns, magnitude, interleaved, q_out=wide[::2, :, 4:4 + d])
    assert torch.equal(wide[::2, :, 4:4 + d], yq) and not wide[1::2].any() and not wide[..., :4].any() and not wide[..., 4 + d:].any()
    expanded = q[:1].expand(T, Hq, d)
    got, _ = O.psa_rotary(expanded, None, dp, turns, magnitude, interleaved)
    within("one token at every position", got, expanded, pos, radians, m, interleaved=interleaved)


@pytest.mark.parametrize("offset,pitch", [(1, 64), (2, 66), (3, 67), (4, 68), (0, 65)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_alignments(dtype, offset, pitch):
    T, H, d, r = 40, 3, 64, 64
    buffer = normal((T * H * pitch + 8,), 1, dtype)
    q = buffer[offset:].as_strided((T, H, d), (H * pitch, pitch, 1), offset)
    turns, magnitude, (radians, m) = tables(r)
    pos = positions(T, 5)
    y, _ = O.psa_rotary(q, None, torch.as_tensor(pos).cuda(), turns, magnitude)
    within("q", y, q, pos, radians, m)
    if offset % 2 == 0 and pitch % 2 == 0:
        y, _ = O.psa_rotary(q, None, torch.as_tensor(pos).cuda(), turns, magnitude, interleaved=True)
        within("interleaved", y, q, pos, radians, m, interleaved=True)


def test_there_and_back():
    turns, magnitude, _ = tables(128, "wavelength")
    q, pos = normal((500, 4, 128), 1, torch.float32), torch.as_tensor(positions(500, 2, 10 ** 6)).cuda()
    there, _ = O.psa_rotary(q, None, pos, turns, magnitude)
    back, _ = O.psa_rotary(there, None, pos, turns, magnitude, inverse=True)
    assert (back - q).abs().max() <= 2.0 ** -21 * 4 * q.abs().max()
    # the gradient's definition: <R a, b> = <a, R' b>
    b = normal((500, 4, 128), 3, torch.float32)
    rb, _ = O.psa_rotary(b, None, pos, turns, magnitude, inverse=True)
    assert abs(float((there.double() * b.double()).sum() - (q.double() * rb.double()).sum())) <= 1e-3


def test_no_tokens_and_bad_values():
    turns, magnitude, _ = tables(64)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    y, _ = O.psa_rotary(q, q, torch.zeros(0, dtype=torch.int32, device="cuda"), turns)
    assert y.shape == q.shape
    x = normal((20, 2, 96), 1, torch.bfloat16)
    clean, _ = O.psa_rotary(x, None, torch.arange(20, dtype=torch.int32, device="cuda"), turns)
    z = x.clone()
    z[7, 1, 3] = float("nan")
    got, _ = O.psa_rotary(z, None, torch.arange(20, dtype=torch.int32, device="cuda"), turns)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[7, 1, 3] = bad[7, 1, 35] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("d", [128])
def test_beyond_2_31_elements(d):
    T, H = 2 ** 21 + 5, 9
    q = torch.zeros((T, H, d), dtype=torch.bfloat16, device="cuda")
    q[-3:] = normal((3, H, d), 1, torch.bfloat16)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    pos[-3:] = torch.tensor([5, 100000, 7], dtype=torch.int32)
    turns, magnitude, (radians, m) = tables(d)
    y, _ = O.psa_rotary(q, None, pos, turns, magnitude, q_out=q.clone())
    within("last", y[-3:], q[-3:], np.array([5, 100000, 7]), radians, m)
    assert not y[:-3].any()
