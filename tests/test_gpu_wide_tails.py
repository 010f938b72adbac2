"""SiLU and GELU of wide layers and their derivatives far from zero, where the functions are small or their exponentials leave fp32's range: W is the identity, so that
every pre-activation is the row's value exactly.

Bounds, in parts of the true value.  An exponential's argument is rounded once after it is multiplied by log2 e (2^-24 of it, and 2^-26 for the constant): SiLU's is z,
GELU's -z^2 / 2, itself rounded once more.  The exponential and the reciprocal instruction are within two units, 2^-22 each, the fit of GELU's tail within 3.4e-7, and a
handful of roundings follow: 2^-20 holds them all."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F = 32
FAR = [13.5, 20.0, 37.0, 60.0, 87.0, 88.5, 89.0, 100.0, 150.0, 1e4, 1e10, 1e20, 3e38]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def relative(name, z):
    return 2.0 ** -20 + (1.25 * z.abs() if name == "silu" else 2.25 * z * z / 2) * 2.0 ** -24


def value(name, z):
    return z * torch.sigmoid(z) if name == "silu" else 0.5 * z * torch.erfc(-z / math.sqrt(2))


def slope_and_bound(name, z):
    """The derivative, and the bound of its terms, each off by the function's part."""
    r = relative(name, z)
    if name == "silu":
        t, rest = torch.sigmoid(z), torch.sigmoid(-z)
        return t * (1 + z * rest), t * (1 + z.abs() * rest) * r + t * z.abs() * (t * r + 2.0 ** -24)
    p, d = 0.5 * torch.erfc(-z / math.sqrt(2)), z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return p + d, (p + d.abs()) * r


def run(B, name, z):
    """act(z), as a layer with a residual and as a gated one give it, and act'(z)."""
    act = B.TMA_ACT_SILU if name == "silu" else B.TMA_ACT_GELU
    eye, one = torch.eye(F, device="cuda"), torch.ones(F, device="cuda")
    y, kept = B.tma_dense_residual_fwd(z, eye, None, act, save=True)
    assert torch.equal(kept, z)
    h, g, u = B.tma_gated_dense_fwd(z, eye, torch.zeros_like(eye), None, one, act)
    assert torch.equal(g, z) and bool((u == 1).all()) and torch.equal(h, y)
    d = B.tma_dense_residual_bwd(torch.zeros_like(z), z, torch.ones_like(z), eye, act)[2]
    dg = B.tma_gated_dense_bwd(torch.zeros_like(z), z, torch.ones_like(z), torch.ones_like(z), eye, torch.zeros_like(eye), act)[4]
    assert torch.equal(d, dg)
    return y, d


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("n", [3, 64, 4000])
def test_over_the_range_of_their_values(B, name, n):
    top = 80.0 if name == "silu" else 12.5          # (their values are normal fp32 numbers up to here)
    z = torch.linspace(-top, top, n * F, device="cuda").view(n, F)
    y, d = run(B, name, z)
    Z = z.double()
    want = value(name, Z)
    assert bool(((y.double() - want).abs() <= want.abs() * relative(name, Z)).all())
    want, bound = slope_and_bound(name, Z)
    assert bool(((d.double() - want).abs() <= bound + 2.0 ** -120).all())       # (parts of gradients below 2^-126 are lost)


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("n", [2, 70])
def test_far_out(B, name, n):
    z = torch.tensor(FAR, device="cuda").repeat(n * F // len(FAR) + 1)[:n * F].view(n, F)
    for sign in (1.0, -1.0):
        y, d = run(B, name, sign * z)
        Z = sign * z.double()
        assert torch.isfinite(y).all() and torch.isfinite(d).all()
        if sign > 0:
            assert bool(((y.double() - Z).abs() <= Z * 2.0 ** -18).all()) and bool(((d.double() - 1).abs() <= 2.0 ** -14).all())
        else:                                       # at most 13.5 e^-13.5 and 13.5 e^(-13.5^2 / 2)
            assert bool(((y.double() - value(name, Z)).abs() <= 2.0 ** -34).all()) and bool((d.double() - slope_and_bound(name, Z)[0]).abs().max() <= 2.0 ** -33)
