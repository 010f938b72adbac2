"""A clipped value is the gradient times max_norm / norm in 64 bits, rounded to the result's type (to bf16 by way of fp32): also where that factor is no normal fp32 number."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scale,bound", [(1.0, 0.3), (1e-3, 1e-9), (1e37, 1.0), (1e37, 1e-3), (1e37, 1e-8), (1e-30, 1e-36), (3e37, 1e36)])
@pytest.mark.parametrize("off", [0, 1])
def test_factors(B, scale, bound, off, dtype):
    n = 40_003
    g = torch.Generator(device="cuda").manual_seed(3)
    flat = (torch.randn(n + off, generator=g, device="cuda").clamp(-3, 3) * scale).to(dtype)
    t = flat[off:]
    out = torch.empty(n + 1, dtype=dtype, device="cuda")[1 - off:n + 1 - off]       # alignments alike and not
    factor = bound / float(t.double().norm())
    assert factor < 1
    want = t.double() * factor
    B.tma_grad_clip([t], bound, out=[out])
    # half a step of fp32, of bf16 with one of fp32 before it, at subnormal numbers of their smallest step; the factor itself is within 2^-40
    u, least = (2.0 ** -8 + 2.0 ** -24, 2.0 ** -134) if dtype == torch.bfloat16 else (2.0 ** -24, 2.0 ** -150)
    assert bool(((out.double() - want).abs() <= want.abs() * (u + 2.0 ** -40) + least * 1.01).all())
    if dtype == torch.float32:
        assert bool((out == want.float()).float().mean() > 0.999)         # (ties and near ties of the 64-bit norm's own roundings)
    B.tma_grad_clip([t], bound)
    assert torch.equal(t, out)
