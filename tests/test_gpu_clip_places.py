"""Clipping where gradients and results lie among each other in one buffer, without an overlap that is refused: each result is its gradient's, whatever the order."""
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


def _close(got, grad, factor, dtype):
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24      # a result's rounding; the norm that the bound was taken from and the factor are off by 2^-22 at most
    want = grad.double() * factor
    return bool(((got.double() - want).abs() <= want.abs() * (u + 2.0 ** -21)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 5, 300])
def test_results_between_gradients(B, count, dtype):
    sizes = [1 + 977 * (k % 7) + 70_000 * (k == 3) for k in range(count)]
    g = torch.Generator(device="cuda").manual_seed(count)
    flat = torch.randn(2 * sum(sizes), generator=g, device="cuda").to(dtype)
    grads, outs, at = [], [], 0
    for k, n in enumerate(sizes):                      # gradient, result, gradient, result ...; every third in place
        grads.append(flat[at:at + n])
        outs.append(grads[-1] if k % 3 == 2 else flat[at + n:at + 2 * n])
        at += 2 * n
    order = torch.randperm(count, generator=torch.Generator().manual_seed(1)).tolist()
    was = [t.clone() for t in grads]
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    B.tma_grad_clip([grads[k] for k in order], norm / 3, out=[outs[k] for k in order])
    for k in range(count):
        assert _close(outs[k], was[k], 1 / 3, dtype)
        assert outs[k] is grads[k] or torch.equal(grads[k], was[k])


def test_a_gradient_read_twice(B):
    t, a, b = torch.randn(5000, device="cuda"), *(torch.empty(5000, device="cuda") for _ in range(2))
    was = t.clone()
    norm = math.sqrt(2) * float(t.double().norm())
    assert abs(float(B.tma_grad_clip([t, t], norm / 2, out=[a, b])) - norm) <= norm * 2.0 ** -23
    assert torch.equal(a, b) and torch.equal(t, was) and _close(a, was, 0.5, torch.float32)


def test_refused_places_are_left_as_they_are(B):
    flat = torch.randn(4000, device="cuda")
    was = flat.clone()
    a, b = flat[:1000], flat[1000:2000]
    for grads, outs, norm_out in (([a, b], [b, a], None), ([a], [flat[1:1001]], None), ([a, a], [a, flat[2000:3000]], None), ([a], None, a[5:6]), ([a], [b], b[-1:])):
        with pytest.raises(B.TmaError, match="overlap"):
            B.tma_grad_clip(grads, 0.1, out=outs, norm_out=norm_out)
    torch.cuda.synchronize()
    assert torch.equal(flat, was)
    B.tma_grad_norm([a, b], norm_out=a[:1])             # read before it is written
    assert abs(float(a[0]) - float(was[:2000].double().norm())) <= 2.0 ** -23 * float(a[0])
