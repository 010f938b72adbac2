"""The global norm of many gradients and clipping by it against fp64.  The norm is a sum of exact squares in 64 bits, rounded once to fp32; a clipped value is
the gradient times the fp32 factor, rounded once."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2305_09887_amd import binding
    binding.lib()
    return binding


def _views(sizes, dtype, seed, gap=0, scale=1.0):
    """Tensors one behind the other in a buffer: they begin anywhere."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = (torch.randn(sum(sizes) + gap * len(sizes) + 1, generator=g, device="cuda") * scale).to(dtype)
    out, at = [], 1
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + gap
    return flat, out


def _norm(grads):
    return math.sqrt(sum(float(t.double().square().sum()) for t in grads))


LISTS = [[1], [7], [16384], [16385], [5, 0, 3, 0, 0, 16390], [100_003], list(range(1, 300)), [3] * 400, [70_000, 1, 33, 16_384, 40_000] * 60, [9_000_001, 5, 2_000_003]]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{sum(s)}")
def test_norm_and_clipping(B, sizes, dtype):
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    flat, grads = _views(sizes, dtype, len(sizes))
    want = _norm(grads)
    got = float(B.tma_grad_norm(grads))
    assert abs(got - want) <= want * 2.0 ** -23
    before = flat.clone()
    out_flat, outs = _views(sizes, dtype, 5, gap=2)
    spare = out_flat.clone()
    for ratio in (0.37, 1.5):
        assert float(B.tma_grad_clip(grads, ratio * want, out=outs)) == got
        assert torch.equal(flat, before)
        for o, t in zip(outs, grads):
            if ratio > 1:
                assert torch.equal(o, t)
            else:
                w = t.double() * ratio
                assert bool(((o.double() - w).abs() <= w.abs() * (u + 2.0 ** -23)).all())
    for o in outs:
        o.fill_(0)
    mask = out_flat != 0
    assert torch.equal(out_flat[mask], spare[mask])               # what lies between the results
    clipped = [o.clone() for o in outs]
    B.tma_grad_clip(grads, 0.37 * want, out=outs)
    B.tma_grad_clip(grads, 0.37 * want)                             # in place
    assert all(torch.equal(o, t) for o, t in zip(outs, grads))
    assert flat[0] == before[0]
    again = flat.clone()
    assert abs(float(B.tma_grad_clip(grads, want)) - 0.37 * want) <= want * (u + 2.0 ** -22)
    assert torch.equal(flat, again)                                 # within the bound: left as it is
    assert all(c.numel() == o.numel() for c, o in zip(clipped, outs))


def test_values_whose_squares_fp32_does_not_hold(B):
    for scale in (1e30, 1e-30):
        _, grads = _views([1000, 3], torch.float32, 1, scale=scale)
        want = _norm(grads)
        assert abs(float(B.tma_grad_norm(grads)) - want) <= want * 2.0 ** -23
        B.tma_grad_clip(grads, want / 2)
        assert abs(_norm(grads) - want / 2) <= want * 2.0 ** -22


def test_norms_of_nothing_of_zero_and_of_no_number(B):
    empty, zeros = torch.empty(0, device="cuda"), torch.zeros(40, device="cuda")
    assert float(B.tma_grad_norm([empty])) == 0 and float(B.tma_grad_clip([empty, empty], 1.0)) == 0
    assert float(B.tma_grad_clip([zeros, empty], 0.0)) == 0 and not zeros.any()
    t = torch.ones(40, device="cuda")
    t[3] = math.inf
    other = torch.ones(5, device="cuda")
    assert float(B.tma_grad_clip([t, other], 1.0)) == math.inf
    assert torch.isnan(t[3]) and not t[:3].any() and not t[4:].any() and not other.any()
    t[3] = math.nan
    other.fill_(1)
    assert math.isnan(float(B.tma_grad_clip([t, other], 1.0)))
    assert torch.isnan(t).all() and torch.isnan(other).all()


def test_more_than_32_bits_of_values(B):
    n = (1 << 31) + 77
    t = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    small = torch.full((5,), 0.5, dtype=torch.bfloat16, device="cuda")
    norm = float(B.tma_grad_norm([small, t]))
    assert abs(norm - 0.5 * math.sqrt(n + 5)) <= 2.0 ** -23 * norm
    B.tma_grad_clip([small, t], norm / 4)
    # 0.5 times a factor within 2^-22 of 1/4: one of bf16's values beside 1/8 at most
    for part in (small, t[:1000], t[n // 2:n // 2 + 1000], t[-1000:]):
        assert bool(((part.float() - 0.125).abs() <= 0.125 * 2.0 ** -7).all())


def test_an_infinite_bound_leaves_gradients_as_they_are(B):
    t = torch.randn(1000, device="cuda")
    was = t.clone()
    B.tma_grad_clip([t], math.inf)
    assert torch.equal(t, was)


def test_refusals(B):
    t = torch.ones(8, device="cuda")
    for bad in (-1.0, math.nan):
        with pytest.raises(B.TmaError, match="max_norm"):
            B.tma_grad_clip([t], bad)
    for grads in ([], [t, t.double()], [t, t.bfloat16()], [torch.ones((4, 4), device="cuda").t()[:2]], [t.cpu()]):
        with pytest.raises(B.TmaError):
            B.tma_grad_norm(grads)
    with pytest.raises(B.TmaError):
        B.tma_grad_clip([t], 1.0, out=[t, t])
    with pytest.raises(B.TmaError):
        B.tma_grad_clip([t], 1.0, out=[torch.ones(7, device="cuda")])
    with pytest.raises(B.TmaError, match="workspace"):
        B.tma_grad_norm([t], ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
